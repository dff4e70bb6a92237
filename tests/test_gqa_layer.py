"""GPU test of the example layer: a training step's gradients, and the same
rows served from the paged cache."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))


@pytest.mark.parametrize("dtype,bound", [("float32", 1e-4), ("bfloat16", 2e-2)])
def test_training_and_serving_agree(dtype, bound):
    """The library's tolerances: 1e-4 in float32, 2e-2 in bf16."""
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import gqa_layer
    off, grads = gqa_layer.main(B=2, N=150, prompt=130, width=128, Hq=6, Hkv=2, D=32,
                                dtype=getattr(torch, dtype))
    assert off <= bound
    assert all(0 < g < float("inf") for g in grads.values())
