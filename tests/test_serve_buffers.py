"""GPU tests of the buffers and streams that a caller of the row calls and the
paged attention may bring."""
import pytest

from paper_2402_07901_amd import fastmax as fm

from test_rows import Rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fm.lib()
    yield
    torch.cuda.synchronize()


def test_allocations_of_the_null_stream():
    """Handle 0 is the null stream, and what the call allocates is its own."""
    import torch
    with fm._owner(0, torch.device("cuda", torch.cuda.current_device())):
        assert torch.cuda.current_stream().cuda_stream == 0
    r = Rows(1, 50, 6, 2, 64, "bf16")
    want = fm.fastmax_rope_fwd(r.q, r.k, r.v, **r.kw())
    torch.cuda.synchronize()
    got = fm.fastmax_rope_fwd(r.q, r.k, r.v, stream=0, **r.kw())
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
