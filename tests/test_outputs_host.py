"""The binding refuses a number of outputs that a call does not have (no GPU needed:
the count is looked at first)."""
import pytest

from paper_2402_07901_amd import fastmax as fm


def calls():
    import torch
    q, k = torch.zeros(1, 8, 4, 64), torch.zeros(1, 8, 2, 64)
    starts = torch.zeros(3, dtype=torch.int32)
    codes, scale = torch.zeros(5, 2, 16, 64, dtype=torch.int8), torch.zeros(5, 2, 16)
    slots = torch.zeros(3, dtype=torch.int64)
    heads = torch.zeros(1, 4, 8, 64)
    return [
        (3, "out", lambda x: fm.fastmax_rope_fwd(q, k, k, None, None, None, out=x)),
        (3, "out", lambda x: fm.fastmax_rope_bwd(q, k, heads, heads, heads, None, None, None, out=x)),
        (2, "out", lambda x: fm.fastmax_cache_read_q8(codes, codes, scale, scale, slots, out=x)),
        (3, "grads", lambda x: fm.fastmax_packed_bwd(q[0], k[0], k[0], starts, q[0], q[0], q[0, ..., 0], grads=x)),
    ]


@pytest.mark.parametrize("i", range(4))
def test_numbers_of_outputs(i):
    import torch
    n, name, call = calls()[i]
    for m in (0, 1, 2, 3, 4):
        if m != n:
            with pytest.raises(ValueError, match=f"{name} must be {n} tensors, got {m}"):
                call([torch.zeros(1)] * m)
    for given in ([torch.zeros(1)] * n, None):
        with pytest.raises(ValueError, match="on a GPU"):
            call(given)
