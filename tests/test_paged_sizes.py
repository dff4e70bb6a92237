"""GPU tests of the sizes that a paged call is given or leaves to their defaults."""
import numpy as np
import pytest

from paper_2402_07901_amd import fastmax as fm

import serve_util as su
from gpu_util import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fm.lib()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("D,dtype", [(32, "bf16"), (16, "bf16"), (32, "f32")])
def test_many_sequences_with_sizes_left_out(D, dtype):
    """1024 prompts of up to 200 tokens in one call that gives neither max_q
    nor max_len: every sequence might have all rows, as far as the call knows."""
    import torch
    say(f"1024 prompts D={D} {dtype}")
    S, Hq, Hkv, page = 1024, 32, 8, 64
    rng = np.random.default_rng(D)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(D)
    news = rng.integers(56, 201, S)
    lens = news + rng.integers(0, 80, S)
    start = np.concatenate([[0], np.cumsum(news)])
    T, cols = int(start[-1]), 5
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]

    def standard(*shape):
        x = torch.randn(shape, generator=gen, device="cuda")
        x = x - x.mean(-1, keepdim=True)
        return (x / x.square().mean(-1, keepdim=True).sqrt()).to(dt)

    k, q = standard(S * cols, Hkv, page, D), standard(T, Hq, D)
    v = torch.randn(k.shape, generator=gen, device="cuda").to(dt)
    table = torch.randperm(S * cols, device="cuda").to(torch.int32).reshape(S, cols)
    dev = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lens, start)]
    out = fm.fastmax_paged_fwd(q, k, v, table, dev[0], q_start=dev[1])
    known = fm.fastmax_paged_fwd(q, k, v, table, dev[0], q_start=dev[1], max_q=200,
                                 max_len=cols * page)
    assert torch.equal(out, known)
    for s in (0, 511, S - 1):
        n, rows = int(lens[s]), slice(int(start[s]), int(start[s + 1]))
        kv = [x[table[s].long()].transpose(0, 1).reshape(Hkv, -1, D)[:, :n] for x in (k, v)]
        for h in (0, Hkv - 1):
            hs = slice(4 * h, 4 * h + 4)
            ref, bound = su.attend(su.np64(q[rows, hs]), su.np64(kv[0][h]), su.np64(kv[1][h]),
                                   np.arange(n - int(news[s]), n), 2, 1.0, 0, 0,
                                   2 if dtype == "bf16" else None)
            su.check(out[rows, hs], ref, su.OUT[dtype] * np.abs(ref) + 1.01 * bound, (s, h))
