"""GPU tests of the sizes that a paged call is given: left to their defaults,
too small, row starts outside q; and chunks and windows at the bound of weights
in two bf16 parts, whatever their rows."""
import numpy as np
import pytest

from paper_2402_07901_amd import fastmax as fm

import serve_util as su
from gpu_util import say
from paged_util import check_rows
from test_paged import Cache

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


@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (17, 4), (64, 16), (100, 200),
                                          (5000, 3)])
def test_chunks_and_windows_at_two_parts(D, dtype, window, sinks):
    """Whole prompts, a few tokens after many and none, through either kernel
    (max_q chooses), held to weights of 16 bits."""
    label = f"paged chunks D={D} {dtype} window={window} sinks={sinks}"
    say(label)
    lens, news = [1, 70, 200, 333, 64, 500, 130, 1000], [1, 70, 5, 200, 0, 129, 64, 90]
    c = Cache(lens, news, 6, 2, D, 32, dtype, seed=D + window)
    kw = dict(window=window, sinks=sinks)
    for max_q in (200, 8, 1):
        c.check(c.run(max_q=max_q, max_len=1000, **kw), (label, max_q), starts=False, **kw)
    c.check(c.run(p=1, scale=1.0 / D, max_q=200, max_len=1, **kw), (label, "p = 1"), p=1,
            tau=1.0 / D, starts=False, **kw)


@pytest.mark.parametrize("max_q", [9, 3])
@pytest.mark.parametrize("Hq,Hkv", [(4, 2), (32, 1)])
def test_odd_starts_write_their_own_rows_only(max_q, Hq, Hkv):
    """Row starts outside q are cut to it: q and out lie in larger buffers, whose
    other rows stay as they are, and so do the rows that no sequence has."""
    import torch
    lens, T, D = [50, 60, 70], 9, 64
    c = Cache(lens, [2, 0, 4], Hq, Hkv, D, 16, "bf16")
    wide = torch.full((T + 8, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    q = wide[4:4 + T]
    q[:] = torch.randn((T, Hq, D), device="cuda").to(torch.bfloat16)
    own = torch.full((T + 8, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    out = own[4:4 + T]
    # rows 0 and 1; none, as its end lies before its start; all rows
    c.q_start = torch.tensor([-5, 2, -10 ** 6, 10 ** 6], dtype=torch.int32, device="cuda")
    c.q, c.start, c.news = q, np.array([0, 2, 0]), [2, 0, T]
    c.run(max_q=max_q, out=out)
    assert (own[:4] == 7.0).all() and (own[4 + T:] == 7.0).all()
    # the first two rows are either's
    check_rows(c, out, 2, np.arange(T) >= 2, "cut starts")
    assert torch.isfinite(out[:2]).all() and (out[:2] != 7.0).any()

    # without an overlap, with rows that nobody has
    own[:] = 7.0
    c.q_start = torch.tensor([-5, 2, 2, 5], dtype=torch.int32, device="cuda")
    c.start, c.news = np.array([0, 2, 2]), [2, 0, 3]
    c.run(max_q=max_q, out=out)
    assert (own[:4] == 7.0).all() and (own[9:] == 7.0).all()
    for s in (0, 2):
        check_rows(c, out, s, np.ones(c.news[s], bool), "rows 0 to 4")
    c.q_start = torch.tensor([5, 5, 5, 10 ** 6], dtype=torch.int32, device="cuda")
    own[:] = 7.0
    c.start, c.news = np.array([5, 5, 5]), [0, 0, 4]
    c.run(max_q=max_q, out=out)
    assert (own[:9] == 7.0).all() and (own[4 + T:] == 7.0).all()
    check_rows(c, out, 2, np.ones(4, bool), "rows 5 to 8")
