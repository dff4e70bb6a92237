"""GPU tests of values that are infinite or not a number in the paged
attention: what the rows that see them get, and that no other row notices."""
import numpy as np
import pytest

from paper_2402_07901_amd import fastmax as fm

import serve_util as su
from gpu_util import say
from paged_util import positions, put, seen
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


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_single_tokens_get_the_infinity_they_see(dtype, D, window, sinks):
    """Lengths that end inside a tile of 16 keys, in an odd number of tiles, in
    one tile and in several splits: lanes without a key of their own read
    another one under weight 0, which must not make a NaN of its infinity."""
    import torch
    say(f"one token and an infinity D={D} {dtype} window={window}")
    lens = [1, 8, 16, 17, 40, 72, 333, 777, 3000]
    for back in (0, 1, 5, 19, 20, 50, 10 ** 6):        # tokens before the last; or the first
        for value in (float("inf"), float("-inf"), float("nan")):
            c = Cache(lens, [1] * len(lens), 4, 2, D, 32, dtype, seed=D)
            want = np.zeros((len(lens), 4, D), bool)
            for s, n in enumerate(lens):
                t = max(0, n - 1 - back)
                put(c, s, t, 1, value, 9)
                want[s, 2:, 9] = seen(n - 1, t, window, sinks)
            out = su.np64(c.run(starts=False, window=window, sinks=sinks))
            assert np.array_equal(~np.isfinite(out), want), (back, value)
            if value == value:
                assert (out[want] == value).all(), (back, value)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("starts", [True, False])
def test_a_weight_of_zero_makes_nan_of_an_infinity(dtype, D, starts):
    """p = 1, scale 1 / D, q^ = -k^ of +-1 entries: the weight is exactly 0 and
    0 times infinity is NaN; where q^ = k^ it is 2."""
    import torch
    n, t = 150, 100
    news = n if starts else 1
    c = Cache([n], [news], 4, 2, D, 32, dtype, seed=D)
    u = torch.ones(D, device="cuda")
    u[::2] = -1.0
    c.k[int(c.table_h[0, t // 32]), 1, t % 32] = u.to(c.k.dtype)
    put(c, 0, t, 1, float("inf"), 9)
    c.q[:, 2], c.q[:, 3] = -u.to(c.q.dtype), u.to(c.q.dtype)
    out = c.run(starts=starts, p=1, scale=1.0 / D, max_q=news)
    see = seen(positions(c, 0), t)
    bad = su.np64(~torch.isfinite(out)) > 0
    assert bad[see, 2:, 9].all() and bad.sum() == 2 * see.sum()
    out = su.np64(out)
    assert np.isnan(out[see, 2, 9]).all()
    assert (out[see, 3, 9] == np.inf).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("n,news,t", [(150, 150, 100), (150, 3, 148), (4000, 100, 3950),
                                      (4000, 100, 17), (4000, 1, 3990)])
def test_first_order_weights_have_a_sign(dtype, D, n, news, t):
    """p = 1: an infinity comes out under its weight's sign, near the diagonal
    and far behind it, in one launch and in splits."""
    say(f"first order and an infinity D={D} {dtype} n={n} new={news} t={t}")
    c = Cache([n], [news], 4, 2, D, 32, dtype, seed=D)
    put(c, 0, t, 1, float("inf"), 9)
    tau = 1.0 / np.sqrt(D)                             # scores of size 1
    out = su.np64(c.run(starts=news > 1, p=1, scale=float(np.float32(tau)), max_q=news))
    see = seen(positions(c, 0), t)
    G = 1.0 + tau * np.einsum("thd,nd->thn", su.np64(c.q)[:, 2:], c.k_h[0][:, 1])
    w = G[..., t]
    G = np.where((np.arange(n) <= positions(c, 0)[:, None])[:, None], G, 0.0).sum(-1)
    bad = ~np.isfinite(out)
    assert bad[see, 2:, 9].all() and bad.sum() == 2 * see.sum()
    # a score near -1 / tau leaves its weight's sign to rounding (D + 8 steps of
    # 2^-24 of a sum of magnitudes up to D), and so does a sum near 0
    sure = see[:, None] & (np.abs(w) > 1e-3) & (np.abs(G) > 1e-3 * n)
    assert sure.any() and (see.sum() < 20 or ((w < 0) & sure).any())
    assert np.array_equal(out[:, 2:, 9][sure], np.sign(w / G)[sure] * np.inf)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinities_in_splits_of_a_chunk(dtype):
    """One sequence whose keys are cut into pieces that are joined: tokens near
    the diagonal, in the last and in an earlier piece."""
    import torch
    n, news, D = 4000, 100, 64
    assert fm.paged_workspace_bytes(1, news, 4, 2, D, news, n, 0, 0,
                                    fm.F32 if dtype == "f32" else fm.BF16) > 0
    for t in (3990, 3950, 3904, 1000):
        for value in (float("inf"), float("-inf"), float("nan")):
            c = Cache([n], [news], 4, 2, D, 32, dtype, seed=t)
            put(c, 0, t, 0, value, 40)
            out = c.run(max_q=news, max_len=n)
            see = seen(positions(c, 0), t)
            bad = su.np64(~torch.isfinite(out)) > 0
            assert bad[see, :2, 40].all() and bad.sum() == 2 * see.sum(), (t, value)
            if value == value:
                assert (su.np64(out)[see, :2, 40] == value).all(), (t, value)
