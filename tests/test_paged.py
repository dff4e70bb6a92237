"""GPU tests of the paged attention against float64: single tokens and chunks,
pages, windows, first tokens, shared heads, rows that see nothing, what unused
slots hold, long caches, strides, streams and graphs."""
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


class Cache:
    """Sequences in a paged cache; unused slots and the rest of the page table
    hold what must not be used."""

    def __init__(self, lens, news, Hq, Hkv, D, page, dtype, seed=0, order="heads", junk="nan",
                 cols=None):
        import torch
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        rng = np.random.default_rng(seed)
        tdt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        S, need = len(lens), [-(-n // page) for n in lens]
        pages = sum(need) + 2
        self.lens_h, self.news, self.page, self.Hkv, self.group = lens, news, page, Hkv, Hq // Hkv
        self.dtype, self.D = dtype, D
        cols = max(need + [1]) + 1 if cols is None else cols
        order_ = rng.permutation(pages)
        self.table_h = np.full((S, cols), -1, np.int32)
        at = 0
        for s, n in enumerate(need):
            self.table_h[s, :n] = order_[at:at + n]
            at += n
        shape = (2, pages, Hkv, page, D) if order == "heads" else (2, pages, page, Hkv, D)
        both = torch.full(shape, float("nan") if junk == "nan" else 3e38, device="cuda").to(tdt)
        if order != "heads":
            both = both.transpose(2, 3)
        self.k, self.v = both[0], both[1]

        def randn(*shape):
            return torch.randn(shape, generator=gen, device="cuda")

        def standard(x):
            x = x - x.mean(-1, keepdim=True)
            return x / x.square().mean(-1, keepdim=True).sqrt()

        self.k_h, self.v_h = [], []
        for s, n in enumerate(lens):
            k = standard(randn(max(n, 1), Hkv, D)).to(tdt)[:n]
            v = randn(max(n, 1), Hkv, D).to(tdt)[:n]
            idx = torch.arange(n, device="cuda")
            pg = torch.from_numpy(self.table_h[s]).cuda().long()[idx // page]
            self.k[pg, :, idx % page] = k
            self.v[pg, :, idx % page] = v
            self.k_h.append(su.np64(k))
            self.v_h.append(su.np64(v))
        self.q = standard(randn(sum(news), Hq, D)).to(tdt)
        self.table = torch.from_numpy(self.table_h).cuda()
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.start = np.concatenate([[0], np.cumsum(news)])
        self.q_start = torch.tensor(self.start, dtype=torch.int32, device="cuda")

    def run(self, starts=True, **kw):
        return fm.fastmax_paged_fwd(self.q, self.k, self.v, self.table, self.lens,
                                    q_start=self.q_start if starts else None, **kw)

    def check(self, out, label, p=2, tau=1.0, window=0, sinks=0, starts=True):
        # chunks of a prompt may hold their weights in one bf16 part
        parts = None if self.dtype == "f32" else 1 if starts else 2
        out64 = su.np64(out)
        for s, n in enumerate(self.lens_h):
            rows = slice(self.start[s], self.start[s + 1])
            pos = n - self.news[s] + np.arange(self.news[s])
            for h in range(self.Hkv):
                hs = slice(h * self.group, (h + 1) * self.group)
                ref, bound = su.attend(su.np64(self.q[rows, hs]), self.k_h[s][:, h],
                                       self.v_h[s][:, h], pos, p, tau, window, sinks, parts)
                su.check(out[rows, hs], ref, su.OUT[self.dtype] * np.abs(ref) + 1.01 * bound,
                         (label, s, h))
        assert out64.shape == tuple(self.q.shape)


LENS = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 255, 300, 777]


@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv", [(3, 3), (8, 1), (14, 2), (40, 1)])
def test_single_tokens(D, dtype, Hq, Hkv):
    label = f"paged one token D={D} {dtype} H={Hq}/{Hkv}"
    say(label)
    c = Cache(LENS, [1] * len(LENS), Hq, Hkv, D, 16 if D < 64 else 64, dtype, seed=D)
    c.check(c.run(starts=False, max_len=777), label, starts=False)
    c.check(c.run(starts=False, p=1, scale=1.0 / D), label, p=1, tau=1.0 / D, starts=False)


@pytest.mark.parametrize("page", [16, 32, 128, 256, 1024])
@pytest.mark.parametrize("order", ["heads", "tokens"])
@pytest.mark.parametrize("junk", ["nan", "big"])
def test_pages_and_orders(page, order, junk):
    label = f"paged page={page} {order} {junk}"
    say(label)
    c = Cache([1, page - 1, page, page + 1, 1500], [1] * 5, 4, 2, 64, page, "bf16", seed=page,
              order=order, junk=junk)
    c.check(c.run(starts=False), label, starts=False)


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("f32", 32), ("bf16", 128)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (17, 4), (33, 31), (64, 16),
                                          (100, 200), (500, 1), (5000, 3)])
def test_windows(dtype, D, window, sinks):
    label = f"paged window={window} sinks={sinks} D={D} {dtype}"
    say(label)
    news = [1, 1, 3, 1, 1, 40, 1, 90]
    lens = [1, 16, 20, 65, 100, 333, 801, 1000]
    c = Cache(lens, news, 6, 2, D, 32, dtype, seed=window)
    c.check(c.run(max_q=90, window=window, sinks=sinks), label, window=window, sinks=sinks)
    one = Cache(lens, [1] * 8, 6, 2, D, 32, dtype, seed=window)
    # pages wholly behind the window are gone: their slots and entries with them
    for s, n in enumerate(lens):
        for i in range(-(-n // 32)):
            if (i + 1) * 32 - 1 <= n - 1 - window and i * 32 >= sinks:
                page = int(one.table_h[s, i])
                one.k[page], one.v[page] = float("nan"), float("inf")
                one.table[s, i] = -1 if i % 2 else 2 ** 31 - 1
    one.check(one.run(starts=False, window=window, sinks=sinks), label, window=window, sinks=sinks,
              starts=False)


@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (4, 1), (9, 3)])
def test_chunks(D, dtype, Hq, Hkv):
    """Chunks of prompts: whole prompts, a few tokens after many, none."""
    label = f"paged chunks D={D} {dtype} H={Hq}/{Hkv}"
    say(label)
    lens, news = [1, 70, 200, 333, 64, 500, 130], [1, 70, 5, 200, 0, 129, 64]
    c = Cache(lens, news, Hq, Hkv, D, 32, dtype, seed=D)
    c.check(c.run(max_q=200, max_len=500), label)
    c.check(c.run(max_q=200, max_len=500, p=1, scale=1.0 / D), label, p=1, tau=1.0 / D)


def test_sizes_that_are_too_small_cost_time_only():
    c = Cache([700, 40, 333], [150, 40, 1], 8, 2, 64, 64, "bf16")
    c.check(c.run(max_q=1, max_len=1), "small max_q and max_len")
    one = Cache([3000, 40, 333], [1, 1, 1], 8, 2, 64, 64, "bf16")
    one.check(one.run(starts=False, max_len=512), "small max_len", starts=False)


def test_rows_that_see_nothing_are_zero():
    """More new tokens than the sequence has, and empty sequences."""
    import torch
    c = Cache([0, 3, 40], [4, 7, 40], 4, 2, 64, 16, "bf16")
    out = torch.full_like(c.q, float("nan"))
    c.check(c.run(max_q=40, out=out), "no keys")
    assert (out[:8] == 0).all() and (out[8:11] != 0).any()
    one = Cache([0, 5], [1, 1], 4, 4, 32, 16, "f32")
    got = one.run(starts=False)
    one.check(got, "no keys", starts=False)
    assert (got[0] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_later_tokens_values_do_not_reach_earlier_rows(dtype):
    """An infinity or a NaN in the value of token t shows in rows from t on and
    in its own channel, nowhere else."""
    import torch
    n, t = 150, 100
    for value in (float("inf"), float("-inf"), float("nan")):
        c = Cache([n], [n], 4, 2, 64, 32, dtype)
        page = int(c.table_h[0, t // 32])
        c.v[page, 1, t % 32, 9] = value
        out = c.run(max_q=n)
        bad = ~torch.isfinite(out)
        assert bad[t:, 2:, 9].all()
        assert bad.sum() == (n - t) * 2
        if value == value:
            assert (out[t:, 2:, 9] == value).all()
        # the others are as without it
        c.v[page, 1, t % 32, 9] = 0.0
        c.v_h[0][t, 1, 9] = 0.0
        c.check(torch.where(bad, c.run(max_q=n), out), "beside the odd value")


def test_key_that_is_not_a_number_stays_behind_the_mask():
    import torch
    c = Cache([90], [90], 4, 2, 64, 32, "bf16")
    page = int(c.table_h[0, 2])
    c.k[page, 0, 6] = float("nan")          # token 70
    out = c.run(max_q=90)
    assert torch.isfinite(out[:70]).all() and torch.isfinite(out[:, 2:]).all()
    assert torch.isnan(out[70:, :2]).all()


def test_bad_pages_and_lengths_are_nan():
    """A page that is not there, a sequence longer than its row of the table."""
    import torch
    for entry in (-1, 10 ** 6, 2 ** 31 - 1, -2 ** 31):
        c = Cache([100, 100], [1, 1], 4, 2, 64, 32, "bf16")
        c.table[0, 1] = entry
        out = c.run(starts=False)
        assert torch.isnan(out[0]).all() and torch.isfinite(out[1]).all()
    c = Cache([100, 100], [1, 1], 4, 2, 64, 32, "bf16", cols=4)
    c.lens[0] = 129
    out = c.run(starts=False, max_len=128)
    assert torch.isnan(out[0]).all() and torch.isfinite(out[1]).all()


def test_odd_starts_stay_inside():
    """Row starts outside q are cut to it."""
    import torch
    c = Cache([50, 60, 70], [2, 3, 4], 4, 2, 64, 16, "bf16")
    c.q_start = torch.tensor([-5, 2, 1, 10 ** 6], dtype=torch.int32, device="cuda")
    out = torch.full_like(c.q, 7.0)
    c.run(max_q=9, out=out)
    assert torch.isfinite(out).all()


def test_large_offsets():
    """A cache whose elements pass 2^32: the last pages, appended and read."""
    import torch
    Hkv, page, D = 8, 64, 128
    pages = (2 ** 32) // (Hkv * page * D) + 3
    kv = torch.empty((2, pages, Hkv, page, D), dtype=torch.bfloat16, device="cuda")
    n = 100
    kv[:, -2:] = float("nan")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    q, k, v = (torch.randn((n, h, D), generator=gen, device="cuda").bfloat16()
               for h in (16, Hkv, Hkv))
    slots = (pages - 1) * page + torch.arange(n, device="cuda") % page
    slots[page:] -= page
    qh = fm.fastmax_cache_append(q, k, v, kv[0], kv[1], slots, None, None, None)
    table = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    out = fm.fastmax_paged_fwd(qh[-1:], kv[0], kv[1], table, lens)
    kc = torch.cat([kv[0, -1], kv[0, -2, :, :n - page]], 1)
    vc = torch.cat([kv[1, -1], kv[1, -2, :, :n - page]], 1)
    for h in range(Hkv):
        ref, bound = su.attend(su.np64(qh[-1:, 2 * h:2 * h + 2]), su.np64(kc[h]), su.np64(vc[h]),
                               np.array([n - 1]), 2, 1.0, 0, 0)
        su.check(out[:, 2 * h:2 * h + 2], ref, su.OUT["bf16"] * np.abs(ref) + 1.01 * bound, h)


def test_strided_queries_another_stream_kept_buffers():
    import torch
    c = Cache([2000, 300], [1, 1], 8, 2, 64, 64, "bf16")
    want = c.run(starts=False)
    wide = torch.zeros((2, 3, 8, 80), dtype=torch.bfloat16, device="cuda")
    wide[:, 1, :, 8:72] = c.q
    c.q = wide[:, 1, :, 8:72]
    need = fm.paged_workspace_bytes(2, 2, 8, 2, 64, 1, 2000, 0, 0, fm.BF16)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out = torch.empty((2, 8, 64), dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = c.run(starts=False, max_len=2000, workspace=ws, out=out)
    side.synchronize()
    assert got.data_ptr() == out.data_ptr()
    c.check(got, "strided", starts=False)
    assert (got.float() - want.float()).abs().max() <= 2.0 ** -7 * want.float().abs().max()


def test_decode_step_in_a_graph():
    """Append and attention captured once, replayed while the sequences grow."""
    import torch
    S, Hq, Hkv, D, page = 3, 8, 2, 64, 16
    kv = torch.zeros((2, 20, Hkv, page, D), dtype=torch.bfloat16, device="cuda")
    table = torch.arange(18, dtype=torch.int32, device="cuda").reshape(S, 6)
    cos, sin = (torch.from_numpy(t).cuda() for t in su.table(96, D))
    lens = torch.tensor([1, 30, 64], dtype=torch.int32, device="cuda")
    rows = torch.randn((S, Hq + 2 * Hkv, D), device="cuda").bfloat16()
    q, k, v = rows.split([Hq, Hkv, Hkv], dim=1)
    slots = torch.empty(S, dtype=torch.int64, device="cuda")
    kv[:, :18] = torch.randn((2, 18, Hkv, page, D), device="cuda").bfloat16()

    def step():
        at = lens.long() - 1
        slots.copy_(table.gather(1, (at // page)[:, None])[:, 0].long() * page + at % page)
        qh = fm.fastmax_cache_append(q, k, v, kv[0], kv[1], slots, lens - 1, cos, sin)
        return fm.fastmax_paged_fwd(qh, kv[0], kv[1], table, lens, max_len=96)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        lens += 1
        rows.copy_(torch.randn_like(rows))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, step()), i


def test_agrees_with_the_attention_itself():
    """Rows through fastmax_rope_fwd and fastmax_fwd, and through the cache one
    chunk and then single tokens: the same attention, in float32."""
    import torch
    N, Hq, Hkv, D, page = 200, 4, 2, 64, 32
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    rows = torch.randn((1, N, Hq + 2 * Hkv, D), generator=gen, device="cuda")
    cos, sin = (torch.from_numpy(t).cuda() for t in su.table(N, D))
    pos = torch.arange(N, dtype=torch.int32, device="cuda")[None]
    q, k, v = rows.split([Hq, Hkv, Hkv], dim=2)
    want, _ = fm.fastmax_fwd(*fm.fastmax_rope_fwd(q, k, v, pos, cos, sin), p=2, causal=True)
    want = want.transpose(1, 2)[0]
    kv = torch.zeros((2, 8, Hkv, page, D), device="cuda")
    table = torch.randperm(8, device="cuda", dtype=torch.int32)[None, :7].contiguous()
    n = torch.arange(N, device="cuda")
    slots = table[0].long()[n // page] * page + n % page
    first = 150
    qh = fm.fastmax_cache_append(q[0, :first], k[0, :first], v[0, :first], kv[0], kv[1],
                                 slots[:first], pos[0, :first], cos, sin)
    start = torch.tensor([0, first], dtype=torch.int32, device="cuda")
    got = [fm.fastmax_paged_fwd(qh, kv[0], kv[1], table,
                                torch.tensor([first], dtype=torch.int32, device="cuda"),
                                q_start=start)]
    for i in range(first, N):
        s = slice(i, i + 1)
        qh = fm.fastmax_cache_append(q[0, s], k[0, s], v[0, s], kv[0], kv[1], slots[s].clone(),
                                     pos[0, s].clone(), cos, sin)
        got.append(fm.fastmax_paged_fwd(qh, kv[0], kv[1], table,
                                        torch.tensor([i + 1], dtype=torch.int32, device="cuda")))
    got = torch.cat(got)
    assert (got - want).abs().max() <= 1e-4 * want.abs().max()   # float32 tolerance


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("size", [1e-30, 1e-6, 1e6, 1e25])
def test_values_of_any_size(D, size):
    """bf16 and float32 values far from 1, some a million times the others: the
    sums keep them (nothing shares a scale) while sum w |v|, up to 1e10 times
    ``size`` here, is a float32 number."""
    import torch
    for dtype in ("bf16", "f32"):
        c = Cache([200, 90], [70, 1], 4, 2, D, 32, dtype, seed=3)
        for s, n in enumerate(c.lens_h):
            grow = torch.ones(n, 1, D, device="cuda")
            grow[::7, :, ::3] = 2.0 ** 20
            idx = torch.arange(n, device="cuda")
            pg = c.table[s].long()[idx // 32]
            v = (torch.from_numpy(c.v_h[s]).cuda().float() * grow * size).to(c.v.dtype)
            c.v[pg, :, idx % 32] = v
            c.v_h[s] = su.np64(v)
        c.check(c.run(max_q=70), (D, size, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_any_size(dtype):
    """q^ and k^ are taken as they are: large ones, whose weights reach 1e12,
    small ones, whose weights are 1."""
    import torch
    for size in (1e3, 1e-20):
        for starts in (True, False):
            news = [60, 1, 33] if starts else [1, 1, 1]
            c = Cache([100, 40, 33], news, 4, 2, 64, 16, dtype, seed=4)
            c.q = (c.q.float() * size).to(c.q.dtype)
            c.check(c.run(starts=starts, max_q=60 if starts else 1), (size, starts), starts=starts)


def test_infinities_in_every_channel_of_one_token():
    """A whole token of infinities (and one of NaN) behind rows that see it and
    rows that do not, in chunks and single tokens."""
    import torch
    for D in (16, 64, 128):
        c = Cache([130], [130], 2, 1, D, 64, "bf16")
        page = int(c.table_h[0, 1])
        c.v[page, 0, 6] = float("-inf")          # token 70
        out = c.run(max_q=130)
        assert torch.isfinite(out[:70]).all()
        assert (out[70:] == float("-inf")).all()
        c.v[page, 0, 8] = float("nan")           # token 72
        out = c.run(max_q=130)
        assert (out[70:72] == float("-inf")).all() and torch.isnan(out[72:]).all()
        one = fm.fastmax_paged_fwd(c.q[:1], c.k, c.v, c.table,
                                   torch.tensor([72], dtype=torch.int32, device="cuda"))
        assert (one == float("-inf")).all()


def test_allocations_belong_to_the_stream():
    """Calls on a stream given as an object or as a handle, with the binding's
    own outputs and workspaces, while the current stream reuses memory."""
    import torch
    c = Cache([3000, 500], [1, 1], 8, 2, 64, 64, "bf16")
    want = c.run(starts=False)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = []
    for i in range(8):
        got.append(c.run(starts=False, stream=side if i % 2 else side.cuda_stream))
        torch.empty(1 << 20, device="cuda").fill_(float("nan"))
    torch.cuda.synchronize()
    for g in got:
        assert torch.equal(g, want)


@pytest.mark.parametrize("Hq,Hkv,lens,news", [(8, 1, [900], [300]), (6, 3, [700], [400]),
                                              (5, 5, [40, 1500], [33, 257]),
                                              (12, 12, [513], [513]),
                                              (16, 2, [2100, 70, 3], [130, 70, 1])])
@pytest.mark.parametrize("dtype,D", [("bf16", 32), ("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_chunks_of_few_heads(Hq, Hkv, lens, news, dtype, D):
    """Chunks whose units (sequence, key head, split) do not divide by the XCDs,
    uneven sequences among them; held to the bound of weights in two bf16 parts."""
    label = f"paged chunk D={D} {dtype} H={Hq}/{Hkv} lens={lens}"
    say(label)
    c = Cache(lens, news, Hq, Hkv, D, 32, dtype, seed=Hq)
    c.check(c.run(max_q=max(news)), label, starts=False)
    c.check(c.run(max_q=max(news), p=1, scale=1.0 / D), label, p=1, tau=1.0 / D, starts=False)
