"""GPU tests of the cache in 8 bits against float64: rows written and read back,
single tokens and chunks over it, pages, windows, what unused slots hold, rows
that are not finite, streams and graphs."""
import numpy as np
import pytest

from paper_2402_07901_amd import fastmax as fm

import q8_util as q8
import serve_util as su
from gpu_util import say
from q8_util import Cache
from test_rows import CASES, Rows, dt

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fm.lib()
    yield
    torch.cuda.synchronize()


def empty(pages, Hkv, page, D, order="heads"):
    """Caches and scales with something in them."""
    import torch
    shape = (2, pages, Hkv, page, D) if order == "heads" else (2, pages, page, Hkv, D)
    both = torch.randint(-127, 128, shape, device="cuda", dtype=torch.int8)
    k, v = both if order == "heads" else both.transpose(2, 3)
    ks, vs = torch.rand((2, pages, Hkv, page), device="cuda")
    return k, v, ks, vs


@pytest.mark.parametrize("T,Hq,Hkv,D,dtype,page,rot,axes,interleaved,norm", CASES)
@pytest.mark.parametrize("order", ["heads", "tokens"])
def test_append(T, Hq, Hkv, D, dtype, page, rot, axes, interleaved, norm, order):
    """q^ as fastmax_cache_append gives it; codes within half a step of the
    float64 rows (and the row's float32 error), other slots as they were."""
    import torch
    label = f"append q8 T={T} H={Hq}/{Hkv} D={D} {dtype} page={page} {order}"
    say(label)
    r = Rows(1, T, Hq, Hkv, D, dtype, rot, axes, interleaved, norm, seed=T)
    kw = r.kw()
    kw["pos"] = None if r.pos is None else r.pos[0]
    pages = -(-T // page) + 2
    cache = empty(pages, Hkv, page, D, order)
    before = [c.cpu().numpy() for c in cache]
    slots = torch.randperm(pages * page, device="cuda")[:T]
    if T > 4:      # padding, and slots that no page has
        slots[1], slots[2], slots[3] = -1, pages * page, 2 ** 62
    q_out = fm.fastmax_cache_append_q8(r.q[0], r.k[0], r.v[0], *cache, slots, **kw)
    plain = [torch.zeros((pages, Hkv, page, D), dtype=dt(dtype), device="cuda") for _ in range(2)]
    assert torch.equal(q_out, fm.fastmax_cache_append(r.q[0], r.k[0], r.v[0], *plain, slots, **kw))

    z, err = r.turned(r.k, r.wk)
    ref = su.standard(z)
    sd = z.std(-1, keepdims=True)
    # the append's float32 error of a row, as in test_rows
    err = (err.max(-1, keepdims=True) * 2 + 40 * np.abs(z).max(-1, keepdims=True)) / sd
    err = su.U * 1.01 * (err * (1.0 + np.abs(ref)) + 20 * np.abs(ref))
    rows = ((ref[0], err[0]), (su.np64(r.v)[0], np.zeros(1)))
    place = slots.cpu().numpy()
    kept = (place >= 0) & (place < pages * page)
    for name, codes, scales, old_c, old_s, (x, e) in zip(
            "kv", cache[:2], cache[2:], before[:2], before[2:], rows):
        codes, scales = codes.cpu().numpy(), scales.cpu().numpy()
        at = (place[kept] // page, slice(None), place[kept] % page)
        want, scale = q8.codes_of(x[kept])
        top = np.abs(x[kept]).max(-1)
        e = np.broadcast_to(e, x.shape)[kept]
        worst = e.max(-1)
        got_s = scales[at]
        assert (np.abs(got_s - scale) <= worst / 127 + 2 * su.U * scale).all(), (label, name)
        # a code's distance from its real value: half a step, the row's error in
        # steps (of the value, and through the scale) and two roundings
        off = (127 / top)[..., None] * (e + worst[..., None] * np.abs(x[kept]) / top[..., None])
        assert (np.abs(codes[at] - want) <= 0.5 + 1.01 * off + 4 * 127 * su.U).all(), (label, name)
        assert (np.abs(codes[at]).max(-1) == 127).all()
        free = np.ones((pages, page), bool)
        free[place[kept] // page, place[kept] % page] = False
        assert np.array_equal(codes.transpose(0, 2, 1, 3)[free], old_c.transpose(0, 2, 1, 3)[free])
        assert np.array_equal(scales.transpose(0, 2, 1)[free], old_s.transpose(0, 2, 1)[free])
    for got_dt in ("f32", "bf16"):
        got = fm.fastmax_cache_read_q8(*cache, slots, dtype=dt(got_dt))
        for x, codes, scales in zip(got, cache[:2], cache[2:]):
            want = torch.zeros((T, Hkv, D), device="cuda")
            inside = (slots >= 0) & (slots < pages * page)
            at = slots[inside]
            want[inside] = (codes[at // page, :, at % page].float()
                            * scales[at // page, :, at % page, None])
            assert torch.equal(x, want.to(dt(got_dt))), (label, got_dt)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [16, 64, 128])
def test_value_rows_of_every_kind(dtype, D):
    """Value rows that are exact in 8 bits, zero, tiny, huge and not finite, and
    codes at half steps (which go to the even one)."""
    import torch
    kinds = torch.zeros((9, 1, D))
    kinds[0] = torch.arange(D) - D // 2
    kinds[0, 0, 0] = 127.0
    kinds[2] = 2.0 ** -110                      # below the least row: zeros
    kinds[3] = 2.0 ** -99
    kinds[4, 0, ::2], kinds[4, 0, 1::2] = 3e38, -1e38
    kinds[5, 0, D - 1] = float("inf")
    kinds[6, 0, 3] = float("nan")
    kinds[7, 0, 5] = float("-inf")
    kinds[8, 0] = 0.5 + torch.arange(D) % 60    # half steps under a scale of 1
    kinds[8, 0, 1] = -127.0
    v = kinds.to(dt(dtype)).cuda()
    q, k = torch.randn((9, 2, D), device="cuda").to(v.dtype), torch.randn((9, 1, D), device="cuda").to(v.dtype)
    cache = empty(1, 1, 16, D)
    slots = torch.arange(9, device="cuda") + 3
    fm.fastmax_cache_append_q8(q, k, v, *cache, slots, None, None, None)
    codes, scale = cache[1][0, 0, 3:12].cpu().numpy(), cache[3][0, 0, 3:12].cpu().numpy()
    assert np.array_equal(codes[0], kinds[0, 0].numpy()) and scale[0] == 1.0
    assert not codes[[1, 2, 5, 6, 7]].any() and (scale[[1, 2]] == 0).all()
    assert np.isnan(scale[[5, 6, 7]]).all()
    assert (codes[3] == 127).all() and scale[3] == np.float32(2.0 ** -99) / np.float32(127)
    assert (codes[4, ::2] == 127).all() and (codes[4, 1::2] == -42).all()
    half = su.np64(v)[8, 0]
    assert scale[8] == 1.0 and np.array_equal(codes[8], np.round(half))
    back = fm.fastmax_cache_read_q8(*cache, slots)[1]
    assert torch.isnan(back[5:8]).all() and torch.isfinite(back[[0, 1, 2, 3, 4, 8]]).all()


def test_key_rows_that_are_not_finite():
    """A constant key row (no deviation) and one with an infinity: NaN scales,
    seen by the rows after them and by no others."""
    import torch
    T, D = 40, 64
    k = torch.randn((T, 1, D), device="cuda")
    k[20], k[30, 0, 5] = 3.0, float("inf")
    q, v = torch.randn((T, 2, D), device="cuda"), torch.randn((T, 1, D), device="cuda")
    cache = empty(3, 1, 16, D)
    slots = torch.arange(T, device="cuda")
    qh = fm.fastmax_cache_append_q8(q, k, v, *cache, slots, None, None, None)
    assert torch.isnan(cache[2].flatten()[[20, 30]]).all()
    assert torch.isfinite(cache[2].flatten()[:T]).sum() == T - 2
    table, lens = torch.arange(3, dtype=torch.int32, device="cuda")[None], torch.tensor([T], dtype=torch.int32, device="cuda")
    start = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    out = fm.fastmax_paged_fwd_q8(qh, *cache, table, lens, q_start=start, max_q=T)
    assert torch.isfinite(out[:20]).all() and torch.isnan(out[20:]).all()
    out = fm.fastmax_paged_fwd_q8(qh, *cache, table, lens, q_start=start, max_q=T, window=5)
    rows = torch.arange(T, device="cuda")
    sees = ((rows >= 20) & (rows < 25)) | ((rows >= 30) & (rows < 35))
    assert torch.isnan(out[sees]).all() and torch.isfinite(out[~sees]).all()


LENS = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 255, 300, 777]


@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv", [(3, 3), (8, 1), (14, 2), (40, 1)])
def test_single_tokens(D, dtype, Hq, Hkv):
    label = f"paged q8 one token D={D} {dtype} H={Hq}/{Hkv}"
    say(label)
    c = Cache(LENS, [1] * len(LENS), Hq, Hkv, D, 16 if D < 64 else 64, dtype, seed=D)
    c.check(c.run(starts=False, max_len=777), label)
    c.check(c.run(starts=False, p=1, scale=1.0 / D), label, p=1, tau=1.0 / D)


@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,lens,news", [(4, 1, [9, 40, 200], [9, 3, 17]), (6, 3, [700], [400]),
                                              (5, 5, [40, 1500], [33, 257]), (12, 12, [513], [513]),
                                              (16, 2, [2100, 70, 3], [130, 70, 1])])
def test_chunks(D, dtype, Hq, Hkv, lens, news):
    label = f"paged q8 chunk D={D} {dtype} H={Hq}/{Hkv} lens={lens}"
    say(label)
    c = Cache(lens, news, Hq, Hkv, D, 32, dtype, seed=Hq + D)
    c.check(c.run(max_q=max(news)), label)
    c.check(c.run(max_q=max(news), p=1, scale=1.0 / D), label, p=1, tau=1.0 / D)


@pytest.mark.parametrize("page", [16, 32, 128, 1024])
@pytest.mark.parametrize("order", ["heads", "tokens"])
@pytest.mark.parametrize("new", [1, 70])
def test_pages_and_orders(page, order, new):
    label = f"paged q8 page={page} {order} new={new}"
    say(label)
    lens = [1, page - 1, page, page + 1, 1500]
    c = Cache(lens, [min(new, n) for n in lens], 4, 2, 64, page, "bf16", seed=page, order=order)
    c.check(c.run(starts=new > 1, max_q=new), label)


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("f32", 32), ("bf16", 128)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (17, 4), (64, 16), (100, 200),
                                          (500, 1), (5000, 3)])
def test_windows(dtype, D, window, sinks):
    label = f"paged q8 window={window} sinks={sinks} D={D} {dtype}"
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
                one.ks[page], one.vs[page] = float("nan"), float("inf")
                one.table[s, i] = -1 if i % 2 else 2 ** 31 - 1
    one.check(one.run(starts=False, window=window, sinks=sinks), label, window=window, sinks=sinks)


@pytest.mark.parametrize("new", [1, 90])
def test_pages_that_are_not_there(new):
    """A row that sees a key whose entry is no page is NaN, the others keep
    their values; so is every row of a sequence longer than its table."""
    import torch
    c = Cache([300, 300, 300], [new] * 3, 4, 2, 64, 32, "bf16", seed=3, cols=10)
    page = 7 if new > 1 else 2                  # chunks: keys 224 .. 255 of 210 .. 299
    c.table[1, page] = c.k.shape[0]
    c.lens[2] = 321
    out = c.run(starts=new > 1, max_q=new)
    pos = 300 - new + np.arange(new)
    bad = np.concatenate([np.zeros(new, bool), pos >= 32 * page, np.ones(new, bool)])
    got = torch.isnan(out).all(-1).all(-1).cpu().numpy()
    assert np.array_equal(got, bad)
    c.check(out, "bad page", keep=~bad)


def test_rows_that_see_nothing_and_rows_of_no_sequence():
    import torch
    c = Cache([5, 0, 40], [9, 2, 30], 4, 1, 32, 16, "f32", seed=8)
    out = torch.full_like(torch.cat([c.q, c.q[:4]]), 7.0)
    c.q = torch.cat([c.q, torch.full_like(c.q[:4], float("nan"))])
    c.run(max_q=30, out=out)
    assert (out[:4] == 0).all() and (out[9:11] == 0).all() and (out[41:] == 7).all()
    assert torch.isfinite(out).all()


def test_query_rows_that_are_not_finite():
    import torch
    for new, starts in ((1, False), (60, True)):
        c = Cache([100, 90], [new, new], 4, 2, 64, 16, "bf16", seed=4)
        c.q[new // 2, 1, 7] = float("nan")
        c.q[new // 2, 2, 9] = float("inf")
        out = c.run(starts=starts, max_q=new)
        odd = torch.zeros(out.shape[:2], dtype=torch.bool, device="cuda")
        odd[new // 2, 1:3] = True
        assert torch.isnan(out[odd]).all() and torch.isfinite(out[~odd]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [1e-25, 1e6, 1e28])
def test_values_of_any_size(dtype, size):
    for new in (1, 70):
        c = Cache([200, 90], [new, 1], 4, 2, 64, 32, dtype, seed=3, size=size)
        c.check(c.run(starts=True, max_q=70 if new > 1 else 1), (dtype, size))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_queries_of_any_size(dtype):
    for size in (1e3, 1e-20):
        for new in (1, 60):
            c = Cache([100, 70], [new, new], 4, 2, 64, 16, dtype, seed=4)
            c.q = (c.q.float() * size).to(c.q.dtype)
            c.check(c.run(max_q=new), (size, new))


def test_offsets_past_32_bits():
    """A cache of more than 2^32 bytes, the pages in use at its end; scales past
    2^25 rows."""
    import torch
    pages, Hkv, page, D = 4200, 8, 1024, 128
    k, v = (torch.zeros((pages, Hkv, page, D), dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros((pages, Hkv, page), device="cuda") for _ in range(2))
    assert k.numel() > 2 ** 32
    small = Cache([1500, 700], [60, 1], 16, Hkv, D, page, "bf16", seed=1)
    used = small.k.shape[0]
    for big, x in zip((k, v, ks, vs), small.cache):
        big[-used:] = x
    table = torch.where(small.table >= 0, small.table + pages - used, small.table)
    out = fm.fastmax_paged_fwd_q8(small.q, k, v, ks, vs, table, small.lens, q_start=small.q_start,
                                  max_q=60)
    small.check(out, "far pages")
    one = fm.fastmax_paged_fwd_q8(small.q[-1:], k, v, ks, vs, table[1:], small.lens[1:].contiguous())
    assert torch.allclose(one, out[-1:], rtol=2.0 ** -7, atol=1e-3)
    slots = torch.tensor([pages * page - 1, (pages - used) * page], device="cuda")
    at = fm.fastmax_cache_read_q8(k, v, ks, vs, slots, dtype=torch.float32)
    for got, codes, scale in zip(at, small.cache[:2], small.cache[2:]):
        want = torch.stack([codes[-1, :, -1].float() * scale[-1, :, -1, None],
                            codes[0, :, 0].float() * scale[0, :, 0, None]])
        assert torch.equal(torch.nan_to_num(got, nan=9.0), torch.nan_to_num(want, nan=9.0))


def test_streams_and_caller_buffers():
    """Another stream, given as an object or a handle; outputs and a workspace of
    the caller's."""
    import torch
    c = Cache([3000, 500], [1, 1], 8, 2, 64, 64, "bf16")
    want = c.run(starts=False)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = []
    for i in range(6):
        got.append(c.run(starts=False, stream=side if i % 2 else side.cuda_stream))
        torch.empty(1 << 20, device="cuda").fill_(float("nan"))
    n = fm.paged_q8_workspace_bytes(2, 2, 8, 2, 64, 1, 3072, 0, 0, fm.BF16)
    out = torch.empty_like(c.q)
    ws = torch.full((n + 16,), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got.append(c.run(starts=False, out=out, workspace=ws, max_len=3072))
    torch.cuda.synchronize()
    for g in got:
        assert torch.equal(g, want)
    rows = fm.fastmax_cache_read_q8(*c.cache, torch.arange(64, device="cuda"), stream=side)
    side.synchronize()
    again = fm.fastmax_cache_read_q8(*c.cache, torch.arange(64, device="cuda"),
                                     out=tuple(torch.empty_like(x) for x in rows))
    for a, b in zip(rows, again):
        assert torch.equal(torch.nan_to_num(a, nan=9.0), torch.nan_to_num(b, nan=9.0))


def test_captured_steps():
    """A captured append and attention, replayed over growing contexts, against
    eager calls between the replays."""
    import torch
    S, Hq, Hkv, D, page = 3, 8, 2, 64, 32
    c = Cache([900, 400, 33], [1] * S, Hq, Hkv, D, page, "bf16", seed=6, cols=40)
    spare = torch.arange(S, device="cuda", dtype=torch.int32) % c.k.shape[0]
    rows = torch.randn((S, Hq + 2 * Hkv, D), device="cuda", dtype=torch.bfloat16)
    cos, sin = (torch.from_numpy(t).cuda() for t in su.table(4096, D))
    lens = c.lens.clone()
    twin = [x.clone() for x in c.cache]

    def step(cache):
        n = lens.long() - 1
        slots = c.table.long().gather(1, (n // page)[:, None])[:, 0] * page + n % page
        q = fm.fastmax_cache_append_q8(*rows.split([Hq, Hkv, Hkv], dim=1), *cache, slots,
                                       n.int(), cos, sin)
        return fm.fastmax_paged_fwd_q8(q, *cache, c.table, lens, max_len=1024)

    for s in range(S):      # a page ahead for each sequence
        used = -(-c.lens_h[s] // page)
        c.table[s, used] = int(spare[s])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(c.cache)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(c.cache)
    step(twin)
    for i in range(4):
        lens += 1
        rows.copy_(torch.randn_like(rows))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, step(twin)), i
        for a, b in zip(c.cache, twin):
            assert torch.equal(torch.nan_to_num(a.float(), nan=9.0), torch.nan_to_num(b.float(), nan=9.0))


@pytest.mark.parametrize("D", [16, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 2), (300, 0)])
def test_what_no_row_sees_may_be_anything(D, dtype, window, sinks):
    """Scales of slots behind the sequences, of any size, and values of a later
    token of the chunk 2^40 times the others': the rows that see neither keep their
    bits."""
    import torch
    label = f"paged q8 unseen slots D={D} {dtype} window={window}"
    say(label)
    kw = {"window": window, "sinks": sinks}
    for news in ([1, 1, 1], [150, 33, 400]):
        c = Cache([203, 40, 777], news, 4, 2, D, 64, dtype, seed=D)
        free = torch.isnan(c.ks)
        want = c.run(max_q=max(news), **kw)
        c.check(want, label, **kw)
        for x in (1e38, float("inf"), -1e30):
            c.ks[free], c.vs[free] = x, -x
            assert torch.equal(c.run(max_q=max(news), **kw), want), (label, x)
        if max(news) == 1:
            continue
        for s, back in ((0, 20), (2, 310)):   # a token that many before the end
            at, (page, place) = c.lens_h[s] - back, c.at(s, c.lens_h[s] - back)
            kept = c.vs[page, :, place].clone()
            c.vs[page, :, place] *= 2.0 ** 40
            got = c.run(max_q=max(news), **kw)
            pos = at - c.lens_h[s] + news[s]      # its row in the chunk
            rows = torch.arange(c.start[-1], device="cuda") - int(c.start[s])
            sees = (rows >= pos) & (rows < news[s])
            if window and pos + c.lens_h[s] - news[s] >= sinks:
                sees &= rows < pos + window
            assert torch.equal(got[~sees], want[~sees]), (label, s, back)
            assert (got[sees].abs().amax((1, 2)) > 2.0 ** 20).all()
            c.vs[page, :, place] = kept
