"""GPU tests of the packed attention, forward and backward, against float64:
lengths, shared heads, both orders, masks, values that are not finite, rows of
any size, strides, streams and graphs."""
import numpy as np
import pytest

from paper_2402_07901_amd import fastmax as fm

import serve_util as su
from gpu_util import say
from packed_util import OUT, Packed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fm.lib()
    yield
    torch.cuda.synchronize()


def forward(x, label, p=2, tau=1.0, causal=True, **kw):
    """The call's O and G, checked; rows of no sequence as they were."""
    import torch
    out = torch.full((x.T, x.Hq, x.D), 7.0, dtype=x.tdt, device="cuda")
    g = torch.full((x.T, x.Hq), 7.0, device="cuda")
    fm.fastmax_packed_fwd(x.q, x.k, x.v, x.starts, p=p, causal=causal, scale=tau, out=out, g=g, **kw)
    for rows, h, hs, head in x.heads(p, tau, causal):
        O, eO, G, eG = head.forward()
        su.check(out[rows, hs], O, OUT[x.dtype] * np.abs(O) + 1.01 * eO, (label, "O", rows, h))
        su.check(g[rows, hs], G, 1.01 * eG, (label, "G", rows, h))
    for rows in (slice(0, x.start[0]), slice(x.start[-1], None)):
        assert (out[rows] == 7).all() and (g[rows] == 7).all(), label
    return out, g


def given(x, p, tau, causal):
    """O and G of the definition in the call's types, for the backward."""
    import torch
    out = torch.zeros((x.T, x.Hq, x.D), dtype=x.tdt, device="cuda")
    g = torch.ones((x.T, x.Hq), device="cuda")
    for rows, _, hs, head in x.heads(p, tau, causal):
        O, _, G, _ = head.forward()
        out[rows, hs] = torch.from_numpy(O).cuda().to(x.tdt)
        g[rows, hs] = torch.from_numpy(G).cuda().float()
    return out, g


def backward(x, label, p=2, tau=1.0, causal=True, **kw):
    import torch
    out, g = given(x, p, tau, causal)
    grads = [torch.full((x.T, h, x.D), 7.0, dtype=x.tdt, device="cuda") for h in (x.Hq, x.Hkv, x.Hkv)]
    fm.fastmax_packed_bwd(x.q, x.k, x.v, x.starts, out, x.dout, g, p=p, causal=causal, scale=tau,
                          grads=grads, **kw)
    do = su.np64(x.dout)
    for rows, h, hs, head in x.heads(p, tau, causal):
        ref = head.backward(do[rows, hs], OUT[x.dtype])
        for name, got, (want, bound) in zip(("dq", "dk", "dv"), (grads[0][rows, hs], grads[1][rows, h], grads[2][rows, h]), ref):
            su.check(got, want, OUT[x.dtype] * (np.abs(want) + bound) + 1.01 * bound, (label, name, rows, h))
    for t in grads:
        assert (t[:x.start[0]] == 7).all() and (t[x.start[-1]:] == 7).all(), label
    return grads


LENS = [1, 2, 0, 31, 32, 33, 63, 0, 64, 65, 127, 128, 129, 257, 0]


@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv", [(3, 3), (8, 2), (7, 1), (40, 1)])
def test_lengths_and_heads(D, dtype, Hq, Hkv):
    label = f"packed D={D} {dtype} H={Hq}/{Hkv}"
    say(label)
    x = Packed(LENS, Hq, Hkv, D, dtype, seed=D + Hq, before=5, after=9)
    forward(x, label)
    forward(x, label, causal=False)
    forward(x, label, p=1, tau=1.0 / D)


@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (6, 2), (7, 1)])
def test_backward(D, dtype, Hq, Hkv):
    label = f"packed backward D={D} {dtype} H={Hq}/{Hkv}"
    say(label)
    x = Packed([2, 0, 31, 33, 64, 1, 129, 257], Hq, Hkv, D, dtype, seed=D + Hq, before=3, after=4)
    backward(x, label)
    backward(x, label, causal=False)
    backward(x, label, p=1, tau=1.0 / D)
    backward(x, label, tau=D ** -0.5)


@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_calls_that_fill_the_gpu(D, dtype):
    """Many heads: workgroups of 128 rows or keys instead of 32."""
    label = f"packed, many heads, D={D} {dtype}"
    say(label)
    x = Packed([33, 0, 128, 300, 1, 129, 400], 64, 32, D, dtype, seed=D, before=2, after=3)
    forward(x, label)
    backward(x, label)
    y = Packed([200, 1, 130, 64], 64, 64, D, dtype, seed=D)
    forward(y, label, causal=False)
    backward(y, label, causal=False)


def test_long_sequences():
    for dtype in ("bf16", "f32"):
        x = Packed([1100, 700], 4, 2, 64, dtype, seed=1)
        forward(x, ("long", dtype))
        backward(x, ("long", dtype))


def test_many_sequences():
    """More sequences than a wave has lanes, many of them empty."""
    rng = np.random.default_rng(5)
    lens = [int(n) for n in rng.integers(0, 4, 5000)]
    x = Packed(lens, 2, 1, 16, "f32", seed=2, after=3)
    out, _ = fm.fastmax_packed_fwd(x.q, x.k, x.v, x.starts, causal=True)
    grads = fm.fastmax_packed_bwd(x.q, x.k, x.v, x.starts, *_step(x, out), causal=True)
    # the same rows, twenty sequences at a time
    for s in range(0, 5000, 977):
        few = x.starts[s:s + 21].contiguous()
        a, b = int(few[0]), int(few[-1])
        again, g = fm.fastmax_packed_fwd(x.q, x.k, x.v, few, causal=True)
        assert (again[a:b] == out[a:b]).all()
        for one, two in zip(fm.fastmax_packed_bwd(x.q, x.k, x.v, few, again, x.dout, g, causal=True), grads):
            assert (one[a:b] == two[a:b]).all()
    forward(Packed(lens[:150], 2, 1, 16, "bf16", seed=2), "many")


def _step(x, out):
    _, g = fm.fastmax_packed_fwd(x.q, x.k, x.v, x.starts, causal=True)
    return out, x.dout, g


def test_gradients_against_differences():
    """The directional derivative of sum(dout * O) from central differences of the
    float64 definition (error about h^2 ~ 1e-8 of its size, and 1e-16 / h)."""
    x = Packed([5, 9, 23], 4, 2, 16, "f32", seed=7)
    out, g = fm.fastmax_packed_fwd(x.q, x.k, x.v, x.starts, causal=True, scale=0.5)
    grads = [su.np64(t) for t in fm.fastmax_packed_bwd(x.q, x.k, x.v, x.starts, out, x.dout, g, causal=True, scale=0.5)]
    leaves, do = [su.np64(t) for t in (x.q, x.k, x.v)], su.np64(x.dout)
    rng = np.random.default_rng(3)

    def loss(q, k, v):
        total = 0.0
        for a, b in zip(x.start, x.start[1:]):
            for h in range(4):
                qh, kh = su.standard(q[a:b, h]), su.standard(k[a:b, h // 2])
                w = np.tril(1 + 0.5 * qh @ kh.T + 0.125 * (qh @ kh.T) ** 2)
                total += (do[a:b, h] * (w @ v[a:b, h // 2] / w.sum(1, keepdims=True))).sum()
        return total

    h = 1e-4
    for i in range(3):
        d = rng.standard_normal(leaves[i].shape)
        hi, lo = ([y + e * d if j == i else y for j, y in enumerate(leaves)] for e in (h, -h))
        slope = (loss(*hi) - loss(*lo)) / (2 * h)
        size = (np.abs(grads[i]) * np.abs(d)).sum()
        assert abs((grads[i] * d).sum() - slope) <= 1e-5 * size, (i, slope, size)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [16, 64, 128])
def test_values_that_are_not_finite(dtype, D):
    """Infinities and NaN in v: not finite in their channel for the rows of their
    sequence that see them, in no other; the other sequences as without them."""
    import torch
    for causal in (True, False):
        x = Packed([40, 150, 70], 4, 2, D, dtype, seed=4)
        want, _ = fm.fastmax_packed_fwd(x.q, x.k, x.v, x.starts, causal=causal)
        x.v[40 + 100, 0, 3] = float("inf")
        x.v[40 + 110, 1, 5] = float("nan")
        x.v[40 + 149, 1, 6] = float("-inf")
        out, _ = fm.fastmax_packed_fwd(x.q, x.k, x.v, x.starts, causal=causal)
        odd = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
        for token, heads, ch in ((100, slice(0, 2), 3), (110, slice(2, 4), 5), (149, slice(2, 4), 6)):
            odd[40 + (token if causal else 0):190, heads, ch] = True
        assert torch.equal(~torch.isfinite(out), odd)
        assert torch.equal(out[:40], want[:40]) and torch.equal(out[190:], want[190:])
        same = (~odd).clone()
        assert torch.allclose(out[same].float(), want[same].float(), rtol=2.0 ** -7, atol=1e-3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", ["q", "k", "v", "dout"])
def test_gradients_of_rows_that_are_not_finite(dtype, what):
    """A token whose row is constant (q, k) or has an infinity (v, dout): the
    gradient rows that depend on it are not finite, the others are, and other
    sequences' are as without it."""
    import torch
    x = Packed([50, 140, 33], 4, 2, 64, dtype, seed=9)
    out, g = fm.fastmax_packed_fwd(x.q, x.k, x.v, x.starts, causal=True)
    want = fm.fastmax_packed_bwd(x.q, x.k, x.v, x.starts, out, x.dout, g, causal=True)
    at = 50 + 75
    row = {"q": x.q, "k": x.k, "v": x.v, "dout": x.dout}[what]
    if what in "qk":
        row[at, 0] = 2.0
    else:
        row[at, 0, 9] = float("inf")
    out, g = fm.fastmax_packed_fwd(x.q, x.k, x.v, x.starts, causal=True)
    dq, dk, dv = fm.fastmax_packed_bwd(x.q, x.k, x.v, x.starts, out, x.dout, g, causal=True)
    for got, old in zip((dq, dk, dv), want):
        assert torch.equal(got[:50], old[:50]) and torch.equal(got[190:], old[190:])
    fine_q, fine_k = torch.ones_like(dq[..., 0], dtype=torch.bool), torch.ones_like(dk[..., 0], dtype=torch.bool)
    if what in ("q", "dout"):
        fine_q[at, 0] = False          # its own row
        fine_k[50:at + 1, 0] = False   # the keys that it sees
    else:
        fine_q[at:190, :2] = False     # the rows that see it
        fine_k[50:190, 0] = False      # the keys that these see
    assert torch.isfinite(dq[fine_q]).all() and torch.isfinite(dk[fine_k]).all()
    assert not torch.isfinite(dq[~fine_q]).all(-1).any()
    assert not torch.isfinite(dk[~fine_k]).all(-1).any()
    assert torch.isfinite(dv[:, 1]).all()
    if what == "dout":
        ch = torch.arange(64, device="cuda") != 9
        assert not torch.isfinite(dv[50:at + 1, 0, 9]).any() and torch.isfinite(dv[at + 1:190, 0]).all()
        assert torch.isfinite(dv[50:190, 0][:, ch]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [1e-30, 1e-6, 1e6, 1e25])
def test_values_of_any_size(dtype, size):
    x = Packed([140, 70], 4, 2, 64, dtype, seed=3, size=size)
    forward(x, ("size", size, dtype))
    if 1e-20 < size < 1e20:
        backward(x, ("size", size, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_beside_much_larger_ones(dtype):
    """Tokens whose values are 2^12 times the others': the sums keep bf16's
    accuracy (per channel: the large rows stand in every third)."""
    import torch
    for order in (1, -1):
        x = Packed([200, 90], 4, 2, 64, dtype, seed=3)
        grow = torch.ones((x.T, 1, 64), device="cuda")
        grow[100::7, :, ::3] = 2.0 ** 12
        x.v.copy_((x.v.float() * (grow if order > 0 else grow.flip(0))).to(x.tdt))
        forward(x, ("large", dtype))
        y = Packed([200, 90], 4, 2, 64, dtype, seed=3)
        y.dout.copy_((y.dout.float() * (grow if order > 0 else grow.flip(0))).to(y.tdt))
        backward(y, ("large", dtype))


def test_zero_values_first():
    """A prefix of zero values (no power of two of its own), then values of any
    size; all of them zero."""
    for size in (1e-10, 1e10):
        x = Packed([200], 2, 1, 64, "bf16", seed=3, size=size)
        x.v[:130] = 0
        forward(x, ("zeros", size))
        backward(x, ("zeros", size))
    x.v.zero_()
    x.dout.zero_()
    out, g = fm.fastmax_packed_fwd(x.q, x.k, x.v, x.starts, causal=True)
    assert (out == 0).all()
    for t in fm.fastmax_packed_bwd(x.q, x.k, x.v, x.starts, out, x.dout, g, causal=True):
        assert (t == 0).all()


def test_starts_outside_the_rows():
    """Starts below 0 and past T count as the bounds."""
    import torch
    x = Packed([40, 60], 2, 1, 32, "f32")
    want, _ = fm.fastmax_packed_fwd(x.q, x.k, x.v, x.starts, causal=True)
    starts = torch.tensor([-2 ** 31, -7, 40, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    got, _ = fm.fastmax_packed_fwd(x.q, x.k, x.v, starts, causal=True)
    assert torch.equal(got, want)


def test_agrees_with_equal_lengths():
    """Sequences of one length: fastmax_fwd and fastmax_bwd on [B, H, N, D]."""
    import torch
    B, N, H, D = 3, 150, 4, 64
    x = Packed([N] * B, H, H, D, "f32", seed=5)
    out, g = fm.fastmax_packed_fwd(x.q, x.k, x.v, x.starts, causal=True)
    got = fm.fastmax_packed_bwd(x.q, x.k, x.v, x.starts, out, x.dout, g, causal=True)
    q, k, v, do = (t.unflatten(0, (B, N)).transpose(1, 2).contiguous() for t in (x.q, x.k, x.v, x.dout))
    o2, g2 = fm.fastmax_fwd(q, k, v, p=2, causal=True)
    want = fm.fastmax_bwd(q, k, v, o2, do, g2, p=2, causal=True)
    for a, b in zip((out, *got), (o2, *want)):
        b = b.transpose(1, 2).flatten(0, 1)
        assert (a - b).abs().max() <= 1e-4 * b.abs().max()
    assert torch.allclose(g, g2.transpose(1, 2).flatten(0, 1), rtol=1e-4)


def test_strides_streams_and_buffers():
    """Heads before tokens, gradients into one buffer, another stream, the
    caller's workspace; equal calls give equal bits."""
    import torch
    x = Packed([100, 45], 6, 2, 64, "bf16", seed=6)
    out, g = fm.fastmax_packed_fwd(x.q, x.k, x.v, x.starts, causal=True)
    want = fm.fastmax_packed_bwd(x.q, x.k, x.v, x.starts, out, x.dout, g, causal=True)
    q, k, v = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in (x.q, x.k, x.v))
    both = torch.empty_like(x.rows)
    n = [fm.packed_workspace_bytes(2, x.T, 6, 2, 64, fm.BF16, b) for b in (False, True)]
    ws = [torch.full((m,), 255, dtype=torch.uint8, device="cuda") for m in n]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o2, g2 = fm.fastmax_packed_fwd(q, k, v, x.starts, causal=True, stream=side, workspace=ws[0])
    got = fm.fastmax_packed_bwd(q, k, v, x.starts, o2, x.dout, g2, causal=True, stream=side,
                                workspace=ws[1], grads=both.split([6, 2, 2], dim=1))
    o3, _ = fm.fastmax_packed_fwd(q, k, v, x.starts, causal=True, want_g=False, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(o2, out) and torch.equal(g2, g) and torch.equal(o3, out)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    with pytest.raises(fm.FastmaxError):
        fm.fastmax_packed_bwd(x.q, x.k, x.v, x.starts, out, x.dout, g, workspace=ws[1][:-256])


def test_captured_step():
    """A captured forward and backward, replayed over other rows and other starts,
    against eager calls between the replays."""
    import torch
    x = Packed([100, 45, 300], 6, 2, 64, "bf16", seed=6)

    def step():
        out, g = fm.fastmax_packed_fwd(x.q, x.k, x.v, x.starts, causal=True)
        return (out, *fm.fastmax_packed_bwd(x.q, x.k, x.v, x.starts, out, x.dout, g, causal=True))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for cut in (100, 7, 210, 100):
        x.rows.copy_(torch.randn_like(x.rows))
        x.starts[1] = cut
        x.starts[2] = cut + 140
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, step()):
            assert torch.equal(a, b), cut


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompts_then_tokens(dtype):
    """Uneven prompts attended packed; their rows appended to the 8-bit cache, then
    single tokens over it against the packed attention of the longer sequences:
    apart by what 8 bits lose, and over the cache in full by rounding alone."""
    import torch
    Hq, Hkv, D, page, new = 6, 2, 64, 32, 3
    tdt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    lens = [70, 1, 200]
    x = Packed([n + new for n in lens], Hq, Hkv, D, dtype, seed=11)
    want, _ = fm.fastmax_packed_fwd(x.q, x.k, x.v, x.starts, causal=True)
    cols = 8
    table = torch.randperm(3 * cols, device="cuda").to(torch.int32).reshape(3, cols)
    codes = torch.zeros((2, 3 * cols, Hkv, page, D), dtype=torch.int8, device="cuda")
    scales = torch.zeros((2, 3 * cols, Hkv, page), device="cuda")
    plain = torch.zeros((2, 3 * cols, Hkv, page, D), dtype=tdt, device="cuda")
    tokens = [torch.arange(int(x.start[s]), int(x.start[s]) + n, device="cuda") for s, n in enumerate(lens)]

    def slots(s, n):
        return table[s].long()[n // page] * page + n % page

    first = torch.cat(tokens)
    at = torch.cat([slots(s, torch.arange(n, device="cuda")) for s, n in enumerate(lens)])
    rows = [t[first] for t in (x.q, x.k, x.v)]
    fm.fastmax_cache_append_q8(*rows, *codes, *scales, at, None, None, None)
    fm.fastmax_cache_append(*rows, *plain, at, None, None, None)
    for i in range(new):
        now = torch.tensor([int(x.start[s]) + n + i for s, n in enumerate(lens)], device="cuda")
        at = torch.stack([slots(s, torch.tensor(n + i, device="cuda")) for s, n in enumerate(lens)])
        rows = [t[now] for t in (x.q, x.k, x.v)]
        ahead = torch.tensor([n + i + 1 for n in lens], dtype=torch.int32, device="cuda")
        q8 = fm.fastmax_cache_append_q8(*rows, *codes, *scales, at, None, None, None)
        q = fm.fastmax_cache_append(*rows, *plain, at, None, None, None)
        assert torch.equal(q8, q)
        full = fm.fastmax_paged_fwd(q, *plain, table, ahead)
        small = fm.fastmax_paged_fwd_q8(q8, *codes, *scales, table, ahead)
        ref = want[now].float()
        tol = {"f32": 1e-4, "bf16": 2e-2}[dtype]      # the library's
        assert (full.float() - ref).abs().max() <= tol * ref.abs().max()
        # a code is off by at most 1/254 of its row's largest, about 3 of a
        # standard normal row's deviations: 7e-3 a channel of k^ and v at rms, so
        # about 7e-3 sqrt(2 D) = 8e-2 of |s| ~ sqrt(D) = 8 in each score and 2e-2 of
        # each weight, averaged over the keys; held to four times that
        assert (small.float() - ref).norm() <= 8e-2 * ref.norm()


@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("heads", [(4, 2), (120, 120)])   # 32 columns to a workgroup, 128
@pytest.mark.parametrize("p", [1, 2])
def test_rows_that_do_not_see_much_larger_ones(D, heads, p):
    """A token's values 2^90 times the others' leave O and dq of the rows before it
    as they are, held to the bounds of the sequence without it; one's dO 2^36 times
    the others' leaves dk and dv of the keys after it."""
    label = f"packed, unseen rows, D={D} p={p} H={heads}"
    say(label)
    tau = 1.0 if p == 2 else 1.0 / D
    n, at = 400, (70, 333)
    for a in at:
        x = Packed([n], *heads, D, "bf16", seed=a)
        x.v[a] *= 2.0 ** 90
        out, g = fm.fastmax_packed_fwd(x.q, x.k, x.v, x.starts, p=p, causal=True, scale=tau)
        dq = fm.fastmax_packed_bwd(x.q, x.k, x.v, x.starts, out, x.dout, g, p=p, causal=True, scale=tau)[0]
        short = Packed([n], *heads, D, "bf16", seed=a)
        short.lens, short.start = [a], np.array([0, a])
        do = su.np64(x.dout)
        for rows, h, hs, head in short.heads(p, tau, True):
            if h > 1:
                break
            O, eO, G, eG = head.forward()
            su.check(out[rows, hs], O, OUT["bf16"] * np.abs(O) + 1.01 * eO, (label, a, "O", h))
            want, bound = head.backward(do[rows, hs], 2 * OUT["bf16"] + eO.max() / np.abs(O).max())[0]
            su.check(dq[rows, hs], want, OUT["bf16"] * (np.abs(want) + bound) + 1.01 * bound, (label, a, "dq", h))

        y = Packed([n], *heads, D, "bf16", seed=a)
        y.dout[a] *= 2.0 ** 36
        out, g = given(y, p, tau, True)
        _, dk, dv = fm.fastmax_packed_bwd(y.q, y.k, y.v, y.starts, out, y.dout, g, p=p, causal=True, scale=tau)
        do = su.np64(y.dout)
        do[:a + 1] = 0
        for rows, h, hs, head in y.heads(p, tau, True):
            if h > 1:
                break
            for name, got, (want, bound) in zip(("dk", "dv"), (dk, dv), head.backward(do[rows, hs], OUT["bf16"])[1:]):
                want, bound = want[a + 1:], bound[a + 1:]
                su.check(got[a + 1:, h], want, OUT["bf16"] * (np.abs(want) + bound) + 1.01 * bound, (label, a, name, h))
