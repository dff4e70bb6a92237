"""GPU tests of the rows around the attention: rotation, norm and head sharing
forward and backward, and the cache append, against float64."""
import numpy as np
import pytest

from paper_2402_07901_amd import fastmax as fm

import serve_util as su
from gpu_util import say

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fm.lib()
    yield
    torch.cuda.synchronize()


def dt(dtype):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]


class Rows:
    """A projection's output with its views, positions, tables and weights."""

    def __init__(self, B, N, Hq, Hkv, D, dtype, rot=None, axes=1, interleaved=False, norm=True,
                 seed=0, table_rows=None):
        import torch
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        rot = D if rot is None else rot
        self.B, self.N, self.Hq, self.Hkv, self.D, self.dtype = B, N, Hq, Hkv, D, dtype
        self.group, self.rot, self.interleaved = Hq // Hkv, rot, interleaved
        self.rows = torch.randn((B, N, Hq + 2 * Hkv, D), generator=gen, device="cuda").to(dt(dtype))
        self.q, self.k, self.v = self.rows.split([Hq, Hkv, Hkv], dim=2)
        half = rot // 2
        self.sections = None
        if axes > 1:
            side = half // axes - (1 if half >= 8 else 0)     # not a multiple of the lane's 8
            self.sections = [side] * (axes - 1) + [half - side * (axes - 1)]
        rows = table_rows or 500
        self.cos_np, self.sin_np = su.table(rows, rot)
        if rot:
            self.cos = torch.from_numpy(self.cos_np).cuda()
            self.sin = torch.from_numpy(self.sin_np).cuda()
            self.pos = torch.randint(0, rows, (B, N, axes), generator=gen, device="cuda",
                                     dtype=torch.int32)
        else:
            self.cos = self.sin = self.pos = None
        self.wq = self.wk = None
        if norm:
            self.wq, self.wk = (1.0 + 0.3 * torch.randn(D, generator=gen, device="cuda")
                                for _ in range(2))

    def kw(self):
        return dict(pos=self.pos, cos=self.cos, sin=self.sin, wq=self.wq, wk=self.wk, eps=EPS,
                    sections=self.sections, interleaved=self.interleaved)

    def turned(self, x, w):
        """(normed and rotated, its error in units of U) in float64."""
        y = su.norm(su.np64(x), None if w is None else su.np64(w), EPS)
        if not self.rot:
            return y, 30 * np.abs(y)
        z = su.turn(y, self.pos.cpu().numpy(), self.cos_np, self.sin_np, self.sections,
                    self.interleaved)
        # norm: a sum of D squares in runs of 16 and three adds, a root, a
        # quotient, two products (30 roundings at most); rotation: two products
        # and a sum
        return z, 34 * su.turn_bound(y, self.rot, self.interleaved)


SHAPES = [
    # B, N, Hq, Hkv, D, dtype, rot, axes, interleaved, norm
    (1, 1, 1, 1, 16, "bf16", None, 1, False, True),
    (2, 37, 4, 4, 32, "f32", None, 1, False, False),
    (3, 65, 6, 2, 64, "bf16", None, 1, False, True),
    (1, 130, 8, 1, 128, "bf16", None, 3, False, True),
    (1, 33, 9, 3, 128, "f32", 64, 2, True, True),
    (2, 19, 5, 5, 64, "bf16", 16, 1, True, False),
    (1, 40, 3, 1, 64, "f32", 48, 4, False, True),
    (2, 21, 17, 1, 16, "f32", None, 3, True, True),
    (1, 300, 2, 2, 32, "bf16", 0, 1, False, True),
]


@pytest.mark.parametrize("B,N,Hq,Hkv,D,dtype,rot,axes,interleaved,norm", SHAPES)
def test_rope_forward(B, N, Hq, Hkv, D, dtype, rot, axes, interleaved, norm):
    label = f"rope fwd B={B} N={N} H={Hq}/{Hkv} D={D} {dtype} rot={rot} axes={axes}"
    say(label)
    r = Rows(B, N, Hq, Hkv, D, dtype, rot, axes, interleaved, norm, seed=N)
    oq, ok, ov = fm.fastmax_rope_fwd(r.q, r.k, r.v, **r.kw())
    for name, got, x, w, group in (("q", oq, r.q, r.wq, 1), ("k", ok, r.k, r.wk, r.group)):
        ref, err = r.turned(x, w)
        ref, err = su.heads(ref, group), su.heads(err, group)
        su.check(got, ref, su.OUT[dtype] * np.abs(ref) + su.U * err * 1.01, (label, name))
    assert np.array_equal(su.np64(ov), su.heads(su.np64(r.v), r.group)), (label, "v")


@pytest.mark.parametrize("B,N,Hq,Hkv,D,dtype,rot,axes,interleaved,norm", SHAPES)
def test_rope_backward(B, N, Hq, Hkv, D, dtype, rot, axes, interleaved, norm):
    import torch
    label = f"rope bwd B={B} N={N} H={Hq}/{Hkv} D={D} {dtype} rot={rot} axes={axes}"
    say(label)
    r = Rows(B, N, Hq, Hkv, D, dtype, rot, axes, interleaved, norm, seed=N)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    gq, gk, gv = (torch.randn((B, Hq, N, D), generator=gen, device="cuda").to(dt(dtype))
                  for _ in range(3))
    # packed gradient rows, as the projection's backward wants them
    rows = torch.empty_like(r.rows)
    out = rows.split([Hq, Hkv, Hkv], dim=2)
    *grads, dwq, dwk = fm.fastmax_rope_bwd(r.q, r.k, gq, gk, gv, out=out, **r.kw())
    again = fm.fastmax_rope_bwd(r.q, r.k, gq, gk, gv, **r.kw())
    for a, b in zip(again, (*grads, dwq, dwk)):
        assert (a is None and b is None) or torch.equal(a, b), (label, "not repeatable")
    for name, got, g, x, w, dw, group in (("q", grads[0], gq, r.q, r.wq, dwq, 1),
                                          ("k", grads[1], gk, r.k, r.wk, dwk, r.group)):
        g = su.np64(g).transpose(0, 2, 1, 3)
        g = g.reshape(B, N, -1, group, D)
        mag, dy = np.abs(g).sum(3), g.sum(3)
        # float32 sums over the group, then the rotation's three roundings
        err = group * mag
        if r.rot:
            pos = r.pos.cpu().numpy()
            dy = su.turn(dy, pos, r.cos_np, r.sin_np, r.sections, interleaved, back=True)
            err = su.turn_bound(err + 3 * mag, r.rot, interleaved)
            mag = su.turn_bound(mag, r.rot, interleaved)
        if w is None:
            su.check(got, dy, su.OUT[dtype] * np.abs(dy) + 1.01 * su.U * err, (label, name))
            continue
        x64, w64 = su.np64(x), su.np64(w)
        dx, ref, terms = su.norm_bwd(x64, w64, EPS, dy)
        rr = 1.0 / np.sqrt((x64 * x64).mean(-1, keepdims=True) + EPS)
        # dx = r (w dy - xr mean(w dy xr)): dy's error and 40 roundings (the
        # norm's 30, two products, the difference, the mean's sums) through
        # either term, taken by magnitude
        wm, xr = np.abs(w64) * (err + 40 * mag), np.abs(x64 * rr)
        bound = rr * (wm + xr * (wm * xr).mean(-1, keepdims=True))
        su.check(got, dx, su.OUT[dtype] * np.abs(dx) + 1.01 * su.U * bound, (label, name))
        ax = (0, 1, 2)
        # terms: dy's error and 35 roundings; sums: at most 8 heads in a run,
        # 6 folds of the wave, 4 waves; partial rows add up in float64
        su.check(dw, ref, su.U * (1.01 * ((err + 55 * mag) * xr).sum(ax) + np.abs(ref) + terms),
                 (label, "dw" + name))
    ref = su.np64(gv).transpose(0, 2, 1, 3).reshape(B, N, Hkv, r.group, D)
    su.check(grads[2], ref.sum(3),
             su.OUT[dtype] * np.abs(ref.sum(3)) + r.group * su.U * np.abs(ref).sum(3) * 1.01,
             (label, "v"))


@pytest.mark.parametrize("D,Hq,Hkv,axes,interleaved", [(32, 4, 2, 1, False), (64, 3, 1, 3, True)])
def test_rope_backward_against_differences(D, Hq, Hkv, axes, interleaved):
    """The directional derivative of sum(outputs * upstream) from central
    differences of the float64 definition (error h^2 ~ 1e-8 of its size, and
    1e-16 / h) against the kernel's float32 gradients."""
    import torch
    r = Rows(2, 11, Hq, Hkv, D, "f32", None, axes, interleaved, True, seed=5)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(8)
    ups = [torch.randn((2, Hq, 11, D), generator=gen, device="cuda") for _ in range(3)]
    grads = [su.np64(g) for g in fm.fastmax_rope_bwd(r.q, r.k, *ups, **r.kw())]
    pos, rng = r.pos.cpu().numpy(), np.random.default_rng(3)
    leaves = [su.np64(t) for t in (r.q, r.k, r.v, r.wq, r.wk)]

    def loss(q, k, v, wq, wk):
        out = [su.turn(su.norm(x, w, EPS), pos, r.cos_np, r.sin_np, r.sections, interleaved)
               for x, w in ((q, wq), (k, wk))] + [v]
        return sum((su.heads(o, 1 if i == 0 else r.group) * su.np64(u)).sum()
                   for i, (o, u) in enumerate(zip(out, ups)))

    h = 1e-4
    for i in range(5):
        d = rng.standard_normal(leaves[i].shape)
        hi = [x + h * d if j == i else x for j, x in enumerate(leaves)]
        lo = [x - h * d if j == i else x for j, x in enumerate(leaves)]
        slope = (loss(*hi) - loss(*lo)) / (2 * h)
        got = (grads[i] * d).sum()
        size = (np.abs(grads[i]) * np.abs(d)).sum()
        assert abs(got - slope) <= 1e-5 * size, (i, got, slope, size)


def test_position_outside_the_table_is_nan():
    import torch
    r = Rows(1, 6, 2, 1, 32, "bf16", 16, 1, False, False, table_rows=50)
    r.pos[0, :, 0] = torch.tensor([0, 49, 50, -1, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    oq, ok, _ = fm.fastmax_rope_fwd(r.q, r.k, r.v, **r.kw())
    for got, x, group in ((oq, r.q, 1), (ok, r.k, 2)):
        got = su.np64(got)
        assert np.isfinite(got[:, :, :2]).all()
        assert np.isnan(got[:, :, 2:, :16]).all()
        # the channels that do not turn are as they were
        assert np.array_equal(got[..., 16:], su.heads(su.np64(x), group)[..., 16:])


def test_rope_other_strides_and_stream():
    """Heads before tokens, a token's rows apart from the next's; another
    stream than the inputs'."""
    import torch
    r = Rows(2, 29, 4, 2, 64, "bf16")
    want = fm.fastmax_rope_fwd(r.q, r.k, r.v, **r.kw())
    q = r.q.transpose(1, 2).contiguous().transpose(1, 2)
    wide = torch.full((2, 29, 2, 2, 96), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[..., 8:72] = torch.stack([r.k, r.v], 2)
    k, v = wide[:, :, 0, :, 8:72], wide[:, :, 1, :, 8:72]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = fm.fastmax_rope_fwd(q, k, v, stream=side, **r.kw())
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


CASES = [
    # T, Hq, Hkv, D, dtype, page, rot, axes, interleaved, norm
    (1, 12, 12, 64, "bf16", 64, None, 1, False, True),
    (5, 1, 1, 16, "f32", 16, None, 1, True, True),
    (77, 8, 2, 128, "bf16", 16, None, 1, False, False),
    (130, 6, 3, 32, "f32", 256, 16, 1, False, True),
    (33, 4, 4, 128, "f32", 1024, None, 3, False, True),
    (64, 7, 1, 16, "bf16", 32, 0, 1, False, False),
]


@pytest.mark.parametrize("T,Hq,Hkv,D,dtype,page,rot,axes,interleaved,norm", CASES)
@pytest.mark.parametrize("order", ["heads", "tokens"])
def test_append(T, Hq, Hkv, D, dtype, page, rot, axes, interleaved, norm, order):
    import torch
    label = f"append T={T} H={Hq}/{Hkv} D={D} {dtype} page={page} {order}"
    say(label)
    r = Rows(1, T, Hq, Hkv, D, dtype, rot, axes, interleaved, norm, seed=T)
    kw = r.kw()
    kw["pos"] = None if r.pos is None else r.pos[0]
    pages = -(-T // page) + 2
    both = torch.randn((2, pages, Hkv, page, D) if order == "heads" else (2, pages, page, Hkv, D),
                       device="cuda").to(dt(dtype))
    caches = [c if order == "heads" else c.transpose(1, 2) for c in both]
    before = [su.np64(c) for c in caches]
    slots = torch.randperm(pages * page, device="cuda")[:T]
    if T > 4:      # padding, and slots that no page has
        slots[1], slots[2], slots[3] = -1, pages * page, 2 ** 62
    q_out = fm.fastmax_cache_append(r.q[0], r.k[0], r.v[0], caches[0], caches[1], slots, **kw)

    def standard(x, w):
        z, err = r.turned(x, w)
        sd = z.std(-1, keepdims=True)
        # the rotated row's error, 40 roundings of its largest channel in mean
        # and deviation, over std; the row's scale: 20 more of the result
        bound = (err.max(-1, keepdims=True) * 2 + 40 * np.abs(z).max(-1, keepdims=True)) / sd
        ref = su.standard(z)
        return ref, bound * (1.0 + np.abs(ref)) + 20 * np.abs(ref)

    ref, err = standard(r.q, r.wq)
    su.check(q_out, ref[0], su.OUT[dtype] * np.abs(ref[0]) + 1.01 * su.U * err[0], (label, "q"))
    ref, err = standard(r.k, r.wk)
    slots = slots.cpu().numpy()
    kb, v64 = su.OUT[dtype] * np.abs(ref[0]) + 1.01 * su.U * err[0], su.np64(r.v)[0]
    want, bound = [b.copy() for b in before], [np.zeros_like(b) for b in before]
    for t in range(T):
        if 0 <= slots[t] < pages * page:
            at = (slots[t] // page, slice(None), slots[t] % page)
            want[0][at], want[1][at] = ref[0, t], v64[t]
            bound[0][at] = kb[t]
    su.check(caches[0], want[0], bound[0], (label, "k"))
    su.check(caches[1], want[1], bound[1], (label, "v"))
