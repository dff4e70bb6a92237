"""Plain float64 forms of the operators around the attention, written from
their definitions with numpy, and the rounding bounds their tests use.

Bounds are elementwise, first order, from the number of roundings: U = 2^-24
is float32's half-ulp relative error; a value rounded once to bf16 (8
significant bits) is off by at most 2^-8 of its magnitude (at the foot of a
binade, 2^-9 elsewhere).
"""
import numpy as np

U = 2.0 ** -24
OUT = {"bf16": 2.0 ** -8, "f32": 2.0 ** -23}


def np64(t):
    return t.detach().double().cpu().numpy()


def table(rows, rot, base=10000.0):
    """float32 cos and sin [rows, rot / 2]."""
    inv = base ** (-np.arange(0, rot, 2) / max(rot, 1))
    a = np.arange(rows)[:, None] * inv[None]
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def axis_of(sections, half):
    return np.repeat(np.arange(len(sections)), sections) if sections else np.zeros(half, int)


def pairs(rot, interleaved):
    j = np.arange(rot // 2)
    return (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)


def norm(x, w, eps):
    if w is None:
        return x
    return w * x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)


def turn(x, pos, cos, sin, sections, interleaved, back=False):
    """x [..., H, D], pos [..., axes]."""
    rot = 2 * cos.shape[1]
    a, b = pairs(rot, interleaved)
    at = pos[..., axis_of(sections, rot // 2)]
    j = np.arange(rot // 2)
    c, s = cos.astype(np.float64)[at, j][..., None, :], sin.astype(np.float64)[at, j][..., None, :]
    s = -s if back else s
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def turn_bound(y, rot, interleaved):
    """|a| + |b| of each channel's pair (an unrotated channel: itself)."""
    a, b = pairs(rot, interleaved)
    m = np.abs(y)
    both = m[..., a] + m[..., b]
    m = m.copy()
    m[..., a] = both
    m[..., b] = both
    return m


def standard(z):
    z = z - z.mean(-1, keepdims=True)
    return z / np.sqrt((z * z).mean(-1, keepdims=True))


def heads(x, group):
    """[B, N, H, D] -> [B, H * group, N, D]."""
    return np.repeat(x, group, axis=2).transpose(0, 2, 1, 3)


def norm_bwd(x, w, eps, dy):
    """(dx, dw, sum |terms of dw|) of y = w x r."""
    D = x.shape[-1]
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    ax = tuple(range(x.ndim - 1))
    terms = dy * x * r
    inner = (x * w * dy).sum(-1, keepdims=True) / D
    return r * (w * dy - x * r * r * inner), terms.sum(ax), np.abs(terms).sum(ax)


def attend(q, k, v, pos, p, tau, window, sinks, parts=2):
    """One sequence and key head: q [t, g, D] at positions pos [t], k and v
    [n, D].  Returns (O, bound): the bound covers the float32 products and
    sums (D + 8 roundings of a score against its sum of magnitudes, n + 64 of
    a sum) and the weights in bf16 parts (2^-8 in one, 2^-16 in two; None:
    float32)."""
    t, g, D = q.shape
    n = np.arange(len(k))
    see = n[None] <= pos[:, None]
    if window:
        see &= (n[None] > pos[:, None] - window) | (n[None] < sinks)
    see = see[:, None, :]
    kz = np.where(np.isfinite(k), k, 0.0)
    s = tau * np.einsum("tgd,nd->tgn", q, kz)
    mag = tau * np.einsum("tgd,nd->tgn", np.abs(q), np.abs(kz))
    w = 1.0 + s + (0.5 * s * s if p == 2 else 0.0)
    part = {None: 0.0, 1: 2.0 ** -8, 2: 2.0 ** -16}[parts]
    e = (D + 8) * U * mag * (1.0 + (np.abs(s) if p == 2 else 0.0))
    e = e + ((len(n) + 64) * U + part) * (1.0 + np.abs(s) + 0.5 * s * s)
    w, e = np.where(see, w, 0.0), np.where(see, e, 0.0)
    G = w.sum(-1, keepdims=True)
    some = see.any(-1, keepdims=True) & np.ones_like(G, bool)
    G = np.where(some, G, 1.0)
    vz = np.where(np.isfinite(v), v, 0.0)
    O = np.einsum("tgn,nd->tgd", w, vz) / G
    bound = np.einsum("tgn,nd->tgd", e, np.abs(vz)) / np.abs(G)
    bound = bound + e.sum(-1, keepdims=True) / np.abs(G) * np.abs(O)
    return np.where(some, O, 0.0), np.where(some, bound, 0.0)


def check(got, ref, bound, label):
    """Elementwise |got - ref| <= bound, NaN nowhere."""
    got = np64(got)
    assert got.shape == ref.shape, (label, got.shape, ref.shape)
    assert np.isfinite(got).all(), (label, "not finite")
    if not got.size:
        return
    over = np.abs(got - ref) - bound
    worst = np.unravel_index(np.argmax(over), over.shape)
    assert over[worst] <= 0, (label, worst, got[worst], ref[worst], bound[worst])
