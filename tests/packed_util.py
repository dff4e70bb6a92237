"""Plain float64 forms of the packed attention, forward and backward, with
elementwise first-order bounds from the count of roundings: U = 2^-24 float32,
H = 2^-11 for the fp16 operands of bf16 calls (q^, k^, weights, T; subnormal
steps of 2^-25 of a wave's largest power besides), none for float32 calls."""
import numpy as np

from serve_util import OUT, U, np64

H = {"bf16": 2.0 ** -11, "f32": 0.0}
SUB = {"bf16": 2.0 ** -25, "f32": 0.0}


def standard(x):
    """x^ and 1 / std."""
    c = x - x.mean(-1, keepdims=True)
    r = 1.0 / np.sqrt((c * c).mean(-1, keepdims=True))
    return c * r, r


def power(x):
    """Powers of two of rows, at least as large as their largest magnitude."""
    top = np.abs(x).max(-1, keepdims=True)
    return 2.0 ** np.ceil(np.log2(np.where(top > 0, top, 1.0)) + 1e-12) * 2.0


class Head:
    """One sequence and key head: q, do [n, g, D], k, v [n, D]."""

    def __init__(self, q, k, v, p, tau, causal, dtype):
        n, g, D = q.shape
        self.n, self.g, self.D, self.p, self.tau, self.dtype = n, g, D, p, tau, dtype
        self.q, self.rq = standard(q)
        self.k, self.rk = standard(k)
        self.v = v
        self.see = (np.tril(np.ones((n, n), bool)) if causal else np.ones((n, n), bool))[:, None]
        s = tau * np.einsum("igd,nd->ign", self.q, self.k)
        # a score: float32 sums and rows (32 roundings of a standardised row), two
        # fp16 operands
        mag = tau * np.einsum("igd,nd->ign", np.abs(self.q), np.abs(self.k))
        self.es = ((D + 72) * U + 2 * H[dtype]) * mag + 40 * U * tau * D
        self.t = np.ones_like(s) if p == 1 else 1.0 + s
        self.et = (0.0 if p == 1 else 1.0) * (self.es + 2 * U * (1 + np.abs(s)))
        w = 1.0 + s if p == 1 else 0.5 * (1.0 + s) ** 2 + 0.5
        size = 1.0 + np.abs(s) + (0.0 if p == 1 else 0.5 * s * s)
        ew = (1.0 if p == 1 else 1.0 + np.abs(s) + self.es) * self.es + 6 * U * size
        self.w, self.ew = np.where(self.see, w, 0.0), np.where(self.see, ew, 0.0)
        self.G = self.w.sum(-1, keepdims=True)
        # (bf16 calls sum the weights that the products take, rounded to fp16)
        self.eG = (self.ew + ((n + 64) * U + H[dtype]) * np.abs(self.w)).sum(-1, keepdims=True)

    def forward(self):
        """O, its bound before the output's rounding, G, its bound."""
        lift = power(self.v).max() / power(self.v)[:, 0]
        O = np.einsum("ign,nd->igd", self.w, self.v) / self.G
        e = self.ew + ((self.n + 64) * U + H[self.dtype]) * np.abs(self.w) + SUB[self.dtype] * lift
        e = np.where(self.see, e, 0.0)
        top = np.broadcast_to(power(self.v) * SUB[self.dtype], self.v.shape)
        bound = np.einsum("ign,nd->igd", e, np.abs(self.v)) + np.einsum("ign,nd->igd", np.abs(self.w), top)
        bound = bound / np.abs(self.G) + (self.eG / np.abs(self.G) + 4 * U) * np.abs(O)
        return O, bound, self.G[..., 0], self.eG[..., 0] + 2 * U * np.abs(self.G[..., 0])

    def backward(self, do, out_error):
        """dq [n, g, D], dk, dv [n, D] and their bounds before the outputs'
        rounding; out_error: the relative error of the O that the call is given
        (its G: float32)."""
        d, D, n, rel = self.dtype, self.D, self.n, H[self.dtype]
        u = 1.0 / self.G
        O = np.einsum("ign,nd->igd", self.w, self.v) * u
        dp = np.einsum("igd,nd->ign", do, self.v)
        delta = (do * O).sum(-1, keepdims=True)
        mag = np.einsum("igd,nd->ign", np.abs(do), np.abs(self.v))
        # the rows of v and do in fp16: 2^-25 of their powers
        sub = SUB[d] * (np.einsum("igo,nd->ign", power(do), np.abs(self.v))
                        + np.einsum("igd,no->ign", np.abs(do), power(self.v)))
        e_dp = (D + 8) * U * mag + sub
        e_delta = ((D + 8) * U + out_error) * (np.abs(do) * np.abs(O)).sum(-1, keepdims=True)
        x = dp - delta
        T = self.t * u * x
        # what a wave shares: powers of the largest v (and delta) of the sequence, of
        # the largest do / G
        top = power(self.v).max() + np.abs(delta).max() / power(do).min()
        tq = SUB[d] * np.abs(u) * power(do) * top * 4
        tk = SUB[d] * (np.abs(u) * power(do)).max() * top * 4
        eT = np.abs(u) * (self.et * np.abs(x) + np.abs(self.t) * (e_dp + e_delta + 4 * U * (np.abs(dp) + np.abs(delta))))
        eT = eT + (rel + 12 * U) * np.abs(T)
        T, eTq, eTk = (np.where(self.see, y, 0.0) for y in (T, eT + tq, eT + tk))
        op = rel + 64 * U                      # k^ and q^ as operands
        acc = (self.n * self.g + 64) * U

        def back(dxh, e, xh, r):
            m1, m2 = dxh.mean(-1, keepdims=True), (dxh * xh).mean(-1, keepdims=True)
            em2 = (e * np.abs(xh)).mean(-1, keepdims=True) + (2 * rel + 80 * U) * (np.abs(dxh) * np.abs(xh)).mean(-1, keepdims=True)
            err = e + e.mean(-1, keepdims=True) + np.abs(xh) * em2 + (rel + 80 * U) * np.abs(xh * m2)
            err = err + 80 * U * (np.abs(dxh) + np.abs(dxh).mean(-1, keepdims=True) + np.abs(xh * m2))
            return (dxh - m1 - xh * m2) * r, err * r

        tau = self.tau
        dq = tau * np.einsum("ign,nd->igd", T, self.k)
        eq = tau * np.einsum("ign,nd->igd", eTq + (op + acc) * np.abs(T), np.abs(self.k)) \
            + 40 * U * tau * np.abs(T).sum(-1, keepdims=True)
        dk = tau * np.einsum("ign,igd->nd", T, self.q)
        ek = tau * np.einsum("ign,igd->nd", eTk + (op + acc) * np.abs(T), np.abs(self.q)) \
            + 40 * U * tau * np.abs(T).sum((0, 1))[:, None]
        W = np.where(self.see, self.w * u, 0.0)
        eW = np.abs(u) * (self.ew + (rel + acc + 8 * U) * np.abs(self.w)) + SUB[d] * (np.abs(u) * power(do)).max() / power(do)
        dv = np.einsum("ign,igd->nd", W, do)
        ev = np.einsum("ign,igd->nd", np.where(self.see, eW, 0.0), np.abs(do)) \
            + np.einsum("ign,igd->nd", np.abs(W), np.broadcast_to(SUB[d] * power(do), do.shape))
        return (back(dq, eq, self.q, self.rq), back(dk, ek, self.k, self.rk), (dv, ev))


class Packed:
    """Rows of packed sequences as views of one projection's output; tokens of no
    sequence before and after them hold NaN."""

    def __init__(self, lens, Hq, Hkv, D, dtype, seed=0, before=0, after=0, size=1.0):
        import torch
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        tdt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        self.lens, self.Hq, self.Hkv, self.D, self.dtype, self.tdt = lens, Hq, Hkv, D, dtype, tdt
        self.group, self.before = Hq // Hkv, before
        self.start = before + np.concatenate([[0], np.cumsum(lens)])
        T = self.T = int(self.start[-1]) + after
        self.rows = torch.randn((T, Hq + 2 * Hkv, D), generator=gen, device="cuda")
        self.rows[:, Hq + Hkv:] *= size
        self.dout = torch.randn((T, Hq, D), generator=gen, device="cuda").to(tdt)
        self.rows = self.rows.to(tdt)
        for x in (self.rows, self.dout):
            x[:before] = x[self.start[-1]:] = float("nan")
        self.q, self.k, self.v = self.rows.split([Hq, Hkv, Hkv], dim=1)
        self.starts = torch.tensor(self.start, dtype=torch.int32, device="cuda")

    def heads(self, p, tau, causal):
        """(tokens, key head, query heads, Head) of every sequence and key head."""
        q, k, v = np64(self.q), np64(self.k), np64(self.v)
        for a, b in zip(self.start, self.start[1:]):
            for h in range(self.Hkv if b > a else 0):
                hs = slice(h * self.group, (h + 1) * self.group)
                yield slice(a, b), h, hs, Head(q[a:b, hs], k[a:b, h], v[a:b, h], p, tau, causal, self.dtype)
