"""Plain float64 forms of the cache in 8 bits, and a paged cache of it whose
unused slots hold what must not be used."""
import numpy as np

from paper_2402_07901_amd import fastmax as fm

import serve_util as su

LEAST = 2.0 ** -100


def codes_of(x):
    """Real-valued codes x 127 / amax and scales amax / 127 of float64 rows."""
    top = np.abs(x).max(-1, keepdims=True)
    live = top >= LEAST
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.where(live, x * (127.0 / top), 0.0)
    return c, np.where(live, top / 127.0, 0.0)[..., 0]


def attend(q, k, v, pos, p, tau, window, sinks, dtype):
    """serve_util.attend over rows k, v (codes times scales), its bound with q's
    whole numbers (an error of 2^-16 of its largest magnitude, float32: 2^-23)
    and the scales' products (3 roundings a score, 3 a value) added.  Chunks: the
    weight, the value's scale and their product are rounded to fp16 (2^-11 each;
    float32: once to two fp16 parts, 2^-22), and the sum G is of the rounded ones."""
    parts = None if dtype == "f32" else 2
    ref, bound = su.attend(q, k, v, pos, p, tau, window, sinks, parts)
    n = np.arange(len(k))
    see = n[None] <= pos[:, None]
    if window:
        see &= (n[None] > pos[:, None] - window) | (n[None] < sinks)
    s = tau * np.einsum("tgd,nd->tgn", q, k)
    whole = 2.0 ** -23 if dtype == "f32" else 2.0 ** -16
    off = tau * whole * np.abs(q).max(-1, keepdims=True) * np.abs(k).sum(-1)
    off = off + 4 * su.U * tau * np.einsum("tgd,nd->tgn", np.abs(q), np.abs(k))
    w = 1.0 + s + (0.5 * s * s if p == 2 else 0.0)
    e = off * (1.0 + (np.abs(s) if p == 2 else 0.0))
    e = e + (3 * su.U + (2.0 ** -22 if dtype == "f32" else 3 * 2.0 ** -11)) * np.abs(w)
    e = np.where(see[:, None, :], e, 0.0)
    G = np.abs(np.where(see[:, None, :], w, 0.0).sum(-1, keepdims=True))
    G = np.where(G > 0, G, 1.0)
    return ref, bound + np.einsum("tgn,nd->tgd", e, np.abs(v)) / G + e.sum(-1, keepdims=True) / G * np.abs(ref)


class Cache:
    """Sequences in a paged 8-bit cache; unused slots have codes 127 and scales
    NaN, the rest of the page table is -1."""

    def __init__(self, lens, news, Hq, Hkv, D, page, dtype, seed=0, order="heads", cols=None,
                 size=1.0):
        import torch
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        rng = np.random.default_rng(seed)
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
        both = torch.full(shape, 127, dtype=torch.int8, device="cuda")
        if order != "heads":
            both = both.transpose(2, 3)
        self.k, self.v = both[0], both[1]
        self.ks, self.vs = (torch.full((pages, Hkv, page), float("nan"), device="cuda")
                            for _ in range(2))

        def standard(x):
            x = x - x.mean(-1, keepdim=True)
            return x / x.square().mean(-1, keepdim=True).sqrt()

        self.k_h, self.v_h = [], []
        for s, n in enumerate(lens):
            rows = torch.randn((2, max(n, 1), Hkv, D), generator=gen, device="cuda")[:, :n]
            idx = torch.arange(n, device="cuda")
            pg = torch.from_numpy(self.table_h[s]).cuda().long()[idx // page]
            held = []
            for x, codes, scales in ((standard(rows[0]), self.k, self.ks),
                                     (rows[1] * size, self.v, self.vs)):
                top = x.abs().amax(-1, keepdim=True)
                c = (x * (127.0 / top)).round().to(torch.int8)
                codes[pg, :, idx % page] = c
                scales[pg, :, idx % page] = top[..., 0] / 127.0
                held.append(su.np64(c) * su.np64(top / 127.0))
            self.k_h.append(held[0])
            self.v_h.append(held[1])
        tdt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        self.q = standard(torch.randn((sum(news), Hq, D), generator=gen, device="cuda")).to(tdt)
        self.table = torch.from_numpy(self.table_h).cuda()
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.start = np.concatenate([[0], np.cumsum(news)])
        self.q_start = torch.tensor(self.start, dtype=torch.int32, device="cuda")

    @property
    def cache(self):
        return self.k, self.v, self.ks, self.vs

    def run(self, starts=True, **kw):
        return fm.fastmax_paged_fwd_q8(self.q, *self.cache, self.table, self.lens,
                                       q_start=self.q_start if starts else None, **kw)

    def at(self, s, n):
        """(page, place) of token n of sequence s."""
        return int(self.table_h[s, n // self.page]), n % self.page

    def check(self, out, label, p=2, tau=1.0, window=0, sinks=0, keep=None):
        """keep: rows of q to look at (None: all)."""
        assert tuple(out.shape) == tuple(self.q.shape)
        for s, n in enumerate(self.lens_h):
            rows = np.arange(self.start[s], self.start[s + 1])
            pos = n - self.news[s] + np.arange(self.news[s])
            if keep is not None:
                rows, pos = rows[keep[rows]], pos[keep[rows]]
            if not len(rows):
                continue
            for h in range(self.Hkv):
                hs = slice(h * self.group, (h + 1) * self.group)
                ref, bound = attend(su.np64(self.q[rows][:, hs]), self.k_h[s][:, h],
                                    self.v_h[s][:, h], pos, p, tau, window, sinks, self.dtype)
                su.check(out[rows][:, hs], ref, su.OUT[self.dtype] * np.abs(ref) + 1.01 * bound,
                         (label, s, h))
