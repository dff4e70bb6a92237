"""Helpers of the paged attention's edge tests, on the Cache of test_paged."""
import numpy as np

import serve_util as su


def put(c, s, t, h, value, channel=slice(None)):
    """Token t of sequence s, key head h: its values in the cache."""
    c.v[int(c.table_h[s, t // c.page]), h, t % c.page, channel] = value


def seen(pos, t, window=0, sinks=0):
    """Whether queries at positions pos see key t."""
    return (t <= pos) & ((t > pos - window) | (t < sinks) if window else t <= pos)


def positions(c, s):
    return c.lens_h[s] - c.news[s] + np.arange(c.news[s])


def check_rows(c, out, s, keep, label, p=2, tau=1.0, window=0, sinks=0):
    """The new tokens ``keep`` (a mask) of sequence s against float64, weights
    to the bound of two bf16 parts."""
    if not keep.any():
        return
    rows = c.start[s] + np.flatnonzero(keep)
    parts = None if c.dtype == "f32" else 2
    for h in range(c.Hkv):
        hs = slice(h * c.group, (h + 1) * c.group)
        ref, bound = su.attend(su.np64(c.q[rows][:, hs]), c.k_h[s][:, h], c.v_h[s][:, h],
                               positions(c, s)[keep], p, tau, window, sinks, parts)
        su.check(out[rows][:, hs], ref, su.OUT[c.dtype] * np.abs(ref) + 1.01 * bound, (label, s, h))
