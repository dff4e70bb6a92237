"""Refusals of the 8-bit cache's calls (no GPU needed): every call here carries at
least one invalid argument, so the library must reject it during host
validation; the fake device pointers are never dereferenced."""
import os

import pytest

from paper_2402_07901_amd import fastmax as fm

from test_serve_host import A, SIZES, rope, strides

pytestmark = pytest.mark.skipif(not os.path.exists(fm.LIB_PATH),
                                reason="libfastmax.so not built")


def append(ptrs=None, st=None, cache=None, T=8, Hq=4, Hkv=2, D=64, pages=4, page=64, r=None,
           dt=fm.BF16):
    p = ptrs or [A] * 9        # q, k, v, q_out, k_cache, v_cache, k_scale, v_scale, slots
    return fm.lib().fastmax_cache_append_q8(*p[:3], st, *p[3:8], cache, p[8], T, Hq, Hkv, D, pages,
                                            page, rope() if r is None else r, dt, None)


def read(ptrs=None, cache=None, T=8, Hkv=2, D=64, pages=4, page=64, dt=fm.BF16):
    p = ptrs or [A] * 7        # k_cache, v_cache, k_scale, v_scale, slots, k, v
    return fm.lib().fastmax_cache_read_q8(*p[:4], cache, *p[4:], T, Hkv, D, pages, page, dt, None)


def paged(ptrs=None, st=None, cache=None, S=2, T=2, Hq=4, Hkv=2, D=64, pages=4, page=64, cols=4,
          max_q=1, max_len=64, p=2, scale=1.0, window=0, sinks=0, dt=fm.BF16, ws=None, wsb=0,
          start=None):
    x = ptrs or [A] * 8        # q, k_cache, v_cache, k_scale, v_scale, table, lens, out
    return fm.lib().fastmax_paged_fwd_q8(x[0], st, *x[1:5], cache, *x[5:7], start, x[7], S, T, Hq,
                                         Hkv, D, pages, page, cols, max_q, max_len, p, scale,
                                         window, sinks, dt, ws, wsb, None)


@pytest.mark.parametrize("kw,code", SIZES + [(dict(T=0), fm.EINVAL), (dict(pages=0), fm.EINVAL),
                                             (dict(page=8), fm.EINVAL), (dict(page=48), fm.EINVAL),
                                             (dict(page=2048), fm.EINVAL), (dict(dt=2), fm.EINVAL)])
def test_append_and_read_sizes(kw, code):
    assert append([0] + [A] * 8, **kw) == code
    if not set(kw) & {"Hq", "Hkv"}:
        assert read([0] + [A] * 6, **kw) == code


def test_read_heads():
    for Hkv in (0, -1, 1 << 17):
        assert read([0] + [A] * 6, Hkv=Hkv) == fm.EINVAL


@pytest.mark.parametrize("kw,code", SIZES + [
    (dict(S=0), fm.EINVAL), (dict(S=65536, T=65536), fm.EINVAL), (dict(T=0), fm.EINVAL),
    (dict(T=3), fm.EINVAL), (dict(max_q=2), fm.EINVAL), (dict(max_len=0), fm.EINVAL),
    (dict(p=0), fm.EINVAL), (dict(scale=0.0), fm.EINVAL), (dict(scale=float("nan")), fm.EINVAL),
    (dict(window=-1), fm.EINVAL), (dict(sinks=-1), fm.EINVAL), (dict(cols=0), fm.EINVAL),
    (dict(cols=1 << 25), fm.EINVAL), (dict(page=24), fm.EINVAL), (dict(dt=2), fm.EINVAL)])
def test_paged_sizes(kw, code):
    assert paged([0] + [A] * 7, **kw) == code


def test_pointers():
    for call, n in ((append, 9), (read, 7), (paged, 8)):
        for i in range(n):
            for bad, code in ((0, fm.ENULL), (A + 2, fm.EALIGN)):
                ptrs = [A] * n
                ptrs[i] = bad
                assert call(ptrs) == code, (call.__name__, i)
    assert paged(start=A + 2) == fm.EALIGN


def test_strides():
    """A row of codes is 16-byte aligned: strides are multiples of 16."""
    for bad, code in ((dict(token=1032), fm.EALIGN), (dict(head=72), fm.EALIGN),
                      (dict(token=-1024), fm.EINVAL), (dict(token=1 << 50), fm.EINVAL)):
        assert append([0] + [A] * 8, cache=strides(1, batch=8192, **bad)) == code
        assert read([0] + [A] * 6, cache=strides(1, batch=8192, **bad)) == code
        assert paged([0] + [A] * 7, cache=strides(1, batch=8192, **bad)) == code
    assert append([0] + [A] * 8, cache=strides(1, batch=0)) == fm.EINVAL
    # rows of q, k, v as ever
    assert append([0] + [A] * 8, st=strides(3, token=1032)) == fm.ENULL
    assert append([0] + [A] * 8, st=strides(3, token=1028)) == fm.EALIGN


def test_workspaces():
    need = fm.paged_q8_workspace_bytes(1, 1, 4, 2, 64, 1, 20000, 0, 0, fm.BF16)
    assert need > 0
    kw = dict(S=1, T=1, cols=400, max_len=20000)
    assert paged(ws=None, wsb=need, **kw) == fm.EWORKSPACE
    assert paged(ws=A, wsb=need - 1, **kw) == fm.EWORKSPACE
    assert paged(ws=A + 4, wsb=need, **kw) == fm.EALIGN
    assert fm.paged_q8_workspace_bytes(1, 1, 4, 3, 64, 1, 20000, 0, 0, fm.BF16) == 0


def test_binding_checks():
    import torch
    q = torch.zeros(3, 4, 64)
    codes = torch.zeros(5, 2, 16, 64, dtype=torch.int8)
    scale = torch.zeros(5, 2, 16)
    ok = fm._cache_q8_of(q, codes, codes, scale, scale, 2)
    assert ok[:2] == (5, 16) and tuple(ok[2]) == (2048, 64, 1024)
    for bad in ((codes.float(), codes, scale, scale), (codes, codes[:4], scale, scale),
                (codes, codes, scale[:4], scale), (codes, codes, scale, scale.double()),
                (codes, codes, scale, scale.transpose(1, 2).contiguous().transpose(1, 2)),
                (codes, torch.zeros(5, 16, 2, 64, dtype=torch.int8).transpose(1, 2), scale, scale)):
        with pytest.raises(ValueError):
            fm._cache_q8_of(q, *bad, 2)
    with pytest.raises(ValueError, match="on a GPU"):
        fm.fastmax_cache_read_q8(codes, codes, scale, scale, torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError, match="on a GPU"):
        fm.fastmax_paged_fwd_q8(q, codes, codes, scale, scale, scale, scale)
    with pytest.raises(ValueError, match=r"\[T, Hq, D\]"):
        fm.fastmax_cache_append_q8(q[0], q, q, codes, codes, scale, scale, None, None, None, None)
