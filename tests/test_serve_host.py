"""Refusals of the row calls and the paged attention (no GPU needed): every
call here carries at least one invalid argument, so the library must reject it
during host validation; the fake device pointers are never dereferenced.  The
binding's own checks are tested with CPU tensors, which it refuses last."""
import ctypes
import os

import pytest

from paper_2402_07901_amd import fastmax as fm

pytestmark = pytest.mark.skipif(not os.path.exists(fm.LIB_PATH),
                                reason="libfastmax.so not built")

A = 0x100000   # 16-byte aligned fake pointer (never dereferenced)


def rope(**kw):
    r = fm.Rope(A, A, A, 100, 64, 1, (ctypes.c_int * 4)(), 0, A, A, 1e-6)
    for name, x in kw.items():
        if name == "sections":
            r.sections[:len(x)] = x
        else:
            setattr(r, name, x)
    return r


def strides(n, batch=0, token=1024, head=64):
    out = (fm.Strides * n)()
    for s in out:
        s.batch, s.token, s.head = batch, token, head
    return out


def rope_fwd(ptrs=None, st=None, B=1, N=8, Hq=4, Hkv=2, D=64, r=None, dt=fm.BF16):
    p = ptrs or [A] * 6
    return fm.lib().fastmax_rope_fwd(*p[:3], st, *p[3:], B, N, Hq, Hkv, D,
                                     rope() if r is None else r, dt, None)


def rope_bwd(ptrs=None, st=None, dst=None, B=1, N=8, Hq=4, Hkv=2, D=64, r=None, dt=fm.BF16,
             ws=None, wsb=0):
    p = ptrs or [A] * 10       # q, k, gq, gk, gv, dq, dk, dv, dwq, dwk
    return fm.lib().fastmax_rope_bwd(*p[:2], st, *p[2:8], dst, *p[8:], B, N, Hq, Hkv, D,
                                     rope() if r is None else r, dt, ws, wsb, None)


def append(ptrs=None, st=None, cache=None, T=8, Hq=4, Hkv=2, D=64, pages=4, page=64, r=None,
           dt=fm.BF16):
    p = ptrs or [A] * 7        # q, k, v, q_out, k_cache, v_cache, slots
    return fm.lib().fastmax_cache_append(*p[:3], st, *p[3:6], cache, p[6], T, Hq, Hkv, D, pages,
                                         page, rope() if r is None else r, dt, None)


def paged(ptrs=None, st=None, cache=None, S=2, T=2, Hq=4, Hkv=2, D=64, pages=4, page=64, cols=4,
          max_q=1, max_len=64, p=2, scale=1.0, window=0, sinks=0, dt=fm.BF16, ws=None, wsb=0,
          start=None):
    x = ptrs or [A] * 6        # q, k_cache, v_cache, table, lens, out
    return fm.lib().fastmax_paged_fwd(x[0], st, x[1], x[2], cache, x[3], x[4], start, x[5], S, T,
                                      Hq, Hkv, D, pages, page, cols, max_q, max_len, p, scale,
                                      window, sinks, dt, ws, wsb, None)


SIZES = [(dict(Hq=0), fm.EINVAL), (dict(Hkv=0), fm.EINVAL), (dict(Hq=4, Hkv=3), fm.EINVAL),
         (dict(Hq=2, Hkv=4), fm.EINVAL), (dict(Hq=1 << 17, Hkv=1), fm.EINVAL),
         (dict(dt=7), fm.EINVAL), (dict(D=48), fm.EUNSUPPORTED), (dict(D=256), fm.EUNSUPPORTED)]


@pytest.mark.parametrize("kw,code", SIZES + [(dict(B=0), fm.EINVAL), (dict(N=-1), fm.EINVAL)])
def test_rope_sizes(kw, code):
    assert rope_fwd([0] + [A] * 5, **kw) == code
    assert rope_bwd([0] + [A] * 9, **kw) == code


@pytest.mark.parametrize("kw,code", SIZES + [(dict(T=0), fm.EINVAL), (dict(pages=0), fm.EINVAL),
                                             (dict(page=8), fm.EINVAL), (dict(page=48), fm.EINVAL),
                                             (dict(page=2048), fm.EINVAL)])
def test_append_sizes(kw, code):
    assert append([0] + [A] * 6, **kw) == code


@pytest.mark.parametrize("kw,code", SIZES + [
    (dict(S=0), fm.EINVAL), (dict(S=65536, T=65536), fm.EINVAL), (dict(T=0), fm.EINVAL),
    (dict(T=3), fm.EINVAL), (dict(max_q=2), fm.EINVAL), (dict(max_q=0), fm.EINVAL),
    (dict(max_len=0), fm.EINVAL), (dict(max_len=(1 << 30) + 1), fm.EINVAL), (dict(p=0), fm.EINVAL),
    (dict(p=3), fm.EINVAL), (dict(scale=0.0), fm.EINVAL), (dict(scale=1.5), fm.EINVAL),
    (dict(scale=float("nan")), fm.EINVAL), (dict(window=-1), fm.EINVAL),
    (dict(sinks=-1), fm.EINVAL), (dict(cols=0), fm.EINVAL), (dict(cols=1 << 25), fm.EINVAL),
    (dict(page=24), fm.EINVAL), (dict(pages=0), fm.EINVAL)])
def test_paged_sizes(kw, code):
    assert paged([0] + [A] * 5, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(rot=24), fm.EINVAL), (dict(rot=80), fm.EINVAL), (dict(rot=-16), fm.EINVAL),
    (dict(axes=0), fm.EINVAL), (dict(axes=5), fm.EINVAL), (dict(table_rows=0), fm.EINVAL),
    (dict(axes=2, sections=[16, 15]), fm.EINVAL), (dict(axes=2, sections=[-1, 33]), fm.EINVAL),
    (dict(interleaved=2), fm.EINVAL), (dict(eps=-1.0), fm.EINVAL),
    (dict(eps=float("nan")), fm.EINVAL), (dict(wq=None), fm.ENULL), (dict(wk=None), fm.ENULL),
    (dict(cos=None), fm.ENULL), (dict(sin=None), fm.ENULL), (dict(pos=None), fm.ENULL),
    (dict(cos=A + 8), fm.EALIGN), (dict(sin=A + 4), fm.EALIGN), (dict(pos=A + 2), fm.EALIGN),
    (dict(wq=A + 4), fm.EALIGN)])
def test_rope_struct(kw, code):
    r = rope(**kw)
    assert rope_fwd([0] + [A] * 5, r=r) == code
    assert rope_bwd([0] + [A] * 9, r=r) == code
    assert append([0] + [A] * 6, r=r) == code
    assert fm.lib().fastmax_rope_fwd(A, A, A, None, A, A, A, 1, 8, 4, 2, 64, None, fm.BF16,
                                     None) == fm.ENULL


def test_pointers():
    for call, n in ((rope_fwd, 6), (rope_bwd, 10), (append, 7), (paged, 6)):
        for i in range(n):
            for bad, code in ((0, fm.ENULL), (A + 2, fm.EALIGN)):
                ptrs = [A] * n
                ptrs[i] = bad
                assert call(ptrs) == code, (call.__name__, i)
    assert paged(start=A + 2) == fm.EALIGN


def test_strides():
    for bad, code in ((dict(token=1025), fm.EALIGN), (dict(head=68), fm.EALIGN),
                      (dict(token=-1024), fm.EINVAL), (dict(token=1 << 50), fm.EINVAL)):
        assert rope_fwd([0] + [A] * 5, st=strides(3, **bad)) == code
        assert rope_bwd([0] + [A] * 9, st=strides(2, **bad)) == code
        assert rope_bwd([0] + [A] * 9, dst=strides(3, **bad)) == code
        assert append([0] + [A] * 6, st=strides(3, **bad)) == code
        assert append([0] + [A] * 6, cache=strides(1, batch=8192, **bad)) == code
        assert paged([0] + [A] * 5, cache=strides(1, batch=8192, **bad)) == code
        assert paged([0] + [A] * 5, st=strides(1, **bad)) == code
    # outputs whose rows would share memory
    assert rope_bwd([0] + [A] * 9, dst=strides(3, token=0)) == fm.EINVAL
    assert append([0] + [A] * 6, cache=strides(1, batch=0)) == fm.EINVAL
    # a stride that no row uses is not looked at
    assert rope_fwd([0] + [A] * 5, st=strides(3, batch=-7)) == fm.ENULL


def test_workspaces():
    need = fm.rope_workspace_bytes(1, 8, 4, 2, 64, True)
    assert need > 0 and fm.rope_workspace_bytes(1, 8, 4, 2, 64, False) == 0
    assert rope_bwd(ws=None, wsb=need) == fm.EWORKSPACE
    assert rope_bwd(ws=A, wsb=need - 1) == fm.EWORKSPACE
    assert rope_bwd(ws=A + 4, wsb=need) == fm.EALIGN
    need = fm.paged_workspace_bytes(1, 1, 4, 2, 64, 1, 20000, 0, 0, fm.BF16)
    assert need > 0
    kw = dict(S=1, T=1, cols=400, max_len=20000)
    assert paged(ws=None, wsb=need, **kw) == fm.EWORKSPACE
    assert paged(ws=A, wsb=need - 1, **kw) == fm.EWORKSPACE
    assert paged(ws=A + 4, wsb=need, **kw) == fm.EALIGN
    # sizes that the calls refuse need none
    assert fm.rope_workspace_bytes(0, 8, 4, 2, 64, True) == 0
    assert fm.paged_workspace_bytes(1, 1, 4, 3, 64, 1, 20000, 0, 0, fm.BF16) == 0


def test_grids_past_the_dispatch_limits():
    """2^34 rows of 64 lanes: refused before the first launch."""
    assert rope_fwd(B=1 << 15, N=1 << 17, D=128, r=rope(rot=128)) == fm.EUNSUPPORTED


def test_binding_checks():
    import torch
    q, k = torch.zeros(1, 8, 4, 64), torch.zeros(1, 8, 2, 64)
    pos, cos = torch.zeros(1, 8, dtype=torch.int32), torch.zeros(10, 32)
    with pytest.raises(ValueError, match="on a GPU"):
        fm.fastmax_rope_fwd(q, k, k, pos, cos, cos)
    with pytest.raises(ValueError, match=r"\[B, N, Hq, D\]"):
        fm.fastmax_rope_fwd(q[0], k, k, pos, cos, cos)
    with pytest.raises(ValueError, match=r"\[T, Hq, D\]"):
        fm.fastmax_cache_append(q, k, k, k, k, pos, pos, cos, cos)
    with pytest.raises(ValueError, match=r"\[T, Hq, D\]"):
        fm.fastmax_paged_fwd(q, k, k, pos, pos)

    # the checks behind that one, on their own
    def build(tokens=(1, 8), pos=pos, cos=cos, sin=cos, wq=None, wk=None, sections=None):
        return fm._rope_of(q, tokens, pos, cos, sin, wq, wk, 1e-6, sections, False)
    assert build().rot == 64 and build(pos=None, cos=None, sin=None).rot == 0
    for kw in (dict(sin=None), dict(pos=None), dict(sin=cos[:5]), dict(cos=cos.double()),
               dict(pos=pos.long()), dict(pos=pos[:, :4]), dict(wq=torch.ones(64)),
               dict(wq=torch.ones(32), wk=torch.ones(64)),
               dict(pos=torch.zeros(1, 8, 5, dtype=torch.int32)),
               dict(pos=torch.zeros(1, 8, 2, dtype=torch.int32)),
               dict(pos=torch.zeros(1, 8, 2, dtype=torch.int32), sections=[32])):
        with pytest.raises(ValueError):
            build(**kw)
    cache = torch.zeros(4, 2, 16, 64)
    assert fm._cache_of(q, cache, cache, 2)[:2] == (4, 16)
    for kc, vc in ((cache[0], cache), (cache, cache[:3]), (cache, cache.bfloat16()),
                   (cache, torch.zeros(4, 16, 2, 64).transpose(1, 2))):
        with pytest.raises(ValueError):
            fm._cache_of(q, kc, vc, 2)


def test_strides_of_single_pages_and_heads():
    """Strides along an axis of size 1 reach nothing: the caches may differ there."""
    import torch
    q = torch.zeros(3, 4, 64)
    whole = torch.zeros(5, 1, 16, 64)
    turned = torch.zeros(5, 16, 1, 64).transpose(1, 2)
    assert whole.stride() != turned.stride()
    for kc, vc in ((whole, turned), (turned, whole)):
        pages, page, st = fm._cache_of(q, kc, vc, 1)
        assert (pages, page) == (5, 16) and tuple(st)[:2] == (1024, 64)
    one, first = torch.zeros(1, 2, 16, 64), torch.zeros(7, 2, 16, 64)[::3][:1]
    assert one.stride() != first.stride()
    for kc, vc in ((one, first), (first, one)):
        pages, page, st = fm._cache_of(q, kc, vc, 2)
        assert (pages, page) == (1, 16) and tuple(st)[1:] == (64, 1024)
    with pytest.raises(ValueError, match="same strides"):
        fm._cache_of(q, torch.zeros(5, 2, 16, 64), torch.zeros(5, 16, 2, 64).transpose(1, 2), 2)


def test_workspaces_are_checked():
    """A workspace with gaps, or in another place than the rows, is refused: the
    library writes its bytes one after the other, on the GPU."""
    import torch
    q, given = torch.zeros(2, 4, 64), torch.zeros(100, dtype=torch.uint8)
    assert fm._workspace(q, given, None, None) == (given, 100)
    assert fm._workspace(q, given.view(torch.int32), None, None)[1] == 100
    assert fm._workspace(q, None, lambda: 0, None) == (None, 0)
    with pytest.raises(ValueError, match="workspace must be contiguous"):
        fm._workspace(q, given[::2], None, None)
    with pytest.raises(ValueError, match="workspace is on meta"):
        fm._workspace(q, given.to("meta")[::2], None, None)
