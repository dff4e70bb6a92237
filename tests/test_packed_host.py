"""Refusals of the packed attention (no GPU needed): every call here carries at
least one invalid argument, so the library must reject it during host
validation; the fake device pointers are never dereferenced."""
import os

import pytest

from paper_2402_07901_amd import fastmax as fm

from test_serve_host import A, SIZES, strides

pytestmark = pytest.mark.skipif(not os.path.exists(fm.LIB_PATH),
                                reason="libfastmax.so not built")
BIG = 1 << 40


def fwd(ptrs=None, g=A, st=None, S=2, T=8, Hq=4, Hkv=2, D=64, p=2, causal=1, scale=1.0, dt=fm.BF16,
        ws=A, wsb=BIG):
    x = ptrs or [A] * 5        # q, k, v, starts, out
    return fm.lib().fastmax_packed_fwd(*x[:3], st, x[3], x[4], g, S, T, Hq, Hkv, D, p, causal, scale,
                                       dt, ws, wsb, None)


def bwd(ptrs=None, st=None, dst=None, S=2, T=8, Hq=4, Hkv=2, D=64, p=2, causal=1, scale=1.0,
        dt=fm.BF16, ws=A, wsb=BIG):
    x = ptrs or [A] * 10       # q, k, v, starts, out, dout, g, dq, dk, dv
    return fm.lib().fastmax_packed_bwd(*x[:3], st, *x[3:], dst, S, T, Hq, Hkv, D, p, causal, scale,
                                       dt, ws, wsb, None)


@pytest.mark.parametrize("kw,code", SIZES + [
    (dict(T=0), fm.EINVAL), (dict(T=-1), fm.EINVAL), (dict(S=0), fm.EINVAL),
    (dict(S=(1 << 20) + 1), fm.EINVAL), (dict(T=1 << 29), fm.EINVAL), (dict(p=0), fm.EINVAL),
    (dict(p=3), fm.EINVAL), (dict(causal=2), fm.EINVAL), (dict(causal=-1), fm.EINVAL),
    (dict(scale=0.0), fm.EINVAL), (dict(scale=1.01), fm.EINVAL),
    (dict(scale=float("nan")), fm.EINVAL)])
def test_sizes(kw, code):
    assert fwd([0] + [A] * 4, **kw) == code
    assert bwd([0] + [A] * 9, **kw) == code


@pytest.mark.parametrize("Hq,Hkv", [(4, 2), (1, 1), (64, 1)])
def test_most_rows_and_sequences(Hq, Hkv):
    """T * Hq = 2^30 and S = 2^20 pass the checks (a NULL q ends the calls), one more
    does not; the size call agrees."""
    most = (1 << 30) // Hq
    for kw, ok in ((dict(T=most), True), (dict(T=most + 1), False), (dict(S=1 << 20), True),
                   (dict(S=(1 << 20) + 1), False), (dict(T=most, S=1 << 20), True)):
        kw = dict(Hq=Hq, Hkv=Hkv, **kw)
        assert fwd([0] + [A] * 4, **kw) == (fm.ENULL if ok else fm.EINVAL)
        assert bwd([0] + [A] * 9, **kw) == (fm.ENULL if ok else fm.EINVAL)
        for backward in (False, True):
            need = fm.packed_workspace_bytes(kw.get("S", 2), kw.get("T", 8), Hq, Hkv, 64, fm.BF16, backward)
            assert (need > 0) == ok


def test_pointers():
    for call, n in ((fwd, 5), (bwd, 10)):
        for i in range(n):
            for bad, code in ((0, fm.ENULL), (A + 2, fm.EALIGN)):
                ptrs = [A] * n
                ptrs[i] = bad
                assert call(ptrs) == code, (call.__name__, i)
    assert fwd(g=A + 4) == fm.EALIGN


def test_strides():
    for bad, code in ((dict(token=1025), fm.EALIGN), (dict(head=68), fm.EALIGN),
                      (dict(token=-1024), fm.EINVAL), (dict(token=1 << 50), fm.EINVAL)):
        assert fwd([0] + [A] * 4, st=strides(3, **bad)) == code
        assert bwd([0] + [A] * 9, st=strides(3, **bad)) == code
        assert bwd([A] * 9 + [0], dst=strides(3, **bad)) == code
    # gradients whose rows would share memory
    assert bwd([A] * 9 + [0], dst=strides(3, token=0)) == fm.EINVAL
    assert fwd([0] + [A] * 4, st=strides(3, token=0)) == fm.ENULL


def test_workspaces():
    for call, backward in ((fwd, False), (bwd, True)):
        need = fm.packed_workspace_bytes(2, 8, 4, 2, 64, fm.BF16, backward)
        assert need > 0
        assert call(ws=None, wsb=need) == fm.EWORKSPACE
        assert call(ws=A, wsb=need - 1) == fm.EWORKSPACE
        assert call(ws=A + 8, wsb=need) == fm.EALIGN
    # sizes that the calls refuse need none
    assert fm.packed_workspace_bytes(0, 8, 4, 2, 64, fm.BF16) == 0
    assert fm.packed_workspace_bytes(2, 8, 4, 3, 64, fm.BF16) == 0
    assert fm.packed_workspace_bytes(2, 8, 4, 2, 48, fm.BF16) == 0
    # past 32 bits
    assert fm.packed_workspace_bytes(1, 1 << 22, 64, 64, 128, fm.F32, True) > 4 * 64 * (128 * 4 << 22)


def test_binding_checks():
    import torch
    q, k = torch.zeros(8, 4, 64), torch.zeros(8, 2, 64)
    starts = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="on a GPU"):
        fm.fastmax_packed_fwd(q, k, k, starts)
    with pytest.raises(ValueError, match=r"\[T, Hq, D\]"):
        fm.fastmax_packed_fwd(q[None], k, k, starts)
    with pytest.raises(ValueError, match="on a GPU"):
        fm.fastmax_packed_bwd(q, k, k, starts, q, q, q[..., 0])
