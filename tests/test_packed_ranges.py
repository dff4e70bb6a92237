"""GPU tests of the packed attention's powers of two (bf16 calls), against float64:
rows beside values of any size that they do not see."""
import copy

import numpy as np
import pytest

from paper_2402_07901_amd import fastmax as fm

import serve_util as su
from gpu_util import say
from packed_util import OUT, Head, Packed

pytestmark = pytest.mark.gpu
LARGEST = (2.0 - 2.0 ** -7) * 2.0 ** 127                       # of bf16
HEADS = [(4, 2), (120, 120)]                                   # 32 columns to a workgroup, 128
SIZES = [(2, 1.0), (2, 0.02), (1, 0.02), (2, 2.0 ** -60)]      # p, the values' deviation


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fm.lib()
    yield
    torch.cuda.synchronize()


def tau_of(p, D):
    return 1.0 if p == 2 else 1.0 / D


def heads_of(x, a, b, p, causal=True):
    """(key head, query heads, Head) of the tokens a .. b - 1 as a sequence, for the
    first two key heads."""
    for h in range(2):
        hs = slice(h * x.group, (h + 1) * x.group)
        yield h, hs, Head(su.np64(x.q[a:b, hs]), su.np64(x.k[a:b, h]), su.np64(x.v[a:b, h]), p,
                          tau_of(p, x.D), causal, x.dtype)


@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("p,size", SIZES)
def test_outputs_beside_the_largest_value(D, heads, p, size):
    """A token's values are the largest that bf16 has: O of the rows before it is held
    to the bounds of the sequence without it, G of all rows and O of the ones that see
    it to the whole sequence's."""
    label = f"packed O beside the largest, D={D} p={p} H={heads} size={size}"
    say(label)
    n = 400
    for a in (70, 333):
        x = Packed([n], *heads, D, "bf16", seed=a, size=size)
        x.v[a] = LARGEST
        x.v[a, :, ::2] *= -1
        out, g = fm.fastmax_packed_fwd(x.q, x.k, x.v, x.starts, p=p, causal=True, scale=tau_of(p, D))
        for h, hs, head in heads_of(x, 0, n, p):
            O, eO, G, eG = head.forward()
            su.check(g[:, hs], G, 1.01 * eG, (label, a, "G", h))
            if p == 2:      # (weights of both signs: an O may be larger than the values)
                su.check(out[a:, hs], O[a:], OUT["bf16"] * np.abs(O[a:]) + 1.01 * eO[a:], (label, a, "later", h))
        for h, hs, head in heads_of(x, 0, a, p):
            O, eO, _, _ = head.forward()
            su.check(out[:a, hs], O, OUT["bf16"] * np.abs(O) + 1.01 * eO, (label, a, "O", h))


def given(x, a, b, p, causal=True):
    """O and G of the tokens a .. b - 1 as a sequence: the definition's for the first
    two key heads, the call's for the others."""
    import torch
    starts = torch.tensor([a, b], dtype=torch.int32, device="cuda")
    out, g = fm.fastmax_packed_fwd(x.q, x.k, x.v, starts, p=p, causal=causal, scale=tau_of(p, x.D))
    for _, hs, head in heads_of(x, a, b, p, causal):
        O, _, G, _ = head.forward()
        out[a:b, hs], g[a:b, hs] = torch.from_numpy(O).cuda().to(x.tdt), torch.from_numpy(G).cuda().float()
    return out, g


@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("p,size", SIZES)
def test_gradients_beside_the_largest_value(D, heads, p, size):
    """The same for dq of the rows before that token."""
    label = f"packed dq beside the largest, D={D} p={p} H={heads} size={size}"
    say(label)
    n = 400
    for a in (70, 333):
        x = Packed([n], *heads, D, "bf16", seed=a, size=size)
        x.v[a] = LARGEST
        x.v[a, :, ::2] *= -1
        out, g = given(x, 0, n, p)
        dq = fm.fastmax_packed_bwd(x.q, x.k, x.v, x.starts, out, x.dout, g, p=p, causal=True,
                                   scale=tau_of(p, D))[0]
        do = su.np64(x.dout)
        for h, hs, head in heads_of(x, 0, a, p):
            want, bound = head.backward(do[:a, hs], OUT["bf16"])[0]
            su.check(dq[:a, hs], want, OUT["bf16"] * (np.abs(want) + bound) + 1.01 * bound, (label, a, h))


def rows_only(head, live):
    """The rows `live` of a Head: what the others add to dk and dv is zero."""
    some = copy.copy(head)
    for name in ("q", "rq", "see", "es", "t", "et", "w", "ew", "G", "eG"):
        x = getattr(head, name)
        setattr(some, name, x[live] if len(x) == len(live) else x)
    return some


@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("power", [0, -16, -24, -30, -90])
def test_gradients_beside_rows_of_zeros(D, heads, causal, power):
    """Tokens without a loss have rows of zeros in dout, the others gradients of any
    size (a mean over many tokens): the zeros are without effect.  The first half of a
    sequence and then every third row, one sequence of nothing else and one of
    nothing but gradients."""
    import torch
    label = f"packed, zero rows of dout, D={D} H={heads} causal={causal} 2^{power}"
    say(label)
    x = Packed([300, 70, 40], *heads, D, "bf16", seed=D)
    zero = torch.zeros(x.T, dtype=torch.bool, device="cuda")
    zero[:150] = zero[:300:3] = zero[300:370] = True
    x.dout *= 2.0 ** power
    x.dout[zero] = 0
    out, g = fm.fastmax_packed_fwd(x.q, x.k, x.v, x.starts, causal=causal)
    for a, b in zip(x.start, x.start[1:]):
        here, gh = given(x, int(a), int(b), 2, causal)
        out[a:b], g[a:b] = here[a:b], gh[a:b]
    dq, dk, dv = fm.fastmax_packed_bwd(x.q, x.k, x.v, x.starts, out, x.dout, g, causal=causal)
    assert (dq[zero] == 0).all() and (dk[300:370] == 0).all() and (dv[300:370] == 0).all()
    do, live = su.np64(x.dout), ~zero.cpu().numpy()
    for a, b in ((0, 300), (370, 410)):
        for h, hs, head in heads_of(x, a, b, 2, causal):
            keep = live[a:b]
            ref = rows_only(head, keep).backward(do[a:b, hs][keep], OUT["bf16"])
            gots = (dq[a:b, hs][~zero[a:b]], dk[a:b, h], dv[a:b, h])
            for name, got, (want, bound) in zip(("dq", "dk", "dv"), gots, ref):
                tol = OUT["bf16"] * (np.abs(want) + bound) + 1.01 * bound
                su.check(got, want, tol, (label, name, a, h))


@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("causal", [True, False])
def test_gradients_of_the_largest_values(D, heads, causal):
    """Values up to bf16's largest, dout along them and small enough for gradients in
    range: dO.O of a row passes float32's range in dO's own power."""
    import torch
    label = f"packed, largest values, D={D} H={heads} causal={causal}"
    say(label)
    x = Packed([1, 2, 150, 40], *heads, D, "bf16", seed=D)
    x.v.copy_((x.v.float() * 2.0 ** 126).clamp(-LARGEST, LARGEST))
    x.dout.copy_((x.dout.abs() * 2.0 ** -30) * x.v.sign().repeat_interleave(x.group, 1))
    out, g = fm.fastmax_packed_fwd(x.q, x.k, x.v, x.starts, causal=causal)
    spans = [(int(a), int(b)) for a, b in zip(x.start, x.start[1:])]
    for a, b in spans:
        here, gh = given(x, a, b, 2, causal)
        out[a:b], g[a:b] = here[a:b], gh[a:b]
    dq, dk, dv = fm.fastmax_packed_bwd(x.q, x.k, x.v, x.starts, out, x.dout, g, causal=causal)
    do = su.np64(x.dout)
    for a, b in spans:
        for h, hs, head in heads_of(x, a, b, 2, causal):
            ref = head.backward(do[a:b, hs], OUT["bf16"])
            for name, got, (want, bound) in zip(("dq", "dk", "dv"), (dq[a:b, hs], dk[a:b, h], dv[a:b, h]), ref):
                su.check(got, want, OUT["bf16"] * (np.abs(want) + bound) + 1.01 * bound, (label, name, a, h))
