"""GPU tests of the packed attention past 32-bit offsets: the most rows that a call
takes, and rows and gradients of more than 2^32 elements, against float64."""
import numpy as np
import pytest

from paper_2402_07901_amd import fastmax as fm

import serve_util as su
from gpu_util import say
from packed_util import OUT, Head

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fm.lib()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


class Far:
    """bf16 rows of T tokens, short sequences at either end, a call's each; the rows
    between are of no sequence and hold anything."""

    def __init__(self, T, Hq, Hkv, D):
        import torch
        self.spans = [(0, 70), (T - 333, T - 33), (T - 33, T)]
        gen = torch.Generator(device="cuda")
        gen.manual_seed(1)

        def rows(H):
            x = torch.empty((T, H, D), dtype=torch.bfloat16, device="cuda")
            for a, b in self.spans:
                x[a:b] = torch.randn((b - a, H, D), generator=gen, device="cuda")
            return x

        self.q, self.k, self.v, self.group = rows(Hq), rows(Hkv), rows(Hkv), Hq // Hkv
        self.rows = rows
        self.calls = [(torch.tensor(s, dtype=torch.int32, device="cuda"), spans)
                      for s, spans in (([0, 70], self.spans[:1]), ([T - 333, T - 33, T], self.spans[1:]))]

    def heads(self, a, b):
        for h in range(self.k.shape[1]):
            hs = slice(h * self.group, (h + 1) * self.group)
            yield h, hs, Head(su.np64(self.q[a:b, hs]), su.np64(self.k[a:b, h]), su.np64(self.v[a:b, h]),
                              2, 1.0, True, "bf16")


def test_most_rows():
    say("packed, 2^30 rows")
    x = Far(1 << 26, 16, 1, 16)
    for starts, spans in x.calls:
        out, g = fm.fastmax_packed_fwd(x.q, x.k, x.v, starts, causal=True)
        for a, b in spans:
            for h, hs, head in x.heads(a, b):
                O, eO, G, eG = head.forward()
                su.check(out[a:b, hs], O, OUT["bf16"] * np.abs(O) + 1.01 * eO, ("2^30 rows", a, h))
                su.check(g[a:b, hs], G, 1.01 * eG, ("2^30 rows", a, h))
        del out, g


def test_gradients_past_32_bits():
    import torch
    say("packed, gradients past 2^32 elements")
    x = Far((1 << 22) + 77, 8, 2, 128)
    assert x.q.numel() > 2 ** 32
    dout = x.rows(8)
    for starts, spans in x.calls:
        out, g = fm.fastmax_packed_fwd(x.q, x.k, x.v, starts, causal=True)
        heads = [(a, b, *y) for a, b in spans for y in x.heads(a, b)]
        for a, b, h, hs, head in heads:
            O, eO, G, eG = head.forward()
            su.check(out[a:b, hs], O, OUT["bf16"] * np.abs(O) + 1.01 * eO, ("far", a, h))
            su.check(g[a:b, hs], G, 1.01 * eG, ("far", a, h))
            # the definition's, for the backward's bounds
            out[a:b, hs], g[a:b, hs] = torch.from_numpy(O).cuda().to(out.dtype), torch.from_numpy(G).cuda().float()
        dq, dk, dv = fm.fastmax_packed_bwd(x.q, x.k, x.v, starts, out, dout, g, causal=True)
        for a, b, h, hs, head in heads:
            ref = head.backward(su.np64(dout[a:b, hs]), OUT["bf16"])
            got = (dq[a:b, hs], dk[a:b, h], dv[a:b, h])
            for name, y, (want, bound) in zip(("dq", "dk", "dv"), got, ref):
                su.check(y, want, OUT["bf16"] * (np.abs(want) + bound) + 1.01 * bound, ("far", name, a, h))
        del out, g, dq, dk, dv
