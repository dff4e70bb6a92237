"""GPU tests of the buffers and streams that a caller of the row calls and the
paged attention may bring, and of calls repeated on the same data."""
import pytest

from paper_2402_07901_amd import fastmax as fm

from gpu_util import say
from test_paged import Cache
from test_rows import Rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fm.lib()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_own_buffers_of_the_rows(dtype):
    import torch
    r = Rows(2, 37, 6, 2, 64, dtype)
    want = fm.fastmax_rope_fwd(r.q, r.k, r.v, **r.kw())
    out = [torch.full_like(w, float("nan")) for w in want]
    got = fm.fastmax_rope_fwd(r.q, r.k, r.v, out=out, **r.kw())
    for a, b, o in zip(got, want, out):
        assert a.data_ptr() == o.data_ptr() and torch.equal(a, b)
    ups = [torch.randn_like(w) for w in want]
    want = fm.fastmax_rope_bwd(r.q, r.k, *ups, **r.kw())
    ws = torch.empty(fm.rope_workspace_bytes(2, 37, 6, 2, 64, True), dtype=torch.uint8,
                     device="cuda")
    got = fm.fastmax_rope_bwd(r.q, r.k, *ups, workspace=ws, **r.kw())
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    with pytest.raises(fm.FastmaxError):
        fm.fastmax_rope_bwd(r.q, r.k, *ups, workspace=ws[:-16], **r.kw())


def test_own_buffers_and_stream_of_the_append():
    import torch
    r = Rows(1, 50, 6, 2, 64, "bf16")
    kw = dict(r.kw(), pos=r.pos[0])
    slots = torch.randperm(128, device="cuda")[:50]
    kv = [torch.zeros((2, 4, 2, 32, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    want = fm.fastmax_cache_append(r.q[0], r.k[0], r.v[0], kv[0][0], kv[0][1], slots, **kw)
    q_out = torch.full_like(want, float("nan"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = fm.fastmax_cache_append(r.q[0], r.k[0], r.v[0], kv[1][0], kv[1][1], slots, q_out=q_out,
                                  stream=side, **kw)
    side.synchronize()
    assert got.data_ptr() == q_out.data_ptr()
    assert torch.equal(got, want) and torch.equal(kv[0], kv[1])


def test_allocations_of_the_null_stream():
    """Handle 0 is the null stream, and what the call allocates is its own."""
    import torch
    with fm._owner(0, torch.device("cuda", torch.cuda.current_device())):
        assert torch.cuda.current_stream().cuda_stream == 0
    r = Rows(1, 50, 6, 2, 64, "bf16")
    want = fm.fastmax_rope_fwd(r.q, r.k, r.v, **r.kw())
    torch.cuda.synchronize()
    got = fm.fastmax_rope_fwd(r.q, r.k, r.v, stream=0, **r.kw())
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_workspaces_in_the_wrong_place_are_refused():
    import torch
    r = Rows(1, 50, 6, 2, 64, "bf16")
    ups = [torch.randn((1, 6, 50, 64), device="cuda").bfloat16() for _ in range(3)]
    need = fm.rope_workspace_bytes(1, 50, 6, 2, 64, True)
    kv = torch.zeros((2, 8, 2, 1024, 64), dtype=torch.bfloat16, device="cuda")
    table = torch.arange(8, dtype=torch.int32, device="cuda")[None]
    lens = torch.full((1,), 8192, dtype=torch.int32, device="cuda")
    paged = fm.paged_workspace_bytes(1, 1, 6, 2, 64, 1, 8192, 0, 0, fm.BF16)
    assert need > 0 and paged > 0
    for bad in (torch.empty(max(need, paged), dtype=torch.uint8),
                torch.empty(2 * max(need, paged), dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError, match="workspace"):
            fm.fastmax_rope_bwd(r.q, r.k, *ups, workspace=bad, **r.kw())
        with pytest.raises(ValueError, match="workspace"):
            fm.fastmax_paged_fwd(r.q[0, :1], *kv, table, lens, workspace=bad)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_equal_calls_give_equal_bits(dtype, D):
    """Splits, joins and pieces add in a fixed order."""
    import torch
    say(f"repeat D={D} {dtype}")
    one = Cache([9000, 777, 40], [1, 1, 1], 8, 2, D, 64, dtype)
    many = Cache([4000, 333], [200, 333], 8, 2, D, 64, dtype)
    first = [one.run(starts=False), many.run(max_q=333)]
    for _ in range(5):
        for a, b in zip(first, (one.run(starts=False), many.run(max_q=333))):
            assert torch.equal(a, b)
