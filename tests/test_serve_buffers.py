"""GPU tests of the buffers and streams that a caller of the row calls and the
paged attention may bring."""
import pytest

from paper_2402_07901_amd import fastmax as fm

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
