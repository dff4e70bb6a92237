"""GPU tests of page tables: entries that are no page, evicted pages under
chunks, sequences longer than their row of the table, views of caches."""
import numpy as np
import pytest

from paper_2402_07901_amd import fastmax as fm

import serve_util as su
from gpu_util import say
from paged_util import check_rows, positions
from test_paged import Cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fm.lib()
    yield
    torch.cuda.synchronize()


CHUNKS = [
    # lens, news, Hq, Hkv, page, entry that is no page, window, sinks
    ([100, 60], [20, 3], 2, 2, 32, 3, 0, 0),          # few rows
    ([110, 60], [30, 1], 2, 1, 32, 2, 8, 0),          # the rows past the window are whole
    ([700, 130], [400, 70], 4, 1, 32, 20, 0, 0),      # many rows
    ([700, 130], [400, 70], 4, 2, 64, 6, 100, 40),
    ([4000, 20], [100, 20], 4, 2, 64, 62, 0, 0),      # splits that are joined
    ([900, 20], [600, 20], 4, 1, 16, 0, 50, 5),       # a page of first tokens: every row
]


@pytest.mark.parametrize("dtype,D", [("bf16", 16), ("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("lens,news,Hq,Hkv,page,i,window,sinks", CHUNKS)
def test_rows_that_see_no_bad_page_are_whole(dtype, D, lens, news, Hq, Hkv, page, i, window,
                                             sinks):
    """A page that is not there makes NaN of the rows that see one of its keys;
    their neighbours in a tile of rows, and other sequences, keep their values."""
    say(f"bad page {i} D={D} {dtype} lens={lens} new={news} window={window}")
    for entry in (-1, 10 ** 6, 2 ** 31 - 1, -2 ** 31):
        c = Cache(lens, news, Hq, Hkv, D, page, dtype, seed=i)
        c.table[0, i] = entry
        out = c.run(max_q=max(news), window=window, sinks=sinks)
        pos = positions(c, 0)
        keys = np.arange(i * page, min((i + 1) * page, lens[0]))
        see = keys[None] <= pos[:, None]
        if window:
            see &= (keys[None] > pos[:, None] - window) | (keys[None] < sinks)
        see = see.any(1)
        assert see.any()
        got = su.np64(out[:news[0]])
        assert np.isnan(got[see]).all(), entry
        check_rows(c, out, 0, ~see, entry, window=window, sinks=sinks)
        check_rows(c, out, 1, np.ones(news[1], bool), entry, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype,D", [("bf16", 16), ("bf16", 64), ("f32", 64)])
def test_chunk_of_a_sequence_longer_than_its_table(dtype, D):
    import torch
    c = Cache([640, 200], [300, 200], 4, 2, D, 32, dtype, cols=20)
    c.lens[0] = 641
    out = c.run(max_q=300, max_len=640)
    assert torch.isnan(out[:300]).all()
    check_rows(c, out, 1, np.ones(200, bool), "the other sequence")


@pytest.mark.parametrize("dtype,D", [("bf16", 16), ("bf16", 64), ("bf16", 128), ("f32", 32),
                                     ("f32", 128)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (33, 0), (64, 16), (100, 33), (500, 1)])
def test_evicted_pages_under_chunks(dtype, D, window, sinks):
    """Pages that no new token of a sequence sees are gone: what they hold and
    their entries are not used, for few rows and for many."""
    say(f"evicted pages D={D} {dtype} window={window} sinks={sinks}")
    lens, news, page = [20, 333, 801, 1000, 1500], [3, 40, 1, 90, 300], 32
    c = Cache(lens, news, 6, 2, D, page, dtype, seed=window)
    for s, (n, new) in enumerate(zip(lens, news)):
        for i in range(-(-n // page)):
            if i * page >= sinks and (i + 1) * page - 1 <= n - new - window:
                gone = int(c.table_h[s, i])
                c.k[gone], c.v[gone] = float("nan"), float("inf")
                c.table[s, i] = -1 if i % 2 else 2 ** 31 - 1
    out = c.run(max_q=300, window=window, sinks=sinks)
    c.check(out, (window, sinks), window=window, sinks=sinks, starts=False)
    few = c.run(max_q=1, window=window, sinks=sinks)
    c.check(few, (window, sinks, "few"), window=window, sinks=sinks, starts=False)


@pytest.mark.parametrize("pages,Hkv", [(6, 1), (1, 2), (1, 1)])
def test_caches_that_differ_where_no_stride_counts(pages, Hkv):
    """One key head, or one page: the caches' strides along it may differ."""
    import torch
    page, D, n = 64, 64, min(pages * 64, 300)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(pages)
    kc = torch.zeros((pages, Hkv, page, D), dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros((3 * pages, Hkv, page, D), dtype=torch.bfloat16, device="cuda")
    vc = vc[::3] if pages == 1 else vc[:pages].reshape(pages, page, Hkv, D).transpose(1, 2)
    assert kc.stride() != vc.stride() and kc.shape == vc.shape
    q, k, v = (torch.randn((n, h, D), generator=gen, device="cuda").bfloat16()
               for h in (4, Hkv, Hkv))
    table = torch.randperm(pages, device="cuda").to(torch.int32)[None]
    at = torch.arange(n, device="cuda")
    slots = table[0].long()[at // page] * page + at % page
    qh = fm.fastmax_cache_append(q, k, v, kc, vc, slots, None, None, None)
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    out = fm.fastmax_paged_fwd(qh[-1:], kc, vc, table, lens)
    rows = [x[table[0].long()].transpose(0, 1).reshape(Hkv, -1, D)[:, :n] for x in (kc, vc)]
    assert torch.equal(rows[1], v.transpose(0, 1))
    g = 4 // Hkv
    for h in range(Hkv):
        hs = slice(g * h, g * h + g)
        ref, bound = su.attend(su.np64(qh[-1:, hs]), su.np64(rows[0][h]), su.np64(rows[1][h]),
                               np.array([n - 1]), 2, 1.0, 0, 0)
        su.check(out[:, hs], ref, su.OUT["bf16"] * np.abs(ref) + 1.01 * bound, h)
