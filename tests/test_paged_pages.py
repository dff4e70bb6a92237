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
