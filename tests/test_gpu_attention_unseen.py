"""Attention over the cache on the GPU: what a row sees reaches it, and what it does not see does not, in every wave of a tile."""
import math

import pytest
import torch

from paper_2403_07221_amd import binding as B
from test_gpu_attention import DTYPES, make_attend, run_attend

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    B.lookupffn_init()


SHAPES = [(128, 128, 1, 1, 64, 16), (200, 130, 4, 2, 64, 32), (140, 140, 2, 2, 128, 16), (90, 20, 4, 2, 128, 64), (150, 100, 3, 3, 192, 128),
          (130, 64, 2, 1, 256, 16), (60, 17, 6, 2, 256, 32), (70, 5, 4, 2, 64, 16)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 40), (False, 30)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_nan_values_reach_all_rows_that_see_them(shape, causal, window, dtype):
    """A NaN value at any key: exactly the rows that see it, and only its column, have a NaN."""
    n, fresh, heads, kv, dim, block = shape
    print("nan", shape, causal, window, dtype, flush=True)
    for key in sorted({0, 5, 20, n - fresh, n - fresh + 1, 63, 64, n // 2, n - 1} & set(range(n))):
        cache, table, starts, q = make_attend(3, [n], [fresh], heads, kv, dim, block, dtype)
        cache.v[table[0][key // block], 0, dim - 3, key % block] = math.nan
        y = run_attend(cache, table, starts, [n], q, causal, window).cpu()
        group = heads // kv
        for i in range(fresh):
            where = n - fresh + i
            sees = (not causal or key <= where) and (not window or where - key < window)
            hit = y[i].isnan()
            assert hit[:group, dim - 3].all() == sees and int(hit.sum()) == (group if sees else 0), (key, i, sees)
