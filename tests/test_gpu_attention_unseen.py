"""Attention over the cache on the GPU: what a row sees reaches it, what it does not see does not, in every wave of a tile and at every
scale (against attention_ref.py in 64 bits)."""
import math

import pytest
import torch

import attention_ref as R
from paper_2403_07221_amd import binding as B
from test_gpu_attention import DTYPES, dev, make_attend, run_attend

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    B.lookupffn_init()


def dense(q, cache, table, starts, lengths, causal, window):
    """R.attend's first three results for caches without NaN among the keys, a request's rows at once."""
    heads, dim, (n_blocks, kv, block, _) = q.shape[1], q.shape[2], cache.k.shape
    y, size, reach = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape[:2])
    for r, n in enumerate(lengths):
        first, end = starts[r], starts[r + 1]
        at = table[r][:-(-n // block)]
        k = (cache.k[at].float().double() * cache.k_scale[at].double()[..., None, None]).transpose(0, 1).reshape(kv, -1, dim)[:, :n]
        v = (cache.v[at].float().double() * cache.v_scale[at].double()[..., None, None]).permute(1, 0, 3, 2).reshape(kv, -1, dim)[:, :n]
        where, j = torch.arange(n - (end - first), n)[:, None], torch.arange(n)[None]
        hidden = (j > where) if causal else torch.zeros(where.shape[0], n, dtype=torch.bool)
        if window:
            hidden = hidden | (where - j >= window)
        for h in range(heads):
            x, kh, vh = q[first:end, h].double(), k[h * kv // heads], v[h * kv // heads]
            p = torch.softmax((x @ kh.T / math.sqrt(dim)).masked_fill(hidden, -math.inf), 1)
            y[first:end, h], size[first:end, h] = p @ vh, p @ vh.abs()
            reach[first:end, h] = ((x.abs() @ kh.abs().T).masked_fill(hidden, 0).amax(1) / math.sqrt(dim)).float()
    return y, size, reach


def check_close(y, cache, table, starts, lengths, q, causal, window, take=None, lost=0.0, plain=None):
    """y against the 64-bit form, with no allowance for what other blocks' scales are; `take` picks rows.  lost: what each of a row's
    probabilities may be off by beside its own bits, relative to the row's largest."""
    ref, size, reach = (plain or R.attend)(q.cpu(), *((cache,) if plain else (cache.k, cache.v, cache.k_scale, cache.v_scale)), table, starts,
                                           lengths, causal, window)[:3]
    bound = R.attend_bound_rows(ref, size, reach, q.dtype, q.shape[2], max(lengths))
    if lost:
        bound = bound + lost * max(lengths) * (448 * cache.v_scale[cache.v_scale.isfinite()].abs().max().double())
    y, at = y.cpu().double(), slice(None) if take is None else take
    err = (y - ref)[at].abs()
    assert (err <= bound[at]).all(), f"off by {float((err / bound[at].clamp(min=1e-300)).max())} of the bound, {float(err.max())}"


def without_nan(cache):
    for c in (cache.k, cache.v):
        c.view(torch.uint8)[c.float().isnan()] = 0x38   # 1.0


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


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("what", [math.inf, math.nan, -math.inf])
@pytest.mark.parametrize("side", ["k", "v"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_scales_that_are_not_finite_reach_only_the_rows_that_see_them(shape, side, what, dtype):
    n, fresh, heads, kv, dim, block = shape
    print("scale", shape, side, what, dtype, flush=True)
    column = (n - fresh // 2) // block
    cache, table, starts, q = make_attend(4, [n], [fresh], heads, kv, dim, block, dtype)
    (cache.k_scale if side == "k" else cache.v_scale)[table[0][column], 0] = what
    y = run_attend(cache, table, starts, [n], q)
    group = heads // kv
    free = torch.ones(fresh, heads, dtype=torch.bool)
    free[max(0, column * block - (n - fresh)):, :group] = False
    check_close(y, cache, table, starts, [n], q, True, 0, take=free)
    if side == "v" or math.isnan(what):   # (infinite keys may have scores of minus infinity)
        assert not y.cpu()[~free].isfinite().any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("large", [2.0 ** 20, 2.0 ** 40, 2.0 ** 100])
@pytest.mark.parametrize("window", [0, 24])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_large_scales_after_a_row_and_before_its_window(shape, window, large, dtype):
    """Blocks with scales far above the others', causally after some rows and before the windows of others."""
    n, fresh, heads, kv, dim, block = shape
    print("large", shape, window, large, dtype, flush=True)
    cache, table, starts, q = make_attend(5, [n], [fresh], heads, kv, dim, block, dtype)
    column = (n - fresh // 2) // block
    where = torch.arange(n - fresh, n)
    free = (where < column * block) | ((where - window + 1 >= (column + 1) * block) & (window > 0))
    cache.v_scale[table[0][column]] *= large
    y = run_attend(cache, table, starts, [n], q, True, window)
    check_close(y, cache, table, starts, [n], q, True, window, take=free if dtype == torch.float16 else None)   # (half ends at 65504)
    cache, table, starts, q = make_attend(5, [n], [fresh], heads, kv, dim, block, dtype)
    cache.k_scale[table[0][column]] *= large
    y = run_attend(cache, table, starts, [n], q, True, window)
    check_close(y, cache, table, starts, [n], q, True, window, take=free)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("fresh,dim", [(1, 64), (80, 64), (20, 128), (70, 128), (40, 256)])
def test_large_values_without_weight(fresh, dim, dtype):
    """A block of large values whose scores lie so far below the others' that its part in the sum is small, and a block of small ones."""
    n, block = 200, 16
    print("weight", fresh, dim, dtype, flush=True)
    cache, table, starts, q = make_attend(6, [n], [fresh], 2, 2, dim, block, dtype)
    q.copy_((torch.rand(q.shape, generator=torch.Generator().manual_seed(1)) + 0.5).to(dtype))
    low = table[0][2]
    cache.k[low] = cache.k[low].float().abs().clamp(min=64).neg().to(cache.k.dtype)   # scores of -50 and less
    cache.k_scale[low] = 64 * math.sqrt(dim) / dim / 64
    cache.v_scale[low] *= 2.0 ** 40
    cache.v_scale[table[0][4]] *= 2.0 ** -30
    y = run_attend(cache, table, starts, [n], q)
    check_close(y, cache, table, starts, [n], q, True, 0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("spread", [7, 8, 9, 15, 16])
@pytest.mark.parametrize("fresh,dim", [(90, 64), (40, 128), (140, 128), (90, 256)])
def test_scales_apart(fresh, dim, spread, dtype):
    """Blocks whose scales are up to 2^spread apart, powers of two, with bytes of all sizes."""
    n, block = 400, 32
    print("apart", fresh, dim, spread, dtype, flush=True)
    cache, table, starts, q = make_attend(7, [n], [fresh], 2, 1, dim, block, dtype)
    for i, b in enumerate(table[0][:-1]):
        cache.k_scale[b] = 2.0 ** (-6 - (i * 5 % (spread + 1)))
        cache.v_scale[b] = 2.0 ** (-6 - (i * 3 % (spread + 1)))
        if i % 3 == 0:   # the smallest bytes too
            cache.v[b, :, :, :block // 2] = (cache.v[b, :, :, :block // 2].float() * 2.0 ** -12).to(cache.v.dtype)
    without_nan(cache)
    cache.k_scale[table[0][spread % 3]] = 2.0 ** -6
    cache.v_scale[table[0][spread % 4]] = 2.0 ** -6
    y = run_attend(cache, table, starts, [n], q)
    check_close(y, cache, table, starts, [n], q, True, 0, lost=2.0 ** -33 if dtype != torch.float32 else 0.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("fresh,dim", [(1, 64), (90, 64), (40, 128), (70, 256)])
def test_scales_of_every_kind_in_several_chunks(fresh, dim, dtype):
    """Chunks with powers of two alone beside others with scales of zero, negative ones, the smallest and any mantissa."""
    n, block = 2500, 16
    print("kinds", fresh, dim, dtype, flush=True)
    cache, table, starts, q = make_attend(8, [n], [fresh], 2, 1, dim, block, dtype)
    for i, b in enumerate(table[0][100:-1]):
        cache.k_scale[b] = (0.0, 0.011, -0.02, 2.0 ** -126, 1e-40, 2.0 ** -8)[i % 6]
        cache.v_scale[b] = (0.013, 0.0, 2.0 ** -7, -0.017, 2.0 ** -126, 1e-40)[i % 6]
    y = run_attend(cache, table, starts, [n], q)
    check_close(y, cache, table, starts, [n], q, True, 0, lost=2.0 ** -33 if dtype != torch.float32 else 0.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv,dim,most", [(1, 1, 64, 3), (4, 4, 64, 40), (2, 2, 128, 70), (4, 1, 256, 10)])
@pytest.mark.parametrize("window", [5, 100])
def test_requests_that_bring_more_than_max_queries(window, heads, kv, dim, most, dtype):
    """The rows inside the bound see all their keys, the others are not written."""
    lengths, fresh = [1400, 900, 70], [1000, 2, 60]
    print("more", window, heads, kv, dim, most, dtype, flush=True)
    cache, table, starts, q = make_attend(9, lengths, fresh, heads, kv, dim, 64, dtype)
    inside = torch.zeros(starts[-1], dtype=torch.bool)
    for a, b in zip(starts, starts[1:]):
        inside[a:min(b, a + most)] = True
    for causal in (True, False):
        y = torch.full_like(q, 7.0, memory_format=torch.contiguous_format)
        B.lookupffn_attend(q, *cache.on_gpu(), dev(table), dev(starts), dev(lengths), y=y, causal=causal, window=window, max_queries=most,
                           max_keys=max(lengths))
        assert (y[~inside.cuda()] == 7).all()
        check_close(y, cache, table, starts, lengths, q, causal, window, take=inside, plain=dense)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("fresh", [2, 80])
@pytest.mark.parametrize("window", [0, 1010])
def test_keys_past_the_table_are_not_there(fresh, window, dtype):
    """A request longer than its row of the table: all slots of its last block are keys, and no more."""
    cache, table, starts, q = make_attend(7, [fresh], [fresh], 4, 4, 64, 16, dtype)
    without_nan(cache)
    cut, lengths = [row[:-(-fresh // 16)] for row in table], [fresh + 1000]
    y = B.lookupffn_attend(q, *cache.on_gpu(), dev(cut), dev(starts), dev(lengths), window=window, max_queries=fresh, max_keys=fresh + 1000)
    check_close(y, cache, cut, starts, lengths, q, True, window)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv,dim", [(8, 4, 64), (8, 2, 128), (4, 2, 256)])
def test_rows_are_the_same_every_time(heads, kv, dim, dtype):
    """No sum's order depends on what runs when."""
    lengths, fresh = [1400, 37, 900, 3], [300, 37, 20, 3]
    cache, table, starts, q = make_attend(11, lengths, fresh, heads, kv, dim, 32, dtype)
    on, ints = cache.on_gpu(), [dev(table), dev(starts), dev(lengths)]
    y = [B.lookupffn_attend(q, *on, *ints, max_queries=300, max_keys=1400) for _ in range(6)]
    assert all(torch.equal(y[0], other) for other in y[1:])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("fresh,dim", [(1, 64), (5, 64), (2, 128), (1, 256), (70, 64), (40, 128)])
def test_nan_values_without_weight(fresh, dim, dtype):
    """A NaN value reaches the rows that see it also where its probability is too small for any type."""
    n, heads, kv = 150, 4, 2
    print("nan without weight", fresh, dim, dtype, flush=True)
    for key in (20, n - fresh, 140):
        if key > n - fresh:
            continue
        cache, table, starts, q = make_attend(12, [n], [fresh], heads, kv, dim, 16, dtype)
        q.copy_(torch.ones_like(q))
        at = table[0][key // 16]
        cache.k[at, 0, key % 16], cache.k_scale[at, 0] = -448.0, 1.0     # a score of -448 sqrt(dim)
        cache.v[at, 0, 3, key % 16] = math.nan
        hit = run_attend(cache, table, starts, [n], q).cpu().isnan()
        assert hit[:, :2, 3].all() and int(hit.sum()) == 2 * fresh, key
