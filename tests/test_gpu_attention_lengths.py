"""Attention over the cache on the GPU with lengths that are none: no content of lengths or starts reaches outside the table, and the other
requests' rows are what they are (the arithmetic itself: test_attention_tile.py, on the CPU)."""
import pytest
import torch

from paper_2403_07221_amd import binding as B
from test_gpu_attention import DTYPES, check_attend, dev, make_attend

pytestmark = pytest.mark.gpu
TOP = (1 << 31) - 1


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    B.lookupffn_init()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window", [0, 1, 190, 2000])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("fresh", [1, 3, 70])
@pytest.mark.parametrize("length", [TOP, TOP - 60, 1 << 30])
def test_lengths_up_to_the_largest_int(length, fresh, causal, window, dtype):
    """A request whose length is far past its blocks has its rows at that end: with a window they see nothing; without, all there is."""
    print("lengths", length, fresh, causal, window, dtype, flush=True)
    held = [2304, 700]
    cache, table, starts, q = make_attend(3, held, [fresh, fresh], 4, 2, 64, 16, dtype)
    table = [row[:144] + [-1] * (144 - len(row[:144])) for row in table]
    lengths = [length, 700]
    y = B.lookupffn_attend(q, *cache.on_gpu(), dev(table), dev(starts), dev(lengths), causal=causal, window=window, max_queries=fresh, max_keys=2304)
    if window:
        assert (y[:fresh] == 0).all()
    ref = [2304 + (fresh if causal else 0), 700]   # (its rows stand past the last key)
    check_attend(y[fresh:], cache, table[1:], [0, fresh], [700], q[fresh:], causal, window)
    if not window:
        check_attend(y[:fresh], cache, table[:1], [0, fresh], ref[:1], q[:fresh], causal, window)


@pytest.mark.parametrize("fresh", [1, 70])
def test_plans_whose_sums_stop(fresh):
    """What plan_cache writes for counts that do not fit an int goes into attention as it is."""
    past, new = dev([TOP, 5]), dev([fresh, fresh])
    table = torch.tensor([[1, 2], [3, 4]], dtype=torch.int32, device="cuda")
    starts, lengths, slots, positions, _ = B.lookupffn_plan_cache(past, new, dev([0]), table, 2 * fresh, 128)
    assert lengths.tolist() == [TOP, 5 + fresh] and (slots[:fresh] == -1).all() and (positions[:fresh] == 0).all()
    cache, _, _, q = make_attend(4, [128] * 5, [fresh, fresh], 4, 2, 64, 128, torch.bfloat16)
    assert cache.n_blocks >= 5
    for window in (0, 1, 60):
        y = B.lookupffn_attend(q, *cache.on_gpu(), table, starts, lengths, window=window, max_queries=fresh, max_keys=256)
        assert window == 0 or (y[:fresh] == 0).all()
