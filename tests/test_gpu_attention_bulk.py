"""Rotation and append of steps large enough for the forms that small ones do not take: several rows to a lane group, streamed outputs, a
block's tokens to a workgroup, many runs in one and runs that cross tiles (against attention_ref.py in 64 bits)."""
import random

import pytest
import torch

import attention_ref as R
from paper_2403_07221_amd import binding as B
from test_gpu_attention import Cache, DTYPES, angle_table, check_append, dev, row_bound, rows, same_bytes, step_slots

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    B.lookupffn_init()


def check_rows(y, x, weight, angles, positions, eps, inter):
    ref = turn_parts(x, weight, angles, positions, eps, inter)
    err, bound = (y.double() - ref).abs(), row_bound(x, ref, weight, x.dtype, eps)
    assert (err <= bound).all(), float((err / bound).max())


def turn_parts(x, weight, angles, positions, eps, inter):
    """R.turn on the GPU, in parts that fit beside each other."""
    return torch.cat([R.turn(x[i:i + 2048], weight, angles, positions[i:i + 2048], eps, inter) for i in range(0, x.shape[0], 2048)])


# tokens, query and key heads, dim, rotated columns: rows over those of a workgroup are 4096 and more
BULK = [(3700, 30, 7, 128, 128), (9500, 21, 7, 64, 32), (4100, 13, 3, 256, 256), (5200, 6, 1, 512, 128), (6600, 17, 5, 80, 48), (15000, 13, 5, 48, 48),
        (3700, 29, 8, 128, 6)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout,inter", [("slice", False), ("slice", True), ("odd", False)])
@pytest.mark.parametrize("shape", BULK, ids=lambda s: "-".join(map(str, s)))
def test_rotate_many_rows(shape, layout, inter, dtype):
    n, h, kv, dim, rot = shape
    print("rotate", shape, inter, layout, dtype, flush=True)
    lanes = 1
    while lanes * 16 < dim:
        lanes *= 2
    assert n * (h + kv) // (256 // lanes) >= 4096
    q, k = rows(1, n, h, dim, dtype, layout), rows(2, n, kv, dim, dtype, layout)
    g = torch.Generator().manual_seed(3)
    qw, kw = [(1 + 0.3 * torch.randn(dim, generator=g)).cuda() for _ in range(2)]
    angles, positions = angle_table(4000, rot).cuda(), torch.randint(0, 4000, (n,), generator=g, dtype=torch.int32).cuda()
    got = B.lookupffn_rotate(q, k, qw, kw, angles, positions, eps=1e-5, interleaved=inter)
    check_rows(got[0], q, qw, angles, positions, 1e-5, inter)
    check_rows(got[1], k, kw, angles, positions, 1e-5, inter)
    want = [t.clone() for t in got]
    q_in, k_in = q.clone(), k.clone()
    B.lookupffn_rotate(q_in, k_in, qw, kw, angles, positions, q_out=q_in, k_out=k_in, eps=1e-5, interleaved=inter)
    assert torch.equal(q_in, want[0]) and torch.equal(k_in, want[1])


def mixed(seed, block, singles, prompts):
    """Requests that bring single tokens, a few, or prompts over several blocks, in any order."""
    rng = random.Random(seed)
    out = [(rng.randrange(block), 1) for _ in range(singles)] + [(rng.randrange(block), rng.randint(2, block // 2)) for _ in range(singles // 8)]
    out += [(rng.randrange(block), rng.randint(block, 4 * block)) for _ in range(prompts)] + [(0, block), (0, 2 * block), (block - 1, 1 + block)]
    rng.shuffle(out)
    return out


# block, dim, query and key heads, rotated columns, pairs of neighbours, single tokens, prompts
STEPS = [(16, 64, 12, 12, 64, False, 340, 6), (32, 128, 32, 8, 128, False, 500, 4), (64, 128, 8, 4, 128, True, 700, 12), (128, 256, 6, 2, 128, False, 300, 14),
         (128, 64, 4, 4, 64, False, 1000, 3), (16, 256, 5, 5, 0, False, 800, 9), (64, 80, 9, 3, 48, True, 100, 15), (128, 16, 9, 9, 4, False, 460, 1)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ["slice", "odd"])
@pytest.mark.parametrize("step", STEPS, ids=lambda s: "-".join(map(str, s)))
def test_append_many_runs(step, layout, dtype):
    block, dim, heads, kv, rot, inter, singles, prompts = step
    print("append", step, layout, dtype, flush=True)
    lengths = mixed(block + dim, block, singles, prompts)
    cache = Cache(5, sum(-(-(p + f) // block) for p, f in lengths) + 3, kv, block, dim)
    slots, positions = step_slots(6, block, cache.n_blocks, lengths)
    n = len(slots)
    assert n * kv * 2 > 8192
    q, k, v = [rows(7 + j, n, h, dim, dtype, layout) for j, h in enumerate((heads, kv, kv))]
    w = 1 + 0.3 * torch.randn(dim, generator=torch.Generator().manual_seed(8))
    angles = angle_table(6 * block, rot) if rot else None
    at = torch.tensor(positions, dtype=torch.int32)
    args = (w.cuda(), w.cuda(), angles.cuda() if rot else None, at.cuda() if rot else None)
    on = cache.on_gpu()
    out = B.lookupffn_rotate_append(q, k, v, *args, dev(slots), *on, interleaved=inter)
    check_rows(out, q, args[0], args[2], at.cuda(), 1e-6, inter)
    want = R.turn(k.cpu(), w, angles, at, 1e-6, inter)
    check_append(cache, on, want, slots, False, row_bound(k.cpu(), want, w, torch.float32, 1e-6))
    check_append(cache, on, v.cpu().double(), slots, True, torch.zeros_like(want))
    again = [t.clone() for t in on]
    B.lookupffn_rotate_append(q, k, v, *args, dev(slots), *again, interleaved=inter)
    assert torch.equal(again[2], on[2]) and torch.equal(again[3], on[3]) and same_bytes(again[0], on[0]) and same_bytes(again[1], on[1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv,dim,inter", [(32, 8, 128, False), (12, 12, 64, True), (6, 2, 256, False)])
def test_append_of_long_prompts(heads, kv, dim, inter, dtype):
    """Prompts whose query rows go several to a lane group, and are streamed, beside the blocks."""
    block, lengths = 64, [(0, 2900), (70, 1), (30, 2800), (63, 5700)]
    if dim == 64:
        lengths = [(0, 9000), (70, 1), (30, 8000), (63, 5700)]
    print("append", heads, kv, dim, inter, dtype, flush=True)
    lengths = [(p % block, f) for p, f in lengths]
    cache = Cache(5, sum(-(-(p + f) // block) for p, f in lengths) + 3, kv, block, dim)
    slots, positions = step_slots(6, block, cache.n_blocks, lengths)
    n = len(slots)
    lanes = dim // 16
    assert n * heads // (256 // lanes) >= 4096
    q, k, v = [rows(7 + j, n, h, dim, dtype, "slice") for j, h in enumerate((heads, kv, kv))]
    w = (1 + 0.3 * torch.randn(dim, generator=torch.Generator().manual_seed(8))).cuda()
    angles, at = angle_table(10000, dim).cuda(), dev(positions)
    on = cache.on_gpu()
    out = B.lookupffn_rotate_append(q, k, v, w, w, angles, at, dev(slots), *on, interleaved=inter)
    check_rows(out, q, w, angles, at, 1e-6, inter)
    want = turn_parts(k, w, angles, at, 1e-6, inter).cpu()
    check_append(cache, on, want, slots, False, row_bound(k.cpu(), want, w.cpu(), torch.float32, 1e-6))
    check_append(cache, on, v.cpu().double(), slots, True, torch.zeros_like(want))
