"""Plain implementations in 64 bits of the entry points beside the layer, on the CPU, with loops over requests: what the tests compare
with.  Written from include/lookupffn.h."""
import math

import torch

U32 = 2.0 ** -24        # half a step of fp32


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def plan(past, fresh, free, table, n_tokens, block):
    """(table, starts, lengths, slots, positions, counts) as lists; the table is a copy."""
    table = [list(row) for row in table]
    starts, lengths, slots, positions, taken = [0], [], [], [], 0
    for r, (p, f) in enumerate(zip(past, fresh)):
        p, f = max(p, 0), max(f, 0)
        have, need = -(-p // block), -(-(p + f) // block)
        for i in range(f):
            at, column = p + i, (p + i) // block
            position, slot = 0, -1
            if column < len(table[r]):
                position = at
                if column < have:
                    slot = table[r][column]
                elif taken + column - have < len(free):
                    slot = free[taken + column - have]
                    if at % block == 0 and len(slots) < n_tokens:
                        table[r][column] = slot
                slot = slot * block + at % block if slot >= 0 else -1
            if len(slots) < n_tokens:
                slots.append(slot)
                positions.append(position)
        taken += need - have
        starts.append(starts[-1] + f)
        lengths.append(p + f)
    left = n_tokens - len(slots)
    return table, starts, lengths, slots + [-1] * left, positions + [0] * left, [taken, starts[-1]]


def turn(x, weight, angles, positions, eps, interleaved):
    """Norm and rotation of x [tokens][heads][dim] in float64."""
    x = x.double()
    if weight is not None:
        x = weight.double() * x / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + eps)
    if angles is None or angles.shape[1] == 0:
        return x
    rot = angles.shape[1]
    row = angles.double()[positions.long().clamp(0, angles.shape[0] - 1)]
    cos, sin = row[:, None, :rot // 2], row[:, None, rot // 2:]
    first = torch.arange(rot // 2) * 2 if interleaved else torch.arange(rot // 2)
    second = first + (1 if interleaved else rot // 2)
    out = x.clone()
    out[..., first] = x[..., first] * cos - x[..., second] * sin
    out[..., second] = x[..., second] * cos + x[..., first] * sin
    return out


def runs(slots, block, n_slots):
    """(first row, rows) of consecutive tokens in consecutive slots of one block."""
    out = []
    for t, s in enumerate(slots):
        if not 0 <= s < n_slots:
            continue
        if out and s % block and slots[t - 1] == s - 1 and out[-1][0] + out[-1][1] == t:
            out[-1][1] += 1
        else:
            out.append([t, 1])
    return out


def scale_for(most):
    if most == 0:
        return 2.0 ** -126
    f, e = math.frexp(most)
    return 2.0 ** max(e - 9 + (f > 0.875), -126)


def attend(q, k_cache, v_cache, k_scale, v_scale, table, starts, lengths, causal, window):
    """(y, weighted mean of |v|, largest sum of |q k| / sqrt(dim), sum of |q| / sqrt(dim) times the request's largest key scale, its largest
    value scale) in float64; keys of blocks that the cache does not have are not seen."""
    n, heads, dim = q.shape
    n_blocks, kv, block, _ = k_cache.shape
    y, size, reach = torch.zeros(n, heads, dim, dtype=torch.float64), torch.zeros(n, heads, dim, dtype=torch.float64), torch.zeros(n, heads)
    coarse_k, coarse_v = torch.zeros(n, heads, dtype=torch.float64), torch.zeros(n, heads, dtype=torch.float64)
    k_all = k_cache.float().double() * k_scale.double()[:, :, None, None]
    v_all = (v_cache.float().double() * v_scale.double()[:, :, None, None]).transpose(2, 3)
    for r, length in enumerate(lengths):
        first, rows = starts[r], starts[r + 1] - starts[r]
        ids = [i for i in table[r][:max(0, -(-length // block))]]
        at = torch.tensor([i if 0 <= i < n_blocks else 0 for i in ids], dtype=torch.long)
        there = torch.tensor([0 <= i < n_blocks for i in ids], dtype=torch.bool).repeat_interleave(block)[:length]
        count = there.numel()
        if rows == 0 or count == 0:
            continue
        k, v = [x[at].transpose(0, 1).reshape(kv, -1, dim)[:, :count] for x in (k_all, v_all)]
        where, j = torch.arange(length - rows, length)[:, None], torch.arange(count)[None]
        seen = there[None].expand(rows, count).clone()
        if causal:
            seen &= j <= where
        if window:
            seen &= where - j < window
        for h in range(heads):
            if there.any():
                used = at[there[::block]]
                coarse_k[first:first + rows, h] = q[first:first + rows, h].double().abs().sum(-1) / math.sqrt(dim) * k_scale[used, h * kv // heads].max()
                coarse_v[first:first + rows, h] = v_scale[used, h * kv // heads].max()
            kh, vh, qh = k[h * kv // heads], v[h * kv // heads], q[first:first + rows, h].double()
            for i in range(rows):
                on = seen[i]
                if not on.any():
                    continue
                s = kh[on] @ qh[i] / math.sqrt(dim)
                p = torch.softmax(s, 0)
                y[first + i, h] = p @ vh[on]
                size[first + i, h] = p @ vh[on].abs()
                reach[first + i, h] = float((kh[on].abs() @ qh[i].abs()).max()) / math.sqrt(dim)
    return y, size, reach, coarse_k, coarse_v


def attend_bound(y, size, reach, coarse_k, coarse_v, dtype, dim, most_keys):
    """How far the kernel's y may be off, element by element.

    Rounding the output; the score's fp32 sum of dim products (off by at most dim u reach, u = 2^-24), its multiplication by the scale and
    the subtraction of the maximum before the power (3 u of a number up to 2 log2(e) reach), which move a probability by that times its
    size, and numerator and denominator both; the rounding of the probabilities (half: 2^-12 of each; fp32 rows 2^-23) and the exponential
    (2 u); the fp32 sums over the keys, 32 products at a time, then four waves and the chunks.  Keys of half rows, and values of 16-bit rows,
    are half numbers relative to a power of two no larger than the largest scale: off by 2^-25 of that."""
    score = (dim + 9) * U32 * reach.double()[..., None]
    if dtype == torch.float16:
        score = score + 2.0 ** -25 * coarse_k[..., None]
    piece = 2.0 ** -23 if dtype == torch.float32 else 2.0 ** -12
    sums = (most_keys / 32 + 40) * U32
    out = half_step(dtype) * y.abs() + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    coarse = 0.0 if dtype == torch.float32 else 2.0 ** -25 * coarse_v[..., None]
    return out + (size * (2 * score + piece + 4 * U32 + 2 * sums) + coarse) * (1 + half_step(dtype))


def attend_bound_rows(y, size, reach, dtype, dim, most_keys):
    """As attend_bound, of rows that no block's scale touches but those they see: nothing is allowed for the largest scale of the request.

    A rounding to half is off by half a step, 2^-11 of the value (the 2^-12 of attend_bound holds at the top of a binade only); two bf16 pieces are off by
    less.  The matrix cores may take a product's factor below 2^-126 as zero, of up to 448 times each key, and fp32 holds no number below that
    with all its bits."""
    score = (dim + 9) * U32 * reach.double()[..., None]
    piece = 2.0 ** -23 if dtype == torch.float32 else 2.0 ** -11
    sums = (most_keys / 32 + 40) * U32
    out = half_step(dtype) * y.abs() + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    return out + size * (2 * score + piece + 4 * U32 + 2 * sums) * (1 + half_step(dtype)) + 449 * most_keys * 2.0 ** -126
