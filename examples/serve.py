"""A few transformer layers whose feed-forward half is a LookupFFN layer, served from an 8-bit cache: ragged prompts, then single tokens.

    python examples/serve.py [--layers 4] [--requests 16] [--prompt 500] [--steps 64]

Random weights (synth.make_layer for the lookup half), synthetic inputs: what a step returns for a request's last token is fed back as its
next one.  A step is lookupffn_plan_cache once, then in every layer lookupffn_rotate_append, lookupffn_attend and lookupffn_forward between
two plain projections.
"""
from __future__ import annotations

import argparse
import sys
import time
from pathlib import Path

import torch

if str(Path(__file__).resolve().parent.parent) not in sys.path:
    sys.path.insert(0, str(Path(__file__).resolve().parent.parent))

from paper_2403_07221_amd import binding as B
from paper_2403_07221_amd import synth


def angle_table(positions: int, rot: int) -> torch.Tensor:
    """[positions, rot] float32: the cosines, then the sines, of position / 10000^(2 i / rot), taken in 64 bits."""
    a = torch.arange(positions, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.cat([a.cos(), a.sin()], 1).float()


class Cache:
    """One layer's keys and values in e4m3, with a scale for each block and head."""

    def __init__(self, n_blocks: int, kv_heads: int, block: int, dim: int):
        self.k = torch.zeros(n_blocks, kv_heads, block, dim, dtype=torch.float8_e4m3fn, device="cuda")
        self.v = torch.zeros(n_blocks, kv_heads, dim, block, dtype=torch.float8_e4m3fn, device="cuda")
        self.k_scale, self.v_scale = torch.zeros(n_blocks, kv_heads, device="cuda"), torch.zeros(n_blocks, kv_heads, device="cuda")

    def __iter__(self):
        return iter((self.k, self.v, self.k_scale, self.v_scale))


class Layer:
    def __init__(self, w: synth.Workload, index: int, heads: int, kv_heads: int, dim: int, n_blocks: int, block: int):
        g = torch.Generator().manual_seed(index)
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        wide = (heads + 2 * kv_heads) * dim
        self.qkv = (torch.randn(w.d, wide, generator=g) / w.d ** 0.5).to(torch.bfloat16).cuda()
        self.out = (torch.randn(heads * dim, w.d, generator=g) / (heads * dim) ** 0.5).to(torch.bfloat16).cuda()
        self.norm = torch.ones(dim, device="cuda")
        _, signs, tables = synth.make_layer(w, index, with_x=False)
        self.signs, self.tables = B.to_device(signs), B.lookupffn_prepare_tables(B.to_device(tables))
        self.cache = Cache(n_blocks, kv_heads, block, dim)

    def __call__(self, x: torch.Tensor, step: Step) -> torch.Tensor:
        n = x.shape[0]
        rows = (torch.nn.functional.rms_norm(x, x.shape[1:]).to(torch.bfloat16) @ self.qkv).view(n, -1, self.dim)
        q, k, v = rows.split([self.heads, self.kv_heads, self.kv_heads], 1)
        q = B.lookupffn_rotate_append(q, k, v, self.norm, self.norm, step.angles, step.positions, step.slots, *self.cache)
        y = B.lookupffn_attend(q, *self.cache, step.table, step.starts, step.lengths, max_queries=step.max_queries, max_keys=step.max_keys)
        x = x + (y.view(n, -1) @ self.out).float()
        return x + B.lookupffn_forward(torch.nn.functional.rms_norm(x, x.shape[1:]), self.signs, self.tables)


class Step:
    """What all layers of a step share."""


class Server:
    def __init__(self, layers: int, requests: int, longest: int, w: synth.Workload = synth.C2, heads: int = 12, kv_heads: int = 12,
                 dim: int = 64, block: int = 16):
        B.lookupffn_init()
        self.block, width = block, -(-longest // block)
        n_blocks = requests * width
        self.layers = [Layer(w, i, heads, kv_heads, dim, n_blocks, block) for i in range(layers)]
        self.table = torch.full((requests, width), -1, dtype=torch.int32, device="cuda")
        self.free = torch.randperm(n_blocks, generator=torch.Generator().manual_seed(0)).to(torch.int32).cuda()
        self.angles = angle_table(longest, dim).cuda()
        self.past = [0] * requests

    def step(self, x: torch.Tensor, fresh: list[int]) -> torch.Tensor:
        """x[sum of fresh, d], the new tokens request by request, through all layers; their keys and values stay in the cache.  A step that
        does not fit is refused before anything changes."""
        if len(fresh) != len(self.past) or min(fresh) < 0 or sum(fresh) != x.shape[0]:
            raise ValueError(f"{len(self.past)} requests bring {fresh}: {x.shape[0]} tokens")
        if max(p + f for p, f in zip(self.past, fresh)) > self.angles.shape[0]:
            raise ValueError(f"a request would be longer than {self.angles.shape[0]} tokens")
        taken = sum(-(-(p + f) // self.block) - -(-p // self.block) for p, f in zip(self.past, fresh))
        if taken > self.free.numel():
            raise ValueError("the cache has too few blocks left")
        s = Step()
        past = torch.tensor(self.past, dtype=torch.int32, device="cuda")
        s.starts, s.lengths, s.slots, s.positions, _ = B.lookupffn_plan_cache(
            past, torch.tensor(fresh, dtype=torch.int32, device="cuda"), self.free, self.table, x.shape[0], self.block)
        self.free = self.free[taken:]
        self.past = [p + f for p, f in zip(self.past, fresh)]
        s.table, s.angles, s.max_queries, s.max_keys = self.table, self.angles, max(fresh), max(self.past)
        for layer in self.layers:
            x = layer(x, s)
        return x


def main() -> None:
    ap = argparse.ArgumentParser()
    for name, value in (("layers", 4), ("requests", 16), ("prompt", 500), ("steps", 64)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    g = torch.Generator().manual_seed(1)
    server = Server(a.layers, a.requests, a.prompt + a.steps)
    fresh = torch.randint(1, a.prompt + 1, (a.requests,), generator=g).tolist()
    x = torch.randn(sum(fresh), synth.C2.d, generator=g).cuda()
    last = torch.tensor(fresh).cumsum(0).cuda() - 1
    x = server.step(x, fresh)[last]
    torch.cuda.synchronize()
    begin = time.perf_counter()
    for _ in range(a.steps):
        x = server.step(x, [1] * a.requests)
    torch.cuda.synchronize()
    took = time.perf_counter() - begin
    print(f"{sum(fresh)} prompt tokens, {a.steps} steps of {a.requests}: {took / a.steps * 1e6:.0f} us a step of {a.layers} layers, "
          f"finite: {bool(torch.isfinite(x).all())}")


if __name__ == "__main__":
    main()
