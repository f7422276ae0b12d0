"""Conversations behind one system prompt over the paged KV cache, one engine step after the other.

The prompt is appended once; its whole pages stand in every conversation's page table, and what is left of it in each one's first page of its
own.  Every step appends its tokens with kv_append_rotated (keys and queries rotated by their positions on the way) and attends with
prefix_attention, layer by layer: a first turn of some tokens for each conversation, then decode steps.  In the end the prompt's
keys are read once for all conversations.

There is no model here: queries, keys and values are random.  What is real is the cache; --check compares every step's attention with plain
products over what should be there.

    python examples/shared_prompt.py [--steps 6] [--check]
"""
import argparse
import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2603_13358_amd as ppd  # noqa: E402

PAGE = 16


class Cache:
    """Pools of all layers and a page table, and what a plain program would hold: rotated K, and V, of every conversation."""

    def __init__(self, layers, hq, hkv, dim, batch, prompt, most, fp8, check):
        self.layers, self.hq, self.hkv, self.dim, self.batch, self.prompt = layers, hq, hkv, dim, batch, prompt
        shared, own = prompt // PAGE, (most + PAGE - 1) // PAGE
        pages = shared + batch * own
        self.ctx = ppd.Context(hq, hkv, dim, pages)
        self.scale = 2.0 ** -5 if fp8 else 1.0
        if fp8:
            self.ctx.set_kv_format(ppd.PPD_KV_FP8_E4M3, self.scale, self.scale)
        self.inv_freq = ppd.ppd_rope_frequencies(dim, 500000.0, ppd.PPD_ROPE_SCALE_BY_PARTS, 4.0, 2048.0)
        self.amplitude = 1.1
        self.ctx.set_rope(self.inv_freq, ppd.PPD_ROPE_HALF, self.amplitude)
        self.pools = torch.zeros((layers, self.ctx.pool_elems()), dtype=torch.uint8 if fp8 else torch.bfloat16, device="cuda")
        perm = np.random.default_rng(0).permutation(pages).astype(np.int32)
        self.table = np.concatenate([np.repeat(perm[None, :shared], batch, 0), perm[shared:].reshape(batch, own)], 1)
        self.table_dev = torch.from_numpy(np.ascontiguousarray(self.table)).cuda()
        self.L = np.zeros(batch, np.int32)
        self.plain = [[[torch.zeros((0, hkv, dim), dtype=torch.float64, device="cuda") for _ in "kv"] for _ in range(batch)] for _ in range(layers)] if check else None

    def slots(self, b, positions):
        return self.table[b, positions // PAGE].astype(np.int64) * PAGE + positions % PAGE

    def turned(self, x, positions):
        """x [row, head, d] rotated in 64 bits."""
        t = torch.from_numpy(positions).cuda().double()[:, None] * torch.from_numpy(self.inv_freq).cuda()
        z = torch.complex(*x.double().chunk(2, -1)) * torch.polar(torch.full_like(t, self.amplitude), t)[:, None]
        return torch.cat([z.real, z.imag], -1)

    def held(self, x):
        """What pages hold of a 64-bit value."""
        if self.scale == 1.0:
            return x.float().to(torch.bfloat16).double()
        return (x / self.scale).float().clamp(-448, 448).to(torch.float8_e4m3fn).double() * self.scale

    def append(self, layer, of, positions):
        """Random rows of a projection for tokens `positions` of conversations `of`: keys and values go to the pages, queries come back
        rotated."""
        rows = torch.randn((len(of), self.hq + 2 * self.hkv, self.dim), device="cuda").to(torch.bfloat16)
        q, k, v = rows[:, :self.hq], rows[:, self.hq:self.hq + self.hkv], rows[:, self.hq + self.hkv:]
        slots = self.slots(of, positions)
        out = torch.empty((len(of), self.hq, self.dim), dtype=torch.bfloat16, device="cuda")
        self.ctx.kv_append_rotated(q, k, v, torch.from_numpy(positions).cuda(), self.pools[layer], torch.from_numpy(slots).cuda(), out)
        return q, k, v, out


def worst_error(cache, layer, n, q, out):
    """Largest difference from plain attention, in units of what the roundings may come to (bf16 queries, probabilities and results)."""
    worst, at, group = 0.0, 0, cache.hq // cache.hkv
    for b in range(cache.batch):
        rows, k, v = int(n[b]), *cache.plain[layer][b]
        seen = torch.arange(len(k), device="cuda")[None] <= int(cache.L[b]) + torch.arange(rows, device="cuda")[:, None]
        for h in range(cache.hq):
            x = q[at:at + rows, h].double()
            s = (x @ k[:, h // group].T) / math.sqrt(cache.dim)
            p = torch.softmax(torch.where(seen, s, -math.inf), -1)
            ref, spread = p @ v[:, h // group], p @ v[:, h // group].abs()
            worst = max(worst, float(((out[at:at + rows, h].double() - ref).abs() / (2.0 ** -8 * (ref.abs() + spread) * 1.01)).max()))
        at += rows
    return worst


def run(steps=6, layers=3, hq=32, hkv=8, dim=128, batch=24, prompt=1500, turn=40, fp8=False, check=False, log=print):
    r = np.random.default_rng(1)
    torch.manual_seed(1)
    cache = Cache(layers, hq, hkv, dim, batch, prompt, turn + steps + PAGE, fp8, check)
    scale = 1.0 / math.sqrt(dim)
    # The prompt: its whole pages once, the rest of it in every conversation's own page.
    common = prompt // PAGE * PAGE
    rest = np.arange(common, prompt)
    for l in range(layers):
        of = np.zeros(prompt, np.int64)
        positions = np.arange(prompt)
        _, k, v, _ = cache.append(l, of, positions)
        for b in range(1, batch):
            if len(rest):
                cache.ctx.kv_append_rotated(None, k[common:], v[common:], torch.from_numpy(rest).cuda(), cache.pools[l], torch.from_numpy(cache.slots(b, rest)).cuda(), None)
        if check:
            held = [cache.held(cache.turned(k, positions)), cache.held(v.double())]
            for b in range(batch):
                cache.plain[l][b] = [x.clone() for x in held]
    cache.L[:] = prompt
    shared = np.full(batch, common, np.int32)
    shared[0] = 0
    worst = 0.0
    for step in range(steps):
        n = r.integers(1, turn + 1, batch).astype(np.int32) if step == 0 else np.ones(batch, np.int32)
        of = np.repeat(np.arange(batch), n)
        positions = (cache.L[of] + np.arange(len(of)) - np.repeat(np.cumsum(n) - n, n)).astype(np.int64)
        out = torch.empty((len(of), hq, dim), dtype=torch.bfloat16, device="cuda")
        for l in range(layers):
            _, k, v, q = cache.append(l, of, positions)
            cache.ctx.prefix_attention(q, cache.pools[l], cache.table_dev, shared, cache.L, n, scale, out)
            if check:
                new = [cache.held(cache.turned(k, positions)), cache.held(v.double())]
                for b in range(batch):
                    cache.plain[l][b] = [torch.cat([old, x[torch.from_numpy(of == b).cuda()]]) for old, x in zip(cache.plain[l][b], new)]
                worst = max(worst, worst_error(cache, l, n, q, out))
        cache.L = cache.L + n
        log("step %d: %d rows, lengths %d to %d" % (step, len(of), cache.L.min(), cache.L.max()))
    flags = cache.ctx.device_error_flags()
    if flags:
        raise RuntimeError("device error flags 0x%x" % flags)
    return worst


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=6)
    ap.add_argument("--fp8", action="store_true", help="FP8 pages")
    ap.add_argument("--check", action="store_true", help="compare with plain attention over the tokens that should be in the cache")
    args = ap.parse_args()
    error = run(steps=args.steps, fp8=args.fp8, check=args.check)
    if args.check:
        print("largest error %.2f of what the roundings may come to" % error)
        sys.exit(error > 1.0)
