"""Speculative decoding with cache eviction over the paged KV cache, one engine step after the other.

Every step drafts a tree of tokens per sequence, appends its K/V, attends for all nodes at once (tree_attention, layer by layer),
accepts one path and moves its tokens to where the sequence ends (kv_compact, all layers in one call).  The token that follows
is decoded with weighted_attention, which also adds up how much every cached token is looked at.  A batch that has outgrown its
budget is cut down to the tokens that matter: kv_select chooses them by these weights for every layer and KV head, kv_compact
moves them, and their weights, to the front.

There is no model here: queries, keys and values are random, and the accepted path is the deepest one.  What is real is the
cache; --check compares the last step's attention with plain products over the tokens that should be there.

    python examples/draft_and_evict.py [--steps 8] [--check]
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
    """Pools of all layers, page tables and lengths, and what a plain program would hold: dense K/V of every sequence."""

    def __init__(self, layers, hq, hkv, dim, batch, most, check):
        self.layers, self.hq, self.hkv, self.dim, self.batch, self.most = layers, hq, hkv, dim, batch, most
        per = (most + PAGE - 1) // PAGE
        self.ctx = ppd.Context(hq, hkv, dim, batch * per)
        self.elems = self.ctx.pool_elems()
        self.pools = torch.zeros((layers, self.elems), dtype=torch.bfloat16, device="cuda")
        self.table = np.random.default_rng(0).permutation(batch * per).astype(np.int32).reshape(batch, per)
        self.table_dev = torch.from_numpy(self.table).cuda()
        self.L = np.zeros(batch, np.int32)
        self.weights = torch.zeros((layers, batch, hkv, most), device="cuda")
        self.dense = [[[torch.zeros((0, hkv, dim), device="cuda") for _ in "kv"] for _ in range(batch)] for _ in range(layers)] if check else None

    def random(self, rows, heads):
        return torch.randn((rows, heads, self.dim), device="cuda").to(torch.bfloat16)

    def append(self, layer, n):
        """K/V of n[b] new tokens behind every sequence; lengths stay as they are until tokens are accepted."""
        rows = int(n.sum())
        k, v = self.random(rows, self.hkv), self.random(rows, self.hkv)
        of = np.repeat(np.arange(self.batch), n)
        pos = self.L[of] + np.arange(rows) - np.repeat(np.cumsum(n) - n, n)
        slots = self.table[of, pos // PAGE].astype(np.int64) * PAGE + pos % PAGE
        self.ctx.kv_append(k, v, self.pools[layer], torch.from_numpy(slots).cuda())
        if self.dense:
            at = 0
            for b, c in enumerate(n):
                for i, x in enumerate((k, v)):
                    self.dense[layer][b][i] = torch.cat([self.dense[layer][b][i][:int(self.L[b])], x[at:at + int(c)].float()])
                at += int(c)

    def keep(self, lists, first, count, weights=None):
        """Token lists[.., i] goes to first + i: the same for all heads and layers ([batch, n]) or every layer's and head's own."""
        self.ctx.kv_compact(self.pools, self.table_dev, lists, first, count, layer_stride_elems=self.elems, num_layers=self.layers, weights=weights)
        if self.dense:
            for l in range(self.layers):
                for b in range(self.batch):
                    f, c = int(first[b]), int(count[b])
                    for i in range(2):
                        x = self.dense[l][b][i]
                        src = (lists[b][None].expand(self.hkv, -1) if lists.dim() == 2 else lists[l, b])[:, :c].long()
                        moved = torch.stack([x[src[h], h] for h in range(self.hkv)], 1) if c else x[:0]
                        self.dense[l][b][i] = torch.cat([x[:f], moved])
        self.L = (first + count).astype(np.int32)


def draft(r, count):
    """A random tree: mask word j has the bits of node j and its ancestors.  Returns the words and the deepest path's nodes."""
    masks, paths = [], []
    for j in range(count):
        parent = int(r.integers(max(-1, j - 6), j)) if j else -1
        paths.append((paths[parent] if parent >= 0 else []) + [j])
        masks.append(sum(1 << k for k in paths[j]))
    return masks, max(paths, key=len)


def worst_error(cache, layer, q, out):
    """Largest difference from plain attention of the decoded tokens, in units of what bf16 results may be off by."""
    worst, group = 0.0, cache.hq // cache.hkv
    for b in range(cache.batch):
        k, v = (x.repeat_interleave(group, 1).double() for x in cache.dense[layer][b])
        p = torch.softmax((q[b].double()[None] * k).sum(-1) / math.sqrt(cache.dim), 0)
        ref, spread = (p[..., None] * v).sum(0), (p[..., None] * v.abs()).sum(0)
        worst = max(worst, float(((out[b].double() - ref).abs() / (2.0 ** -8 * (ref.abs() + spread) * 1.01)).max()))
    return worst


def run(steps=8, layers=4, hq=32, hkv=8, dim=128, batch=6, prompt=900, budget=512, limit=960, check=False, log=print):
    r = np.random.default_rng(1)
    torch.manual_seed(1)
    scale = 1.0 / math.sqrt(dim)
    cache = Cache(layers, hq, hkv, dim, batch, limit + 64, check)
    n = r.integers(prompt // 2, prompt + 1, batch).astype(np.int32)
    for l in range(layers):
        cache.append(l, n)
    cache.L = n
    worst = 0.0
    for step in range(steps):
        # a tree per sequence, all nodes in one pass
        n = r.integers(8, 33, batch).astype(np.int32)
        trees = [draft(r, int(c)) for c in n]
        mask = torch.from_numpy(np.array(sum((t[0] for t in trees), []), np.uint64).view(np.int64)[:, None]).cuda()
        out = torch.empty((int(n.sum()), hq, dim), dtype=torch.bfloat16, device="cuda")
        for l in range(layers):
            cache.append(l, n)
            cache.ctx.tree_attention(cache.random(len(out), hq), cache.pools[l], cache.table_dev, cache.L, n, mask, scale, out)
        # the accepted path's tokens become the sequence's end
        accepted = np.full((batch, max(len(t[1]) for t in trees)), -1, np.int32)
        for b, (_, path) in enumerate(trees):
            accepted[b, :len(path)] = cache.L[b] + np.array(path)
        cache.weights.masked_fill_(torch.arange(cache.most, device="cuda") >= torch.from_numpy(cache.L).cuda()[:, None, None], 0.0)
        cache.keep(torch.from_numpy(accepted).cuda(), cache.L, np.array([len(t[1]) for t in trees], np.int32))
        # the next token, with the cache watched
        one = np.ones(batch, np.int32)
        out = torch.empty((batch, hq, dim), dtype=torch.bfloat16, device="cuda")
        for l in range(layers):
            cache.append(l, one)
            q = cache.random(batch, hq)
            cache.ctx.weighted_attention(q, cache.pools[l], cache.table_dev, cache.L, one, scale, out, cache.weights[l])
            if check:
                worst = max(worst, worst_error(cache, l, q, out))
        cache.L = cache.L + one
        # too long: every layer and head keeps the tokens it looked at
        evict = bool((cache.L > limit - 40).any())
        if evict:
            lists = torch.full((layers, batch, hkv, budget), -1, dtype=torch.int32, device="cuda")
            for l in range(layers):
                cache.ctx.kv_select(cache.weights[l], cache.L, budget, 4, 64, lists[l])
            cache.keep(lists, np.zeros(batch, np.int32), np.minimum(cache.L, budget), weights=cache.weights)
        log("step %d: %d drafted, %d accepted%s, lengths %s" % (step, int(n.sum()), sum(len(t[1]) for t in trees), ", cut down" if evict else "", cache.L.tolist()))
    flags = cache.ctx.device_error_flags()
    if flags:
        raise RuntimeError("device error flags 0x%x" % flags)
    return worst


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--check", action="store_true", help="compare with plain attention over the tokens that should be in the cache")
    args = ap.parse_args()
    error = run(steps=args.steps, check=args.check)
    if args.check:
        print("largest error %.2f of what bf16 results may be off by" % error)
        sys.exit(error > 1.0)
