"""Tree attention, weighted attention, kv_select and kv_compact on the GPU against plain computations in 64 bits on the CPU.

Tolerances follow from the roundings.  A probability p enters the product with V as a bf16 number (off by 2^-8 of itself at most) and
the result is rounded to bf16: |error| <= 2^-8 |o| + 2^-8 sum p|v|, and on top what p itself is off by.  A score is a sum of D
products in 32 bits, off by (D + 8) 2^-24 of the sum of their magnitudes at most, its exponent in units of log2 by two more
roundings, the exponential by about a unit in the last place: relative error of p below eta = (D + 64) 2^-23 (1 + max sum |q k| scale),
once in the numerator and once in the sum."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2603_13358_amd as ppd  # noqa: E402

PAGE = 16
SCALE8 = 2.0 ** -4


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def bf16(x):
    """float64 array of the nearest bf16 numbers."""
    return torch.from_numpy(np.asarray(x, np.float64)).to(torch.float32).to(torch.bfloat16).double().numpy()


class Batch:
    """K/V of a batch of sequences, a pool of pages that holds them, and queries; everything else in the pool is NaN."""

    def __init__(self, L, n, hq, hkv, dim, fp8=False, seed=0, q_scale=1.0, slack=3, kv=None, num_pages=None, first_page=0):
        r = np.random.default_rng(seed)
        self.L, self.n = np.array(L, np.int32), np.array(n, np.int32)
        self.hq, self.hkv, self.dim, self.fp8 = hq, hkv, dim, fp8
        total = self.L + self.n
        need = (total + PAGE - 1) // PAGE
        self.num_pages = int(need.sum()) + slack if num_pages is None else num_pages
        perm = (first_page + r.permutation(int(need.sum()) + slack)).astype(np.int32)
        self.table = np.full((len(total), int(need.max()) + 2), -7, np.int32)
        at = 0
        for i, c in enumerate(need):
            self.table[i, :c] = perm[at:at + c]
            at += c
        self.k, self.v = ([bf16(r.standard_normal((t, hkv, dim))) for t in total] for _ in range(2))
        self.q = bf16(r.standard_normal((int(self.n.sum()), hq, dim)) * q_scale)
        self.scale = 1.0 / math.sqrt(dim)
        if kv:
            kv(self)
        self.ctx = ppd.Context(hq, hkv, dim, self.num_pages)
        if fp8:
            self.ctx.set_kv_format(ppd.PPD_KV_FP8_E4M3, SCALE8, SCALE8)
            self.pool = torch.full((self.ctx.pool_elems(),), 0x7F, dtype=torch.uint8, device="cuda")
            quantised = lambda x: [torch.from_numpy(a / SCALE8).float().clamp(-448, 448).to(torch.float8_e4m3fn).double().numpy() * SCALE8 for a in x]  # noqa: E731
        elif num_pages is None:
            self.pool = torch.full((self.ctx.pool_elems(),), float("nan"), dtype=torch.bfloat16, device="cuda")
            quantised = lambda x: x  # noqa: E731
        else:
            self.pool = torch.empty((self.ctx.pool_elems(),), dtype=torch.bfloat16, device="cuda")
            quantised = lambda x: x  # noqa: E731
        for i, t in enumerate(total):
            pos = np.arange(t)
            slots = self.table[i, pos // PAGE].astype(np.int64) * PAGE + pos % PAGE
            self.ctx.kv_append(dev(self.k[i]).to(torch.bfloat16), dev(self.v[i]).to(torch.bfloat16), self.pool, dev(slots))
        self.k, self.v = quantised(self.k), quantised(self.v)
        self.q_dev, self.table_dev = dev(self.q).to(torch.bfloat16), dev(self.table)

    def sees(self, i, mask=None):
        """[row, token] of sequence i: by mask words, or causal."""
        n, L = int(self.n[i]), int(self.L[i])
        seen = np.ones((n, L + n), bool)
        j = np.arange(n)
        if mask is None:
            seen[:, L:] = j[None] <= j[:, None]
        else:
            r0 = int(self.n[:i].sum())
            words = mask[r0:r0 + n]
            seen[:, L:] = (words[:, j // 64] >> (j % 64).astype(np.uint64)) & np.uint64(1) == 1
        return seen

    def reference(self, mask=None, scale=None):
        """(results, bounds) [row, head, d] and per sequence (weights, bounds) [KV head, token], in 64 bits."""
        scale = self.scale if scale is None else scale
        G = self.hq // self.hkv
        outs, bounds, weights = [], [], []
        for i in range(len(self.L)):
            r0, n = int(self.n[:i].sum()), int(self.n[i])
            seen = self.sees(i, mask)
            out, bound = np.zeros((n, self.hq, self.dim)), np.zeros((n, self.hq, self.dim))
            w, wb = np.zeros((self.hkv, seen.shape[1])), np.zeros((self.hkv, seen.shape[1]))
            for h in range(self.hq):
                q, k, v = self.q[r0:r0 + n, h], self.k[i][:, h // G], self.v[i][:, h // G]
                s = np.where(seen, (q @ k.T) * scale, -np.inf)
                eta = (self.dim + 64) * 2.0 ** -23 * (1 + float((np.abs(q) @ np.abs(k).T).max()) * scale)
                top = s.max(1, keepdims=True)
                p = np.exp(s - np.where(np.isfinite(top), top, 0))
                p /= np.maximum(p.sum(1, keepdims=True), 1e-300)
                out[:, h] = p @ v
                spread = p @ np.abs(v)
                bound[:, h] = 2.0 ** -8 * (np.abs(out[:, h]) + spread) * (1 + 2 * eta) + 2 * eta * spread
                w[h // G] += p.sum(0)
                wb[h // G] += p.sum(0) * (2 * eta + (n * G + 4) * 2.0 ** -23)
            outs.append(out)
            bounds.append(bound)
            weights.append((w, wb))
        return np.concatenate(outs), np.concatenate(bounds), weights

    def tree(self, mask, scale=None, out=None, stream=None):
        out = torch.full((len(self.q), self.hq, self.dim), float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
        self.ctx.tree_attention(self.q_dev, self.pool, self.table_dev, self.L, self.n, dev(mask.view(np.int64)), self.scale if scale is None else scale, out, stream=stream)
        return out

    def weighted(self, weights, out=None, stream=None):
        out = torch.full((len(self.q), self.hq, self.dim), float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
        self.ctx.weighted_attention(self.q_dev, self.pool, self.table_dev, self.L, self.n, self.scale, out, weights, stream=stream)
        return out

    def flags(self):
        return self.ctx.device_error_flags(torch.cuda.current_stream().cuda_stream)


def random_mask(b, words, seed, density=0.4, self_bit=True):
    r = np.random.default_rng(seed)
    mask = np.zeros((len(b.q), words), np.uint64)
    for bit in range(64):
        mask |= (r.random(mask.shape) < density).astype(np.uint64) << np.uint64(bit)  # bits beyond the nodes among them
    at = 0
    for n in b.n:
        for j in range(int(n)):
            if self_bit:
                mask[at, j // 64] |= np.uint64(1) << np.uint64(j % 64)
            at += 1
    return mask


def within(got, ref, bound):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all()
    over = np.abs(got - ref) - bound
    assert over.max() <= 1e-30, "off by %.3e more than allowed at %s" % (over.max(), np.unravel_index(over.argmax(), over.shape))


TREES = [  # L, n, query heads, KV heads, head_dim, FP8 pages, mask words
    ([0], [1], 8, 8, 64, False, 1),
    ([1], [2], 4, 1, 128, False, 1),
    ([37], [5], 8, 2, 64, False, 1),
    ([31, 32, 33], [1, 31, 33], 8, 1, 128, False, 1),
    ([100, 0, 17], [64, 1, 40], 10, 2, 128, False, 1),
    ([127, 128, 129], [7, 9, 3], 14, 2, 64, True, 1),
    ([300, 5], [65, 128], 4, 2, 128, False, 2),
    ([95, 250], [200, 13], 6, 1, 64, False, 4),
    ([40], [1000], 1, 1, 64, False, 16),
    ([700, 3, 64], [17, 64, 30], 12, 2, 128, True, 1),
    ([5000, 2100], [24, 61], 8, 1, 128, False, 1),
    ([9001], [3], 8, 1, 64, True, 3),
]


@pytest.mark.parametrize("L,n,hq,hkv,dim,fp8,words", TREES, ids=lambda x: str(x).replace(" ", ""))
def test_tree_attention_matches_the_definition(L, n, hq, hkv, dim, fp8, words):
    b = Batch(L, n, hq, hkv, dim, fp8, seed=len(L) + sum(L))
    mask = random_mask(b, words, seed=5)
    ref, bound, _ = b.reference(mask)
    got = b.tree(mask)
    within(got, ref, bound)
    assert torch.equal(got, b.tree(mask))  # the same from run to run, bit for bit
    assert b.flags() == 0


@pytest.mark.parametrize("fp8", [False, True])
def test_tree_rows_that_see_little_or_nothing(fp8):
    b = Batch([0, 40, 0], [6, 3, 33], 8, 2, 64, fp8, seed=1)
    mask = np.zeros((len(b.q), 1), np.uint64)
    mask[1] = 1 << 4          # one node and not itself
    mask[9 + 32] = 1 << 32    # the last node alone
    mask[2] = ~np.uint64(0x3F)  # bits of nodes that are not there
    ref, bound, _ = b.reference(mask)
    got = b.tree(mask)
    within(got, ref, bound)
    for row in [0, 2, 3, 9, 40]:
        assert not got[row].any(), "a row that sees nothing gives zeros"
    for h in range(8):  # a row that sees one node is that node's V
        assert np.array_equal(got[1, h].double().cpu().numpy(), b.v[0][4, h // 4])
        assert np.array_equal(got[41, h].double().cpu().numpy(), b.v[2][32, h // 4])


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("long", [False, True])
def test_what_a_row_does_not_see_does_not_reach_it(bad, long):
    L, n = ([2500], [40]) if long else ([20], [40])
    fill = dict(k=lambda b: b.k[0].__setitem__((L[0] + 7, 0, 5), bad), v=lambda b: b.v[0].__setitem__((L[0] + 7, 0, slice(3, 9)), bad))

    def both(b):
        fill["k"](b)
        fill["v"](b)
    clean = Batch(L, n, 8, 2, 128, seed=3)
    dirty = Batch(L, n, 8, 2, 128, seed=3, kv=both)
    mask = random_mask(clean, 1, seed=4, density=0.5)
    blind = (mask[:, 0] & np.uint64(1 << 7)) == 0
    assert 5 < blind.sum() < 35
    a, b = clean.tree(mask), dirty.tree(mask)
    assert torch.equal(a[dev(blind)], b[dev(blind)])
    assert torch.equal(a[:, 4:], b[:, 4:])  # the other KV head's queries
    # an element that is seen counts: V alone is infinite or NaN, its row finite elsewhere
    only_v = Batch(L, n, 8, 2, 128, seed=3, kv=fill["v"])
    c = only_v.tree(mask).double().cpu().numpy()
    seeing = c[~blind][:, :4]
    assert np.array_equal(np.isnan(seeing[..., 3:9]), np.full(seeing[..., 3:9].shape, np.isnan(bad)))
    assert np.isnan(bad) or (seeing[..., 3:9] == bad).all()
    assert np.isfinite(seeing[..., :3]).all() and np.isfinite(seeing[..., 9:]).all() and np.isfinite(c[blind]).all()


@pytest.mark.parametrize("n", [8, 40])
@pytest.mark.parametrize("fp8", [False, True])
def test_a_row_is_rounded_by_what_it_sees_itself(n, fp8):
    b = Batch([900], [n], 8, 2, 128, fp8, seed=17)
    mask = random_mask(b, 1, seed=18)
    before = b.tree(mask)
    b.q_dev[3] *= 64.0  # far larger scores: its reference is raised again and again
    after = b.tree(mask)
    others = [j for j in range(n) if j != 3]
    assert torch.equal(before[others], after[others]) and not torch.equal(before[3], after[3])


def test_tree_scale_zero_and_sharp_scores():
    b = Batch([70], [9], 8, 1, 128, seed=6, q_scale=12.0)
    mask = random_mask(b, 1, seed=7)
    ref, bound, _ = b.reference(mask)
    within(b.tree(mask), ref, bound)
    ref, bound, _ = b.reference(mask, scale=0.0)
    within(b.tree(mask, scale=0.0), ref, bound)


def test_a_chain_is_causal_attention():
    b = Batch([1200, 64], [48, 17], 32, 8, 128, seed=8)
    j = np.concatenate([np.arange(n) for n in b.n]).astype(np.uint64)
    mask = ((np.uint64(2) << j) - np.uint64(1))[:, None]
    ref, bound, _ = b.reference()
    got = b.tree(mask)
    within(got, ref, bound)
    mixed = torch.empty_like(got)
    b.ctx.mixed_attention(b.q_dev, b.pool, b.table_dev, b.L, b.n, b.scale, mixed)
    within(mixed, got.double().cpu().numpy(), 2 * bound)


def test_tree_offsets_beyond_32_bits():
    pages = 2 ** 31 // (2 * 8 * 16 * 128) + 400  # element offsets pass 2^31, byte offsets 2^32
    b = Batch([90], [20], 8, 8, 128, seed=9, num_pages=pages, first_page=pages - 20)
    mask = random_mask(b, 1, seed=10)
    ref, bound, weights = b.reference(mask)
    within(b.tree(mask), ref, bound)
    ref, bound, weights = b.reference()
    w = torch.zeros((1, 8, 110), device="cuda")
    within(b.weighted(w), ref, bound)
    within(w[0], *weights[0])
    before = b.pool.view(-1, 2 * 8 * 16 * 128)[pages - 20:].clone()
    keep = dev(np.array([[3, 50, 109]], np.int32))
    b.ctx.kv_compact(b.pool, b.table_dev, keep, np.array([1], np.int32), np.array([3], np.int32))
    after = b.pool.view(-1, 2 * 8 * 16 * 128)[pages - 20:]
    expect = moved(before.cpu().view(torch.int16).numpy(), b.table - (pages - 20), keep.cpu().numpy(), [1], [3], 8, 128)
    assert np.array_equal(after.cpu().view(torch.int16).numpy(), expect)


def test_tree_page_ids_outside_the_pool_raise_the_flag():
    b = Batch([50], [4], 8, 2, 64, seed=11)
    b.table_dev[0, 1] = b.num_pages
    b.table_dev[0, 2] = -5
    b.tree(random_mask(b, 1, seed=1))
    assert b.flags() == 2 and b.flags() == 0
    b.weighted(torch.zeros((1, 2, 64), device="cuda"))
    assert b.flags() == 2


def test_tree_and_weighted_on_streams_and_in_graphs():
    b = Batch([900, 30], [12, 5], 32, 8, 128, seed=12)
    mask = random_mask(b, 1, seed=13)
    mask_dev = dev(mask.view(np.int64))
    eager = b.tree(mask)
    w0 = torch.rand((2, 8, 1000), device="cuda")
    w_eager = w0.clone()
    out_eager = b.weighted(w_eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out, w = torch.empty_like(eager), w0.clone()
        b.ctx.tree_attention(b.q_dev, b.pool, b.table_dev, b.L, b.n, mask_dev, b.scale, out, stream=side.cuda_stream)
        w_out = b.weighted(w, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(out, eager) and torch.equal(w, w_eager) and torch.equal(w_out, out_eager)
    keep = torch.full((2, 8, 40), -1, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    pool0 = b.pool.clone()
    lengths = (b.L + b.n).astype(np.int32)
    with torch.cuda.graph(graph, stream=side):
        s = torch.cuda.current_stream().cuda_stream
        b.weighted(w, out=w_out, stream=s)
        b.ctx.kv_select(w, lengths, 30, 2, 5, keep, stream=s)
        b.ctx.kv_compact(b.pool, b.table_dev, keep, np.zeros(2, np.int32), np.array([30, 30], np.int32), weights=w, stream=s)
    w_ref, keep_ref = w_eager.clone(), torch.full_like(keep, -1)
    b.ctx.kv_select(w_ref, lengths, 30, 2, 5, keep_ref)
    b.ctx.kv_compact(b.pool, b.table_dev, keep_ref, np.zeros(2, np.int32), np.array([30, 30], np.int32), weights=w_ref)
    pool_ref = b.pool.clone()
    for _ in range(4):
        b.pool.copy_(pool0)
        w.copy_(w0)
        keep.fill_(-1)
        w_out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(w_out, out_eager) and torch.equal(keep, keep_ref) and torch.equal(w, w_ref)
        assert torch.equal(b.pool.view(torch.int16), pool_ref.view(torch.int16))
    assert b.flags() == 0


WEIGHTED = [  # L, n, query heads, KV heads, head_dim, FP8 pages
    ([0], [1], 8, 8, 64, False),
    ([0, 1], [3, 1], 4, 1, 128, False),
    ([100, 0, 500], [1, 1, 1], 32, 8, 128, False),
    ([255, 256, 257], [1, 2, 33], 10, 2, 64, False),
    ([4000], [1], 8, 1, 128, False),
    ([1023, 70], [5, 90], 12, 2, 128, True),
    ([333], [1], 8, 2, 64, True),
    ([2050, 31], [32, 1], 5, 1, 128, False),
    ([3000, 700], [4, 4], 8, 1, 128, False),         # 32 columns, whose scores fill a tile's LDS at 512 keys
    ([5000], [2], 16, 2, 128, True),
    ([2600, 40, 1200], [2, 50, 1], 10, 2, 64, False),  # kept scores, scores computed again, and row blocks in one batch
    ([9000], [3], 4, 2, 64, False),
]


@pytest.mark.parametrize("L,n,hq,hkv,dim,fp8", WEIGHTED, ids=lambda x: str(x).replace(" ", ""))
def test_weighted_attention_matches_the_definition(L, n, hq, hkv, dim, fp8):
    b = Batch(L, n, hq, hkv, dim, fp8, seed=20 + len(L))
    ref, bound, weights = b.reference()
    stride = int((b.L + b.n).max()) + 5
    start = torch.rand((len(L), hkv, stride), device="cuda")
    w = start.clone()
    for i, t in enumerate(b.L):  # what stands at the new tokens before does not count
        w[i, :, int(t):int(t + b.n[i])] = float("nan")
    within(b.weighted(w), ref, bound)
    for i, (ww, wb) in enumerate(weights):
        t, total = int(b.L[i]), int(b.L[i] + b.n[i])
        old = start[i].double().cpu().numpy()
        old[:, t:] = 0
        within(w[i, :, :total], old[:, :total] + ww, wb + 2.0 ** -23 * (old[:, :total] + ww))
        assert torch.equal(w[i, :, total:], start[i, :, total:])
        got = w[i, :, :total].double().cpu().numpy() - old[:, :total]
        assert abs(got.sum() / (hq * int(b.n[i])) - 1) < 1e-3  # every row's probabilities add up to one
    again = start.clone()
    b.weighted(again)
    assert all(torch.equal(again[i, :, :int(b.L[i] + b.n[i])], w[i, :, :int(b.L[i] + b.n[i])]) for i in range(len(L)))
    assert b.flags() == 0


def test_weighted_masked_keys_that_are_not_finite():
    def fill(b):
        b.k[0][101, 0, :] = np.nan
        b.v[0][101, 0, :] = np.inf
    clean, dirty = Batch([100], [4], 4, 1, 64, seed=30), Batch([100], [4], 4, 1, 64, seed=30, kv=fill)
    w = torch.zeros((2, 1, 1, 104), device="cuda")
    a, b = clean.weighted(w[0]), dirty.weighted(w[1])
    assert torch.equal(a[0], b[0])  # only later rows see token 101
    assert torch.isnan(b[1:]).all()
    assert torch.isnan(w[1]).any()


def chosen(w, length, budget, sinks, recent):
    """Positions to keep, written apart from the kernel: sort by (held, weight descending, position)."""
    t = np.arange(length)
    if length <= budget:
        return t
    key = [(0 if i < sinks or i >= length - recent else 1, 0 if np.isnan(x) else 1, -x if not np.isnan(x) else 0.0, i) for i, x in enumerate(w[:length].astype(np.float64))]
    return np.sort(np.array(sorted(key))[:budget, 3].astype(np.int64))


SELECTS = [  # lengths, KV heads, budget, sinks, recent
    ([1], 1, 1, 0, 0),
    ([0, 5, 2], 2, 3, 1, 1),
    ([64, 63, 65, 66], 2, 64, 0, 0),
    ([700], 8, 128, 4, 32),
    ([1500, 10, 1024, 1025], 3, 512, 4, 64),
    ([5000, 129], 2, 129, 100, 29),
    ([3000], 2, 100, 100, 0),
    ([3000], 2, 100, 0, 100),
    ([8193, 8192], 1, 8192, 3, 0),
    ([40000], 2, 5001, 16, 100),
    ([70001, 300], 1, 30000, 0, 1),
]


@pytest.mark.parametrize("lengths,hkv,budget,sinks,recent", SELECTS, ids=lambda x: str(x).replace(" ", ""))
@pytest.mark.parametrize("kind", ["heavy", "ties", "odd"])
def test_select_keeps_the_heaviest(lengths, hkv, budget, sinks, recent, kind):
    r = np.random.default_rng(sum(lengths) + budget)
    stride = max(lengths) + 3
    w = np.exp(2 * r.standard_normal((len(lengths), hkv, stride))).astype(np.float32)
    if kind == "ties":
        w = r.integers(0, 3, w.shape).astype(np.float32) * 0.25
    elif kind == "odd":
        w = r.choice(np.array([0.0, -0.0, 1e-42, -1.5, 2.5, np.inf, -np.inf, np.nan, -np.nan, 3e38], np.float32), w.shape)
    ctx = ppd.Context(hkv, hkv, 64, 4)
    keep = torch.full((len(lengths), hkv, budget + 2), -9, dtype=torch.int32, device="cuda")
    ctx.kv_select(dev(w), np.array(lengths, np.int32), budget, sinks, recent, keep)
    keep = keep.cpu().numpy()
    for i, n in enumerate(lengths):
        for h in range(hkv):
            want = chosen(w[i, h], n, budget, sinks, recent)
            assert np.array_equal(keep[i, h, :len(want)], want)
            assert (keep[i, h, len(want):] == -9).all()


def test_select_of_more_sequences_than_one_launch_takes():
    r = np.random.default_rng(2)
    lengths = r.integers(0, 90, 1100).astype(np.int32)
    w = r.random((1100, 2, 90)).astype(np.float32)
    ctx = ppd.Context(4, 2, 64, 4)
    keep = torch.full((1100, 2, 40), -1, dtype=torch.int32, device="cuda")
    ctx.kv_select(dev(w), lengths, 40, 1, 8, keep)
    keep = keep.cpu().numpy()
    for i in range(0, 1100, 7):
        for h in range(2):
            want = chosen(w[i, h], int(lengths[i]), 40, 1, 8)
            assert np.array_equal(keep[i, h, :len(want)], want) and (keep[i, h, len(want):] == -1).all()


def offsets(table_row, h, pos, hkv, dim, value):
    """[position, d]: (page, element within the page) by the layout's formulas."""
    pos, d = np.asarray(pos)[:, None], np.arange(dim)[None]
    tok = pos % PAGE
    if value:
        at = hkv * PAGE * dim + h * PAGE * dim + tok // 8 * (dim * 8) + d * 8 + tok % 8
    else:
        at = h * PAGE * dim + d // 8 * (PAGE * 8) + tok * 8 + d % 8
    return np.broadcast_to(table_row[pos // PAGE], at.shape), at


def moved(pool, table, keep, first, count, hkv, dim):
    """The pool [page, element] after the move; keep: [sequence, n] or [sequence, KV head, n]."""
    out = pool.copy()
    for b in range(len(first)):
        for h in range(hkv):
            src = (keep[b] if keep.ndim == 2 else keep[b, h])[:count[b]]
            dst = first[b] + np.arange(count[b])
            for value in (False, True):
                out[offsets(table[b], h, dst, hkv, dim, value)] = pool[offsets(table[b], h, src, hkv, dim, value)]
    return out


COMPACTS = [  # tokens of every sequence, first, count, KV heads, head_dim, FP8 pages, layers, lists: shared, by head, by layer
    ([20], [0], [1], 1, 64, False, 1, "shared"),
    ([50], [13], [5], 2, 128, False, 3, "shared"),
    ([300, 17, 64], [3, 0, 40], [90, 0, 24], 2, 64, False, 1, "head"),
    ([1000, 129], [0, 0], [400, 129], 3, 128, False, 1, "head"),
    ([700, 260], [0, 5], [300, 130], 2, 128, True, 2, "layer"),
    ([333], [7], [200], 8, 64, True, 1, "head"),
    ([2000] * 40, list(range(40)), [500 + 7 * i for i in range(40)], 8, 128, False, 1, "head"),
    ([60] * 300, [20] * 300, [i % 9 for i in range(300)], 1, 64, False, 4, "shared"),
]


@pytest.mark.parametrize("tokens,first,count,hkv,dim,fp8,layers,lists", COMPACTS, ids=lambda x: str(x).replace(" ", "")[:24])
@pytest.mark.parametrize("with_weights", [False, True])
def test_compact_moves_tokens_bit_for_bit(tokens, first, count, hkv, dim, fp8, layers, lists, with_weights):
    r = np.random.default_rng(sum(tokens))
    need = [(t + PAGE - 1) // PAGE for t in tokens]
    pages = sum(need) + 4
    table = np.full((len(tokens), max(need) + 1), -1, np.int32)
    perm, at = r.permutation(pages).astype(np.int32), 0
    for i, c in enumerate(need):
        table[i, :c] = perm[at:at + c]
        at += c
    elems = 2 * hkv * PAGE * dim
    pool = r.integers(0, 256 if fp8 else 65536, (layers, pages, elems)).astype(np.uint8 if fp8 else np.uint16)
    most = max(max(count), 1)
    shape = {"shared": (1, len(tokens), 1), "head": (1, len(tokens), hkv), "layer": (layers, len(tokens), hkv)}[lists]
    keep = np.full(shape + (most + 1,), -1, np.int32)
    for l in range(shape[0]):
        for b, t in enumerate(tokens):
            for h in range(shape[2]):
                keep[l, b, h, :count[b]] = first[b] + np.sort(r.permutation(t - first[b])[:count[b]])
    full = np.broadcast_to(keep, (layers, len(tokens), hkv, most + 1))
    weights = r.random((layers, len(tokens), hkv, max(tokens) + 2)).astype(np.float32) if with_weights else None
    ctx = ppd.Context(hkv, hkv, dim, pages)
    if fp8:
        ctx.set_kv_format(ppd.PPD_KV_FP8_E4M3, 1.0, 1.0)
    got, got_w = dev(pool if fp8 else pool.view(np.int16)), dev(weights) if with_weights else None
    arg = dev({"shared": keep[0, :, 0], "head": keep[0], "layer": keep}[lists])
    ctx.kv_compact(got, dev(table), arg, np.array(first, np.int32), np.array(count, np.int32), layer_stride_elems=pages * elems, num_layers=layers, weights=got_w)
    for l in range(layers):
        assert np.array_equal(got[l].cpu().numpy().view(pool.dtype), moved(pool[l], table, full[l], first, count, hkv, dim))
    if with_weights:
        want = weights.copy()
        for l in range(layers):
            for b in range(len(tokens)):
                for h in range(hkv):
                    want[l, b, h, first[b]:first[b] + count[b]] = weights[l, b, h, full[l, b, h, :count[b]]]
        assert np.array_equal(got_w.cpu().numpy(), want)
    assert ctx.device_error_flags() == 0


def test_compact_entries_out_of_order_stay_and_raise_the_flag():
    r = np.random.default_rng(1)
    pool = r.integers(0, 65536, (8, 2 * 16 * 64)).astype(np.uint16)
    table = np.arange(8, dtype=np.int32)[None]
    ctx = ppd.Context(1, 1, 64, 8)
    #                 ok  repeated  below its place  beyond the pages  ok
    keep = np.array([[5, 5, 1, 128, 90]], np.int32)
    got = dev(pool.view(np.int16))
    ctx.kv_compact(got, dev(table), dev(keep), np.array([2], np.int32), np.array([5], np.int32))
    assert ctx.device_error_flags() == 8
    want = moved(pool, table, np.array([[5]]), [2], [1], 1, 64)
    assert np.array_equal(got.cpu().numpy().view(np.uint16), want)  # 90 does not ascend from 128
    for bad in (8, -1):  # a page outside the pool: from there, and to there
        table = np.array([[0, bad, 2, 3, 4, 5, 6, 7]], np.int32)
        got = dev(pool.view(np.int16))
        keep = np.array([[20, 40, 70]], np.int32)
        ctx.kv_compact(got, dev(table), dev(keep), np.array([14], np.int32), np.array([3], np.int32))
        assert ctx.device_error_flags() == 2
        safe = np.array([[0, 0, 2, 3, 4, 5, 6, 7]], np.int32)
        assert np.array_equal(got.cpu().numpy().view(np.uint16), moved(pool, safe, np.array([[40]]), [15], [1], 1, 64))


def test_refusals_reach_python():
    b = Batch([30], [4], 8, 2, 64, seed=40)
    mask = random_mask(b, 1, seed=1)
    with pytest.raises(ppd.PPDError) as e:
        b.ctx.tree_attention(b.q_dev, b.pool, b.table_dev[:, :2].contiguous(), b.L, b.n, dev(mask.view(np.int64)), b.scale, torch.empty_like(b.q_dev))
    assert e.value.status == -4
    with pytest.raises(ppd.PPDError) as e:
        b.weighted(torch.zeros((1, 2, 33), device="cuda"))
    assert e.value.status == -3
    keep = torch.zeros((1, 2, 4), dtype=torch.int32, device="cuda")
    with pytest.raises(ppd.PPDError) as e:
        b.ctx.kv_select(torch.zeros((1, 2, 34), device="cuda"), np.array([34]), 5, 0, 0, keep)
    assert e.value.status == -3
    with pytest.raises(ppd.PPDError) as e:
        b.ctx.kv_compact(b.pool, b.table_dev, keep, np.array([0]), np.array([5]))
    assert e.value.status == -3
    with pytest.raises(ppd.PPDError) as e:
        b.ctx.tree_attention(b.q_dev, b.pool, b.table_dev, b.L, np.array([4, 4]), dev(mask.view(np.int64)), b.scale, torch.empty_like(b.q_dev))
    assert e.value.status == -3
