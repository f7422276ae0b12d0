"""Attention over shared prefixes on the GPU against a plain computation in 64 bits on the CPU.

Tolerances follow from the roundings, as in test_gpu_operators: a probability enters the product with V as a bf16 number (off by 2^-8 of itself at
most) and the result is rounded to bf16, |error| <= 2^-8 |o| + 2^-8 sum p|v|, and on top what p itself is off by: a score is a sum of D
products in 32 bits, its exponent two more roundings, the exponential about a unit in the last place, partials joined by as many
factors as there are: relative error of p below eta = (D + 64 + partials) 2^-23 (1 + max sum |q k| scale), in the numerator and in the sum."""
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
    return torch.from_numpy(np.asarray(x, np.float64)).float().to(torch.bfloat16).double().numpy()


class Batch:
    """Sequences of which neighbours have `common` leading tokens in common, in the same pages where these are whole; the rest of the pool is NaN."""

    def __init__(self, common, L, n, hq, hkv, dim, fp8=False, seed=0, q_scale=1.0, change=None, num_pages=None, first_page=0):
        r = np.random.default_rng(seed)
        self.L, self.n = np.array(L, np.int32), np.array(n, np.int32)
        self.shared = (np.array(common, np.int32) // PAGE * PAGE).astype(np.int32)
        self.hq, self.hkv, self.dim, self.fp8, self.scale = hq, hkv, dim, fp8, 1.0 / math.sqrt(dim)
        total = self.L + self.n
        need = (total + PAGE - 1) // PAGE
        same = self.shared // PAGE
        self.num_pages = int((need - same).sum()) + 3 if num_pages is None else num_pages
        perm = (first_page + r.permutation(int((need - same).sum()) + 3)).astype(np.int32)
        self.table = np.full((len(total), int(need.max()) + 2), -7, np.int32)
        self.k, self.v = [], []
        at = 0
        for i, c in enumerate(need):
            k, v = (bf16(r.standard_normal((total[i], hkv, dim))) for _ in range(2))
            if i:
                self.table[i, :same[i]] = self.table[i - 1, :same[i]]
                k[:common[i]], v[:common[i]] = self.k[i - 1][:common[i]], self.v[i - 1][:common[i]]
            self.table[i, same[i]:c] = perm[at:at + c - same[i]]
            at += c - same[i]
            self.k.append(k)
            self.v.append(v)
        self.q = bf16(r.standard_normal((int(self.n.sum()), hq, dim)) * q_scale)
        if change:
            change(self)
        self.ctx = ppd.Context(hq, hkv, dim, self.num_pages)
        if fp8:
            self.ctx.set_kv_format(ppd.PPD_KV_FP8_E4M3, SCALE8, SCALE8)
            self.pool = torch.full((self.ctx.pool_elems(),), 0x7F, dtype=torch.uint8, device="cuda")
        elif num_pages is None:
            self.pool = torch.full((self.ctx.pool_elems(),), float("nan"), dtype=torch.bfloat16, device="cuda")
        else:
            self.pool = torch.empty((self.ctx.pool_elems(),), dtype=torch.bfloat16, device="cuda")
        for i, t in enumerate(total):
            pos = np.arange(self.shared[i], t)
            slots = self.table[i, pos // PAGE].astype(np.int64) * PAGE + pos % PAGE
            self.ctx.kv_append(dev(self.k[i][pos]).to(torch.bfloat16), dev(self.v[i][pos]).to(torch.bfloat16), self.pool, dev(slots))
        if fp8:
            self.k, self.v = ([torch.from_numpy(a / SCALE8).float().clamp(-448, 448).to(torch.float8_e4m3fn).double().numpy() * SCALE8 for a in x] for x in (self.k, self.v))
        self.q_dev, self.table_dev = dev(self.q).to(torch.bfloat16), dev(self.table)

    def reference(self, scale=None, partials=600):
        scale = self.scale if scale is None else scale
        G = self.hq // self.hkv
        outs, bounds = [], []
        for i in range(len(self.L)):
            r0, n, L = int(self.n[:i].sum()), int(self.n[i]), int(self.L[i])
            seen = np.arange(L + n)[None] <= L + np.arange(n)[:, None]
            out, bound = np.zeros((n, self.hq, self.dim)), np.zeros((n, self.hq, self.dim))
            for h in range(self.hq):
                q, k, v = self.q[r0:r0 + n, h], self.k[i][:, h // G], self.v[i][:, h // G]
                s = np.where(seen, (q @ k.T) * scale, -np.inf)
                eta = (self.dim + 64 + partials) * 2.0 ** -23 * (1 + float((np.abs(q) @ np.abs(k).T).max()) * scale)
                top = s.max(1, keepdims=True)
                p = np.exp(s - np.where(np.isfinite(top), top, 0))
                p /= np.maximum(p.sum(1, keepdims=True), 1e-300)
                out[:, h] = p @ v
                spread = p @ np.abs(v)
                bound[:, h] = 2.0 ** -8 * (np.abs(out[:, h]) + spread) * (1 + 2 * eta) + 2 * eta * spread
            outs.append(out)
            bounds.append(bound)
        return np.concatenate(outs), np.concatenate(bounds)

    def attend(self, scale=None, out=None, stream=None, shared=None):
        out = torch.full((len(self.q), self.hq, self.dim), float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
        self.ctx.prefix_attention(self.q_dev, self.pool, self.table_dev, self.shared if shared is None else shared, self.L, self.n,
                                  self.scale if scale is None else scale, out, stream=stream)
        return out

    def flags(self):
        return self.ctx.device_error_flags(torch.cuda.current_stream().cuda_stream)


def within(got, ref, bound):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all()
    over = np.abs(got - ref) - bound
    assert over.max() <= 1e-30, "off by %.3e more than allowed at %s" % (over.max(), np.unravel_index(over.argmax(), over.shape))


def uniform(B, common, own, new=1):
    """B sequences with the same prefix."""
    return [0] + [common] * (B - 1), [common + own + 3 * i for i in range(B)], [new] * B


CASES = {  # common, L, n, query heads, KV heads, head_dim, FP8 pages
    "one": ([0], [0], [1], 8, 8, 64, False),
    "two_alone": ([0, 0], [5, 70], [1, 2], 4, 1, 128, False),
    "short_prefix": (*uniform(3, 50, 0), 8, 2, 64, False),          # below a step: nothing is shared
    "little_to_save": (*uniform(3, 120, 7), 8, 2, 64, False),
    "samples": (*uniform(3, 200, 0), 8, 2, 64, False),
    "only_new_tokens_of_their_own": ([0, 320, 320, 320, 320, 320], [320] * 6, [1, 3, 1, 2, 1, 1], 8, 1, 128, False),
    "cols_32": (*uniform(8, 640, 33), 32, 8, 128, False),
    "cols_33": (*uniform(11, 300, 1), 6, 2, 64, True),
    "cols_64": (*uniform(8, 1030, 40), 16, 2, 128, True),
    "cols_65": (*uniform(13, 257, 2), 5, 1, 64, False),
    "cols_128": (*uniform(16, 777, 60), 8, 1, 128, False),
    "cols_129_and_more": (*uniform(43, 500, 5), 6, 2, 64, False),
    "seven_heads": (*uniform(40, 400, 20), 7, 1, 128, True),
    "many_rows_each": (*uniform(5, 900, 30, 17), 10, 2, 128, False),  # 85 columns of one sequence, 425 of all
    "row_blocks": (*uniform(4, 700, 100, 70), 8, 2, 128, False),
    "row_blocks_fp8": (*uniform(3, 1300, 10, 150), 5, 1, 64, True),
    "prompts_alone_and_behind": ([0, 0, 512, 512, 0], [0, 512, 600, 512, 3], [300, 40, 1, 200, 1], 4, 2, 128, False),
    "nested": ([0, 600, 1500, 1500, 600, 1400, 1400, 600, 0, 64], [1500, 1600, 1501, 2000, 1400, 1400, 1477, 700, 64, 90], [1, 2, 1, 1, 3, 1, 1, 1, 1, 1], 8, 2, 128, False),
    "chain": ([0] + [64 * (i + 1) for i in range(21)], [64 * (i + 2) for i in range(22)], [1] * 22, 8, 2, 64, False),
    "chain_down": ([0] + [64 * (21 - i) for i in range(21)], [64 * (22 - i) for i in range(22)], [1] * 22, 8, 1, 64, True),
    "long": (*uniform(6, 9000, 300), 8, 1, 128, False),              # split ranges on both sides
    "long_wide": (*uniform(40, 20011, 900), 8, 1, 64, True),
    "long_row_blocks": (*uniform(3, 17000, 400, 90), 4, 1, 64, False),
}


@pytest.mark.parametrize("case", list(CASES))
def test_prefix_attention_matches_the_definition(case):
    b = Batch(*CASES[case], seed=len(case))
    ref, bound = b.reference()
    got = b.attend()
    within(got, ref, bound)
    assert torch.equal(got, b.attend())  # the same from run to run, bit for bit
    mixed = torch.empty_like(got)
    b.ctx.mixed_attention(b.q_dev, b.pool, b.table_dev, b.L, b.n, b.scale, mixed)
    within(mixed, got.double().cpu().numpy(), 2 * bound)
    assert b.flags() == 0


def test_the_same_batch_shared_less():
    """Nothing depends on how much of what is in common is named."""
    b = Batch(*CASES["nested"], seed=1)
    ref, bound = b.reference()
    for shared in (np.zeros_like(b.shared), np.minimum(b.shared, 100), b.shared // 2, b.shared):
        within(b.attend(shared=shared.astype(np.int32)), ref, bound)


def test_scale_zero_and_sharp_scores():
    b = Batch(*uniform(9, 800, 40), 8, 1, 128, seed=6, q_scale=12.0)
    within(b.attend(), *b.reference())
    within(b.attend(scale=0.0), *b.reference(scale=0.0))


@pytest.mark.parametrize("rows", [3, 40])
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_what_a_row_does_not_see_does_not_reach_it(bad, rows):
    """A new token that is not finite, K and V: only rows from it on see it."""
    args = (*uniform(5, 300, 20, rows), 8, 2, 64)

    def change(b):
        b.k[2][b.L[2] + 1, 0, 5] = bad
        b.v[2][b.L[2] + 1, 0, 3:9] = bad

    def v_alone(b):
        b.v[2][b.L[2] + 1, 0, 3:9] = bad
    clean, dirty, only_v = Batch(*args, seed=3), Batch(*args, seed=3, change=change), Batch(*args, seed=3, change=v_alone)
    a, b = clean.attend(), dirty.attend()
    seeing = np.zeros((len(clean.q), 8), bool)
    seeing[2 * rows + 1:3 * rows, :4] = True
    assert torch.equal(a[dev(~seeing)], b[dev(~seeing)])
    c = only_v.attend().double().cpu().numpy()
    assert torch.equal(a[dev(~seeing)].cpu(), torch.from_numpy(c[~seeing]).to(torch.bfloat16))
    touched = c[seeing][:, 3:9]
    assert np.isnan(touched).all() if np.isnan(bad) else (touched == bad).all()
    assert np.isfinite(c[seeing][:, :3]).all() and np.isfinite(c[seeing][:, 9:]).all()


@pytest.mark.parametrize("hq,n", [(2, 1), (8, 3), (8, 40)])
def test_a_row_whose_every_score_is_minus_infinity_gives_zeros(hq, n):
    def change(b):
        b.q[0, :, 5] = 1.0
        for k in b.k:
            k[:, :, 5] = np.where(np.arange(len(k))[:, None] < 321, -np.inf, 0.0)
    b = Batch([0, 320, 320, 320], [320, 330, 340, 350], [n] * 4, hq, 2, 64, seed=7, change=change)  # row 0 sees the prefix and itself
    b.q_dev[1:, :, 5] = 0.0
    b.q[1:, :, 5] = 0.0
    out = b.attend()
    assert not out[0].any()


def test_page_ids_outside_the_pool_raise_the_flag():
    b = Batch(*uniform(6, 640, 40), 8, 2, 64, seed=11)
    for row, column, bad in ((0, 3, b.num_pages), (4, 41, -5)):  # of the shared range, of a sequence's own
        keep = int(b.table_dev[row, column])
        b.table_dev[row, column] = bad
        b.attend()
        assert b.flags() == 2 and b.flags() == 0
        b.table_dev[row, column] = keep
    within(b.attend(), *b.reference())


def test_offsets_beyond_32_bits():
    pages = 2 ** 31 // (2 * 8 * 16 * 128) + 400  # element offsets pass 2^31, byte offsets 2^32
    b = Batch(*uniform(9, 400, 30), 16, 8, 128, seed=9, num_pages=pages, first_page=pages - 60)
    within(b.attend(), *b.reference())


def test_rows_behind_the_last_sequence_stay():
    b = Batch(*uniform(9, 400, 30, 2), 8, 2, 64, seed=10)
    out = torch.full((30, 8, 64), -3.0, dtype=torch.bfloat16, device="cuda")
    b.q_dev = torch.cat([b.q_dev, torch.full((12, 8, 64), float("nan"), dtype=torch.bfloat16, device="cuda")])
    b.attend(out=out)
    within(out[:18], *b.reference())
    assert (out[18:] == -3.0).all()


def test_streams_graphs_and_plans():
    b = Batch(*CASES["nested"], seed=12)
    first = torch.cuda.CUDAGraph()
    out = torch.zeros((len(b.q), 8, 128), dtype=torch.bfloat16, device="cuda")
    mark = torch.zeros(1, device="cuda")
    with torch.cuda.graph(first):  # nothing is planned yet
        with pytest.raises(ppd.PPDError) as e:
            b.attend(out=out, stream=torch.cuda.current_stream().cuda_stream)
        assert e.value.status == -3 and "capture" in str(e.value)
        mark.add_(1)
    first.replay()
    torch.cuda.synchronize()
    assert mark.item() == 1 and not out.any()
    eager = b.attend()
    side = torch.cuda.Stream()
    other = torch.zeros_like(out)
    side.wait_stream(torch.cuda.current_stream())
    b.attend(out=other, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(other, eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = torch.cuda.current_stream().cuda_stream
        b.attend(out=out, stream=s)
        with pytest.raises(ppd.PPDError):  # another batch: refused, and the capture goes on
            b.attend(out=out, stream=s, shared=np.zeros_like(b.shared))
    # other attention calls, eager calls of the same batch, and their waits between the replays
    for i in range(4):
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        assert torch.equal(b.attend(), eager)
        if i == 1:
            b.ctx.mixed_attention(b.q_dev, b.pool, b.table_dev, b.L, b.n, b.scale, torch.empty_like(out))
        if i == 2:
            weights = torch.zeros((len(b.L), 2, 2100), device="cuda")
            b.ctx.weighted_attention(b.q_dev, b.pool, b.table_dev, b.L, b.n, b.scale, torch.empty_like(out), weights)
    # plans that follow one another without a wait
    b.attend(shared=np.zeros_like(b.shared))
    for shared in (b.shared, b.shared // 2, b.shared, np.zeros_like(b.shared), b.shared, b.shared // 3, b.shared):
        last = b.attend(shared=shared.astype(np.int32))
    assert torch.equal(last, eager) and b.flags() == 0


def test_the_page_format_changes_between_calls_of_one_plan():
    b, c = (Batch(*CASES["nested"][:6], seed=13, fp8=fp8) for fp8 in (False, True))
    want = b.attend(), c.attend()
    ctx = b.ctx
    for fp8 in (True, False, True):  # one context, whose plan is that of the same lengths
        ctx.set_kv_format(*((ppd.PPD_KV_FP8_E4M3, SCALE8, SCALE8) if fp8 else (ppd.PPD_KV_BF16, 1.0, 1.0)))
        it = c if fp8 else b
        out = torch.empty_like(want[fp8])
        ctx.prefix_attention(it.q_dev, it.pool, it.table_dev, it.shared, it.L, it.n, it.scale, out)
        within(out, *it.reference())


def test_an_empty_batch_does_nothing():
    ctx = ppd.Context(8, 2, 64, 4)
    none, zero = torch.zeros((0, 8, 64), dtype=torch.bfloat16, device="cuda"), np.zeros(0, np.int32)
    ctx.prefix_attention(none, none, torch.zeros((0, 1), dtype=torch.int32, device="cuda"), zero, zero, zero, 1.0, none)
