"""The rotation by positions, on its own and on the way into the pages, on the GPU against the definition in exact angles and 64 bits.

Tolerances follow from the roundings.  An angle is off by |position| 2^-64 turns (the frequency as a fraction of 2^64; the frequencies here
are at most one radian) + 2^-32 (what is cut off) + 2^-26 (the rest as a binary32 number), the sine and cosine by 2^-22 as documented, their
product with the amplitude by 2^-24 of itself.  With eps the sum of these in radians, a rotated element A (a c - b s) is off by
A (|a| + |b|) (eps + 2^-22) before the last rounding (two more in binary32), and by 2^-8 of itself after it (bf16; FP8 codes of x / scale: 2^-4 of
themselves, or half of the smallest step, 2^-10)."""
import math
from fractions import Fraction

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2603_13358_amd as ppd  # noqa: E402

PAGE = 16
PI = Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def bf16(x):
    return torch.from_numpy(np.asarray(x)).float().to(torch.bfloat16)


def angles(positions, inv_freq):
    """Radians without whole turns, [position, pair], from exact products."""
    turn = [Fraction(float(f)) / (2 * PI) for f in inv_freq]
    return np.array([[float(int(p) * t % 1) for t in turn] for p in positions]).reshape(len(positions), len(turn)) * 2 * math.pi


def pairs(rotary, layout):
    i = np.arange(rotary // 2)
    return (i, i + rotary // 2) if layout == ppd.PPD_ROPE_HALF else (2 * i, 2 * i + 1)


def rotated(x, positions, inv_freq, layout, amplitude=1.0, transpose=False):
    """(result before its last rounding, bound of what binary32 is off by) of x [row, head, d] in 64 bits; elements that are not rotated as they are."""
    x = x.double().cpu().numpy()
    t = angles(positions, inv_freq)[:, None] * (-1 if transpose else 1)
    first, second = pairs(2 * len(inv_freq), layout)
    a, b = x[..., first], x[..., second]
    y, bound = x.copy(), np.zeros_like(x)
    y[..., first], y[..., second] = amplitude * (a * np.cos(t) - b * np.sin(t)), amplitude * (b * np.cos(t) + a * np.sin(t))
    far = np.abs(np.asarray(positions, np.float64))[:, None, None]
    eps = (far * 2.0 ** -64 + 2.0 ** -32 + 2.0 ** -26) * 2 * math.pi + 2.0 ** -22 + 2.0 ** -22
    bound[..., first] = bound[..., second] = abs(amplitude) * (np.abs(a) + np.abs(b)) * eps
    return y, bound


def near(got, y, bound, rotary_elements):
    got = got.double().cpu().numpy()
    allowed = bound + np.where(rotary_elements, 2.0 ** -8 * (np.abs(y) + bound), 0.0)
    over = np.abs(got - y) - allowed
    assert np.isfinite(got).all() and over.max() <= 0, "off by %.3e more than allowed at %s" % (over.max(), np.unravel_index(over.argmax(), over.shape))


CASES = [  # rows, heads, head_dim, rotary_dim, layout, amplitude, transpose
    (1, 1, 64, 64, 0, 1.0, False),
    (1, 8, 128, 128, 1, 1.0, True),
    (5, 3, 64, 32, 0, 1.25, False),
    (7, 6, 64, 24, 0, 1.0, False),     # halves of 12: no whole granules
    (3, 5, 128, 2, 0, -0.5, True),
    (9, 2, 128, 126, 0, 1.0, False),
    (6, 7, 128, 126, 1, 1.0, False),
    (130, 40, 128, 64, 0, 1.0, False),
    (33, 33, 64, 20, 1, 1.1, False),
    (1000, 9, 128, 128, 0, 1.0, True),
    (2, 4096, 64, 64, 1, 1.0, False),
]


@pytest.mark.parametrize("T,heads,dim,rotary,layout,amplitude,transpose", CASES)
def test_rope_matches_the_definition(T, heads, dim, rotary, layout, amplitude, transpose):
    r = np.random.default_rng(T + heads)
    ctx = ppd.Context(8, 2, dim, 4)
    inv_freq = ppd.ppd_rope_frequencies(rotary, 10000.0)
    ctx.set_rope(inv_freq, layout, amplitude)
    positions = r.integers(0, 200000, T)
    x = bf16(r.standard_normal((T, heads, dim))).cuda()
    out = torch.full((T, heads, dim), float("nan"), dtype=torch.bfloat16, device="cuda")
    ctx.rope(x, dev(positions), out, transpose=transpose)
    y, bound = rotated(x, positions, inv_freq, layout, amplitude, transpose)
    near(out, y, bound, np.arange(dim) < rotary)
    assert torch.equal(out[..., rotary:].view(torch.int16), x[..., rotary:].view(torch.int16))
    in_place = x.clone()
    ctx.rope(in_place, dev(positions), in_place, transpose=transpose)
    assert torch.equal(in_place, out)


def test_rope_of_far_and_negative_positions():
    ctx = ppd.Context(8, 2, 128, 4)
    inv_freq = ppd.ppd_rope_frequencies(128, 500000.0)
    ctx.set_rope(inv_freq)
    positions = np.array([0, 1, -1, 2 ** 24 + 1, 2 ** 31 - 1, 2 ** 31, 2 ** 32 + 12345, 2 ** 40 + 7, -2 ** 35 - 3, 2 ** 53 + 1])
    x = bf16(np.random.default_rng(1).standard_normal((len(positions), 4, 128))).cuda()
    out = torch.empty_like(x)
    ctx.rope(x, dev(positions), out)
    near(out, *rotated(x, positions, inv_freq, 0), True)
    assert torch.equal(out[0], x[0])
    # all of int64: angles are those of the position modulo 2^64 turns' units, and whatever they are, lengths of pairs stay
    ends = dev(np.array([-2 ** 63, 2 ** 63 - 1] * 5))
    ctx.rope(x, ends, out)
    before, after = (t.double()[..., :64].square() + t.double()[..., 64:].square() for t in (x, out))
    assert ((after - before).abs() <= before * (2 * 2.0 ** -8 * 1.01) + 1e-30).all()


def test_rope_of_strided_rows_touches_nothing_else():
    ctx = ppd.Context(6, 2, 64, 4)
    inv_freq = ppd.ppd_rope_frequencies(48, 10000.0)
    ctx.set_rope(inv_freq)
    r = np.random.default_rng(2)
    whole = bf16(r.standard_normal((20, 10, 64))).cuda()  # queries, keys, values side by side
    positions = r.integers(0, 5000, 17)
    target = torch.full((20, 9, 64), -7.0, dtype=torch.bfloat16, device="cuda")
    ctx.rope(whole[:, :6], dev(positions), target[:, 2:8])  # rows behind the 17 positions are not rotated
    near(target[:17, 2:8], *rotated(whole[:17, :6], positions, inv_freq, 0), np.arange(64) < 48)
    rest = target.clone()
    rest[:17, 2:8] = -7.0
    assert (rest == -7.0).all()
    before = whole.clone()
    ctx.rope(whole[:, 6:8], dev(positions), whole[:, 6:8])  # keys, in place
    near(whole[:17, 6:8], *rotated(before[:17, 6:8], positions, inv_freq, 0), np.arange(64) < 48)
    whole[:17, 6:8] = before[:17, 6:8]
    assert torch.equal(whole, before)


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("rotary", [24, 32])
def test_elements_that_are_not_rotated_keep_their_bits(layout, rotary):
    """All bit patterns, NaN of every kind among them; infinities beside them do not reach other pairs."""
    ctx = ppd.Context(2, 2, 64, 8)
    ctx.set_rope(ppd.ppd_rope_frequencies(rotary), layout)
    bits = np.arange(65536, dtype=np.uint16).reshape(-1, 1, 64).view(np.int16)
    x = dev(bits).view(torch.bfloat16)
    out = torch.zeros_like(x)
    ctx.rope(x, dev(np.arange(len(bits)) * 37), out)
    assert torch.equal(out[..., rotary:].view(torch.int16), x[..., rotary:].view(torch.int16))
    y = torch.ones((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    first, second = pairs(rotary, layout)
    y[0, 0, first[3]] = float("inf")
    ctx.rope(y, dev(np.array([5])), y)
    finite = np.isfinite(y.double().cpu().numpy()[0, 0])
    assert not finite[first[3]] and not finite[second[3]] and finite.sum() == 62


def test_the_transpose_is_the_gradient():
    """Against the formula (autograd of a plain rotation in 64 bits) and against differences of the plain function."""
    ctx = ppd.Context(8, 2, 64, 4)
    inv_freq = ppd.ppd_rope_frequencies(32, 100.0, ppd.PPD_ROPE_SCALE_LINEAR, 2.0)
    r = np.random.default_rng(3)
    positions = r.integers(0, 3000, 6)
    for layout in (0, 1):
        ctx.set_rope(inv_freq, layout, 1.5)
        x, g = (bf16(r.standard_normal((6, 8, 64))).cuda() for _ in range(2))
        grad = torch.empty_like(x)
        ctx.rope(g, dev(positions), grad, transpose=True)
        first, second = (torch.from_numpy(i).cuda() for i in pairs(32, layout))
        t = dev(angles(positions, inv_freq))[:, None]

        def plain(v):
            a, b = v[..., first], v[..., second]
            y = v.clone()
            y[..., first], y[..., second] = 1.5 * (a * t.cos() - b * t.sin()), 1.5 * (b * t.cos() + a * t.sin())
            return y
        leaf = x.double().requires_grad_()
        (plain(leaf) * g.double()).sum().backward()
        _, bound = rotated(g, positions, inv_freq, layout, 1.5, True)
        near(grad, leaf.grad.cpu().numpy(), bound, np.arange(64) < 32)
        step = torch.zeros((6, 8, 64), dtype=torch.float64, device="cuda")
        step[2, 5, 7] = 2.0 ** -10  # the function is linear: a difference is exact but for 64-bit rounding
        slope = float(((plain(x.double() + step) - plain(x.double() - step)) * g.double()).sum()) / 2.0 ** -9
        assert abs(float(grad[2, 5, 7]) - slope) <= 2.0 ** -8 * abs(slope) * 1.01 + float(bound[2, 5, 7]) + 1e-9


def test_rope_beyond_32_bit_offsets():
    ctx = ppd.Context(8, 2, 128, 4)
    inv_freq = ppd.ppd_rope_frequencies(128)
    ctx.set_rope(inv_freq)
    rows, stride = 5, 2 ** 30 + 2 ** 28 + 8  # the last rows start behind 2^32 elements
    whole = torch.empty(rows * stride, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(whole, (rows, 2, 128), (stride, 128, 1))
    x.copy_(bf16(np.random.default_rng(4).standard_normal((rows, 2, 128))))
    before = x.clone()
    positions = np.arange(rows) * 1001
    ctx.rope(x, dev(positions), x)
    near(x, *rotated(before, positions, inv_freq, 0), True)


def test_rope_of_more_rows_than_one_dimension_of_a_launch_has_threads():
    """2^26 rows and some, four to a workgroup of 256 threads: more than 2^32 threads.  Rows around each 2^24 (and the ends) are checked, those between
    are zeros and stay so."""
    T = 2 ** 26 + 5
    ctx = ppd.Context(8, 2, 64, 4)
    inv_freq = ppd.ppd_rope_frequencies(64)
    ctx.set_rope(inv_freq)
    rows = np.unique(np.concatenate([at + np.arange(-6, 6) for at in range(0, T + 8, 2 ** 24)] + [np.arange(T - 6, T)]))
    rows = rows[(rows >= 0) & (rows < T)]
    x = torch.zeros((T, 1, 64), dtype=torch.bfloat16, device="cuda")
    before = bf16(np.random.default_rng(6).standard_normal((len(rows), 1, 64))).cuda()
    x[dev(rows)] = before
    ctx.rope(x, torch.arange(T, device="cuda"), x)
    near(x[dev(rows)], *rotated(before, rows, inv_freq, 0), True)
    x[dev(rows)] = 0
    assert not any(part.any() for part in x.split(2 ** 22))


# ---- the append ----

def pool_bits(ctx, fp8):
    r = np.random.default_rng(9)
    bits = r.integers(0, 256, ctx.pool_elems()).astype(np.uint8) if fp8 else r.integers(0, 65536, ctx.pool_elems()).astype(np.uint16).view(np.int16)
    return dev(bits)


def offsets(slots, h, hkv, dim, value):
    """[token, d]: element offsets in a pool, from the layout's formulas."""
    t, d = np.asarray(slots)[:, None], np.arange(dim)[None]
    base = t // PAGE * (2 * hkv * PAGE * dim) + h * PAGE * dim
    tok = t % PAGE
    if value:
        return base + hkv * PAGE * dim + tok // 8 * (dim * 8) + d * 8 + tok % 8
    return base + d // 8 * (PAGE * 8) + tok * 8 + d % 8


def slots_of(kind, T, pages, r):
    """Runs that start anywhere, single tokens of many sequences, or any order; some skipped, one beyond the pool."""
    if kind == "run":
        return np.arange(T) + 5
    if kind == "decodes":
        return r.permutation(pages)[:T] * PAGE + r.integers(0, PAGE, T)
    s = r.permutation(pages * PAGE)[:T]
    s[r.random(T) < 0.2] = -1
    return s


APPENDS = [  # tokens, query heads, KV heads, head_dim, rotary_dim, layout, FP8 pages, slots
    (1, 8, 2, 64, 64, 0, False, "run"),
    (1, 6, 6, 128, 128, 0, True, "decodes"),
    (7, 8, 8, 64, 24, 0, False, "run"),
    (7, 8, 8, 64, 24, 0, True, "any"),
    (30, 40, 8, 128, 64, 1, False, "any"),
    (100, 12, 4, 128, 128, 0, True, "run"),
    (130, 5, 1, 64, 32, 1, True, "any"),
    (500, 32, 8, 128, 128, 0, False, "decodes"),
    (1100, 16, 8, 64, 64, 0, False, "run"),    # 16 tokens to a workgroup
    (1100, 8, 8, 128, 126, 0, True, "any"),
    (8200, 1, 1, 128, 128, 1, False, "any"),
]


@pytest.mark.parametrize("T,hq,hkv,dim,rotary,layout,fp8,kind", APPENDS)
@pytest.mark.parametrize("packed", [False, True])
def test_rotated_append_matches_the_definition(T, hq, hkv, dim, rotary, layout, fp8, kind, packed):
    r = np.random.default_rng(T)
    pages = T + 10 if kind == "decodes" else T // PAGE + 12
    ctx = ppd.Context(hq, hkv, dim, pages)
    if fp8:
        ctx.set_kv_format(ppd.PPD_KV_FP8_E4M3, 2.0 ** -5, 0.3)
    inv_freq = ppd.ppd_rope_frequencies(rotary, 10000.0, ppd.PPD_ROPE_SCALE_BASE if rotary > 2 else 0, 2.0)
    ctx.set_rope(inv_freq, layout, 1.25)
    whole = bf16(r.standard_normal((T, hq + 2 * hkv, dim))).cuda()
    q, k, v = whole[:, :hq], whole[:, hq:hq + hkv], whole[:, hq + hkv:]
    if not packed:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    positions, slots = r.integers(0, 100000, T), slots_of(kind, T, pages, r)
    beyond = T >= 30 and kind == "any"
    if beyond:
        slots[T // 2] = pages * PAGE
    pool = pool_bits(ctx, fp8)
    want = pool.cpu().numpy().copy()
    out = torch.full((T, hq, dim), float("nan"), dtype=torch.bfloat16, device="cuda")
    ctx.kv_append_rotated(q, k, v, dev(positions), pool, dev(slots), out)
    assert ctx.device_error_flags() == (1 if beyond else 0)
    near(out, *rotated(q, positions, inv_freq, layout, 1.25), np.arange(dim) < rotary)
    got = pool.cpu().numpy()
    good = (slots >= 0) & (slots < pages * PAGE)
    y, bound = rotated(k, positions, inv_freq, layout, 1.25)
    # what ppd_rope and ppd_kv_append do one after the other: values, and on bf16 pages keys, to the bit
    two = pool_bits(ctx, fp8)
    k_rot = torch.empty((T, hkv, dim), dtype=torch.bfloat16, device="cuda")
    ctx.rope(k, dev(positions), k_rot)
    quiet = slots.copy()
    quiet[~good] = -1
    ctx.kv_append(k_rot, v.contiguous(), two, dev(quiet))
    two = two.cpu().numpy()
    written = np.zeros(want.shape, bool)
    for h in range(hkv):
        at = offsets(slots[good], h, hkv, dim, True)
        assert np.array_equal(got[at], two[at])
        written[at] = True
        at = offsets(slots[good], h, hkv, dim, False)
        written[at] = True
        if not fp8:
            assert np.array_equal(got[at], two[at])
        else:
            codes = torch.from_numpy(got[at]).view(torch.float8_e4m3fn).double().numpy()
            x, b = y[good, h] / 2.0 ** -5, bound[good, h] / 2.0 ** -5
            assert (np.abs(codes - np.clip(x, -448, 448)) <= b + np.maximum(2.0 ** -4 * (np.abs(x) + b), 2.0 ** -10)).all()
    assert np.array_equal(got[~written], want[~written])
    # without queries: the same pool
    alone = pool_bits(ctx, fp8)
    ctx.kv_append_rotated(None, k, v, dev(positions), alone, dev(quiet), None)
    assert np.array_equal(alone.cpu().numpy(), got)


def test_rotated_append_takes_queries_in_place_and_padded_batches():
    ctx = ppd.Context(8, 2, 128, 8)
    inv_freq = ppd.ppd_rope_frequencies(128)
    ctx.set_rope(inv_freq)
    r = np.random.default_rng(5)
    q, k, v = (bf16(r.standard_normal((12, h, 128))).cuda() for h in (8, 2, 2))
    before = q.clone()
    positions = np.arange(20, 32)
    pool = pool_bits(ctx, False)
    ctx.kv_append_rotated(q, k, v, dev(positions), pool, dev(np.arange(9) + 40), q)  # nine slots: the rows behind are padding
    near(q[:9], *rotated(before[:9], positions[:9], inv_freq, 0), True)
    assert torch.equal(q[9:], before[9:])
    pool2 = pool_bits(ctx, False)
    ctx.kv_append_rotated(None, k[:9], v[:9], dev(positions[:9]), pool2, dev(np.arange(9) + 40), None)
    assert torch.equal(pool, pool2)


def test_fp8_keys_saturate_and_keep_nan():
    ctx = ppd.Context(2, 2, 64, 2)
    ctx.set_kv_format(ppd.PPD_KV_FP8_E4M3, 2.0 ** -8, 2.0 ** -8)
    ctx.set_rope(ppd.ppd_rope_frequencies(32))
    k = torch.ones((1, 2, 64), dtype=torch.bfloat16, device="cuda")
    k[0, 0, 1], k[0, 0, 18], k[0, 0, 40], k[0, 0, 41], k[0, 0, 42] = float("nan"), float("inf"), float("-inf"), float("nan"), 1000.0
    pool = torch.zeros(ctx.pool_elems(), dtype=torch.uint8, device="cuda")
    ctx.kv_append_rotated(None, k, k.clone(), dev(np.array([0])), pool, dev(np.array([3])), None)
    codes = pool.view(torch.float8_e4m3fn).double().cpu().numpy()
    got = codes[offsets([3], 0, 2, 64, False)][0]
    # position 0: a turn of nothing, but infinity times a sine of zero is no number, nor is what NaN is paired with
    nan = np.zeros(64, bool)
    nan[[1, 17, 2, 41]] = True
    assert np.array_equal(np.isnan(got), nan)
    assert got[18] == 448 and got[40] == -448 and got[42] == 448 and got[0] == 256


def test_settings_hold_for_calls_that_were_made_and_captured_under_them():
    ctx = ppd.Context(8, 2, 64, 4)
    a, b = ppd.ppd_rope_frequencies(64, 10000.0), ppd.ppd_rope_frequencies(32, 500.0)
    r = np.random.default_rng(6)
    x = bf16(r.standard_normal((50, 8, 64))).cuda()
    positions = r.integers(0, 9000, 50)
    p = dev(positions)
    first, second, eager = (torch.empty_like(x) for _ in range(3))
    ctx.set_rope(a)
    ctx.rope(x, p, first)  # the first launch is not a captured one
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = torch.cuda.current_stream().cuda_stream
        ctx.set_rope(a)
        ctx.rope(x, p, first, stream=s)
        ctx.set_rope(b, ppd.PPD_ROPE_INTERLEAVED)
        ctx.rope(x, p, second, stream=s)
    for i in range(3):
        for t in (first, second):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        ctx.set_rope(b if i % 2 else a)
        ctx.rope(x, p, eager)
        torch.cuda.synchronize()
        near(first, *rotated(x, positions, a, 0), True)
        near(second, *rotated(x, positions, b, 1), np.arange(64) < 32)
        near(eager, *rotated(x, positions, b if i % 2 else a, 0), np.arange(64) < (32 if i % 2 else 64))


def test_append_on_streams_and_in_graphs():
    ctx = ppd.Context(16, 4, 128, 40)
    ctx.set_rope(ppd.ppd_rope_frequencies(128), ppd.PPD_ROPE_INTERLEAVED)
    r = np.random.default_rng(7)
    whole = bf16(r.standard_normal((60, 24, 128))).cuda()
    q, k, v = whole[:, :16], whole[:, 16:20], whole[:, 20:]
    positions, slots = dev(r.integers(0, 9000, 60)), dev(r.permutation(640)[:60])
    ref, ref_out = pool_bits(ctx, False), torch.empty((60, 16, 128), dtype=torch.bfloat16, device="cuda")
    ctx.kv_append_rotated(q, k, v, positions, ref, slots, ref_out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    pool, out = pool_bits(ctx, False), torch.zeros_like(ref_out)
    side.wait_stream(torch.cuda.current_stream())
    ctx.kv_append_rotated(q, k, v, positions, pool, slots, out, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(pool, ref) and torch.equal(out, ref_out)
    clean = pool_bits(ctx, False)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.kv_append_rotated(q, k, v, positions, pool, slots, out, stream=torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        pool.copy_(clean)
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(pool, ref) and torch.equal(out, ref_out)


def test_an_empty_call_does_nothing():
    ctx = ppd.Context(8, 2, 64, 4)
    ctx.set_rope(ppd.ppd_rope_frequencies(64))
    none = torch.zeros((0, 8, 64), dtype=torch.bfloat16, device="cuda")
    kv, idx = none[:, :2], torch.zeros(0, dtype=torch.int64, device="cuda")
    pool = pool_bits(ctx, False)
    before = pool.clone()
    ctx.rope(none, idx, none)
    ctx.kv_append_rotated(none, kv, kv, idx, pool, idx, none)
    assert torch.equal(pool, before) and ctx.device_error_flags() == 0
