"""The rotation of many rows, of which a workgroup has four, on the GPU against the definition in exact angles and 64 bits (tolerances of
test_gpu_positions): heads that run over into the next row, and halves whose partners other lanes have, among them."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2603_13358_amd as ppd  # noqa: E402
from test_gpu_positions import bf16, dev, near, rotated  # noqa: E402


@pytest.mark.parametrize("T", [2047, 2048, 2051])  # one row to a workgroup, four, four and a rest
@pytest.mark.parametrize("heads", [1, 3, 9, 33])
@pytest.mark.parametrize("dim,rotary,layout", [(64, 64, 0), (64, 24, 0), (64, 20, 1), (128, 128, 0), (128, 32, 0), (128, 126, 0), (128, 40, 0), (128, 128, 1)])
def test_many_rows_match_the_definition(T, heads, dim, rotary, layout):
    if heads == 33 and T != 2051:
        heads = 2
    r = np.random.default_rng(T + heads + rotary)
    ctx = ppd.Context(8, 2, dim, 4)
    inv_freq = ppd.ppd_rope_frequencies(rotary, 10000.0)
    ctx.set_rope(inv_freq, layout, 1.25)
    kinds = r.integers(-50, 200000, 64)  # positions, so that exact angles are few
    of = r.integers(0, 64, T)
    x = bf16(r.standard_normal((T, heads + 2, dim))).cuda()[:, 1:heads + 1]  # parts of wider rows
    whole = torch.full((T, heads + 1, dim), -7.0, dtype=torch.bfloat16, device="cuda")
    out = whole[:, :heads]
    ctx.rope(x, dev(kinds[of]), out, transpose=bool(T & 1))
    for first in range(0, T, 700):  # the reference is in 64 bits, row by row
        part = slice(first, min(T, first + 700))
        y, bound = rotated(x[part], kinds[of[part]], inv_freq, layout, 1.25, bool(T & 1))
        near(out[part], y, bound, np.arange(dim) < rotary)
    assert torch.equal(out[..., rotary:], x[..., rotary:]) and (whole[:, heads:] == -7.0).all()
    in_place = x.contiguous()
    ctx.rope(in_place, dev(kinds[of]), in_place, transpose=bool(T & 1))
    assert torch.equal(in_place, out)


@pytest.mark.parametrize("hq,hkv,dim,rotary,layout,fp8", [(6, 3, 64, 24, 0, False), (9, 9, 128, 126, 0, False), (8, 2, 128, 40, 0, True), (5, 5, 64, 64, 0, False)])
def test_an_append_of_many_rows_is_the_rotation_and_the_append(hq, hkv, dim, rotary, layout, fp8):
    T = 2051
    r = np.random.default_rng(T + hq)
    ctx = ppd.Context(hq, hkv, dim, T // 16 + 3)
    if fp8:
        ctx.set_kv_format(ppd.PPD_KV_FP8_E4M3, 2.0 ** -5, 0.3)
    ctx.set_rope(ppd.ppd_rope_frequencies(rotary), layout)
    rows = bf16(r.standard_normal((T, hq + 2 * hkv, dim))).cuda()
    q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    positions, slots = dev(r.integers(0, 9000, T)), dev(r.permutation((T // 16 + 3) * 16)[:T])
    pools = [torch.zeros(ctx.pool_elems(), dtype=torch.uint8 if fp8 else torch.bfloat16, device="cuda") for _ in range(2)]
    out, q_rot = (torch.empty((T, hq, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ctx.kv_append_rotated(q, k, v, positions, pools[0], slots, out)
    ctx.rope(q, positions, q_rot)
    assert torch.equal(out, q_rot)
    k_rot = torch.empty((T, hkv, dim), dtype=torch.bfloat16, device="cuda")
    ctx.rope(k, positions, k_rot)
    ctx.kv_append(k_rot, v.contiguous(), pools[1], slots)
    if not fp8:
        assert torch.equal(pools[0], pools[1])
    else:  # keys are rounded once, not to bf16 first: codes differ by a step at most, values' codes not at all
        a, b = (p.view(-1, 2, hkv * 16 * dim) for p in pools)
        assert torch.equal(a[:, 1], b[:, 1]) and ((a[:, 0].int() & 127) - (b[:, 0].int() & 127)).abs().max() <= 1
    assert ctx.device_error_flags() == 0
