"""Tree and weighted attention and kv_compact on the GPU at inputs where a token or a row drops out."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2603_13358_amd as ppd  # noqa: E402
from test_gpu_operators import Batch, dev, moved, within  # noqa: E402


@pytest.mark.parametrize("layers", [1, 2])
def test_weights_of_tokens_that_stay_stay_as_well(layers):
    r = np.random.default_rng(60)
    pool = r.integers(0, 65536, (layers, 8, 2 * 2 * 16 * 64)).astype(np.uint16)
    weights = r.random((layers, 1, 2, 120)).astype(np.float32)
    ctx = ppd.Context(2, 2, 64, 8)

    def compact(table, keep, first, good, flag):
        """`good`: the entries that move."""
        got, w = dev(pool.view(np.int16)), dev(weights)
        ctx.kv_compact(got, dev(table), dev(np.array([keep], np.int32)), np.array([first], np.int32), np.array([len(keep)], np.int32),
                       layer_stride_elems=pool[0].size, num_layers=layers, weights=w)
        assert ctx.device_error_flags() == flag
        want_pool, want_w = pool.copy(), weights.copy()
        for i in good:
            for l in range(layers):
                want_pool[l] = moved(want_pool[l], table.clip(0, 7), np.array([[keep[i]]]), [first + i], [1], 2, 64)
            want_w[:, :, :, first + i] = weights[:, :, :, keep[i]]
        assert np.array_equal(got.cpu().numpy().view(np.uint16), want_pool)
        assert np.array_equal(w.cpu().numpy(), want_w)

    whole = np.arange(8, dtype=np.int32)[None]
    compact(whole, [5, 5, 1, 125, 90], 2, [0], 8)  # repeated, below its place, beyond the weights, not above the one before
    compact(whole, [20, 40, 70], 14, [0, 1, 2], 0)
    for bad in (8, -1):  # the page of token 20 and of place 16
        table = whole.copy()
        table[0, 1] = bad
        compact(table, [20, 40, 70], 14, [1], 2)
    # many steps of a long list, every second page missing
    table = whole.copy()
    table[0, 1::2] = 1 << 30
    keep = list(range(30, 110))
    compact(table, keep, 3, [i for i, t in enumerate(keep) if t // 16 % 2 == 0 and (3 + i) // 16 % 2 == 0], 2)


@pytest.mark.parametrize("n,hq,dim", [(1, 8, 64), (8, 8, 128), (40, 8, 128), (70, 2, 64), (300, 2, 128)])
def test_a_row_whose_every_score_is_minus_infinity_gives_zeros_and_no_weight(n, hq, dim):
    def fill(b):
        b.q[..., 5] = 1.0
        b.k[0][0, :, 5] = -np.inf
    b = Batch([0], [n], hq, 2, dim, seed=61, kv=fill)  # row 0 sees token 0 alone
    w = torch.full((1, 2, n), float("nan"), device="cuda")
    out = b.weighted(w)
    b.k[0][0] = 0.0

    def sees(i):
        seen = np.tril(np.ones((n, n), bool))
        seen[:, 0] = False
        return seen
    b.sees = lambda i, mask=None: sees(i)
    ref, bound, weights = b.reference()
    assert not ref[0].any() and not out[0].any()
    within(out, ref, bound)
    within(w[0], *weights[0])


@pytest.mark.parametrize("L,n,hq,hkv,dim,fp8", [([9000], [70], 8, 1, 128, False), ([5000, 3], [130, 60], 10, 2, 64, True),
                                                ([3000, 200, 2500], [300, 1, 290], 2, 1, 64, False)], ids=["d128", "fp8", "d64"])
def test_weights_of_split_ranges_and_several_row_blocks(L, n, hq, hkv, dim, fp8):
    """Every row's reference comes from the join of its own block's partials."""
    b = Batch(L, n, hq, hkv, dim, fp8, seed=62)
    ref, bound, weights = b.reference()
    w = torch.zeros((len(L), hkv, int((b.L + b.n).max())), device="cuda")
    within(b.weighted(w), ref, bound)
    for i, (ww, wb) in enumerate(weights):
        within(w[i, :, :L[i] + n[i]], ww, wb + 2.0 ** -23 * ww)
    assert b.flags() == 0
