"""Scores that are not a number, in attention whose key ranges are cut and joined: a row that sees a key with NaN, or whose query has one, is NaN
in every tile shape and wherever the key lies, as by the definition; the others are what they were, bit for bit."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import test_gpu_operators as operators  # noqa: E402
import test_gpu_prefix as prefix  # noqa: E402


def nan_rows(out):
    """[row, head]: whether a result is NaN, which it is as a whole or not at all."""
    bad = torch.isnan(out)
    assert torch.equal(bad.all(-1), bad.any(-1))
    return bad.all(-1).cpu().numpy()


def dev_mask(a):
    return torch.from_numpy(a).cuda()


def mixed(b):
    out = torch.empty((len(b.q), b.hq, b.dim), dtype=torch.bfloat16, device="cuda")
    b.ctx.mixed_attention(b.q_dev, b.pool, b.table_dev, b.L, b.n, b.scale, out)
    return out


# More shapes than prefix.CASES has: one sequence's columns in a tile of each kind that writes its rows itself, and one new token that is alone in
# what a wave, or a sequence, has of its own.
ALONE = {
    "wave_32": ([0], [96], [1], 8, 1, 64, False),
    "wave_32_fp8": ([0], [32], [1], 8, 2, 128, True),
    "wave_64": ([0], [96], [9], 5, 1, 128, False),
    "direct_64": ([0], [70], [50], 1, 1, 64, False),
    "direct_128": ([0], [70], [100], 2, 2, 128, False),
    "direct_row_block": ([0], [0], [290], 1, 1, 64, False),
    "split": ([0], [9000], [1], 8, 1, 128, False),
    "split_128": ([0], [9000], [100], 1, 1, 64, True),
    "own_token_64": (*prefix.uniform(7, 1280, 0), 8, 1, 64, False),
    "own_token_128": (*prefix.uniform(14, 1280, 0), 8, 1, 128, True),
}
SHAPES = {**ALONE, **prefix.CASES}


@pytest.mark.parametrize("case", list(SHAPES))
def test_prefix_rows_whose_query_is_nan(case):
    clean = prefix.Batch(*SHAPES[case], seed=len(case))
    want = clean.attend()
    bad = np.zeros((len(clean.q), clean.hq), bool)
    bad[0, 0] = bad[-1, -1] = bad[len(bad) // 2, clean.hq // 2] = True
    clean.q_dev[dev_mask(bad)] = float("nan")
    got = clean.attend()
    assert np.array_equal(nan_rows(got), bad) and np.array_equal(nan_rows(mixed(clean)), bad)
    assert torch.equal(got[dev_mask(~bad)], want[dev_mask(~bad)])


@pytest.mark.parametrize("case,which", [(case, which) for which in ("new", "cached") for case, (_, L, *_) in SHAPES.items() if which == "new" or L[len(L) // 2] > 0])
def test_prefix_rows_that_see_a_key_with_nan(case, which):
    args = SHAPES[case]
    i = len(args[1]) // 2
    at = args[1][i] + (args[2][i] - 1) // 2 if which == "new" else args[1][i] - 1  # of sequence i; cached: its last, which others may share

    def change(b):
        b.k[i][at, 0, 7] = np.nan
        first = i
        while which == "cached" and at < b.shared[first]:  # written by the first sequence that has the page
            first -= 1
            b.k[first][at, 0, 7] = np.nan
    clean, dirty = prefix.Batch(*args, seed=len(case)), prefix.Batch(*args, seed=len(case), change=change)
    seq = np.repeat(np.arange(len(clean.L)), clean.n)
    has = np.zeros(len(clean.L), bool)
    has[i] = True
    for other in range(i + 1, len(has)):
        has[other] = has[other - 1] and at < clean.shared[other]
    for other in range(i - 1, -1, -1):
        has[other] = has[other + 1] and at < clean.shared[other + 1]
    row = np.arange(len(seq)) - (np.cumsum(clean.n) - clean.n)[seq]
    bad = np.zeros((len(seq), clean.hq), bool)
    bad[:, :clean.hq // clean.hkv] = (has[seq] & (at <= clean.L[seq] + row))[:, None]
    assert bad.any()
    got = dirty.attend()
    assert np.array_equal(nan_rows(got), bad) and np.array_equal(nan_rows(mixed(dirty)), bad)
    assert torch.equal(got[dev_mask(~bad)], clean.attend()[dev_mask(~bad)])


@pytest.mark.parametrize("rows", [3, 40])
def test_prefix_rows_that_see_a_new_token_of_nan(rows):
    """K and V of it, in a batch where most rows do not see it."""
    args = (*prefix.uniform(5, 300, 20, rows), 8, 2, 64)

    def change(b):
        b.k[2][b.L[2] + 1, 0, 5] = b.v[2][b.L[2] + 1, 0, 3] = np.nan
    dirty = prefix.Batch(*args, seed=3, change=change)
    bad = np.zeros((len(dirty.q), 8), bool)
    bad[2 * rows + 1:3 * rows, :4] = True
    assert np.array_equal(nan_rows(dirty.attend()), bad)


@pytest.mark.parametrize("L,n,hq,hkv,dim,fp8,words", operators.TREES, ids=lambda x: str(x).replace(" ", ""))
@pytest.mark.parametrize("what", ["query", "key", "node"])
def test_tree_rows_with_a_score_that_is_nan(L, n, hq, hkv, dim, fp8, words, what):
    """A NaN query; NaN in the last cached key, which all rows of the sequence see; NaN in a node, which some see."""
    i, G = len(L) - 1, hq // hkv
    at = L[i] + n[i] // 2 if what == "node" else max(L[i] - 1, 0)

    def fill(b):
        if what != "query":
            b.k[i][at, 0, 7] = np.nan
    clean, dirty = (operators.Batch(L, n, hq, hkv, dim, fp8, seed=40, kv=kv) for kv in (None, fill))
    mask = operators.random_mask(clean, words, seed=41)
    bad = np.zeros((len(clean.q), hq), bool)
    if what == "query":
        bad[0, 0] = bad[-1, -1] = True
        dirty.q_dev[dev_mask(bad)] = float("nan")
    else:
        bad[int(clean.n[:i].sum()):, :G] = clean.sees(i, mask)[:, at, None]
    got = dirty.tree(mask)
    assert np.array_equal(nan_rows(got), bad)
    assert torch.equal(got[dev_mask(~bad)], clean.tree(mask)[dev_mask(~bad)])


@pytest.mark.parametrize("L,n,hq,hkv,dim,fp8", operators.WEIGHTED, ids=lambda x: str(x).replace(" ", ""))
@pytest.mark.parametrize("what", ["query", "key"])
def test_weights_of_rows_with_a_score_that_is_nan(L, n, hq, hkv, dim, fp8, what):
    """Keys that such a row sees have no weight that is a number; other KV heads and sequences keep theirs."""
    i, G = len(L) - 1, hq // hkv
    row = int(n[i]) - 1  # of the sequence: it sees all keys
    at = L[i] + row

    def fill(b):
        if what == "key":
            b.k[i][at, 0, 7] = np.nan
    clean, dirty = (operators.Batch(L, n, hq, hkv, dim, fp8, seed=42, kv=kv) for kv in (None, fill))
    bad = np.zeros((len(clean.q), hq), bool)
    bad[-1, :G if what == "key" else 1] = True
    if what == "query":
        dirty.q_dev[dev_mask(bad)] = float("nan")
    want, w = (torch.zeros((len(L), hkv, max(x + y for x, y in zip(L, n))), device="cuda") for _ in range(2))
    clean_out, got = clean.weighted(want), dirty.weighted(w)
    assert np.array_equal(nan_rows(got), bad)
    assert torch.equal(got[dev_mask(~bad)], clean_out[dev_mask(~bad)])
    assert torch.isnan(w[i, 0, :at + 1]).all()
    assert torch.equal(w[:i], want[:i]) and torch.equal(w[i, 1:], want[i, 1:])
