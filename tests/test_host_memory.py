"""What the calls of positions and shared prefixes refuse in Python: tensors in memory that the GPU does not reach (the entry point is a stand-in that
counts what is passed on, the context an address that nothing reads), and integers of more than 64 bits."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2603_13358_amd as ppd  # noqa: E402
from paper_2603_13358_amd import binding  # noqa: E402

PASSED_ON = 77


def handle(address):
    h = ctypes.c_void_p(address)
    h.num_q_heads, h.num_kv_heads, h.head_dim = 8, 2, 64
    return h


class Elsewhere:
    """A tensor that says it is on the GPU, or in pinned memory."""

    def __init__(self, tensor, is_cuda, pinned=False):
        self.tensor, self.is_cuda, self.pinned = tensor, is_cuda, pinned
        self.dtype, self.shape = tensor.dtype, tensor.shape

    def is_pinned(self):
        return self.pinned

    def stride(self):
        return self.tensor.stride()

    def is_contiguous(self):
        return self.tensor.is_contiguous()

    def data_ptr(self):
        return self.tensor.data_ptr()


def rows(n, heads):
    return torch.zeros(n, heads, 64, dtype=torch.bfloat16)


def index(n):
    return torch.zeros(n, dtype=torch.int64)


S, L, N = np.array([0, 16], np.int32), np.array([30, 20], np.int32), np.array([2, 3], np.int32)
CALLS = {
    "rope": dict(x=lambda: rows(5, 8), positions=lambda: index(5), out=lambda: rows(5, 8)),
    "append": dict(q=lambda: rows(5, 8), k=lambda: rows(5, 2), v=lambda: rows(5, 2), positions=lambda: index(5), slot_mapping=lambda: index(5), q_out=lambda: rows(5, 8)),
    "prefix": dict(q=lambda: rows(5, 8), page_tables=lambda: torch.zeros(2, 3, dtype=torch.int32), out=lambda: rows(5, 8)),
}


@pytest.fixture
def passed_on(monkeypatch):
    """Entry points that count their calls and read nothing."""
    ppd.load_library()
    calls = []

    def stand_in(*_):
        calls.append(1)
        return PASSED_ON
    fn = ctypes.CFUNCTYPE(ctypes.c_int32)(stand_in)  # its arguments are the caller's to clear away
    for name in ("_fn_rope", "_fn_append_rotated", "_fn_prefix"):
        monkeypatch.setattr(binding, name, ctypes.cast(fn, ctypes.c_void_p).value)
    monkeypatch.setattr(binding, "ppd_last_error", lambda ctx=None: "")
    calls.append(fn)
    yield lambda: len(calls) - 1


def call(kind, h, a):
    with pytest.raises(ppd.PPDError) as e:
        if kind == "rope":
            ppd.ppd_rope(h, a["x"], a["positions"], a["out"])
        elif kind == "append":
            ppd.ppd_kv_append_rotated(h, a["q"], a["k"], a["v"], a["positions"], 1 << 20, a["slot_mapping"], a["q_out"])
        else:
            ppd.ppd_prefix_attention(h, a["q"], 1 << 20, a["page_tables"], S, L, N, 1.0, a["out"])
    return e.value


@pytest.mark.parametrize("kind", list(CALLS))
def test_tensors_of_the_host_are_refused(kind, passed_on):
    h = handle(1 << 20)
    good = {name: Elsewhere(make(), True) for name, make in CALLS[kind].items()}
    assert call(kind, h, good).status == PASSED_ON and passed_on() == 1
    for name, make in CALLS[kind].items():
        e = call(kind, h, dict(good, **{name: make()}))
        assert e.status == -3 and str(e).endswith(name + " has to be on the GPU")
        assert passed_on() == 1
    for name, make in CALLS[kind].items():  # pinned memory is reached
        assert call(kind, h, dict(good, **{name: Elsewhere(make(), False, True)})).status == PASSED_ON
    addresses = dict(good, **{name: 1 << 21 for name in good if name in ("out", "q_out", "page_tables")})
    if kind == "append":
        assert call(kind, h, addresses).status == PASSED_ON


@pytest.mark.parametrize("far", [1 << 63, (1 << 64) + 5, -(1 << 63) - 1])
def test_integers_are_not_cut_to_64_bits(far):
    """Counts and strides; the context is NULL, which the library itself would refuse with PPD_ERR_NULL."""
    def refused(what, f, *args, **kw):
        with pytest.raises(ppd.PPDError) as e:
            f(None, *args, **kw)
        return e.value.status == -3 and what in str(e.value)
    address = 1 << 20
    assert refused("T", ppd.ppd_rope, rows(5, 8), index(5), rows(5, 8), T=far)
    assert refused("T", ppd.ppd_kv_append_rotated, None, rows(5, 2), rows(5, 2), index(5), address, index(5), None, T=far)
    assert refused("stride", ppd.ppd_rope, address, index(5), address, heads=8, x_stride=far, out_stride=512)
    assert refused("stride", ppd.ppd_rope, address, index(5), address, heads=8, x_stride=512, out_stride=far)
    assert refused("stride", ppd.ppd_kv_append_rotated, None, address, address, index(5), address, index(5), None, k_stride=128, v_stride=far)
