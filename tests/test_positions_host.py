"""Host side of the rotation by positions and of the append with it on the CPU: their code compiled against a stand-in for the HIP runtime
(tests/native/host_runtime), launches recorded, under AddressSanitizer + UndefinedBehaviorSanitizer; and what their Python calls refuse."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2603_13358_amd as ppd  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    path = str(tmp_path_factory.mktemp("positions_host") / "positions_host")
    native = os.path.join(ROOT, "tests", "native")
    csrc = os.path.join(ROOT, "paper_2603_13358_amd", "csrc")
    subprocess.check_call(["g++", "-std=c++17", "-w", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                           "-fno-omit-frame-pointer", "-I", os.path.join(native, "host_runtime"), os.path.join(native, "positions_host.cpp"),
                           os.path.join(csrc, "ppd_plan.cpp"), "-pthread", "-o", path])
    return path


@pytest.mark.parametrize("what", ["frequencies", "settings", "rope", "append"])
def test_host_side(exe, what):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0")
    env.pop("LD_PRELOAD", None)
    res = subprocess.run([exe, what], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=120)
    assert res.returncode == 0 and "ok" in res.stdout, res.stdout[-3000:]


# The context is NULL, or a handle of none: the library itself refuses it with PPD_ERR_NULL once everything has been passed on.
def handle():
    h = ctypes.c_void_p()
    h.num_q_heads, h.num_kv_heads, h.head_dim = 8, 2, 64
    return h


def rows(n, heads, dim=64, dtype=torch.bfloat16):
    return torch.zeros(n, heads, dim, dtype=dtype)


def rope(h=None, **kw):
    ppd.ppd_rope(h, **dict(dict(x=rows(5, 3), positions=torch.zeros(5, dtype=torch.int64), out=rows(5, 3)), **kw))


def append(h=None, **kw):
    idx = torch.zeros(5, dtype=torch.int64)
    ppd.ppd_kv_append_rotated(h, **dict(dict(q=rows(5, 8), k=rows(5, 2), v=rows(5, 2), positions=idx, kv_pages=torch.zeros(64), slot_mapping=idx, q_out=rows(5, 8)), **kw))


def status(call, *args, **kw):
    with pytest.raises(ppd.PPDError) as e:
        call(*args, **kw)
    return e.value.status


def refused(call, what, *args, **kw):
    with pytest.raises(ppd.PPDError) as e:
        call(*args, **kw)
    return e.value.status == -3 and what in str(e.value)


@pytest.mark.parametrize("h", [None, handle()], ids=["address", "handle"])
def test_good_arguments_are_passed_on(h):
    assert status(rope, h) == -1 and status(append, h) == -1
    assert status(append, h, q=None, q_out=None) == -1
    packed = rows(5, 12)
    assert status(append, h, q=packed[:, :8], k=packed[:, 8:10], v=packed[:, 10:]) == -1
    assert status(rope, h, x=packed[:, 1:4], out=packed[:, 4:7]) == -1
    assert status(rope, h, x=rows(9, 3), out=rows(7, 3)) == -1  # rows behind the positions
    assert status(rope, h, x=1 << 20, heads=3, x_stride=192, out=1 << 21, out_stride=192, positions=1 << 22, T=5) == -1
    assert status(append, h, q=1 << 20, q_stride=512, k=1 << 21, k_stride=128, v=1 << 22, v_stride=128, slot_mapping=1 << 23, T=5, q_out=1 << 24) == -1
    assert status(rope, h, x=rows(5, 3, dtype=torch.int16), out=rows(5, 3, dtype=torch.int16)) == -1  # the bits of bf16 numbers


@pytest.mark.parametrize("h", [None, handle()], ids=["address", "handle"])
def test_tensors_that_are_not_as_the_call_takes_them_are_refused(h):
    for dtype in (torch.float32, torch.float16, torch.int32):
        for name, heads in (("x", 3), ("out", 3)):
            assert refused(rope, name, h, **{name: rows(5, heads, dtype=dtype)})
        for name, heads in (("q", 8), ("k", 2), ("v", 2), ("q_out", 8)):
            assert refused(append, name, h, **{name: rows(5, heads, dtype=dtype)})
    for dtype in (torch.int32, torch.float64):
        assert refused(rope, "positions", h, positions=torch.zeros(5, dtype=dtype))
        assert refused(append, "positions", h, positions=torch.zeros(5, dtype=dtype))
        assert refused(append, "slot_mapping", h, slot_mapping=torch.zeros(5, dtype=dtype))
    every_second = torch.zeros(10, dtype=torch.int64)[::2]
    assert refused(rope, "positions", h, positions=every_second)
    assert refused(append, "positions", h, positions=every_second) and refused(append, "slot_mapping", h, slot_mapping=every_second)
    assert refused(append, "positions", h, positions=torch.zeros(4, dtype=torch.int64))
    for bad in (rows(4, 3), rows(5, 2), rows(5, 3)[0], rows(5, 6)[:, ::2], rows(5, 3, 128)[..., ::2], rows(3, 5).transpose(0, 1)):
        assert refused(rope, "out", h, out=bad)
    assert refused(rope, "x", h, x=rows(4, 3)) and refused(rope, "x", h, heads=4)
    for name, heads in (("q", 8), ("k", 2), ("v", 2), ("q_out", 8)):
        assert refused(append, name, h, **{name: rows(4, heads)})
        assert refused(append, name, h, **{name: rows(5, 2 * heads)[:, ::2]})
    assert refused(append, "v", h, v=rows(5, 3)) and refused(append, "q_out", h, q_out=rows(5, 7))
    assert refused(append, "q_out", h, q_out=rows(5, 10)[:, :8])
    if h is not None:
        assert refused(rope, "x", h, x=rows(5, 3, 128), out=rows(5, 3, 128))
        assert refused(append, "q", h, q=rows(5, 9), q_out=rows(5, 9)) and refused(append, "k", h, k=rows(5, 3), v=rows(5, 3))


def test_addresses_need_what_a_tensor_would_say():
    assert refused(rope, "stride", x=1 << 20, heads=3) and refused(rope, "stride", out=1 << 20)
    assert refused(rope, "T", positions=1 << 20) and refused(append, "T", slot_mapping=1 << 20)
    assert refused(append, "stride", k=1 << 20)
    assert refused(rope, "stride", x_stride=192)  # a tensor's is its own
    assert refused(rope, "heads", heads=1 << 40)


def test_frequencies_and_settings():
    f = ppd.ppd_rope_frequencies(64, 10000.0)
    assert f.dtype == np.float64 and f.shape == (32,) and f[0] == 1.0 and abs(f[16] - 0.01) < 1e-16
    for dim in (0, 3, 130, -2):
        assert status(ppd.ppd_rope_frequencies, dim) == -2
    with pytest.raises(ppd.PPDError) as e:
        ppd.ppd_rope_frequencies(64, -1.0)
    assert e.value.status == -3 and "base" in str(e.value)
    assert status(ppd.ppd_set_rope, None, f) == -1


def test_a_stretched_base_beyond_the_largest_number():
    """base * factor^(d / (d - 2)) is 1e300 * 1e10^(8/6), more than a binary64 holds; the frequencies are not.  Each is a product of two powers:
    some roundings, and exponents' roundings times |ln base| < 700: 1e-12 is far above 700 * 2^-52."""
    f = ppd.ppd_rope_frequencies(8, 1e300, ppd.PPD_ROPE_SCALE_BASE, 1e10)
    want = 10.0 ** np.array([-(300.0 * 2 * i / 8 + 10.0 * 2 * i / 6) for i in range(4)])
    np.testing.assert_allclose(f, want, rtol=1e-12)
