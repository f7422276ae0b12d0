"""Host side of attention over shared prefixes on the CPU: its code compiled against a stand-in for the HIP runtime (tests/native/host_runtime),
launches recorded, under AddressSanitizer + UndefinedBehaviorSanitizer; and what its Python call refuses."""
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
    path = str(tmp_path_factory.mktemp("prefix_host") / "prefix_host")
    native = os.path.join(ROOT, "tests", "native")
    csrc = os.path.join(ROOT, "paper_2603_13358_amd", "csrc")
    subprocess.check_call(["g++", "-std=c++17", "-w", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                           "-fno-omit-frame-pointer", "-I", os.path.join(native, "host_runtime"), os.path.join(native, "prefix_host.cpp")] +
                          [os.path.join(csrc, f) for f in ("ppd_plan.cpp", "ppd_tree_plan.cpp", "ppd_prefix_plan.cpp")] + ["-pthread", "-o", path])
    return path


@pytest.mark.parametrize("what", ["refusals", "plans", "streams", "staircase"])
def test_host_side(exe, what):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0")
    env.pop("LD_PRELOAD", None)
    res = subprocess.run([exe, what], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=300)
    assert res.returncode == 0 and "ok" in res.stdout, res.stdout[-3000:]


def handle():
    h = ctypes.c_void_p()
    h.num_q_heads, h.num_kv_heads, h.head_dim = 8, 2, 64
    return h


S, L, n = np.array([0, 16], np.int32), np.array([30, 20], np.int32), np.array([2, 3], np.int32)


def rows(count, heads=8, dim=64, dtype=torch.bfloat16):
    return torch.zeros(count, heads, dim, dtype=dtype)


def prefix(h=None, **kw):
    a = dict(q=rows(5), kv_pages=torch.zeros(64), page_tables=torch.zeros(2, 3, dtype=torch.int32), shared=S, L=L, n=n, scale=1.0, out=rows(5))
    ppd.ppd_prefix_attention(h, **dict(a, **kw))


def status(*args, **kw):
    with pytest.raises(ppd.PPDError) as e:
        prefix(*args, **kw)
    return e.value.status


def refused(what, *args, **kw):
    with pytest.raises(ppd.PPDError) as e:
        prefix(*args, **kw)
    return e.value.status == -3 and what in str(e.value)


@pytest.mark.parametrize("h", [None, handle()], ids=["address", "handle"])
def test_python_call(h):
    assert status(h) == -1  # a NULL context: everything was passed on
    for name, good in (("shared", S), ("L", L), ("n", n)):
        for same in (good.astype(np.int64), good.astype(np.float64), list(map(int, good)), torch.from_numpy(good)):
            assert status(h, **{name: same}) == -1
        for far in (np.array([(1 << 32), 5]), np.array([0.5, 5.0])):
            assert refused("32-bit", h, **{name: far})
        assert refused("length", h, **{name: good[:1]}) and refused("length", h, **{name: np.append(good, good)})
    assert status(h, q=rows(7), out=rows(6)) == -1
    assert status(h, q=1 << 20, out=1 << 21, page_tables=1 << 22, max_pages=3) == -1
    for name in ("q", "out"):
        assert refused(name, h, **{name: rows(4)}) and refused(name, h, **{name: rows(5, dtype=torch.float16)})
        assert refused(name, h, **{name: rows(5, 16)[:, :8]}) and refused(name, h, **{name: rows(5)[0]})
        if h is not None:
            assert refused(name, h, **{name: rows(5, 9)}) and refused(name, h, **{name: rows(5, 8, 128)})
    assert refused("page_tables", h, page_tables=torch.zeros(2, 3, dtype=torch.int64)) and refused("page_tables", h, page_tables=torch.zeros(1, 3, dtype=torch.int32))
    assert refused("page_tables", h, page_tables=torch.zeros(2, 5, dtype=torch.int32)[:, :3])
    assert refused("max_pages", h, max_pages=1 << 33)
