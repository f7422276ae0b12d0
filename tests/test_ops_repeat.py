"""What a call of tree or weighted attention or of kv_select leaves behind for the calls and captured graphs after it: their host code
against the stand-in HIP runtime, under AddressSanitizer + UndefinedBehaviorSanitizer."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    path = str(tmp_path_factory.mktemp("ops_repeat") / "ops_repeat_host")
    native = os.path.join(ROOT, "tests", "native")
    csrc = os.path.join(ROOT, "paper_2603_13358_amd", "csrc")
    subprocess.check_call(["g++", "-std=c++17", "-w", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                           "-fno-omit-frame-pointer", "-I", os.path.join(native, "host_runtime"), os.path.join(native, "ops_repeat_host.cpp"),
                           os.path.join(csrc, "ppd_plan.cpp"), os.path.join(csrc, "ppd_tree_plan.cpp"), "-pthread", "-o", path])
    return path


@pytest.mark.parametrize("what", ["first_call_under_capture", "kinds", "longest", "split_blocks"])
def test_host_side(exe, what):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0")
    env.pop("LD_PRELOAD", None)
    res = subprocess.run([exe, what], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=120)
    assert res.returncode == 0 and "ok" in res.stdout, res.stdout[-3000:]
