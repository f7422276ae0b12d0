"""Partials of the attention calls in the workspace on the CPU: where the plans put them, under AddressSanitizer + UndefinedBehaviorSanitizer."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    path = str(tmp_path_factory.mktemp("partials_host") / "partials_host")
    csrc = os.path.join(ROOT, "paper_2603_13358_amd", "csrc")
    subprocess.check_call(["g++", "-std=c++17", "-w", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer",
                           os.path.join(ROOT, "tests", "native", "partials_host.cpp")] +
                          [os.path.join(csrc, f) for f in ("ppd_plan.cpp", "ppd_tree_plan.cpp", "ppd_prefix_plan.cpp")] + ["-o", path])
    return path


@pytest.mark.parametrize("what", ["alignment"])
def test_plans(exe, what):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0")
    env.pop("LD_PRELOAD", None)
    res = subprocess.run([exe, what], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=300)
    assert res.returncode == 0 and "ok" in res.stdout, res.stdout[-3000:]
