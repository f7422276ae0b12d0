"""Partials of the attention calls in the workspace on the CPU: where the plans put them and how much they take, under AddressSanitizer +
UndefinedBehaviorSanitizer (the calls' host code compiled against a stand-in for the HIP runtime, tests/native/host_runtime)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def build(tmp_path_factory, name):
    path = str(tmp_path_factory.mktemp(name) / name)
    native = os.path.join(ROOT, "tests", "native")
    csrc = os.path.join(ROOT, "paper_2603_13358_amd", "csrc")
    subprocess.check_call(["g++", "-std=c++17", "-w", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer",
                           "-I", os.path.join(native, "host_runtime"), os.path.join(native, name + ".cpp")] +
                          [os.path.join(csrc, f) for f in ("ppd_plan.cpp", "ppd_tree_plan.cpp", "ppd_prefix_plan.cpp")] + ["-pthread", "-o", path])
    return path


def run(exe, what):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0")
    env.pop("LD_PRELOAD", None)
    res = subprocess.run([exe, what], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=300)
    assert res.returncode == 0 and "ok" in res.stdout, res.stdout[-3000:]


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    return build(tmp_path_factory, "partials_host")


@pytest.fixture(scope="module")
def parts(tmp_path_factory):
    return build(tmp_path_factory, "prefix_parts_host")


@pytest.mark.parametrize("what", ["alignment"])
def test_plans(plans, what):
    run(plans, what)


@pytest.mark.parametrize("what", ["bound", "memory"])
def test_prefix_batches_whose_partials_do_not_fit(parts, what):
    run(parts, what)
