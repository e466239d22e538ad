"""The planner of linear_chunk_attn (paper_2608_11152_amd/csrc/plan.cpp) built with g++ under the address and
undefined-behaviour sanitizers and driven by randomized calls (tests/host_linear_plan_check.cpp): coverage, states before
each item, the workspace that linear_chunk_workspace_size promises.  CPU only; no HIP code is built here."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


@pytest.fixture(scope="module")
def checker(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("g++ is not available")
    exe = str(tmp_path_factory.mktemp("sanitized") / "host_linear_plan_check")
    cmd = [cxx, "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", f"-I{os.path.join(ROOT, 'include')}",
           os.path.join(HERE, "host_linear_plan_check.cpp"),
           os.path.join(ROOT, "paper_2608_11152_amd", "csrc", "plan.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return exe


@pytest.mark.parametrize("seed", ["1", "2", "3"])
def test_randomized_plans_under_sanitizers(checker, seed):
    r = subprocess.run([checker, "2000", seed], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "ok:" in r.stdout and "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr


def test_checker_rejects_planted_mistakes(checker):
    r = subprocess.run([checker, "self-test"], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "planted mistakes rejected" in r.stdout
