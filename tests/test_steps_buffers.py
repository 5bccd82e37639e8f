"""The library's own workspace of the tree attention is freed only after both launches
that use it (steps_buffers.cpp, which stands in for the HIP runtime; no GPU)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2506_03296_amd", "libapex_steps.so")


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    if not os.path.exists(LIB):
        from paper_2506_03296_amd import build
        build.build(quiet=True)
    exe = str(tmp_path_factory.mktemp("buffers") / "steps_buffers")
    subprocess.run(["g++", "-std=c++17", "-O1", "-rdynamic", "-pthread", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "steps_buffers.cpp"), "-o", exe, "-ldl"],
                   check=True, capture_output=True)
    return exe


@pytest.mark.parametrize("launch", ["1", "2"])
@pytest.mark.parametrize("other", ["grow", "release"])
def test_freed_after_both_launches(program, launch, other):
    r = subprocess.run([program, LIB, launch, other], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
