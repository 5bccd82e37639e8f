"""The libraries' own workspaces are freed only after the launches that use them
(library_buffers.cpp, which stands in for the HIP runtime; no GPU)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PACKAGE = os.path.join(ROOT, "paper_2506_03296_amd")


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    for lib in ("libapex_kv4.so", "libapex_decode.so"):
        if not os.path.exists(os.path.join(PACKAGE, lib)):
            from paper_2506_03296_amd import build
            build.build(quiet=True)
    exe = str(tmp_path_factory.mktemp("buffers") / "library_buffers")
    subprocess.run(["g++", "-std=c++17", "-O1", "-rdynamic", "-pthread", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "library_buffers.cpp"), "-o", exe, "-ldl"],
                   check=True, capture_output=True)
    return exe


@pytest.mark.parametrize("other", ["grow", "release"])
@pytest.mark.parametrize("lib,call", [("libapex_kv4.so", "attention"), ("libapex_kv4.so", "evict"),
                                      ("libapex_decode.so", "decode")])
def test_freed_after_the_launch(program, lib, call, other):
    r = subprocess.run([program, os.path.join(PACKAGE, lib), call, other], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
