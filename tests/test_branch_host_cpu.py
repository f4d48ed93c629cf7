"""Host code of generation that branches without a GPU, over the stand-in for the CUDA runtime (tests/host): the kernel
that a call goes to, scratch in captured calls, and calls for which there is no memory."""
import glob
import os
import subprocess

import pytest


@pytest.fixture(scope="module")
def program(repo_root, tmp_path_factory):
    import __graft_entry__ as g
    g.build()
    from paper_2607_17715_gb300 import build as b
    host = os.path.join(repo_root, "tests", "host")
    exe = str(tmp_path_factory.mktemp("host") / "branch_paths")
    cuda = os.path.join(os.path.dirname(os.path.dirname(b._nvcc())), "include")
    cmd = ["g++", "-std=c++17", "-O1", "-I", b.INCLUDE, "-I", host, "-I", cuda, "-o", exe,
           os.path.join(host, "fake_cudart.cpp"), os.path.join(host, "branch_paths.cpp"),
           *sorted(glob.glob(os.path.join(b.BUILD_DIR, "*.o")))]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    return exe


@pytest.mark.parametrize("scenario", ["tree_routes", "tree_capture", "tree_no_memory", "moves"])
def test_scenario(program, scenario):
    res = subprocess.run([program, scenario], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0, res.stdout + res.stderr
