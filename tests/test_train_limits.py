"""Sizes at the limits of the norm, of 8-bit rows and of the cross entropy, on the host."""
import os
import subprocess

import paper_2005_04680_amd as pk


def test_every_launch_is_one_that_hip_takes(tmp_path):
    """By a driver that checks the library's launches instead of making them."""
    if not os.path.exists(pk.LIB_PATH):
        import paper_2005_04680_amd.build as b
        b.build()
    here = os.path.dirname(os.path.abspath(__file__))
    inc = os.path.join(os.path.dirname(here), "include")
    rocm, exe = "/opt/rocm", str(tmp_path / "launches")
    r = subprocess.run(["g++", "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-rdynamic", "-I", inc, "-I",
                        os.path.join(rocm, "include"), os.path.join(here, "train_launch_driver.cpp"), pk.LIB_PATH,
                        "-L", os.path.join(rocm, "lib"), "-lamdhip64", "-Wl,-rpath," + os.path.dirname(pk.LIB_PATH),
                        "-Wl,-rpath," + os.path.join(rocm, "lib"), "-Wno-unused-result", "-o", exe],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.stdout[-2000:], r.stderr[-4000:])
    assert "all launches fit" in r.stdout


def test_workspaces_grow_with_a_piece_not_with_the_scores():
    f = pk.embbag_xent_workspace_bytes
    small, large = (f(4096, v, 1024, pk.EMBBAG_BF16, True) for v in (1 << 18, 1 << 24))
    assert large < small + (1 << 30) and large < 1 << 31
