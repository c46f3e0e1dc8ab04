"""Sizes at and past the output head's limits, on the host: what the binding hands to the C ABI."""
import os
import subprocess
from types import SimpleNamespace

import pytest
import torch

import paper_2005_04680_amd as pk
from paper_2005_04680_amd import head

FAKE = 1 << 20


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(pk.LIB_PATH):
        import paper_2005_04680_amd.build as b
        b.build()
    head._lib()


class Fake:
    """What the binding looks at of a GPU tensor of contiguous rows."""
    is_cuda, dtype = True, torch.float32

    def __init__(self, *shape):
        self.shape = shape

    def stride(self):
        return (self.shape[1], 1)

    def data_ptr(self):
        return FAKE


def test_no_workspace_for_sizes_past_32_bits():
    for past in (2 ** 32 + 100, 2 ** 31, 2 ** 33 + 64, -2 ** 31 - 1, -2 ** 32 + 100):
        for f in (pk.embbag_mx4_matmul_workspace_bytes, pk.embbag_mx4_matmul_grad_workspace_bytes):
            assert f(past, 70000, 256) == 0 and f(100, 70000, past) == 0
        assert f(100, 70000, 256) > 0
        assert pk.embbag_distill_workspace_bytes(past, 200003, 8) == 0
        assert pk.embbag_distill_workspace_bytes(2, past, 8) == 0
        assert pk.embbag_distill_workspace_bytes(2, 200003, past) == 0
    assert pk.embbag_distill_workspace_bytes(2, 2 ** 31 - 1, 8) > 0


@pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="dummy pointers: run where no GPU is visible")
@pytest.mark.parametrize("m", [2 ** 32 + 3, 2 ** 31, 2 ** 33])
def test_calls_of_more_rows_than_32_bits_are_refused(m):
    t = SimpleNamespace(dim=64, rows=20, codes_ptr=FAKE, scales_ptr=FAKE)
    assert pk.embbag_mx4_matmul(Fake(m, 64), t, Fake(m, 20), None, stream=0) == pk.EMBBAG_ERR_INVALID_ARG
    assert pk.embbag_mx4_matmul_grad(Fake(m, 20), t, Fake(m, 64), None, stream=0) == pk.EMBBAG_ERR_INVALID_ARG


def test_a_table_wider_than_32_bits_is_refused():
    dim = 2 ** 32 + 64
    with pytest.raises(ValueError):
        pk.Mx4Table(Fake(1, pk.mx4_code_bytes(dim)), Fake(1, pk.mx4_scale_bytes(dim)), dim)


def test_every_launch_is_one_that_hip_takes(tmp_path):
    """At the limits of every size, by a driver that counts the library's launches instead of making them."""
    here = os.path.dirname(os.path.abspath(__file__))
    inc = os.path.join(os.path.dirname(here), "include")
    rocm, exe = "/opt/rocm", str(tmp_path / "launches")
    r = subprocess.run(["g++", "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-rdynamic", "-I", inc, "-I",
                        os.path.join(rocm, "include"), os.path.join(here, "launch_driver.cpp"), pk.LIB_PATH,
                        "-L", os.path.join(rocm, "lib"), "-lamdhip64", "-Wl,-rpath," + os.path.dirname(pk.LIB_PATH),
                        "-Wl,-rpath," + os.path.join(rocm, "lib"), "-Wno-unused-result", "-o", exe],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.stdout[-2000:], r.stderr[-4000:])
    assert "all launches fit" in r.stdout
