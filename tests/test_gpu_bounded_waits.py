"""Waits inside kernels that run out: they end, tell, and ask for nothing more.  The probes wait for barriers that nothing completes, with
limits of a millisecond and no copy under way."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2306_06098_b200 import binding, build

pytestmark = pytest.mark.gpu

SOURCE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "csrc", "bounded_waits.cu")


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("probes") / "libprobes.so")
    subprocess.run([os.environ.get("NVCC", "nvcc"), "-std=c++17", "-O2", "-gencode", "arch=compute_100a,code=sm_100a", "-shared",
                    "-Xcompiler", "-fPIC", "-I", build.INCLUDE, "-I", build.CSRC, "-o", lib, SOURCE], check=True)
    call = ctypes.CDLL(lib).probe
    call.argtypes = [ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]

    def run(which):
        x, out = torch.zeros(4, 256, device="cuda"), torch.full((4,), -1, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        assert call(which, x.data_ptr(), out.data_ptr()) == 0
        return out.tolist()
    return run


def test_a_wait_ends(probe):
    assert probe(0) == [1, 0, 1, 0]


def test_a_ring_asks_for_nothing_when_a_wait_has_run_out(probe):
    """The place's copies may still be under way, and its barrier takes one arrival for each phase."""
    assert probe(2) == [0, 1, 0, 1]


def test_a_wait_that_runs_out_late_is_told(probe):
    assert probe(1)[:2] == [binding.ETIMEOUT, 0]


def test_the_status_raises(monkeypatch):
    class Library:
        code = binding.OK

        def __getattr__(self, name):
            return (lambda: self.code) if name == "efcp_operators_status" else getattr(library, name)

    library, fake = binding._lib, Library()
    monkeypatch.setattr(binding, "_lib", fake)
    binding.operators_status()
    fake.code = binding.ETIMEOUT
    with pytest.raises(binding.EfcpError) as raised:
        binding.operators_status()
    assert raised.value.code == binding.ETIMEOUT
