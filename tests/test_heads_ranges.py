"""Which temperatures distillation and which eps the norm take: those whose scales and largest r are numbers in fp32 (no device is touched)."""
import ctypes

import numpy as np
import pytest

from paper_2312_08656_amd import binding, build

INVALID = -1
p = ctypes.c_void_p(0x1000)  # never dereferenced: calls have no rows, and refuse all the same


@pytest.fixture(scope="module")
def lib():
    if not binding.lib_path().exists():
        build.build()
    return binding.load_library()


def distill(lib, temperature):
    need = lib.maxk_classes_workspace(1, 100000, 0)
    calls = (lib.maxk_distill(p, 0, 0, 100000, p, 0, p, 4, 5, temperature, p, p, need, None),
             lib.maxk_distill_grad(p, 0, 0, 100000, p, 0, p, 4, 5, temperature, p, p, p, p, need, None))
    assert calls[0] == calls[1]
    return calls[0]


def test_temperatures(lib):
    top = float(np.finfo(np.float32).max)
    # log2(e) / temperature is what logits are taken times: past fp32's range from a temperature of log2(e) / 2^128 = 4.2398e-39 down, where 1 / temperature is not yet
    for temperature in (4.239e-39, 4e-39, 3.5e-39, 2.9388e-39, 2.9e-39, 1e-45, 5e-324, 3.5e38, 1e40, 1e44, 1e300):
        assert distill(lib, temperature) == INVALID, temperature
    for temperature in (4.241e-39, 1e-38, 1e-6, 1.0, 1e6, 1e38, top):
        assert distill(lib, temperature) == 0, temperature


def norm(lib, eps):
    return lib.maxk_rms_norm(p, None, 0, 0, 8, p, eps, None, p, 0, None, None, None, None)


def test_eps(lib):
    # of a row of zeros r = 1 / sqrt(eps): past fp32's range from eps = 2^-256 = 8.636e-78 down, and 0 r is not 0 there
    for eps in (8.6e-78, 1e-80, 1e-100, 1e-300, 5e-324):
        assert norm(lib, eps) == INVALID, eps
    for eps in (8.7e-78, 1e-76, 1e-38, 1e-6, 1.0, 1e300):
        assert norm(lib, eps) == 0, eps
