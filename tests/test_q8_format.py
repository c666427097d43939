"""The 8-bit cache format on the host: the accuracy that cmc.h states, on the oracle, and the sizes
that its calls take."""

import ctypes

import numpy as np
import pytest
import torch

import paper_2609_25537_gb300 as cmc
from paper_2609_25537_gb300.build import build

SHAPE, RANGE = 2, 3
FAKE = 0x10000

host_only = pytest.mark.skipif(torch.cuda.is_available(),
                               reason="fake-pointer argument checks run only without a GPU")


@pytest.fixture(scope="module")
def L():
    build()
    return cmc.lib()


@host_only
def test_no_rows_of_an_empty_cache(L):
    def quantize(N, k, idx=0):
        return L.cmc_quantize_cache(0, 0, idx, 0, ctypes.byref(cmc.CmcDims(2, 1, 2, 2, 64, N, k, 1)), 0, 0, 0, None)

    def dequantize(N, k, idx=0):
        return L.cmc_dequantize_cache(0, 0, idx, ctypes.byref(cmc.CmcDims(2, 1, 2, 2, 64, N, k, 1)), 0, 0, 0, None)
    for f in (quantize, dequantize):
        assert f(0, 0) == f(0, 0, FAKE) == f(5, 0) == 0
        assert f(0, 1) == f(0, 1, FAKE) == f(-1, 0) == f(1 << 25, 0) == SHAPE
        assert f(0, -1) in (SHAPE, RANGE) and f(3, -1) == RANGE
