"""The 8-bit cache format on the host: the accuracy that cmc.h states, on the oracle, and the sizes
that its calls take."""

import ctypes

import numpy as np
import pytest
import torch

import paper_2609_25537_gb300 as cmc
from oracle import q8
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


@pytest.mark.parametrize("amax", [224.0 * (1 + 2.0 ** -10), 225.0, 256.0, 300.0, 343.0, 447.0, 448.0])
@pytest.mark.parametrize("exponent", [-118, -20, 0, 100])
def test_accuracy_of_a_value_quantised_once(amax, exponent):
    """e4m3 rounds to 2^-4 of a value down to 2^-6, and to 2^-10 below; a block's amax is at most 448 and above 224 in
    these units: 2^-6 is at most 2^-13 of it, and 2^-10 at most 2^-17."""
    amax = amax * 2.0 ** exponent
    x = amax * np.concatenate([2.0 ** -np.linspace(0.0, 24.0, 20001), [1.0]])
    c = q8.block_byte(amax)
    assert c == 127 + exponent  # amax is above 224 and at most 448 times 2^exponent
    err = np.abs(q8.E4M3[q8.round_e4m3(x / q8.power(c))] * q8.power(c) - x)
    large = x >= 2.0 ** -13 * amax
    assert (err[large] <= 2.0 ** -4 * x[large]).all() and (err[~large] <= 2.0 ** -17 * amax).all()


def test_accuracy_where_the_power_of_two_is_the_smallest():
    x = 448.0 * 2.0 ** -127 * 2.0 ** -np.linspace(0.0, 30.0, 20001)
    err = np.abs(q8.E4M3[q8.round_e4m3(x / q8.power(0))] * q8.power(0) - x)
    assert (err <= np.maximum(2.0 ** -4 * x, 2.0 ** -137)).all()


@pytest.mark.parametrize("seed", range(6))
def test_accuracy_of_values_rounded_again(seed):
    """Tokens that grow by up to 2^3 a step, so that a block's power of two rises again and again.

    A code that falls below 2^-6 is rounded to half of 2^-9 then, at P = 2^(c - 127), and again at every larger P:
    2^-10 (P + P / 2 + P / 4 ...) in all; before, it was off by 2^-4 of the value, at most 2^-10 of the first of
    these P, since the largest code below 2^-6 is 15/16 of it.  Together no more than 2^-9 of the last P.  A
    code that stays above 2^-6 is off by 2^-4 of the value alone."""
    rng = np.random.default_rng(seed)
    W, d = 64, 64
    codes = np.zeros((1, 1, 1, 2, W, d), dtype=np.uint8)
    scales = np.zeros((1, 1, 1, 2, q8.scale_bytes(W)), dtype=np.uint8)
    pos = np.zeros(1, dtype=np.int64)
    x, most = np.zeros((2, W, d)), np.zeros((2, W))  # the tokens; their block's largest power of two since
    size = 1e-3
    for t in range(3 * W):
        slot = t % W
        size = size * 2.0 ** rng.uniform(0.0, 3.0) if t % 32 else 1e-3
        row = size * rng.uniform(-1.0, 1.0, (2, d)) * 2.0 ** rng.uniform(-16.0, 0.0, (2, d))
        q8.append(codes, scales, pos, row[None, None, 0, None], row[None, None, 1, None])
        x[:, slot], most[:, slot] = row, 0.0
        block = slice(slot // 32 * 32, slot // 32 * 32 + 32)
        power = np.array([q8.power(c) for c in scales[0, 0, 0, :, slot // 32]])
        most[:, block] = np.maximum(most[:, block], power[:, None])
        err = np.abs(q8.values(codes, scales)[0, 0, 0] - x)
        assert (err <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -9 * most[..., None])).all(), t
