"""The 8-bit cache on the host: pins of its oracle, and the refusals of its entry points."""

import ctypes

import numpy as np
import pytest
import torch

import paper_2609_25537_gb300 as cmc
from oracle import q8
from paper_2609_25537_gb300.build import build

NULL, SHAPE, RANGE, ALIGN, WORKSPACE = 1, 2, 3, 4, 5
FAKE = 0x10000

host_only = pytest.mark.skipif(torch.cuda.is_available(),
                               reason="fake-pointer argument checks run only without a GPU")


@pytest.fixture(scope="module")
def L():
    build()
    return cmc.lib()


# ---- pins of the oracle ----

def test_e4m3_table_is_torchs():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).to(torch.float64).numpy()
    np.testing.assert_array_equal(q8.E4M3, want)


def test_rounding_is_torchs():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(4000) * 2.0 ** rng.integers(-12, 8, 4000),
                        q8.E4M3[:127], (q8.E4M3[:126] + q8.E4M3[1:127]) / 2,  # values and midpoints
                        [0.0, -0.0, 2.0 ** -10, -2.0 ** -10, 448.0, -448.0]])
    x = x[np.abs(x) <= 448.0].astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(q8.round_e4m3(x), want)
    assert q8.round_e4m3(np.array([np.inf, -np.inf, np.nan])).tolist() == [127, 127, 127]


@pytest.mark.parametrize("amax", [0.0, 1e-39, 2.0 ** -119, 1.0, 1.75, 1.7500001, 448.0, 449.0, 3e38])
def test_block_byte_is_the_smallest_that_holds(amax):
    c = q8.block_byte(amax)
    assert amax <= 448.0 * q8.power(c)
    assert c == 0 or amax > 448.0 * q8.power(c - 1)


def _relative(codes, scales, x):
    v = q8.values(codes, scales)
    return np.abs(v - x) / np.abs(x)


def test_quantisation_error_is_half_a_step():
    rng = np.random.default_rng(1)
    x = rng.uniform(1.0, 2.0, (2, 2, 1, 2, 100, 16)) * 2.0 ** rng.integers(-6, 8, (2, 2, 1, 2, 100, 16))
    codes, scales = q8.quantize(x[:, :, :, 0], x[:, :, :, 1], np.ones((2, 100), dtype=bool))
    assert _relative(codes, scales, x).max() <= 2.0 ** -4  # e4m3: half of 2^-3


def test_append_in_order_equals_quantising_the_block_when_the_largest_comes_first():
    """The block's power of two is set by its first token here, so nothing is rounded twice."""
    rng = np.random.default_rng(2)
    x = rng.uniform(0.1, 1.0, (1, 1, 1, 2, 32, 8))
    x[0, 0, 0, :, 0] *= 50.0
    codes = np.full((1, 1, 1, 2, 32, 8), 0x7F, dtype=np.uint8)
    scales = np.full((1, 1, 1, 2, 4), 0xFF, dtype=np.uint8)
    pos = np.zeros(1, dtype=np.int64)
    for t in range(32):
        q8.append(codes, scales, pos, x[:, :, :, 0, t], x[:, :, :, 1, t])
    want, wscales = q8.quantize(x[:, :, :, 0], x[:, :, :, 1], np.ones((1, 32), dtype=bool))
    np.testing.assert_array_equal(codes, want)
    np.testing.assert_array_equal(scales[..., :1], wscales[..., :1])
    assert pos[0] == 32


def test_append_sets_a_block_anew_at_its_first_slot():
    codes = np.zeros((1, 1, 1, 2, 40, 4), dtype=np.uint8)
    scales = np.zeros((1, 1, 1, 2, 4), dtype=np.uint8)
    pos = np.zeros(1, dtype=np.int64)
    for t in range(41):
        big = 1000.0 if t == 0 else 1.0
        q8.append(codes, scales, pos, np.full((1, 1, 1, 4), big), np.full((1, 1, 1, 4), big))
    # the 41st token took the place of the large one: the block needs no more than 1.0 does
    assert scales[0, 0, 0, 0, 0] == q8.block_byte(1.0)
    np.testing.assert_array_equal(q8.values(codes, scales)[0, 0, 0, 0, :32], 1.0)


def test_attention_of_equal_keys_is_the_mean_value():
    v = np.arange(12.0).reshape(1, 1, 1, 3, 4)
    tier = np.concatenate([np.zeros((1, 1, 1, 3, 4))[:, :, :, None], v[:, :, :, None]], axis=3)
    ring = np.zeros((1, 1, 1, 2, 2, 4))
    out, mag = q8.attention(np.ones((1, 1, 2, 4)), tier, ring, np.array([0]), 1.0)
    np.testing.assert_allclose(out[0, 0, 0], v[0, 0, 0].mean(axis=0))
    np.testing.assert_allclose(mag, out)


# ---- refusals ----

def _dims(**kw):
    base = dict(B=2, L=3, Hq=8, Hkv=2, d=128, N=100, k=10, W=16)
    base.update(kw)
    return cmc.CmcDims(*(base[f] for f, _ in cmc.CmcDims._fields_))


def test_scale_bytes(L):
    for rows in (0, 1, 31, 32, 128, 129, 4096):
        assert L.cmc_q8_scale_bytes(rows) == cmc.q8_scale_bytes(rows) == q8.scale_bytes(rows)
    assert L.cmc_q8_scale_bytes(-1) == 0


def test_attention_workspace_size(L):
    # a 256-byte status header, 8 bytes per sequence padded to 256
    def f(**kw):
        return L.cmc_decode_attn_q8_workspace_size(ctypes.byref(_dims(**kw)))
    assert f() == f(L=65, k=100, W=5000, d=64) == 256 + 256
    assert f(B=40) == 256 + 512
    assert f(d=96) == 0


@host_only
def test_quantize_cache_argument_checks(L):
    def f(k=FAKE, idx=0, count=0, kv=FAKE, scales=FAKE, status=0, **kw):
        return L.cmc_quantize_cache(k, FAKE, idx, count, ctypes.byref(_dims(**kw)), kv, scales, status,
                                    None)
    assert f(k=0) == f(kv=0) == f(scales=0) == NULL
    assert f(k=FAKE + 8) == f(kv=FAKE + 8) == f(idx=FAKE + 2) == f(count=FAKE + 4) == ALIGN
    assert f(status=FAKE + 2) == f(scales=FAKE + 4) == ALIGN
    assert f(k=FAKE, N=5) == RANGE
    assert f(d=96) == f(B=0) == f(N=0) == SHAPE
    assert f(k=0, kv=0, scales=0, **{"Hq": 3}) == NULL  # query heads are ignored
    assert L.cmc_quantize_cache(0, 0, 0, 0, ctypes.byref(_dims(k=0)), 0, 0, 0, None) == 0
    assert L.cmc_quantize_cache(FAKE, FAKE, 0, 0, None, FAKE, FAKE, 0, None) == NULL


@host_only
def test_dequantize_cache_argument_checks(L):
    def f(kv=FAKE, scales=FAKE, idx=0, out=FAKE, status=0, **kw):
        return L.cmc_dequantize_cache(kv, scales, idx, ctypes.byref(_dims(**kw)), out, FAKE, status, None)
    assert f(kv=0) == f(scales=0) == f(out=0) == NULL
    assert f(kv=FAKE + 8) == f(scales=FAKE + 8) == f(out=FAKE + 8) == f(idx=FAKE + 1) == ALIGN
    assert f(k=101) == RANGE
    assert f(d=32) == SHAPE
    assert L.cmc_dequantize_cache(0, 0, 0, ctypes.byref(_dims(k=0)), 0, 0, 0, None) == 0


@host_only
def test_window_append_q8_argument_checks(L):
    def f(ring=FAKE, scales=FAKE, pos=FAKE, k_new=FAKE, **kw):
        return L.cmc_window_append_q8(ring, scales, pos, k_new, FAKE, ctypes.byref(_dims(**kw)), None)
    assert f(ring=0) == f(scales=0) == f(pos=0) == f(k_new=0) == NULL
    assert f(ring=FAKE + 8) == f(scales=FAKE + 8) == f(pos=FAKE + 4) == f(k_new=FAKE + 8) == ALIGN
    assert f(d=32) == f(W=0) == f(B=0) == SHAPE


@host_only
def test_attention_q8_argument_checks(L):
    def f(q=FAKE, t1=FAKE, t1s=FAKE, ring=FAKE, rs=FAKE, pos=FAKE, out=FAKE, ws=FAKE, wsb=1 << 30, **kw):
        return L.cmc_two_tier_decode_attn_q8(q, t1, t1s, ring, rs, pos, ctypes.byref(_dims(**kw)), 0.0,
                                             out, ws, wsb, None)
    assert f(q=0) == f(ring=0) == f(rs=0) == f(pos=0) == f(out=0) == NULL
    assert f(t1=0) == f(t1s=0) == NULL
    assert f(t1=0, t1s=0, k=0) not in (NULL, SHAPE, RANGE, ALIGN, WORKSPACE)
    assert f(q=FAKE + 8) == f(t1=FAKE + 8) == f(t1s=FAKE + 4) == f(ring=FAKE + 8) == ALIGN
    assert f(rs=FAKE + 4) == f(pos=FAKE + 4) == f(out=FAKE + 8) == f(ws=FAKE + 8) == ALIGN
    assert f(d=96) == f(Hq=6) == f(Hq=32) == f(W=0) == SHAPE
    assert f(k=101) == RANGE
    assert f(ws=0) == f(wsb=16) == WORKSPACE


@host_only
def test_decode_step_q8_argument_checks(L):
    def f(theta=0.0, off=0, k_new=FAKE, ring=FAKE, wsb=1 << 30, **kw):
        return L.cmc_decode_step_q8(FAKE, FAKE, FAKE, ring, FAKE, FAKE, k_new, FAKE,
                                    ctypes.byref(_dims(**kw)), 0.0, theta, off, FAKE, FAKE, wsb, None)
    assert f(k_new=0) == f(ring=0) == NULL
    assert f(k_new=FAKE + 8) == ALIGN
    assert f(d=96) == f(Hq=32) == SHAPE
    assert f(k=101) == f(theta=-1.0) == f(theta=float("inf")) == f(theta=float("nan")) == RANGE
    assert f(theta=1e4, off=-1) == f(theta=1e4, off=2 ** 32 + 1) == RANGE
    assert f(wsb=16) == WORKSPACE


def test_decode_attn_q8_plan_argument_checks(L):
    ctas = ctypes.c_int(0)
    def f(dims, a=ctypes.byref(ctas)):
        return L.cmc_decode_attn_q8_plan(dims, 1, a)
    assert f(None) == f(ctypes.byref(_dims()), None) == NULL
    assert f(ctypes.byref(_dims(d=96))) == SHAPE
    assert f(ctypes.byref(_dims(k=101))) == RANGE


def test_binding_refuses_cpu_tensors():
    kv = torch.zeros(1, 1, 1, 2, 32, 64).to(torch.float8_e4m3fn)
    scales = torch.zeros(1, 1, 1, 2, 4, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    bank = torch.zeros(1, 1, 1, 32, 64, dtype=torch.bfloat16)
    pos = torch.zeros(1, dtype=torch.int64)
    row = torch.zeros(1, 1, 1, 64, dtype=torch.bfloat16)
    for call in (lambda: cmc.quantize_cache(bank, bank), lambda: cmc.dequantize_cache(kv, scales),
                 lambda: cmc.window_append_q8(kv, scales, pos, row, row),
                 lambda: cmc.two_tier_decode_attn_q8(row, kv, scales, kv, scales, pos),
                 lambda: cmc.decode_step_q8(row, kv, scales, kv, scales, pos, row, row)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
