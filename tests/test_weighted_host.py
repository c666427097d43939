"""The cache with weights on the host: pins of its oracle, and the refusals of its entry points."""

import ctypes

import numpy as np
import pytest
import torch

import paper_2609_25537_gb300 as cmc
from oracle import weighted as ow
from paper_2609_25537_gb300.build import build
from paper_2609_25537_gb300._lib import CmcQkPrep

OK, NULL, SHAPE, RANGE, ALIGN, WORKSPACE = 0, 1, 2, 3, 4, 5
FAKE = 0x10000  # 16-byte aligned, never dereferenced: these calls fail before any launch
BIG = 1 << 40

host_only = pytest.mark.skipif(torch.cuda.is_available(),
                               reason="fake-pointer argument checks run only without a GPU")


@pytest.fixture(scope="module")
def L():
    build()
    return cmc.lib()


# ---- pins of the oracle ----

def test_bf16_rounding_is_torchs():
    rng = np.random.default_rng(0)
    x = (rng.standard_normal(4000) * 2.0 ** rng.integers(-140, 60, 4000)).astype(np.float32)
    x = np.concatenate([x, np.float32([0.0, 1.00390625, 1.01171875, 2.0 ** -133, 1.5 * 2.0 ** -133])])
    want = torch.from_numpy(x).to(torch.bfloat16).to(torch.float64).numpy()
    np.testing.assert_array_equal(ow.to_bf16(x), want)


def test_norm_closed_forms():
    x = np.array([[3.0, 4.0, 0.0, 0.0]])
    np.testing.assert_allclose(ow.heads(x, np.ones(4), eps=0.0), x / 2.5)
    np.testing.assert_allclose(ow.heads(x, np.array([1.0, 2.0, 3.0, 4.0]), eps=0.0), [[1.2, 3.2, 0.0, 0.0]])
    np.testing.assert_allclose(ow.heads(np.zeros((1, 4)), np.ones(4)), 0.0)
    x = np.random.default_rng(0).standard_normal((5, 3, 64))
    want = torch.nn.functional.rms_norm(torch.from_numpy(x), (64,), eps=1e-6).numpy()
    np.testing.assert_allclose(ow.heads(x, np.ones((5, 64))), want, rtol=1e-12)


def test_rotation_is_a_complex_product():
    rng = np.random.default_rng(1)
    x, p = rng.standard_normal((6, 2, 64)), np.array([0, 1, -5, 1000, 123456, 2 ** 31])
    got = ow.heads(x, theta=1e4, p=p)
    for n, at in enumerate(p):
        for i in range(32):
            z = (x[n, :, i] + 1j * x[n, :, i + 32]) * np.exp(1j * (float(at) * 1e4 ** (-i / 32)))
            # the angle itself is rounded in this form: at * 2^-52
            tol = 1e-12 + abs(float(at)) * 2.0 ** -50
            np.testing.assert_allclose(got[n, :, i], z.real, atol=tol * 4)
            np.testing.assert_allclose(got[n, :, i + 32], z.imag, atol=tol * 4)
    np.testing.assert_allclose(got[0], x[0])


def test_prefill_is_a_run_of_appends():
    k = np.arange(6.0).reshape(1, 1, 6, 1, 1)
    ring, ringv, w, pos = np.zeros((1, 1, 1, 4, 1)), np.zeros((1, 1, 1, 4, 1)), np.ones((1, 1, 1, 4)), np.array([3])
    ow.prefill(k, -k, ring, ringv, w, pos, np.array([6]))
    assert pos[0] == 9 and not w.any()  # tokens 2 .. 5 are numbers 5 .. 8
    np.testing.assert_array_equal(ring.ravel(), [5, 2, 3, 4])
    np.testing.assert_array_equal(ringv.ravel(), [-5, -2, -3, -4])
    w[:] = 1
    ow.prefill(k, k, ring, ringv, w, pos, np.array([2]))
    np.testing.assert_array_equal(ring.ravel(), [5, 0, 1, 4])
    np.testing.assert_array_equal(w.ravel(), [1, 0, 0, 1])


def test_weights_grow_by_one_per_query():
    rng = np.random.default_rng(2)
    q = rng.standard_normal((2, 1, 4, 8))
    t1 = [rng.standard_normal((2, 1, 2, 3, 8)) for _ in range(2)] + [np.zeros((2, 1, 2, 3))]
    ring = [rng.standard_normal((2, 1, 2, 5, 8)) for _ in range(2)] + [np.zeros((2, 1, 2, 5))]
    out, _, _, _ = ow.attend(q, t1, ring, np.array([2, 9]), 0.3)
    np.testing.assert_allclose(t1[2].sum(-1) + ring[2].sum(-1), 2.0)
    assert not ring[2][0, ..., 2:].any()
    k = torch.from_numpy(np.concatenate([t1[0], ring[0]], axis=3))[1, 0].repeat_interleave(2, 0)
    v = torch.from_numpy(np.concatenate([t1[1], ring[1]], axis=3))[1, 0].repeat_interleave(2, 0)
    want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q[1, 0])[:, None], k, v, scale=0.3)
    np.testing.assert_allclose(out[1, 0], want[:, 0].numpy(), rtol=1e-12)


def test_eviction_by_hand():
    w = np.float32([[[[5, 1, 4, 1, 3]]]])
    idx, held = ow.evict(w, 3)
    assert idx.ravel().tolist() == [0, 2, 4] and held.tolist() == [3]
    assert ow.evict(w, 4)[0].ravel().tolist() == [0, 1, 2, 4]  # equal weights: the older
    assert ow.evict(w, 3, recent=2)[0].ravel().tolist() == [0, 3, 4]
    assert ow.evict(w, 3, recent=2, pos=np.array([4]))[0].ravel().tolist() == [0, 2, 3]
    assert ow.evict(w, 3, pos=np.array([2]))[0].ravel().tolist() == [0, 1, -1]
    # wrapped: tokens 2 .. 6 in rows 2, 3, 4, 0, 1
    assert ow.evict(w, 3, recent=1, pos=np.array([7]))[0].ravel().tolist() == [2, 0, 1]
    assert ow.evict(w, 2, pos=np.array([7]))[0].ravel().tolist() == [2, 0]
    assert ow.evict(np.float32([[[[np.nan, -np.inf, -0.0, 0.0]]]]), 2)[0].ravel().tolist() == [2, 3]
    assert ow.evict(np.float32([[[[np.nan, -np.inf, -0.0, 0.0]]]]), 3)[0].ravel().tolist() == [1, 2, 3]


# ---- refusals ----

def _dims(**kw):
    base = dict(B=2, L=3, Hq=8, Hkv=2, d=128, N=100, k=10, W=16)
    base.update(kw)
    return ctypes.byref(cmc.CmcDims(*(base[f] for f, _ in cmc.CmcDims._fields_)))


def test_workspace_sizes(L):
    # a 256-byte status header, 8 bytes per sequence padded to 256
    assert L.cmc_cache_workspace_size(2) == 512 and L.cmc_cache_workspace_size(40) == 768
    assert L.cmc_cache_workspace_size(0) == L.cmc_cache_workspace_size(65536) == 0

    def f(**kw):
        return L.cmc_decode_attn_weighted_workspace_size(_dims(**kw))
    assert f() == f(L=65, k=100, W=5000, d=64) == 512
    assert f(d=96) == 0 and f(Hq=6) == 0 and f(k=101) == 0
    # G = 4: 18,432 keys fit a cluster's shared memory; beyond, 4 (G + 1) bytes a key, rounded up to 128 keys a CTA
    assert f(k=0, W=18432) == f(N=16000, k=8192, W=10240) == 512
    assert f(k=0, W=18433) == 512 + 2 * 3 * 2 * 8 * 19 * 128 * 20
    assert f(k=0, W=9216, Hq=16) == 512
    assert f(k=0, W=9217, Hq=16) == 512 + 2 * 3 * 2 * 8 * 10 * 128 * 36
    assert f(k=0, W=30720, Hq=4) == f(k=0, W=46080, Hq=2) == 512
    assert f(k=0, W=30721, Hq=4) > 512 and f(k=0, W=46081, Hq=2) > 512


def _prep(**kw):
    base = dict(q_weight=0, k_weight=0, evicted=0, rope_theta=1e4, rope_offset=0, eps=1e-6)
    base.update(kw)
    return ctypes.byref(CmcQkPrep(**base))


def _norm(L, q=BIG, qs=1024, k=2 * BIG, ks=256, T=4, pos=FAKE, dims=None, prep=None, oq=3 * BIG, ok=4 * BIG):
    return L.cmc_qk_norm_rope(q, qs, k, ks, T, pos, dims or _dims(), prep, oq, ok, None)


@host_only
def test_norm_argument_checks(L):
    assert _norm(L, T=0) == OK  # nothing to do
    assert _norm(L, T=-1) == SHAPE
    assert _norm(L, T=(1 << 24) + 1) == SHAPE
    assert _norm(L, T=1 << 24, dims=_dims(L=8)) == SHAPE
    for name in ("q", "k", "pos", "oq", "ok"):
        assert _norm(L, **{name: 0}) == NULL
        assert _norm(L, **{name: FAKE + 4}) == ALIGN
    assert _norm(L, dims=_dims(d=96)) == SHAPE
    assert _norm(L, dims=_dims(Hq=6)) == SHAPE
    assert _norm(L, qs=1016) == SHAPE and _norm(L, ks=248) == SHAPE and _norm(L, qs=-1024) == SHAPE
    assert _norm(L, qs=1028) == ALIGN and _norm(L, ks=260) == ALIGN
    for theta in (-1.0, float("inf"), float("nan")):
        assert _norm(L, prep=_prep(rope_theta=theta)) == RANGE
    for offset in (-1, (1 << 32) + 1):
        assert _norm(L, prep=_prep(rope_offset=offset)) == RANGE
    for eps in (-1.0, float("inf"), float("nan")):
        assert _norm(L, prep=_prep(q_weight=FAKE, eps=eps)) == RANGE
        assert _norm(L, prep=_prep(k_weight=FAKE, eps=eps)) == RANGE
    assert _norm(L, prep=_prep(q_weight=FAKE + 4)) == ALIGN
    assert _norm(L, prep=_prep(k_weight=FAKE + 4)) == ALIGN
    assert _norm(L, prep=_prep(evicted=FAKE + 4)) == ALIGN
    assert L.cmc_qk_norm_rope(FAKE, 1024, FAKE, 256, 4, FAKE, None, None, FAKE, FAKE, None) == NULL
    # outputs that meet inputs (24 tokens of 2,048 and 512 bytes), but for heads prepared where they are
    bad = _prep(rope_theta=-1.0)
    evil = _prep(q_weight=FAKE + 4)  # refused after these
    for change in (dict(oq=BIG + 2048), dict(oq=BIG - 16), dict(oq=BIG, qs=1536), dict(oq=2 * BIG), dict(ok=BIG + 24 * 2048 - 16),
                   dict(ok=2 * BIG, ks=264), dict(ok=3 * BIG), dict(oq=4 * BIG - 24 * 2048 + 16)):
        assert _norm(L, prep=evil, **change) == RANGE
    for change in (dict(oq=BIG, ok=2 * BIG), dict(oq=BIG + 24 * 2048), dict(ok=BIG + 24 * 2048), dict(oq=4 * BIG - 24 * 2048),
                   dict(q=BIG, k=BIG + 2048, qs=1536, ks=1536), dict(k=BIG)):
        assert _norm(L, prep=evil, **change) == ALIGN
        assert _norm(L, prep=bad, **change) == RANGE


def _prefill(L, q=BIG, qs=1024, k=2 * BIG, ks=256, v=3 * BIG, vs=256, T=4, rk=4 * BIG, rv=5 * BIG, rw=FAKE, pos=FAKE,
             count=FAKE, dims=None, prep=None, oq=6 * BIG, ws=FAKE, wsb=512):
    return L.cmc_window_prefill(q, qs, k, ks, v, vs, T, rk, rv, rw, pos, count, dims or _dims(), prep, oq, ws,
                                wsb, None)


@host_only
def test_prefill_argument_checks(L):
    assert _prefill(L, T=0) == OK
    assert _prefill(L, T=0, q=0, oq=0, rw=0, count=0) == OK
    for name in ("k", "v", "rk", "rv", "pos", "oq"):
        assert _prefill(L, **{name: 0}) == NULL
    for name in ("q", "k", "v", "rk", "rv", "pos", "oq", "count", "ws"):
        assert _prefill(L, **{name: FAKE + 4}) == ALIGN
    assert _prefill(L, rw=FAKE + 2) == ALIGN
    assert _prefill(L, dims=_dims(W=0)) == SHAPE
    assert _prefill(L, vs=248) == SHAPE and _prefill(L, vs=260) == ALIGN
    assert _prefill(L, ws=0) == WORKSPACE and _prefill(L, wsb=511) == WORKSPACE
    assert _prefill(L, prep=_prep(rope_theta=-1.0)) == RANGE
    evil = _prep(q_weight=FAKE + 4)
    for change in (dict(rk=2 * BIG), dict(rv=3 * BIG + 512), dict(rk=5 * BIG), dict(oq=5 * BIG + 16), dict(rv=BIG), dict(oq=3 * BIG),
                   dict(oq=BIG, qs=1536)):
        assert _prefill(L, prep=evil, **change) == RANGE
    for change in (dict(oq=BIG), dict(v=2 * BIG), dict(q=0, oq=0), dict(rv=4 * BIG + 2 * 3 * 2 * 16 * 256)):
        assert _prefill(L, prep=evil, **change) == ALIGN


@host_only
def test_prefill_refuses_a_ring_in_the_values(L):
    """Prepared keys over values that other warps have not read yet: dense, as many slots as tokens."""
    evil = _prep(q_weight=FAKE + 4)  # refused after these
    for change in (dict(rk=3 * BIG), dict(rv=3 * BIG), dict(rk=2 * BIG), dict(rv=2 * BIG), dict(rk=3 * BIG + 512)):
        assert _prefill(L, T=16, prep=evil, **change) == RANGE
    assert _prefill(L, T=16, prep=evil) == ALIGN and _prefill(L, T=16, prep=evil, oq=BIG) == ALIGN


@host_only
def test_prefill_and_norm_overlaps(L):
    """Weights, positions, counts, gains and the workspace: 24 tokens, rings of 16 slots, 49,152 bytes each, weights 768."""
    CUDA = 6  # all checks passed: no device
    a = dict(rw=7 * BIG, pos=8 * BIG, count=8 * BIG + 64, ws=9 * BIG)
    prep = dict(q_weight=10 * BIG, k_weight=10 * BIG + 1536, evicted=8 * BIG + 16, rope_theta=1e4)
    assert _prefill(L, prep=_prep(**prep), **a) == CUDA
    assert _prefill(L, **{**a, "count": 0, "rw": 0}) == CUDA
    for change in (dict(count=8 * BIG), dict(count=8 * BIG + 8), dict(rw=4 * BIG), dict(rw=5 * BIG + 49148), dict(rw=6 * BIG),
                   dict(rw=BIG), dict(rw=3 * BIG + 8), dict(rw=8 * BIG - 764), dict(rw=9 * BIG + 508), dict(pos=4 * BIG),
                   dict(pos=9 * BIG + 504), dict(pos=2 * BIG), dict(pos=6 * BIG + 8), dict(ws=5 * BIG), dict(ws=BIG), dict(count=4 * BIG),
                   dict(count=7 * BIG + 760), dict(ws=8 * BIG + 64)):
        assert _prefill(L, prep=_prep(**prep), **{**a, **change}) == RANGE, change
    for change in (dict(evicted=8 * BIG), dict(evicted=7 * BIG), dict(evicted=9 * BIG), dict(q_weight=4 * BIG), dict(k_weight=7 * BIG - 1520),
                   dict(q_weight=6 * BIG), dict(k_weight=9 * BIG + 16)):
        assert _prefill(L, prep=_prep(**{**prep, **change}), **a) == RANGE, change
    assert _prefill(L, prep=_prep(**{**prep, "k_weight": 10 * BIG, "evicted": 8 * BIG + 64}), **a) == CUDA  # what is read may meet
    assert _norm(L) == CUDA and _norm(L, pos=BIG) == CUDA
    for change in (dict(pos=3 * BIG), dict(pos=4 * BIG + 24 * 512 - 8)):
        assert _norm(L, **change) == RANGE
    for change in (dict(q_weight=3 * BIG), dict(k_weight=4 * BIG + 16), dict(evicted=3 * BIG + 8)):
        assert _norm(L, prep=_prep(**change)) == RANGE


def _attend(L, q=FAKE, tk=FAKE, tv=FAKE, tw=FAKE, rk=FAKE, rv=FAKE, rw=FAKE, pos=FAKE, dims=None, out=FAKE,
            ws=FAKE, wsb=512):
    return L.cmc_two_tier_decode_attn_weighted(q, tk, tv, tw, rk, rv, rw, pos, dims or _dims(), 0.0, out, ws,
                                               wsb, None)


def _step(L, q=FAKE, tk=FAKE, tv=FAKE, tw=FAKE, rk=FAKE, rv=FAKE, rw=FAKE, pos=FAKE, kn=FAKE, vn=FAKE, dims=None,
          prep=None, out=FAKE, ws=FAKE, wsb=512):
    return L.cmc_decode_step_weighted(q, tk, tv, tw, rk, rv, rw, pos, kn, vn, dims or _dims(), 0.0, prep, out, ws,
                                      wsb, None)


@host_only
@pytest.mark.parametrize("call", [_attend, _step])
def test_weighted_attention_argument_checks(L, call):
    names = ["q", "tk", "tv", "tw", "rk", "rv", "rw", "pos", "out"] + (["kn", "vn"] if call is _step else [])
    for name in names:
        assert call(L, **{name: 0}) == NULL
        assert call(L, **{name: FAKE + 2}) == ALIGN
    assert call(L, dims=_dims(k=0), tk=0, tv=0, tw=0, ws=0) == WORKSPACE  # none of Tier-1 is looked at
    assert call(L, ws=0) == WORKSPACE and call(L, wsb=511) == WORKSPACE and call(L, ws=FAKE + 8) == ALIGN
    assert call(L, dims=_dims(k=101)) == RANGE
    for bad in (dict(B=0), dict(d=32), dict(Hq=6), dict(Hq=32), dict(W=0), dict(N=0, k=0)):
        assert call(L, dims=_dims(**bad)) == SHAPE
    assert call(L, dims=_dims(W=40000), wsb=512) == WORKSPACE


@host_only
@pytest.mark.parametrize("call", [_attend, _step])
def test_weighted_attention_overlaps(L, call):
    """48 query heads' rows, 12,288 bytes; Tier-1 of 12 x 100 rows, 307,200 and 4,800; rings of 12 x 16, 49,152 and 768; new rows
    a quarter of the queries'."""
    CUDA = 6  # all checks passed: no device
    a = dict(q=BIG, tk=2 * BIG, tv=3 * BIG, tw=4 * BIG, rk=5 * BIG, rv=6 * BIG, rw=7 * BIG, pos=8 * BIG, out=9 * BIG, ws=10 * BIG)
    step = call is _step
    if step:
        a.update(kn=11 * BIG, vn=12 * BIG)
    assert call(L, **a) == CUDA
    bad = [dict(out=BIG + 16), dict(out=BIG - 16), dict(out=2 * BIG), dict(out=3 * BIG + 307184), dict(out=4 * BIG), dict(out=5 * BIG),
           dict(out=6 * BIG + 49136), dict(out=7 * BIG), dict(out=10 * BIG + 496), dict(out=8 * BIG), dict(rw=4 * BIG), dict(rw=4 * BIG + 4796),
           dict(tw=2 * BIG), dict(tw=6 * BIG), dict(rw=BIG), dict(rw=8 * BIG - 764), dict(rw=3 * BIG), dict(tw=10 * BIG), dict(ws=5 * BIG),
           dict(ws=8 * BIG), dict(ws=2 * BIG + 307184)]
    ring_reads = [dict(rk=6 * BIG), dict(rk=2 * BIG), dict(rv=3 * BIG + 307184), dict(rk=BIG), dict(pos=BIG), dict(pos=2 * BIG)]
    good = [dict(out=BIG), dict(out=BIG + 12288), dict(rw=4 * BIG + 4800), dict(rw=8 * BIG - 768), dict(tk=3 * BIG),
            dict(dims=_dims(k=0), tk=9 * BIG, tv=9 * BIG, tw=9 * BIG), dict(out=10 * BIG + 512)]
    if step:
        bad += ring_reads + [dict(kn=5 * BIG), dict(vn=6 * BIG + 49136), dict(kn=9 * BIG), dict(vn=7 * BIG), dict(kn=10 * BIG),
                             dict(prep=_prep(evicted=8 * BIG)), dict(prep=_prep(q_weight=9 * BIG)), dict(prep=_prep(k_weight=7 * BIG)),
                             dict(prep=_prep(evicted=4 * BIG))]
        good += [dict(kn=12 * BIG), dict(vn=BIG), dict(prep=_prep(q_weight=BIG, evicted=8 * BIG + 16))]
    else:
        good += ring_reads
    for change in bad:
        assert call(L, **{**a, **change}) == RANGE, change
    for change in good:
        assert call(L, **{**a, **change}) == CUDA, change


@host_only
def test_step_prep_checks(L):
    assert _step(L, prep=_prep(rope_theta=float("nan"))) == RANGE
    assert _step(L, prep=_prep(rope_offset=-1)) == RANGE
    assert _step(L, prep=_prep(q_weight=FAKE, eps=-1.0)) == RANGE
    assert _step(L, prep=_prep(evicted=FAKE + 2)) == ALIGN


def _evict(L, k=BIG, v=2 * BIG, w=3 * BIG, pos=0, dims=None, recent=0, ok=4 * BIG, ov=5 * BIG, ow=6 * BIG, idx=7 * BIG,
           op=0, ev=0, ws=FAKE, wsb=512):
    return L.cmc_evict_cache(k, v, w, pos, dims or _dims(), recent, ok, ov, ow, idx, op, ev, ws, wsb, None)


@host_only
def test_evict_argument_checks(L):
    for name in ("k", "v", "w", "ok", "ov", "ow", "idx"):
        assert _evict(L, **{name: 0}) == NULL
    for name in ("k", "v", "ok", "ov", "ws"):
        assert _evict(L, **{name: FAKE + 8}) == ALIGN
    for name in ("w", "ow", "idx"):
        assert _evict(L, **{name: FAKE + 2}) == ALIGN
    for name in ("pos", "op", "ev"):
        assert _evict(L, **{name: FAKE + 4}) == ALIGN
    for bad in (dict(k=0), dict(k=101), dict(W=9), dict(k=-1)):
        assert _evict(L, dims=_dims(**bad)) == RANGE
    assert _evict(L, recent=-1) == RANGE and _evict(L, recent=11) == RANGE
    assert _evict(L, dims=_dims(d=96)) == SHAPE and _evict(L, dims=_dims(N=0, k=0)) == SHAPE
    assert _evict(L, ws=0) == WORKSPACE and _evict(L, wsb=511) == WORKSPACE
    # in place: all three or none, and as many rows
    assert _evict(L, ok=BIG) == RANGE and _evict(L, ov=2 * BIG) == RANGE and _evict(L, ow=3 * BIG) == RANGE
    assert _evict(L, ok=BIG, ov=2 * BIG, ow=3 * BIG) == RANGE  # W != N
    # part of the input
    assert _evict(L, ok=BIG + 256) == RANGE and _evict(L, ow=3 * BIG + 4) == RANGE and _evict(L, ov=BIG + 512) == RANGE


@host_only
def test_evict_overlaps(L):
    """What is written meets nothing else; idx, which is read back as the rows to copy, above all.  units = 12: k and v 307,200
    bytes, weight 4,800; outputs of 16 rows 49,152 and 768, idx 480."""
    CUDA = 6  # all checks passed: no device
    assert _evict(L) == CUDA
    rows, ws = 12 * 16 * 256, dict(ws=8 * BIG)
    for at in (BIG, 2 * BIG + 307200 - 4, 3 * BIG + 4796, 4 * BIG, 5 * BIG + rows - 4, 6 * BIG + 764, 4 * BIG - 476):
        assert _evict(L, idx=at) == RANGE
    assert _evict(L, ok=4 * BIG, ov=4 * BIG) == RANGE and _evict(L, ov=4 * BIG + rows - 16) == RANGE
    for at in (BIG, 2 * BIG + 16, 4 * BIG + rows - 4, 5 * BIG - 764):
        assert _evict(L, ow=at) == RANGE
    assert _evict(L, ok=3 * BIG) == RANGE and _evict(L, ov=3 * BIG + 4784) == RANGE
    for name in ("op", "ev"):
        for at in (BIG, 2 * BIG, 3 * BIG + 8, 4 * BIG, 5 * BIG, 6 * BIG + 760, 7 * BIG + 472):
            assert _evict(L, pos=9 * BIG, **{name: at}) == RANGE
    assert _evict(L, pos=9 * BIG, ev=9 * BIG) == RANGE and _evict(L, pos=9 * BIG, op=9 * BIG + 8) == RANGE
    assert _evict(L, op=9 * BIG, ev=9 * BIG + 8) == RANGE and _evict(L, op=9 * BIG, ev=9 * BIG) == RANGE
    assert _evict(L, pos=9 * BIG, idx=9 * BIG + 12) == RANGE and _evict(L, pos=9 * BIG, ok=9 * BIG) == RANGE
    for change in (dict(pos=8 * BIG + 504), dict(op=8 * BIG), dict(idx=8 * BIG - 476), dict(k=8 * BIG), dict(ow=8 * BIG + 508)):
        assert _evict(L, **{**ws, **change}) == RANGE
    # side by side, in place, pos in place, inputs that are one another
    for change in (dict(idx=4 * BIG + rows), dict(idx=4 * BIG - 480), dict(ov=4 * BIG + rows), dict(ow=5 * BIG - 768),
                   dict(pos=9 * BIG, op=9 * BIG), dict(pos=9 * BIG, op=9 * BIG, ev=9 * BIG + 16), dict(k=2 * BIG),
                   dict(v=BIG + 256), dict(dims=_dims(W=100), ok=BIG, ov=2 * BIG, ow=3 * BIG),
                   dict(dims=_dims(W=100), k=2 * BIG, ok=2 * BIG, ov=2 * BIG, ow=3 * BIG)):
        assert _evict(L, **change) == CUDA
    place = dict(dims=_dims(W=100), ok=BIG, ov=2 * BIG, ow=3 * BIG)
    for change in (dict(idx=BIG + 307200 - 4), dict(idx=3 * BIG), dict(v=BIG + 256, ov=BIG + 256), dict(w=BIG + 512, ow=BIG + 512),
                   dict(op=2 * BIG), dict(ev=3 * BIG)):
        assert _evict(L, **{**place, **change}) == RANGE


@host_only
def test_plan_argument_checks(L):
    assert L.cmc_decode_attn_weighted_plan(None, 1, ctypes.byref(ctypes.c_int())) == NULL
    assert L.cmc_decode_attn_weighted_plan(_dims(), 1, None) == NULL
    assert L.cmc_decode_attn_weighted_plan(_dims(d=32), 0, ctypes.byref(ctypes.c_int())) == SHAPE


def test_tensors_on_the_host_are_refused(L):
    x = torch.zeros(1, 1, 2, 4, 64, dtype=torch.bfloat16)
    w, pos = torch.zeros(1, 1, 2, 4), torch.zeros(1, dtype=torch.int64)
    q = torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16)
    row = q[:, :, :2].contiguous()
    for call in (lambda: cmc.qk_norm_rope(q, row, pos), lambda: cmc.window_prefill(q, row, row, x, x, pos),
                 lambda: cmc.two_tier_decode_attn_weighted(q, None, None, None, x, x, w, pos),
                 lambda: cmc.decode_step_weighted(q, x, x, w, x, x, w, pos, row, row),
                 lambda: cmc.evict_cache(x, x, w, 2)):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()
    for call in (lambda: cmc.qk_norm_rope(None, row, pos), lambda: cmc.qk_norm_rope(q, "k", pos),
                 lambda: cmc.window_prefill(q, None, row, x, x, pos),
                 lambda: cmc.window_prefill(q, row, 3, x, x, pos),
                 lambda: cmc.two_tier_decode_attn_weighted(None, None, None, None, x, x, w, pos),
                 lambda: cmc.evict_cache([1], x, w, 2)):
        with pytest.raises(TypeError):
            call()
