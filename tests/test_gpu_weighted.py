"""The cache with weights on the GPU against its fp64 oracle: norm and rotation, prefill of the ring, attention that
accumulates what each key receives, eviction by weight, and all of them in a run.

Tolerances.  u = 2^-24 is half a step of fp32, 2^-8 of bf16, relative to the value.
  norm, rotation  a sum of d <= 128 squares in 16 fused steps and 3 additions, a square root, a division, two
                  products: below 2^-19 of the value; sines and cosines off by 1e-7 < 2^-23, a product and a fused
                  step: all in all 2^-18 (|y_i| + |y_(i+h)|) with room, then the rounding to bf16
  probabilities   a product q . k in fp32 is off by at most d u sum |q||k| (that of a prepared q, held as two bf16
                  of 2^-8 each, by 2^-16 of it more), and so is the maximum; 2^x is off by 2^-22 of
                  itself, the sum of n of them by the additions on its way, at most 2 per block of a warp and 20 to
                  merge: 2^-17 for all of that up to 50 blocks
  weights         what p is off by, and one rounding of the sum of the heads and one of the weight: 2^-22
  outputs         p, rounded to bf16 for the product (2^-8), times |v|, and the output's rounding
"""

import math

import numpy as np
import pytest
import torch

import paper_2609_25537_gb300 as cmc
from oracle import weighted as ow
from _gpu_helpers import to_f64

pytestmark = pytest.mark.gpu

THETA = 5e5


def gen(dev, seed):
    return torch.Generator(device=dev).manual_seed(seed)


def randn(g, *shape, scale=1.0):
    return (torch.randn(shape, generator=g, device=g.device) * scale).to(torch.bfloat16)


def f64(t):
    return None if t is None else (to_f64(t) if t.is_floating_point() else t.cpu().numpy())


def check_heads(got, x, weight, p, what, theta=THETA, eps=1e-6):
    """got [B, L, T, H, d] against the norm and rotation of x."""
    w = None if weight is None else f64(weight)[None, :, None]
    y = ow.heads(x, w, eps)
    want = y if p is None else ow.heads(y, None, 0.0, theta, np.broadcast_to(p[:, None], x.shape[:3]))
    mag = np.abs(y)
    h = y.shape[-1] // 2
    if p is not None:
        mag = np.concatenate([mag[..., :h] + mag[..., h:]] * 2, axis=-1)
    tol = 2.0 ** -8 * np.abs(want) + (1 + 2.0 ** -8) * 2.0 ** -18 * mag + 2.0 ** -133
    err = np.abs(f64(got) - want)
    assert (err <= tol).all(), f"{what}: {np.max(err - tol)} over"
    return want


# ----------------------------------------------------------------------------
# Norm and rotation
# ----------------------------------------------------------------------------

HEADS = [  # B, L, T, Hkv, G, d
    (1, 1, 1, 2, 4, 64), (1, 1, 1, 1, 1, 128), (2, 3, 5, 1, 8, 128), (1, 2, 17, 3, 2, 64), (3, 1, 130, 8, 4, 128),
    (2, 1, 33, 5, 1, 64), (1, 32, 1, 8, 4, 128), (1, 1, 700, 7, 8, 64),
]


@pytest.mark.parametrize("form", ["both", "norm", "rope", "neither", "q norm only"])
@pytest.mark.parametrize("case", HEADS)
def test_norm_and_rotation(cuda_device, case, form):
    B, L, T, H, G, d = case
    g = gen(cuda_device, 1)
    packed = randn(g, B, L, T, H * (G + 2), d, scale=2.0)
    q, k = packed[..., :H * G, :], packed[..., H * G:H * (G + 1), :]
    pos = torch.randint(-5, 10 ** 9, (B,), generator=g, device=cuda_device)
    evicted = torch.randint(0, 10 ** 6, (B,), generator=g, device=cuda_device)
    qw = 1 + torch.randn(L, d, generator=g, device=cuda_device) if form in ("both", "norm", "q norm only") else None
    kw = 1 + torch.randn(L, d, generator=g, device=cuda_device) if form in ("both", "norm") else None
    rope = {"rope_theta": THETA, "rope_offset": 37, "evicted": evicted} if form in ("both", "rope") else {}
    before = packed.clone()
    oq, ok = cmc.qk_norm_rope(q, k, pos, q_weight=qw, k_weight=kw, **rope)
    torch.cuda.synchronize()
    assert torch.equal(packed, before) and oq.is_contiguous() and ok.is_contiguous()
    p = ow.positions(f64(pos), f64(evicted), 37, T) if rope else None
    check_heads(oq, f64(q), qw, p, f"q {form}")
    check_heads(ok, f64(k), kw, p, f"k {form}")
    if form == "neither":
        assert torch.equal(oq, q) and torch.equal(ok, k)
    # dense, in place
    q2, k2 = q.clone(memory_format=torch.contiguous_format), k.clone(memory_format=torch.contiguous_format)
    r = cmc.qk_norm_rope(q2, k2, pos, q_weight=qw, k_weight=kw, out_q=q2, out_k=k2, **rope)
    assert r[0] is q2 and torch.equal(q2, oq) and torch.equal(k2, ok)
    if T == 1:  # one token's form
        a, b = cmc.qk_norm_rope(q[:, :, 0], k[:, :, 0], pos, q_weight=qw, k_weight=kw, **rope)
        assert a.shape == (B, L, H * G, d) and torch.equal(a, oq[:, :, 0]) and torch.equal(b, ok[:, :, 0])


def test_norm_of_extreme_rows(cuda_device):
    """Zeros, one element, values near bf16's ends, NaN and infinity stay within their rows."""
    x = torch.zeros(1, 1, 6, 2, 64, dtype=torch.bfloat16, device=cuda_device)
    x[0, 0, 1, 0, 5] = 3.0
    x[0, 0, 2] = 1e-20
    x[0, 0, 3] = 1e15
    x[0, 0, 4, 0] = float("nan")
    x[0, 0, 5, 1, 3] = float("inf")
    w = torch.ones(1, 64, device=cuda_device)
    pos = torch.zeros(1, dtype=torch.int64, device=cuda_device)
    got, _ = cmc.qk_norm_rope(x, x, pos, q_weight=w, k_weight=w)
    got = got.float().cpu()
    assert not got[0, 0, 0].any()
    assert got[0, 0, 1, 0, 5] == 8.0 and got[0, 0, 1].abs().sum() == 8.0
    check_heads(got[:, :, 2:4], f64(x)[:, :, 2:4], w, None, "small and large")
    assert got[0, 0, 4, 0].isnan().all() and not got[0, 0, 4, 1].isnan().any()
    assert not got[0, 0, 5, 0].any()


def test_layouts_of_tokens_that_are_refused(cuda_device):
    q = torch.zeros(2, 3, 4, 8, 64, dtype=torch.bfloat16, device=cuda_device)
    k = q[:, :, :, :2].contiguous()
    pos = torch.zeros(2, dtype=torch.int64, device=cuda_device)
    w = torch.zeros(3, 64, device=cuda_device)
    for bad in (q.transpose(0, 1), q.transpose(2, 3), q[..., ::2, :], q[:, :, ::2], q[:, :2], q[..., :32],
                q[:1].expand(2, 3, 4, 8, 64), q[:, :, :, None]):
        with pytest.raises((ValueError, TypeError)):
            cmc.qk_norm_rope(bad, k, pos)
    for kw in (dict(q_weight=w[:2]), dict(k_weight=w.double()), dict(q_weight=w.cpu()), dict(rope_theta=0.0),
               dict(rope_theta=-1.0), dict(rope_theta=float("nan")), dict(rope_theta=1e4, evicted=pos[:1]),
               dict(rope_theta=1e4, evicted=pos.int()), dict(out_q=q[:, :, :, :4]), dict(out_k=q)):
        with pytest.raises((ValueError, TypeError)):
            cmc.qk_norm_rope(q, k, pos, **kw)
    for kw in (dict(rope_theta=float("inf")), dict(rope_theta=1e4, rope_offset=-1), dict(q_weight=w, eps=-1.0),
               dict(rope_theta=1e4, rope_offset=2 ** 64 + 5)):
        with pytest.raises(cmc.CmcError, match="RANGE"):
            cmc.qk_norm_rope(q, k, pos, **kw)
    with pytest.raises(ValueError):
        cmc.qk_norm_rope(q, k, pos[:1])
    with pytest.raises(cmc.CmcError, match="ALIGN"):  # tokens 12 elements apart, and a row that starts off 16 bytes
        x = torch.zeros(2 * 3 * 4 * 520 + 8, dtype=torch.bfloat16, device=cuda_device)
        cmc.qk_norm_rope(x[4:4 + 2 * 3 * 4 * 512].view(2, 3, 4, 8, 64), k, pos)
    empty = q[:, :, :0]
    a, b = cmc.qk_norm_rope(empty, k[:, :, :0], pos, rope_theta=1e4)
    assert a.shape == (2, 3, 0, 8, 64) and b.shape == (2, 3, 0, 2, 64)


# ----------------------------------------------------------------------------
# Prefill
# ----------------------------------------------------------------------------

PREFILL = [  # B, L, T, Hkv, G, d, W, counts (None: all)
    (1, 1, 1, 2, 4, 64, 5, None), (2, 2, 7, 2, 2, 128, 5, None), (3, 1, 40, 1, 8, 64, 33, [0, 17, 40]),
    (4, 3, 130, 2, 1, 128, 130, [130, -3, 500, 1]), (2, 1, 300, 8, 4, 128, 64, [65, 300]),
    (5, 1, 9, 3, 4, 64, 1, [0, 1, 2, 9, 8]), (1, 2, 33, 2, 4, 128, 100, [20]),
]


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("case", PREFILL)
def test_prefill(cuda_device, case, packed):
    B, L, T, H, G, d, W, counts = case
    g = gen(cuda_device, 2)
    x = randn(g, B, L, T, H * (G + 2), d)
    q, k, v = x.split([H * G, H, H], dim=3)
    if not packed:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    ring_k, ring_v = randn(g, B, L, H, W, d), randn(g, B, L, H, W, d)
    ring_w = torch.rand(B, L, H, W, generator=g, device=cuda_device) + 1
    pos = torch.randint(0, 3 * W + 2, (B,), generator=g, device=cuda_device)
    evicted = torch.randint(0, 99, (B,), generator=g, device=cuda_device)
    kw = 1 + torch.randn(L, d, generator=g, device=cuda_device)
    count = None if counts is None else torch.tensor(counts, device=cuda_device)
    o = [f64(t).copy() for t in (ring_k, ring_v, ring_w)] + [f64(pos).copy()]
    pos0 = o[3].copy()
    out = torch.full((B, L, T, H * G, d), 7.0, dtype=torch.bfloat16, device=cuda_device)
    r = cmc.window_prefill(q, k, v, ring_k, ring_v, pos, ring_weight=ring_w, count=count, k_weight=kw,
                           rope_theta=THETA, rope_offset=3, evicted=evicted, out_q=out)
    torch.cuda.synchronize()
    assert r is out
    p = ow.positions(pos0, f64(evicted), 3, T)
    n = np.full(B, T) if counts is None else np.clip(counts, 0, T)
    for b in range(B):
        check_heads(out[b:b + 1, :, :n[b]], f64(q)[b:b + 1, :, :n[b]], None, p[b:b + 1, :n[b]], f"q {b}")
        assert (out[b, :, n[b]:] == 7.0).all()
    # the ring's keys: the bf16 of the library where it wrote one (checked as heads), the old ones elsewhere
    _, ok = cmc.qk_norm_rope(q, k, torch.from_numpy(pos0).to(cuda_device), k_weight=kw, rope_theta=THETA, rope_offset=3,
                             evicted=evicted)
    check_heads(ok, f64(k), kw, p, "k")
    ow.prefill(f64(ok), f64(v), *o[:3], o[3], n)
    for got, want in zip((ring_k, ring_v, ring_w, pos), o):
        np.testing.assert_array_equal(f64(got), want)


def test_prefill_is_a_run_of_appends(cuda_device):
    """Without norm and rotation: the ring that as many calls of window_append leave."""
    g = gen(cuda_device, 3)
    B, L, T, H, d, W = 3, 2, 21, 2, 64, 8
    k, v = randn(g, B, L, T, H, d), randn(g, B, L, T, H, d)
    rings = [[randn(g, B, L, H, W, d) for _ in range(2)] + [torch.tensor([0, 5, 100], device=cuda_device)]]
    rings.append([x.clone() for x in rings[0]])
    assert cmc.window_prefill(None, k, v, *rings[0]) is None
    for t in range(T):
        cmc.window_append(*rings[1], k[:, :, t].contiguous(), v[:, :, t].contiguous())
    for a, b in zip(*rings):
        assert torch.equal(a, b)


def test_prefill_of_a_sequence_without_a_position(cuda_device):
    g = gen(cuda_device, 4)
    B, L, T, H, d, W = 3, 1, 6, 2, 128, 4
    q, k, v = randn(g, B, L, T, 4, d), randn(g, B, L, T, H, d), randn(g, B, L, T, H, d)
    ring_k, ring_v = randn(g, B, L, H, W, d), randn(g, B, L, H, W, d)
    w = torch.ones(B, L, H, W, device=cuda_device)
    pos = torch.tensor([2, -1, 0], device=cuda_device)
    before = [x.clone() for x in (ring_k, ring_v, w)]
    out = torch.zeros_like(q)
    dims = cmc.CmcDims(B, L, 4, H, d, 1, 0, W)
    for ws in (None, cmc.DecodeWorkspace(dims, cuda_device, weighted=True), cmc.DecodeWorkspace(dims, cuda_device)):
        pos.copy_(torch.tensor([2, -1, 0]))
        cmc.weighted_cache_status()
        cmc.window_prefill(q, k, v, ring_k, ring_v, pos, ring_weight=w, out_q=out, workspace=ws)
        assert pos.tolist() == [8, -1, 6]
        status = cmc.weighted_cache_status() if ws is None else ws.status()
        assert status == cmc.DEVFLAG_BAD_POS
        if ws is not None:
            assert not ws.buf[256:256 + 8 * B].any()
        for x, y in zip((ring_k, ring_v, w), before):
            assert torch.equal(x[1], y[1])
        assert not w[0].any() and torch.equal(out[0], q[0]) and not out[1].any()


def test_prefill_refusals(cuda_device):
    B, L, T, H, d, W = 2, 1, 3, 2, 64, 4
    q = torch.zeros(B, L, T, 4, d, dtype=torch.bfloat16, device=cuda_device)
    k = torch.zeros(B, L, T, H, d, dtype=torch.bfloat16, device=cuda_device)
    ring = torch.zeros(B, L, H, W, d, dtype=torch.bfloat16, device=cuda_device)
    pos = torch.zeros(B, dtype=torch.int64, device=cuda_device)
    w = torch.zeros(B, L, H, W, device=cuda_device)
    args = dict(q=q, k=k, v=k.clone(), ring_k=ring, ring_v=ring.clone(), pos=pos)
    for change in (dict(v=k[:, :, :2]), dict(v=q), dict(ring_v=ring[..., :3, :]), dict(ring_k=ring[:, :, :1]),
                   dict(pos=pos.int()), dict(pos=pos[:1]), dict(ring_weight=w[..., :3]), dict(ring_weight=w.half()),
                   dict(count=pos[:1]), dict(count=pos.int()), dict(q=None, out_q=q), dict(q=q[:, :, :2]),
                   dict(q=q.float()), dict(out_q=k), dict(rope_theta=0.0)):
        a = {**args, **change}
        with pytest.raises((ValueError, TypeError)):
            cmc.window_prefill(a.pop("q"), a.pop("k"), a.pop("v"), a.pop("ring_k"), a.pop("ring_v"), a.pop("pos"), **a)
    with pytest.raises(cmc.CmcError, match="SHAPE"):  # three query heads to a KV head
        cmc.window_prefill(torch.cat([q, k], dim=3), k, k.clone(), ring, ring.clone(), pos)
    assert not pos.any()


# ----------------------------------------------------------------------------
# Attention
# ----------------------------------------------------------------------------

ATTEND = [  # B, L, Hkv, G, d, k, W, positions (cycled)
    (1, 1, 2, 4, 64, 32, 128, [500]), (2, 1, 1, 1, 128, 1, 1, [0, 3]), (1, 1, 1, 8, 64, 0, 1, [1]),
    (3, 2, 2, 2, 128, 15, 17, [0, 16, 17]), (4, 1, 8, 4, 128, 16, 33, [1, 15, 16, 32]), (2, 3, 1, 8, 128, 17, 130, [129, 131]),
    (5, 1, 2, 1, 64, 0, 300, [0, -1, 299, 2 ** 33 + 5, 7]), (1, 1, 3, 4, 128, 700, 900, [900]),
    (1, 1, 1, 4, 64, 2048, 2000, [1999]), (40, 2, 8, 4, 64, 30, 40, [3, 39, 40, 100]), (2, 1, 1, 8, 128, 3000, 1, [0, 1]),
    (1, 1, 1, 2, 128, 100, 20000, [19983]),
    # many short units: a warp each
    (60, 1, 8, 8, 128, 40, 70, [0, 1, 69, 70, 2 ** 35, -7]), (20, 3, 8, 1, 128, 0, 33, [32, 31, 64]),
    (58, 1, 8, 2, 64, 250, 220, [219, 5, 64]),
    # two warps each
    (60, 1, 8, 4, 128, 40, 70, [0, 1, 69, 70, 2 ** 35, -7]), (31, 3, 8, 8, 64, 100, 200, [199, 31, 200, 3, -1]),
    (465, 1, 1, 1, 128, 3, 500, [0, 499, 5000, 80]), (250, 1, 2, 2, 128, 0, 20, [5, 19, 20]),
    # several waves, which start with the longest sequences: up to 128 sequences, a CTA a unit and a cluster
    (61, 1, 8, 1, 64, 200, 400, [3, 399, -5, 400, 77, 0, 2 ** 40, 210]), (128, 1, 4, 2, 64, 40, 520, [100, 519, 7, 520, -1, 33]),
    (129, 2, 2, 1, 64, 30, 540, [100, 539, 7, 540, -1]), (120, 1, 1, 8, 64, 100, 4400, [17, 4399, 0, 9999, 300, -2, 2222]),
]


def attention_problem(dev, case, seed, poison=True):
    B, L, H, G, d, k, W, positions = case
    g = gen(dev, seed)
    pos = torch.tensor([positions[b % len(positions)] for b in range(B)], device=dev)
    ring = [randn(g, B, L, H, W, d, scale=0.7), randn(g, B, L, H, W, d)]
    w = torch.rand(B, L, H, W, generator=g, device=dev) * 8
    if poison:  # slots that hold no token may hold anything
        dead = (torch.arange(W, device=dev) >= pos.clamp(min=0)[:, None])[:, None, None].expand(w.shape)
        for x, bad in zip(ring, (float("nan"), float("inf"))):
            x.masked_fill_(dead[..., None], bad)
        w.masked_fill_(dead, float("nan"))
    t1 = [None] * 3
    if k:
        t1 = [randn(g, B, L, H, k, d, scale=0.7), randn(g, B, L, H, k, d), torch.rand(B, L, H, k, generator=g, device=dev)]
    return randn(g, B, L, H * G, d, scale=1.5), t1, ring + [w], pos, g


def check_attention(out, t1_w, ring_w, q, t1, ring, pos, scale, prepared=False, new=None):
    """Against the oracle on q, t1, ring as the call found them (K, V, weights in float64; the new slots' weights 0)."""
    d = q.shape[-1]
    dead = np.arange(ring[0].shape[3]) >= np.clip(pos, 0, None)[:, None]
    stale = np.broadcast_to(dead[:, None, None], ring[2].shape)
    ring = [np.where(stale[..., None], 0.0, ring[0]), np.where(stale[..., None], 0.0, ring[1]),
            np.where(stale, 0.0, ring[2])]
    want, mag, grew, size = ow.attend(q, None if t1[0] is None else t1, ring, pos, scale)
    rel = 2 * size * (d * 2.0 ** -24 + (2.0 ** -16 if prepared else 0.0)) + 2.0 ** -17
    rel_q = np.repeat(rel, q.shape[2] // ring[0].shape[2], axis=2)[..., None]
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2 * rel_q) * mag + 2.0 ** -130
    err = np.abs(f64(out) - want)
    assert (err <= tol).all(), f"output: {np.max(err - tol)} over"
    for got, w, gr, skip in ((t1_w, None if t1[0] is None else t1[2], grew[0], None), (ring_w, ring[2], grew[1], stale)):
        if w is None:
            continue
        got = f64(got)
        if skip is not None:
            got = np.where(skip, 0.0, got)
        tol = 2 * rel[..., None] * gr + 2.0 ** -22 * np.abs(w) + 1e-37
        err = np.abs(got - w)
        assert (err <= tol).all(), f"weights: {np.max(err - tol)} over"


@pytest.mark.parametrize("scale", [None, 0.5])
@pytest.mark.parametrize("case", ATTEND)
def test_attention_and_its_weights(cuda_device, case, scale):
    q, t1, ring, pos, _ = attention_problem(cuda_device, case, 5)
    before = [None if x is None else x.clone() for x in (q, *t1, *ring, pos)]
    out = cmc.two_tier_decode_attn_weighted(q, *t1, *ring, pos, scale=scale)
    torch.cuda.synchronize()
    for x, y in zip((q, t1[0], t1[1], ring[0], ring[1], pos), [before[i] for i in (0, 1, 2, 4, 5, 7)]):
        assert x is None or torch.equal(x.view(torch.int16) if x.dtype == torch.bfloat16 else x,
                                        y.view(torch.int16) if x.dtype == torch.bfloat16 else y)
    # weights of slots without a token are as they were
    B, W, n = q.shape[0], ring[2].shape[3], f64(pos)
    for b in range(B):
        live = max(0, min(int(n[b]), W))
        assert torch.equal(ring[2][b, ..., live:].view(torch.int32), before[6][b, ..., live:].view(torch.int32))
    s = scale or 1 / math.sqrt(q.shape[-1])
    check_attention(out, t1[2], ring[2], f64(before[0]), [f64(x) for x in before[1:4]], [f64(x) for x in before[4:7]], n, s)
    again = [None if x is None else x.clone() for x in before]
    out2 = cmc.two_tier_decode_attn_weighted(again[0], *again[1:4], *again[4:7], again[7], scale=scale, out=torch.ones_like(q))
    assert torch.equal(out, out2)  # in a fixed order: the same bits
    assert torch.equal(again[6].view(torch.int32), ring[2].view(torch.int32))


@pytest.mark.parametrize("form", ["plain", "rope", "norm", "both"])
@pytest.mark.parametrize("case", [c for c in ATTEND if c[5] + c[6] < 5000])
def test_step(cuda_device, case, form):
    B, L, H, G, d, k, W, _ = case
    q, t1, ring, pos, g = attention_problem(cuda_device, case, 6)
    k_new, v_new = randn(g, B, L, H, d), randn(g, B, L, H, d)
    evicted = torch.randint(0, 999, (B,), generator=g, device=cuda_device)
    qw = kw = None
    if form in ("norm", "both"):
        qw, kw = (1 + 0.5 * torch.randn(L, d, generator=g, device=cuda_device) for _ in range(2))
    opts = dict(q_weight=qw, k_weight=kw, eps=1e-5)
    if form in ("rope", "both"):
        opts.update(rope_theta=THETA, rope_offset=k, evicted=evicted)
    before = [f64(x) for x in (q, *t1, *ring, pos)]
    bits = [x.view(torch.int16).clone() for x in ring[:2]]
    pos0 = pos.clone()
    out = cmc.decode_step_weighted(q, *t1, *ring, pos, k_new, v_new, **opts)
    torch.cuda.synchronize()
    n = before[7]
    np.testing.assert_array_equal(f64(pos), np.where(n < 0, n, n + 1))
    # the stored key (two evaluations in fp32 may round to either side of a border, so it is the formula's, not
    # qk_norm_rope's bit for bit), and everything else as it was
    p = ow.positions(n, f64(evicted), k, 1) if "rope_theta" in opts else None
    for b in range(B):
        if n[b] < 0:
            continue
        s = int(n[b] % W)
        if form == "plain":
            assert torch.equal(ring[0][b, :, :, s], k_new[b])
        else:
            check_heads(ring[0][b:b + 1, :, None, :, s], f64(k_new)[b:b + 1, :, None], kw, None if p is None else p[b:b + 1],
                        "new key", eps=1e-5)
        for i, x in enumerate((ring[0], v_new)):
            bits[i][b, :, :, s] = (x[b, :, :, s] if i == 0 else x[b]).view(torch.int16)
        before[6][b, :, :, s] = 0.0
    for x, y in zip(ring, bits):
        assert torch.equal(x.view(torch.int16), y)
    qq = before[0]
    if form != "plain":
        w = None if qw is None else f64(qw)[None, :]
        qq = ow.heads(qq, w, 1e-5)
        if "rope_theta" in opts:
            qq = ow.heads(qq, None, 0.0, THETA, np.broadcast_to(p, qq.shape[:2]))
    check_attention(out, t1[2], ring[2], qq, before[1:4], [f64(ring[0]), f64(ring[1]), before[6]], f64(pos),
                    1 / math.sqrt(d), prepared=form != "plain")


def test_step_as_append_and_attend(cuda_device):
    """Bit for bit the append followed by the attention, and its outputs those of decode_step's within both's rounding."""
    q, t1, ring, pos, g = attention_problem(cuda_device, (6, 2, 2, 4, 128, 30, 130, [0, 50, 129, 130, 400, 7]), 7, poison=False)
    k_new, v_new = randn(g, 6, 2, 2, 128), randn(g, 6, 2, 2, 128)
    a = [x.clone() for x in (*t1, *ring, pos)]
    slot = pos % 130
    out = cmc.decode_step_weighted(q, *t1, *ring, pos, k_new, v_new)
    cmc.window_append(a[3], a[4], a[6], k_new, v_new)
    a[5][torch.arange(6, device=cuda_device), :, :, slot] = 0.0
    out2 = cmc.two_tier_decode_attn_weighted(q, *a)
    assert torch.equal(out, out2)
    for x, y in zip((*t1, *ring, pos), a):
        assert torch.equal(x, y)
    plain = cmc.two_tier_decode_attn(q, a[0], a[1], None, a[3], a[4], a[6])
    err = (plain.float() - out.float()).abs()
    assert (err <= 2.0 ** -6 * (plain.float().abs() + 4.0)).all()


def test_nan_among_the_keys_reaches_its_kv_head_only(cuda_device):
    q, t1, ring, pos, _ = attention_problem(cuda_device, (2, 1, 2, 4, 64, 40, 100, [100]), 8, poison=False)
    clean = [x.clone() for x in (*t1, *ring)]
    t1[0][0, 0, 1, 3, 5] = float("nan")
    want = cmc.two_tier_decode_attn_weighted(q, *clean, pos)
    out = cmc.two_tier_decode_attn_weighted(q, *t1, *ring, pos)
    assert out[0, 0, 4:].isnan().all() and t1[2][0, 0, 1].isnan().all() and ring[2][0, 0, 1].isnan().all()
    assert torch.equal(out[0, 0, :4], want[0, 0, :4]) and torch.equal(out[1], want[1])
    assert torch.equal(t1[2][1], clean[2][1]) and torch.equal(ring[2][0, 0, 0], clean[5][0, 0, 0])


@pytest.mark.parametrize("B, G", [(1, 4), (480, 1), (480, 2)])
def test_scores_and_values_that_are_not_finite(cuda_device, B, G):
    """In a CTA's and in a warp's unit: what they reach, and what they leave as it was."""
    q, t1, ring, pos, _ = attention_problem(cuda_device, (B, 1, 2, G, 64, 40, 50, [50]), 8, poison=False)
    clean = [x.clone() for x in (*t1, *ring)]
    want = cmc.two_tier_decode_attn_weighted(q, *clean, pos)

    def run(change):
        x = [y.clone() for y in (q, *t1, *ring)]
        change(x)
        return cmc.two_tier_decode_attn_weighted(*x, pos), x[3], x[6]

    def same(out, w1, w2, heads, kv):
        """The outputs of `heads`, and the weights of the KV heads `kv`, of sequence 0; everything of the others."""
        for h in heads:
            assert torch.equal(out[0, 0, h], want[0, 0, h])
        for g in kv:
            assert torch.equal(w1[0, 0, g], clean[2][0, 0, g]) and torch.equal(w2[0, 0, g], clean[5][0, 0, g])
        assert torch.equal(out[1:], want[1:]) and torch.equal(w1[1:], clean[2][1:]) and torch.equal(w2[1:], clean[5][1:])

    def nan_query(x):
        x[0][0, 0, 0, 7] = float("nan")
    out, w1, w2 = run(nan_query)
    assert out[0, 0, 0].isnan().all() and w1[0, 0, 0].isnan().all() and w2[0, 0, 0].isnan().all()
    same(out, w1, w2, range(1, 2 * G), [1])

    def infinite_scores(sign):
        def change(x):
            x[0][0, 0, :, 3] = 1.0
            x[1][0, 0, 0, 5, :] = 0.0
            x[1][0, 0, 0, 5, 3] = sign * float("inf")
            x[0][0, 0, :, 4:] = 0.0  # so that no infinity meets a zero of the keys, nor an infinity the other sign
        return change
    out, w1, w2 = run(infinite_scores(1.0))
    assert out[0, 0, :G].isnan().all() and w1[0, 0, 0].isnan().all() and not out[0, 0, G:].isnan().any()
    out, w1, w2 = run(infinite_scores(-1.0))
    assert not out.isnan().any() and w1[0, 0, 0, 5] == t1[2][0, 0, 0, 5] and (w1[0, 0, 0, :5] > t1[2][0, 0, 0, :5]).all()

    def nan_value(x):
        x[5][0, 0, 1, 4, 9] = float("nan")
    out, w1, w2 = run(nan_value)
    assert out[0, 0, G:, 9].isnan().all() and not out[0, 0, G:, :9].isnan().any()
    same(out, w1, w2, range(G), [0, 1])


@pytest.mark.parametrize("B, H", [(2, 1), (5, 4)])
def test_units_whose_products_go_to_the_workspace(cuda_device, B, H):
    """G = 8: more than 9,216 keys a unit; with up to a CTA an SM they stay in shared memory all the same."""
    case = (B, 1, H, 8, 64, 6000, 5000, [4999, 5])
    dims = cmc.CmcDims(B, 1, 8 * H, H, 64, 6000, 6000, 5000)
    assert cmc.decode_attn_weighted_workspace_size(dims) > B * H * 11000 * 36
    assert cmc.decode_attn_weighted_plan(dims) == B * H * 8
    q, t1, ring, pos, g = attention_problem(cuda_device, case, 9)
    before = [f64(x) for x in (q, *t1, *ring, pos)]
    ws = cmc.DecodeWorkspace(dims, cuda_device, weighted=True)
    out = cmc.two_tier_decode_attn_weighted(q, *t1, *ring, pos, workspace=ws)
    check_attention(out, t1[2], ring[2], before[0], before[1:4], before[4:7], before[7], 1 / 8)
    assert ws.status() == 0
    with pytest.raises(cmc.CmcError, match="WORKSPACE"):
        cmc.two_tier_decode_attn_weighted(q, *t1, *ring, pos,
                                          workspace=cmc.DecodeWorkspace(cmc.CmcDims(2, 1, 8, 1, 64, 1, 1, 1), cuda_device, weighted=True))


def test_offsets_past_32_bits(cuda_device):
    """Caches of more than 2^32 elements: the last unit's rows, in attention and in eviction."""
    B, H, d, W = 1, 40, 128, 1 << 20
    ring = [torch.zeros(B, 1, H, W, d, dtype=torch.bfloat16, device=cuda_device) for _ in range(2)]
    w = torch.zeros(B, 1, H, W, device=cuda_device)
    g = gen(cuda_device, 10)
    n = 50
    small = [randn(g, B, 1, H, n, d) for _ in range(2)]
    for x, y in zip(ring, small):
        x[..., :n, :] = y
    pos = torch.tensor([n], device=cuda_device)
    q = randn(g, B, 1, H * 2, d)
    sw = torch.zeros(B, 1, H, n, device=cuda_device)
    want = cmc.two_tier_decode_attn_weighted(q, None, None, None, *small, sw, pos)
    out = cmc.two_tier_decode_attn_weighted(q, None, None, None, *ring, w, pos)
    assert (out.float() - want.float()).abs().max() <= 2.0 ** -5  # split over other CTAs: rounded elsewhere
    assert (w[..., :n] - sw).abs().max() <= 2.0 ** -16 and not w[..., n:].any()
    k2, v2, w2, idx, held = cmc.evict_cache(*ring, w, 7, pos=pos, recent=2)
    ref, _ = ow.evict(w[..., :n].cpu().numpy(), 7, 2)
    np.testing.assert_array_equal(idx.cpu().numpy(), ref)
    rows = torch.from_numpy(ref).to(cuda_device)
    assert torch.equal(v2, torch.gather(small[1], 3, rows[..., None].expand(B, 1, H, 7, d)))
    assert held.tolist() == [7]


def test_attention_refusals(cuda_device):
    q, t1, ring, pos, _ = attention_problem(cuda_device, (2, 1, 2, 4, 64, 8, 16, [3]), 11, poison=False)
    row = q[:, :, :2].contiguous()
    calls = [[q, *t1, *ring, pos], [q, None, None, None, *ring, pos]]
    for args in calls:
        for i, x in enumerate(args):
            if x is None:
                bads = [t1[0] if i < 3 else t1[2]]  # a part of Tier-1
            else:
                bads = [None, x[:1], x.double() if x.is_floating_point() else x.int(), x.cpu(), [0]]
            for bad in bads:
                a = list(args)
                a[i] = bad
                with pytest.raises((ValueError, TypeError)):
                    cmc.two_tier_decode_attn_weighted(*a)
                with pytest.raises((ValueError, TypeError)):
                    cmc.decode_step_weighted(*a, row, row)
    for new in ((row[:1], row), (row, row[:, :, :1]), (row, row.float()), (row, None)):
        with pytest.raises((ValueError, TypeError)):
            cmc.decode_step_weighted(*calls[0], *new)
    for kw in (dict(out=row), dict(q_weight=row), dict(rope_theta=-1.0), dict(evicted=pos[:1], rope_theta=1e4),
               dict(workspace=cmc.DecodeWorkspace(cmc.CmcDims(2, 1, 8, 2, 64, 8, 8, 16), torch.device("cpu"), weighted=True))):
        with pytest.raises((ValueError, TypeError)):
            cmc.decode_step_weighted(*calls[0], row, row, **kw)
    with pytest.raises(ValueError):
        cmc.DecodeWorkspace(cmc.CmcDims(2, 1, 8, 2, 64, 8, 8, 16), cuda_device, q8=True, weighted=True)
    assert pos.tolist() == [3, 3]


# ----------------------------------------------------------------------------
# Eviction
# ----------------------------------------------------------------------------

EVICT = [  # B, L, Hkv, d, T, keep, recent, positions (None: all rows)
    (1, 1, 1, 64, 1, 1, 0, None), (1, 1, 2, 64, 2, 1, 1, None), (1, 1, 1, 128, 63, 62, 0, None), (2, 1, 3, 128, 64, 64, 5, None),
    (2, 2, 2, 64, 65, 1, 0, None), (3, 1, 2, 128, 130, 65, 64, [130, 0, 64]), (5, 1, 2, 64, 100, 40, 10, [39, 40, 41, 100, 357]),
    (2, 1, 2, 128, 640, 333, 333, [1281, 700]), (1, 1, 2, 128, 4097, 2050, 17, None), (1, 1, 1, 64, 16384, 5000, 100, [16384]),
    (1, 1, 2, 64, 16385, 300, 0, [40000]), (2, 1, 1, 128, 30000, 29999, 1, [30000, 29999]), (30, 4, 8, 64, 33, 16, 3, [33, 20, 70]),
    (2, 1, 1, 64, 50, 20, 4, [-1, 2 ** 40 + 3]),
    # keys that fill shared memory, and that do not fit; more units than SMs
    (1, 1, 2, 64, 49152, 100, 7, None), (1, 1, 2, 64, 49153, 20000, 64, [49153]), (2, 1, 1, 64, 100000, 65, 0, [170001, 90000]),
    (500, 1, 1, 64, 3000, 64, 9, [2999, 70, 5000]),
]


def weights_of(g, kind, *shape):
    dev = g.device
    if kind == "heavy tail":
        return torch.exp(3 * torch.randn(shape, generator=g, device=dev))
    if kind == "ties":
        return torch.randint(0, 4, shape, generator=g, device=dev).float() * 0.25
    if kind == "equal":
        return torch.full(shape, 0.5, device=dev)
    x = torch.randn(shape, generator=g, device=dev)  # odd values
    odd = torch.tensor([float("nan"), float("inf"), -float("inf"), 0.0, -0.0, 1e-45, -1e-45], device=dev)
    return torch.where(torch.rand(shape, generator=g, device=dev) < 0.5, x, odd[torch.randint(0, 7, shape, generator=g, device=dev)])


@pytest.mark.parametrize("kind", ["heavy tail", "ties", "equal", "odd"])
@pytest.mark.parametrize("case", EVICT)
def test_eviction(cuda_device, case, kind):
    B, L, H, d, T, keep, recent, positions = case
    g = gen(cuda_device, 12)
    k, v = randn(g, B, L, H, T, d), randn(g, B, L, H, T, d)
    w = weights_of(g, kind, B, L, H, T)
    pos = None if positions is None else torch.tensor([positions[b % len(positions)] for b in range(B)], device=cuda_device)
    evicted = torch.arange(B, device=cuda_device)
    R = keep + 3
    outs = [torch.full((B, L, H, R, d), 9.0, dtype=torch.bfloat16, device=cuda_device) for _ in range(2)]
    outs.append(torch.full((B, L, H, R), 9.0, device=cuda_device))
    before = [x.clone() for x in (k, v, w)]
    r = cmc.evict_cache(k, v, w, keep, pos=pos, recent=recent, evicted=evicted, out_k=outs[0], out_v=outs[1], out_weight=outs[2])
    torch.cuda.synchronize()
    assert all(a is b for a, b in zip(r, outs))
    for x, y in zip((k, v, w), before):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))
    idx, held = ow.evict(w.cpu().numpy(), keep, recent, None if pos is None else f64(pos))
    np.testing.assert_array_equal(r[3].cpu().numpy(), idx)
    np.testing.assert_array_equal(f64(r[4]), held)
    p = np.full(B, T) if pos is None else f64(pos)
    np.testing.assert_array_equal(f64(evicted), np.arange(B) + np.where(p < 0, 0, p - held))
    rows = torch.from_numpy(idx).to(cuda_device)
    live = rows >= 0
    for got, x in zip(outs, (k, v, w)):
        at = rows.clamp(min=0)
        want = torch.gather(x, 3, at if x.dim() == 4 else at[..., None].expand(*at.shape, d))
        m = live if x.dim() == 4 else live[..., None]
        want = torch.where(m, want, torch.full_like(want, 9.0))
        assert torch.equal(got[:, :, :, :keep].contiguous().view(torch.int16), want.view(torch.int16))
        assert (got[:, :, :, keep:] == 9.0).all()
    # tensors of its own
    r2 = cmc.evict_cache(k, v, w, keep, pos=pos, recent=recent)
    assert r2[0].shape == (B, L, H, keep, d) and torch.equal(r2[3], r[3]) and torch.equal(r2[4], r[4])


@pytest.mark.parametrize("case", EVICT)
def test_eviction_in_place(cuda_device, case):
    B, L, H, d, T, keep, recent, positions = case
    g = gen(cuda_device, 13)
    k, v = randn(g, B, L, H, T, d), randn(g, B, L, H, T, d)
    w = weights_of(g, "ties", B, L, H, T)
    pos = torch.tensor([(positions or [T])[b % len(positions or [T])] for b in range(B)], device=cuda_device)
    evicted = torch.zeros(B, dtype=torch.int64, device=cuda_device)
    before = [x.clone() for x in (k, v, w, pos)]
    dims = cmc.CmcDims(B, L, H, H, d, T, keep, T)
    ws = cmc.DecodeWorkspace(dims, cuda_device, weighted=True)
    r = cmc.evict_cache(k, v, w, keep, pos=pos, recent=recent, evicted=evicted, out_k=k, out_v=v, out_weight=w, out_pos=pos, workspace=ws)
    torch.cuda.synchronize()
    p = f64(before[3])
    stays = (p < 0) | ((p > T) & (p % T != 0))  # a ring that starts elsewhere
    idx, held = ow.evict(before[2].cpu().numpy(), keep, recent, p)
    idx[stays] = -1
    held[stays] = p[stays]
    np.testing.assert_array_equal(r[3].cpu().numpy(), idx)
    np.testing.assert_array_equal(f64(pos), held)
    np.testing.assert_array_equal(f64(evicted), p - held)
    assert ws.status() == (cmc.DEVFLAG_BAD_POS if stays.any() else 0) and not ws.buf[256:256 + 8 * B].any()
    for x, y in zip((k, v, w), before):
        for b in range(B):
            m = 0 if stays[b] else int(held[b])
            rows = torch.from_numpy(idx[b:b + 1, :, :, :m]).to(cuda_device)
            want = torch.gather(y[b:b + 1], 3, rows if y.dim() == 4 else rows[..., None].expand(*rows.shape, d))
            assert torch.equal(x[b:b + 1, :, :, :m], want) and torch.equal(x[b, :, :, max(m, keep):], y[b, :, :, max(m, keep):])


def test_eviction_refusals(cuda_device):
    k = torch.zeros(2, 1, 2, 10, 64, dtype=torch.bfloat16, device=cuda_device)
    v, w = k.clone(), torch.zeros(2, 1, 2, 10, device=cuda_device)
    pos = torch.full((2,), 10, device=cuda_device)
    for keep, recent in ((0, 0), (11, 0), (-1, 0), (5, 6), (5, -1), (2 ** 32 + 5, 0), (5, 2 ** 32 + 1)):
        with pytest.raises(cmc.CmcError, match="RANGE"):
            cmc.evict_cache(k, v, w, keep, recent=recent)
    with pytest.raises(cmc.CmcError, match="RANGE"):  # in place in part
        cmc.evict_cache(k, v, w, 5, out_k=k, out_v=torch.zeros_like(k), out_weight=torch.zeros_like(w))
    with pytest.raises(cmc.CmcError, match="RANGE"):  # fewer rows than are kept
        cmc.evict_cache(k, v, w, 5, out_k=k[..., :4, :].contiguous(), out_v=v[..., :4, :].contiguous(), out_weight=w[..., :4].contiguous())
    for kw in (dict(pos=pos.int()), dict(pos=pos[:1]), dict(evicted=pos[:1]), dict(out_pos=pos[:1]), dict(out_pos=pos.float()),
               dict(out_k=k[..., :6, :]), dict(out_weight=w[..., :5]), dict(out_v=[1]),
               dict(workspace=cmc.DecodeWorkspace(cmc.CmcDims(2, 1, 2, 2, 64, 1, 1, 1), torch.device("cpu"), q8=True))):
        with pytest.raises((ValueError, TypeError)):
            cmc.evict_cache(k, v, w, 5, **kw)
    for a in ((k, v[:1], w), (k, v, w[..., :9]), (k, v, w.double()), (k.float(), v, w), (k, v.cpu(), w)):
        with pytest.raises((ValueError, TypeError)):
            cmc.evict_cache(*a, 5)
    with pytest.raises(cmc.CmcError, match="WORKSPACE"):
        big = torch.zeros(40, 1, 2, 10, 64, dtype=torch.bfloat16, device=cuda_device)
        cmc.evict_cache(big, big.clone(), torch.zeros(40, 1, 2, 10, device=cuda_device), 5,
                        workspace=cmc.DecodeWorkspace(cmc.CmcDims(2, 1, 2, 2, 64, 1, 1, 1), cuda_device, weighted=True))


# ----------------------------------------------------------------------------
# A run of them
# ----------------------------------------------------------------------------

class Decoder:
    """One request batch: prefill, decode steps, and eviction whenever the ring is full."""

    def __init__(self, dev, seed, B=3, L=2, H=2, G=4, d=64, k=9, W=40):
        g = gen(dev, seed)
        self.B, self.k, self.W, self.dev = B, k, W, dev
        self.t1 = [randn(g, B, L, H, k, d), randn(g, B, L, H, k, d), torch.zeros(B, L, H, k, device=dev)]
        self.ring = [randn(g, B, L, H, W, d), randn(g, B, L, H, W, d), torch.full((B, L, H, W), float("nan"), device=dev)]
        self.pos, self.evicted = torch.zeros(B, dtype=torch.int64, device=dev), torch.zeros(B, dtype=torch.int64, device=dev)
        self.qw, self.kw = (1 + 0.3 * torch.randn(L, d, generator=g, device=dev) for _ in range(2))
        self.x = randn(g, B, L, 31, H * (G + 2), d)
        self.count = torch.tensor([31, 20, 31][:B], device=dev)
        self.parts = [H * G, H, H]
        self.new = [randn(g, 12, B, L, H * (G + 2), d)]
        self.opts = dict(q_weight=self.qw, k_weight=self.kw, rope_theta=THETA, rope_offset=k, evicted=self.evicted)

    def state(self):
        return [*self.t1, *self.ring, self.pos, self.evicted]

    def prefill(self):
        q, k, v = self.x.split(self.parts, dim=3)
        return cmc.window_prefill(q, k, v, self.ring[0], self.ring[1], self.pos, ring_weight=self.ring[2], count=self.count, **self.opts)

    def step(self, i):
        q, k, v = (y.contiguous() for y in self.new[0][i].split(self.parts, dim=2))
        return cmc.decode_step_weighted(q, *self.t1, *self.ring, self.pos, k, v, **self.opts)

    def evict(self):
        return cmc.evict_cache(*self.ring, 25, pos=self.pos, recent=6, evicted=self.evicted, out_k=self.ring[0],
                               out_v=self.ring[1], out_weight=self.ring[2], out_pos=self.pos)[3]

    def run(self):
        outs = [self.prefill()]
        for i in range(9):
            outs.append(self.step(i))
        outs.append(self.evict())
        for i in range(9, 12):
            outs.append(self.step(i))
        return outs


def test_a_run_of_prefill_steps_and_eviction(cuda_device):
    """Each call against the oracle on what the call before it left."""
    r = Decoder(cuda_device, 20)
    r.prefill()
    assert r.pos.tolist() == [31, 20, 31]
    for i in range(12):
        if i == 9:
            old = [x.clone() for x in r.ring]
            assert r.pos.tolist() == [40, 29, 40]
            idx = r.evict()
            want, held = ow.evict(old[2].cpu().numpy(), 25, 6, np.array([40, 29, 40]))
            np.testing.assert_array_equal(idx.cpu().numpy(), want)
            assert r.pos.tolist() == held.tolist() == [25, 25, 25] and r.evicted.tolist() == [15, 4, 15]
            rows = torch.from_numpy(want).to(cuda_device)
            assert torch.equal(r.ring[2][..., :25], torch.gather(old[2], 3, rows))
        before = [f64(x) for x in r.state()]
        out = r.step(i)
        n = before[6]
        for b in range(r.B):
            before[5][b, :, :, int(n[b] % r.W)] = 0.0
        q = f64(r.new[0][i][:, :, :r.parts[0]])
        p = ow.positions(n, before[7], r.k, 1)
        np.testing.assert_array_equal(p[:, 0], r.k + np.array([31, 20, 31]) + i)  # the token's number, whatever was evicted
        q = ow.heads(ow.heads(q, f64(r.qw)[None], 1e-6), None, 0.0, THETA, np.broadcast_to(p, q.shape[:2]))
        check_attention(out, r.t1[2], r.ring[2], q, before[:3], [f64(r.ring[0]), f64(r.ring[1]), before[5]], n + 1,
                        1 / 8, prepared=True)
    total = (torch.nan_to_num(r.t1[2]).sum(-1) + torch.nan_to_num(r.ring[2]).sum(-1))
    assert (total <= 12 * 4 + 1e-3).all()


@pytest.mark.parametrize("given", [True, False])
def test_a_captured_run(cuda_device, given):
    """The same bits from a graph replayed twice, beside eager calls on another stream."""
    eager = Decoder(cuda_device, 21)
    start = [x.clone() for x in eager.state()]
    want = eager.run()
    end = [x.clone() for x in eager.state()]
    r = Decoder(cuda_device, 21)
    if given:
        dims = cmc.CmcDims(r.B, 2, 8, 2, 64, r.k, r.k, r.W)
        ws = cmc.DecodeWorkspace(dims, cuda_device, weighted=True)
        prefill, step, evict = cmc.window_prefill, cmc.decode_step_weighted, cmc.evict_cache
        r.prefill = lambda: prefill(*r.x.split(r.parts, dim=3), r.ring[0], r.ring[1], r.pos, ring_weight=r.ring[2], count=r.count, workspace=ws, **r.opts)
        r.step = lambda i: step(*[y.contiguous() for y in r.new[0][i].split(r.parts, dim=2)][:1], *r.t1, *r.ring, r.pos,
                                *[y.contiguous() for y in r.new[0][i].split(r.parts, dim=2)][1:], workspace=ws, **r.opts)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            got = r.run()
    other = Decoder(cuda_device, 22)
    stream = torch.cuda.Stream()
    for _ in range(2):
        for x, y in zip(r.state(), start):
            x.copy_(y)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(stream):
            other.step(0)
        torch.cuda.synchronize()
        for x, y in zip(r.state(), end):
            assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))
        for i, (x, y) in enumerate(zip(got, want)):
            if i == 0:  # rows past count are not written
                x, y = x[:, :, :20], y[:, :, :20]
            assert torch.equal(x, y), i
    if given:
        assert ws.status() == 0 and not ws.buf.any()


def test_a_rotation_first_asked_for_in_a_capture(cuda_device):
    """A frequency that the device has no table of yet: the captured call carries its own, and gives the bits of the
    eager ones after it."""
    g = gen(cuda_device, 23)
    q, k = randn(g, 2, 1, 5, 8, 64), randn(g, 2, 1, 5, 2, 64)
    pos = torch.tensor([3, 10 ** 6], device=cuda_device)
    case = (2, 1, 2, 4, 64, 8, 16, [3, 20])
    args, t1, ring, p, _ = attention_problem(cuda_device, case, 24, poison=False)
    new = [randn(g, 2, 1, 2, 64) for _ in range(2)]
    state = [x.clone() for x in (*t1, *ring, p)]
    ws = cmc.DecodeWorkspace(cmc.CmcDims(2, 1, 8, 2, 64, 8, 8, 16), cuda_device, weighted=True)
    theta = 12345.678
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        a = cmc.qk_norm_rope(q, k, pos, rope_theta=theta)
        b = cmc.decode_step_weighted(args, *t1, *ring, p, *new, rope_theta=theta, workspace=ws)
    graph.replay()
    torch.cuda.synchronize()
    c = cmc.qk_norm_rope(q, k, pos, rope_theta=theta)
    d = cmc.decode_step_weighted(args, *state, *new, rope_theta=theta)
    for x, y in zip((*a, b, *t1, *ring, p), (*c, d, *state)):
        assert torch.equal(x, y)
    assert ws.status() == 0


def test_streams_have_workspaces_of_their_own(cuda_device):
    runs = [Decoder(cuda_device, 30 + i, B=2) for i in range(4)]
    alone = [Decoder(cuda_device, 30 + i, B=2) for i in range(4)]
    want = [r.run() for r in alone]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    got = []
    for r, s in zip(runs, streams):
        with torch.cuda.stream(s):
            got.append(r.run())
    torch.cuda.synchronize()
    for a, b, x, y in zip(got, want, runs, alone):
        for i, j in zip(a[1:], b[1:]):
            assert torch.equal(i, j)
        for i, j in zip(x.state(), y.state()):
            assert torch.equal(i.contiguous().view(torch.uint8), j.contiguous().view(torch.uint8))
    assert cmc.weighted_cache_status() & ~cmc.DEVFLAG_BAD_POS == 0
