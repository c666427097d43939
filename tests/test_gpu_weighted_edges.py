"""The calls over a cache with weights on the GPU at their edges: new tokens at every place of a block, in every variant of
the step's kernel.  Tolerances as in test_gpu_weighted.py, whose helpers check."""

import math

import numpy as np
import pytest
import torch

import paper_2609_25537_gb300 as cmc
from oracle import weighted as ow
from test_gpu_weighted import THETA, attention_problem, check_attention, check_heads, f64, gen, randn

pytestmark = pytest.mark.gpu


def prepared_queries(q, weight, eps, p):
    """The formula's norm (where gains are given) and rotation of one token's query heads at positions p [B, 1]."""
    q = ow.heads(f64(q), None if weight is None else f64(weight)[None, :], eps)
    return q if p is None else ow.heads(q, None, 0.0, THETA, np.broadcast_to(p, q.shape[:2]))


def check_step(dev, case, prepared, seed, workspace=None):
    """A fused step, plain or with norm and rotation, against the oracle on the ring that it left, and the ring."""
    B, L, H, G, d, k, W, _ = case
    q, t1, ring, pos, g = attention_problem(dev, case, seed)
    k_new, v_new = randn(g, B, L, H, d), randn(g, B, L, H, d)
    opts = {}
    if prepared:
        qw, kw = (1 + 0.5 * torch.randn(L, d, generator=g, device=dev) for _ in range(2))
        opts = dict(q_weight=qw, k_weight=kw, eps=1e-5, rope_theta=THETA, rope_offset=k)
    before = [f64(x) for x in (q, *t1, *ring, pos)]
    bits = [x.view(torch.int16).clone() for x in ring[:2]]
    out = cmc.decode_step_weighted(q, *t1, *ring, pos, k_new, v_new, workspace=workspace, **opts)
    torch.cuda.synchronize()
    n = before[7]
    np.testing.assert_array_equal(f64(pos), np.where(n < 0, n, n + 1))
    for b in range(B):
        if n[b] < 0:
            assert not out[b].any()
            continue
        s = int(n[b] % W)
        if not prepared:
            assert torch.equal(ring[0][b, :, :, s], k_new[b])
        bits[0][b, :, :, s] = ring[0][b, :, :, s].view(torch.int16)
        bits[1][b, :, :, s] = v_new[b].view(torch.int16)
        before[6][b, :, :, s] = 0.0
    for x, y in zip(ring, bits):
        assert torch.equal(x.view(torch.int16), y)
    p = ow.positions(n, None, k, 1)
    if prepared:
        for b in np.flatnonzero(n >= 0):
            check_heads(ring[0][b:b + 1, :, None, :, int(n[b] % W)], f64(k_new)[b:b + 1, :, None], kw, p[b:b + 1], "new key",
                        eps=1e-5)
    qq = prepared_queries(q, qw, 1e-5, p) if prepared else before[0]
    check_attention(out, t1[2], ring[2], qq, before[1:4], [f64(ring[0]), f64(ring[1]), before[6]], f64(pos), 1 / math.sqrt(d),
                    prepared=prepared)


# What the rule takes for a unit: B, Hkv, rows of Tier-1; rings of 70 slots, of which sequence b holds b
PLACES = {"a CTA": (40, 1, 20), "a cluster": (70, 1, 600), "two warps": (70, 8, 20), "a warp": (70, 16, 20),
          "the longest first": (70, 8, 500)}


@pytest.mark.parametrize("prepared", [False, True])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("unit", list(PLACES))
def test_new_tokens_at_every_place_of_a_block(cuda_device, unit, d, G, prepared):
    """The lanes that store a new token, a half or a quarter of a warp, are joined by the others before the products; blocks
    partly filled, in each of the kernel's variants."""
    B, H, k = PLACES[unit]
    ctas = cmc.decode_attn_weighted_plan(cmc.CmcDims(B, 1, H * G, H, d, k, k, 70))
    assert ctas == B * H * (2 if unit == "a cluster" else 1)
    check_step(cuda_device, (B, 1, H, G, d, k, 70, list(range(70))), prepared, 40)
