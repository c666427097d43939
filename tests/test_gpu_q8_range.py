"""Attention over the cache in 8 bits where blocks' values differ by much, or lie near the ends of
bf16's range: every form of the launch (a warp, a CTA, a cluster per unit, the longest first), with
several blocks a warp, against the fp64 oracle."""

import numpy as np
import pytest
import torch

import paper_2609_25537_gb300 as cmc
from oracle import q8
from _gpu_helpers import to_f64

pytestmark = pytest.mark.gpu

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu

# form: B, L, Hkv, G, d, k, W, warps that share a unit's blocks, grid
FORMS = {
    "warp": (150, 1, 8, 2, 128, 64, 256, 1, 300),
    "warp64": (230, 1, 8, 4, 64, 64, 256, 1, 460),
    "cta": (29, 1, 8, 4, 128, 256, 512, 4, 232),
    "cta64": (55, 1, 8, 8, 64, 256, 512, 4, 440),
    "cta3": (39, 1, 8, 4, 128, 256, 512, 4, 312),  # three an SM, two stages a warp
    "ordered": (64, 1, 8, 2, 128, 32, 480, 4, 512),  # several waves, the longest first
    "cluster": (1, 1, 8, 4, 128, 2048, 2048, 32, 64),
}


def rounds(T1, T2, warps):
    """Which block of its warp each block is: Tier-1's, the ring's."""
    n1, n2 = (T1 + 31) // 32, (T2 + 31) // 32
    j = np.arange(n1 + n2) // warps
    return j[:n1], j[n1:]


def make(rng, form, byte_of, key_of=None, most=448.0):
    """A problem of full rings whose V blocks have the bytes byte_of(unit, round), None for a block of
    zeros; key_of(unit, round) gives element 0 of the block's keys.  Values of V are up to `most` times the
    power of two; keys are about 1."""
    B, L, H, G, d, k, W, warps, grid = FORMS[form]
    dims = cmc.CmcDims(B, L, G * H, H, d, k, k, W)
    for fused in (False, True):
        assert cmc.decode_attn_q8_plan(dims, fused) == grid
    caches = []
    for T, r in zip((k, W), rounds(k, W, warps)):
        x = rng.standard_normal((B, L, H, 2, T, d), dtype=np.float32)
        x[:, :, :, 0] *= 64.0
        x[:, :, :, 1] *= most / 4
        x = x.clip(-most, most)
        scales = np.full((B, L, H, 2, q8.scale_bytes(T)), 0xFF, dtype=np.uint8)
        scales[:, :, :, 0] = 121
        for b in range(B):
            for h in range(H):
                for j, i in enumerate(r):
                    byte = byte_of(b * H + h, i)
                    rows = slice(32 * j, 32 * j + 32)
                    if byte is None:
                        x[b, 0, h, 1, rows] = 0.0
                    scales[b, 0, h, 1, j] = byte or 0
                    if key_of is not None:
                        x[b, 0, h, 0, rows, 0] = key_of(b * H + h, i) * 64.0
        codes = torch.from_numpy(x).to(E4M3).view(torch.uint8).numpy()
        caches.append((codes, scales))
    q = torch.from_numpy(rng.standard_normal((B, L, G * H, d)).astype(np.float32)).to(torch.bfloat16)
    return q, *caches, np.full(B, 2 * W + 3, dtype=np.int64)


def device_args(dev, q, t1, ring, pos):
    def put(codes, scales):
        return (torch.from_numpy(codes).to(dev).view(E4M3), torch.from_numpy(scales).to(dev).view(E8M0))
    return [q.to(dev), *put(*t1), *put(*ring), torch.from_numpy(pos).to(dev)]


def run(dev, *problem, scale=None):
    return cmc.two_tier_decode_attn_q8(*device_args(dev, *problem), scale=scale)


def check(got, q, t1, ring, units, what, scale=None):
    """Against the oracle, each output within what the roundings on the way to it may do:

    * the output is rounded to bf16, 2^-8 of it (2^-134 where it is subnormal);
    * a probability is rounded to fp16, 2^-11 of it or, relative to the largest, 2^-29, but for one
      that becomes 0 by no more than itself;
    * what lies 2^-64 below the largest of a head's tokens (their probability times their block's power of
      two times 448) may be lost;
    * a score is off by what fp16 leaves of the query and by fp32's roundings (2^-23 each; 2^x by 2^-21):
      an error e of all scores changes the quotient by at most 2 e (1 + e) of the sum of p |v|.
    """
    B, L, Hq, d = q.shape
    H = ring[0].shape[2]
    G = Hq // H
    scale = 1 / np.sqrt(d) if scale is None else scale
    got, q = to_f64(got), to_f64(q)
    for u in units:
        b, g = u // H, u % H
        x = [q8.values(c[b:b + 1, :, g:g + 1], s[b:b + 1, :, g:g + 1])[0, 0, 0] for c, s in (t1, ring)]
        K, V = (np.concatenate([y[i] for y in x]) for i in range(2))
        top = np.concatenate([np.repeat(np.array([q8.power(c) for c in s[b, 0, g, 1]]), 32)[:c.shape[4]]
                              for c, s in (t1, ring)]) * 448.0
        for h in range(g * G, g * G + G):
            s = K @ q[b, 0, h] * scale
            p = np.exp(s - s.max())
            out, mag = (p @ y / p.sum() for y in (V, np.abs(V)))
            a = np.abs(q[b, 0, h])
            e = scale * (2.0 ** -30 * a.max() * np.abs(K).sum(axis=1)
                         + (d + 8) * 2.0 ** -23 * (np.abs(K) @ a)).max()
            bound = (2.0 ** -8 * np.abs(out) + 2.0 ** -134
                     + (2.0 ** -11 + 2 * (e + 2.0 ** -21) * (1 + e)) * mag
                     + (np.minimum(p, 2.0 ** -29) @ np.abs(V) + 2.0 ** -64 * (p * top).max()) / p.sum())
            err = np.abs(got[b, 0, h] - out)
            assert (err <= bound).all(), (what, u, h, got[b, 0, h, :4], out[:4])


# Bytes of V's blocks in the order in which a warp takes them (None: a block of zeros), repeated.
PATTERNS = {
    "zeros after 2^10": [128, None, 126, None],
    "zeros after 2^62": [180, None, 176, None],
    "zeros after 2^74": [192, None, 190, None],
    "zeros after 2^122": [240, None, 240, None],
    "zeros first": [None, 240, None, 120],
    "rising": [40, 90, 150, 210],
    "falling": [240, 170, 100, 30],
    "forth and back": [240, 90, 90, 245],
}


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("form", FORMS)
def test_values_far_apart(cuda_device, form, fused):
    """Neighbouring blocks of a warp with values 2^10 to 2^240 apart, and blocks of zeros between them; in the
    fused step over the cache that it leaves."""
    rng = np.random.default_rng(1)
    lists = list(PATTERNS.values())
    q, t1, ring, pos = make(rng, form, lambda u, i: lists[u % len(lists)][i % 4])
    if fused:
        B, L, H, _, d = FORMS[form][:5]
        new = [torch.from_numpy(rng.standard_normal((B, L, H, d)).astype(np.float32)).to(torch.bfloat16)
               for _ in range(2)]
        args = device_args(cuda_device, q, t1, ring, pos)
        got = cmc.decode_step_q8(*args, *(x.to(cuda_device) for x in new))
        ring = [x.view(torch.uint8).cpu().numpy() for x in args[3:5]]
    else:
        got = run(cuda_device, q, t1, ring, pos)
    for u, name in enumerate(PATTERNS):
        check(got, q, t1, ring, [u], name)


@pytest.mark.parametrize("order", [1, -1])
@pytest.mark.parametrize("form", FORMS)
def test_large_values_behind_small_probabilities(cuda_device, form, order):
    """Every other block's values are 2^106 times as large, and its keys turn away from the first query
    of each KV head, so that they count nothing for it (their probabilities are 2^-245 of the largest), and from no
    other, for which nothing else counts."""
    rng = np.random.default_rng(2)
    q, t1, ring, pos = make(rng, form, lambda u, i: (227, 121)[::order][i % 2],
                            lambda u, i: (-7.0, 0.0)[::order][i % 2])
    G, d = FORMS[form][3:5]
    q[..., 0] = 0.0
    q[:, :, ::G, 0] = 280.0 * np.sqrt(d / 128)  # 280 * 7 / sqrt(128) = 173, 250 octaves
    check(run(cuda_device, q, t1, ring, pos), q, t1, ring, range(2), "")


@pytest.mark.parametrize("byte", [226, 233, 240, 247])
@pytest.mark.parametrize("form", FORMS)
def test_values_near_the_largest(cuda_device, form, byte):
    """Sums of many large values, which times the probabilities' 2^15 are beyond fp32, and whose mean is not
    (for byte 247 codes go up to 240: 2^128 is the first power of two that bf16 lacks)."""
    rng = np.random.default_rng(3)
    problem = make(rng, form, lambda u, i: byte, most=448.0 if byte < 247 else 240.0)
    problem[0][...] = 0.0  # all keys count alike
    for c, _ in problem[1:3]:
        c[:, :, :, 1] &= 0x7F  # and no sum cancels
    got = run(cuda_device, *problem)
    assert torch.isfinite(got).all()
    check(got, *problem[:3], range(2), "")


@pytest.mark.parametrize("byte", [0, 3, 12])
@pytest.mark.parametrize("form", FORMS)
def test_values_near_the_smallest(cuda_device, form, byte):
    """Means around 2^-120, of which the smallest are subnormal in bf16."""
    rng = np.random.default_rng(4)
    problem = make(rng, form, lambda u, i: byte)
    check(run(cuda_device, *problem), *problem[:3], range(2), "")


@pytest.mark.parametrize("form", FORMS)
def test_nan_reaches_what_it_touches_alone(cuda_device, form):
    """A query with a NaN or an infinity: its head. A block whose byte for K or V is NaN, the last of a warp or all of
    them: the heads of its unit. A NaN among the values: its column."""
    rng = np.random.default_rng(6)
    q, t1, ring, pos = make(rng, form, lambda u, i: 120 + i % 3)
    G = FORMS[form][3]
    q[0, 0, 0, 5] = float("nan")
    q[0, 0, G + 1, 0] = -float("inf")  # (unit 1)
    ring[1][0, 0, 2, 0, (ring[0].shape[4] - 1) // 32] = 255
    ring[1][0, 0, 3, 1, (ring[0].shape[4] - 1) // 32] = 255
    t1[1][0, 0, 4, 1, 0] = 255
    t1[1][0, 0, 5] = ring[1][0, 0, 5] = 255
    ring[0][0, 0, 6, 1, 40, 7] = 0xFF
    got = run(cuda_device, q, t1, ring, pos)
    want = torch.zeros(got.shape, dtype=torch.bool)
    want[0, 0, 0] = want[0, 0, G + 1] = True
    want[0, 0, 2 * G:6 * G] = True
    want[0, 0, 6 * G:7 * G, 7] = True
    assert torch.equal(torch.isnan(got).cpu(), want)
    q[0, 0, 0, 5] = q[0, 0, G + 1, 0] = 0.0
    ring[0][0, 0, 6, 1, 40, 7] = 0  # unit 7 has nothing of them, the others' heads without one are as ever
    check(run(cuda_device, q, t1, ring, pos), q, t1, ring, [0, 1, 6, 7], "")
    check(got, q, t1, ring, [7], "")


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("form", FORMS)
def test_large_scores(cuda_device, form, sign):
    """Scores of two million, whose products are exact: tokens of the largest one share the output."""
    rng = np.random.default_rng(5)
    q, t1, ring, pos = make(rng, form, lambda u, i: 118 + u % 3)
    q[...] = 0.0
    q[..., 0] = sign * 2.0 ** 14
    H = ring[0].shape[2]
    for c, s in (t1, ring):
        # keys of 64 to 120 in element 0 alone, for the negative sign -64 and up; scores in steps of 2^17
        step = rng.integers(0, 8, c.shape[:3] + c.shape[4:5])
        c[:, :, :, 0] = 0
        c[:, :, :, 0, :, 0] = torch.from_numpy((64.0 + 8 * step).astype(np.float32)).to(E4M3).view(
            torch.uint8).numpy()
        s[:, :, :, 0] = 127
    got = to_f64(run(cuda_device, q, t1, ring, pos, scale=1.0))
    for u in range(3):
        b, g = u // H, u % H
        x = [q8.values(c[b:b + 1, :, g:g + 1], s[b:b + 1, :, g:g + 1])[0, 0, 0] for c, s in (t1, ring)]
        K, V = (np.concatenate([y[i] for y in x]) for i in range(2))
        best = K[:, 0] == (K[:, 0].max() if sign > 0 else K[:, 0].min())
        want, mag = (y[best].mean(axis=0) for y in (V, np.abs(V)))
        G = q.shape[2] // H
        # equal scores get equal probabilities: roundings to fp16 and of the sums, then to bf16
        assert (np.abs(got[b, 0, g * G:g * G + G] - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * mag).all()


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_append_beside_the_largest_values(cuda_device, d, fused):
    """A block set anew keeps tokens that bf16's largest value (255 * 2^120) rounded up to 2^128, and those
    of the largest powers of two that the format has."""
    W = 70
    k = torch.randn(4, 1, 1, W, d).to(torch.bfloat16)
    k[0, ..., 5, 3] = torch.finfo(torch.bfloat16).max
    k[1, ..., 33:60, :] = -torch.finfo(torch.bfloat16).max
    codes, scales = q8.quantize(to_f64(k), to_f64(k.flip(-1)), np.ones((4, W), dtype=bool))
    scales[2, ..., :2], scales[3, ..., :2] = 250, 254
    codes[2:, ..., 6, 1] = codes[2:, ..., 40, 1] = 0x7E  # 448
    pos = np.array([2 * W, W + 32, 3 * W, 5 * W + 32], dtype=np.int64)  # first slots of blocks
    row = torch.full((4, 1, 1, d), 0.25, dtype=torch.bfloat16)
    q = torch.zeros(4, 1, 2, d, dtype=torch.bfloat16)
    args = device_args(cuda_device, q, (codes[..., :0, :], scales[..., :0]), (codes, scales), pos)
    if fused:
        cmc.decode_step_q8(args[0], None, None, *args[3:], row.to(cuda_device), row.to(cuda_device))
    else:
        cmc.window_append_q8(*args[3:], row.to(cuda_device), row.to(cuda_device))
    q8.append(codes, scales, pos, to_f64(row), to_f64(row))
    assert scales[0, 0, 0, 0, 0] == scales[1, 0, 0, 1, 1] == 247
    np.testing.assert_array_equal(args[4].view(torch.uint8).cpu().numpy(), scales)
    np.testing.assert_array_equal(args[3].view(torch.uint8).cpu().numpy(), codes)
