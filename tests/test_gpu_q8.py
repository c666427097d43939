"""The two-tier cache in 8 bits on the GPU against the fp64 oracle.

Codes and powers of two are compared bit for bit.  Attention outputs are held to a bound
computed for each output (see attn_bound)."""

import numpy as np
import pytest
import torch

import oracle
import paper_2609_25537_gb300 as cmc
from oracle import q8
from _gpu_helpers import to_f64

pytestmark = pytest.mark.gpu

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def rows_bf16(rng, *shape, spread=3.0):
    """Rows whose magnitude varies from block to block by some powers of two, as bf16."""
    x = rng.standard_normal(shape) * 2.0 ** rng.uniform(-spread, spread, shape[:-1] + (1,))
    return torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16)


def bytes_of(t):
    return t.view(torch.uint8).cpu().numpy()


def to_dev(codes, scales, dev):
    return (torch.from_numpy(codes).to(dev).view(E4M3), torch.from_numpy(scales).to(dev).view(E8M0))


def used(scales, T):
    return scales[..., :(T + 31) // 32]


def cache(rng, B, L, H, T, d, live=None):
    """Random rows quantised by the oracle; where no row lives the codes are NaN and the powers of
    two of blocks without a token NaN, as unwritten memory may be."""
    k, v = (to_f64(rows_bf16(rng, B, L, H, T, d)) for _ in range(2))
    live = np.ones((B, T), dtype=bool) if live is None else live
    codes, scales = q8.quantize(k, v, live)
    codes[~np.broadcast_to(live[:, None, None, None, :], codes.shape[:-1])] = 0x7F
    scales[..., (T + 31) // 32:] = 0xFF
    for b in range(B):
        for j in range((T + 31) // 32):
            if not live[b, 32 * j:32 * j + 32].any():
                scales[b, ..., j] = 0xFF
    return codes, scales


# ---- writing and reading back ----

SHAPES = [  # B, L, Hkv, N, d
    (1, 1, 1, 1, 64), (2, 1, 2, 31, 128), (1, 3, 2, 32, 64), (3, 2, 1, 33, 128), (2, 1, 1, 128, 64),
    (1, 2, 3, 129, 128), (2, 1, 2, 300, 128)]


@pytest.mark.parametrize("B,L,H,N,d", SHAPES)
def test_quantize_whole(cuda_device, B, L, H, N, d):
    rng = np.random.default_rng(N)
    k, v = (rows_bf16(rng, B, L, H, N, d) for _ in range(2))
    kv, scales = cmc.quantize_cache(k.to(cuda_device), v.to(cuda_device))
    codes, want = q8.quantize(to_f64(k), to_f64(v), np.ones((B, N), dtype=bool))
    np.testing.assert_array_equal(bytes_of(scales), want)  # the padding, zeroed, among it
    np.testing.assert_array_equal(bytes_of(kv), codes)


@pytest.mark.parametrize("B,L,H,N,d,k", [(2, 2, 2, 50, 128, 1), (1, 1, 2, 300, 64, 33), (3, 1, 1, 7, 128, 40),
                                         (2, 1, 2, 129, 64, 128)])
def test_quantize_rows_by_index_with_counts(cuda_device, B, L, H, N, d, k):
    rng = np.random.default_rng(k)
    bank_k, bank_v = (rows_bf16(rng, B, L, H, N, d) for _ in range(2))
    idx = rng.integers(0, N, (B, k)).astype(np.int32)  # any order, the same row more than once
    count = np.array([k // 2, -3, 10 ** 12][:B])
    kv, scales = cmc.quantize_cache(bank_k.to(cuda_device), bank_v.to(cuda_device),
                                    torch.from_numpy(idx).to(cuda_device),
                                    count=torch.from_numpy(count).to(cuda_device))
    rows = [np.stack([to_f64(x)[b][:, :, idx[b]] for b in range(B)]) for x in (bank_k, bank_v)]
    codes, want = q8.quantize(*rows, np.arange(k)[None] < count[:, None])
    np.testing.assert_array_equal(bytes_of(scales), want)
    np.testing.assert_array_equal(bytes_of(kv), codes)


def test_quantize_special_values(cuda_device):
    """Zeros, infinities, NaN, bf16's largest, smallest normal and subnormal values, and magnitudes on both
    sides of 1.75 times a power of two, each with a block of its own or with others."""
    x = torch.zeros(1, 1, 1, 320, 64)
    top = torch.finfo(torch.bfloat16).max
    x[..., 32, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), 3.0])
    x[..., 64, 5], x[..., 65, 5] = top, -top
    x[..., 96, 1], x[..., 97, 1] = 2.0 ** -126, -(2.0 ** -133)
    x[..., 128, 2], x[..., 160, 2], x[..., 192, 2] = 1.75, 1.7578125, 448.0
    x[..., 224, 0], x[..., 225, 0] = 1.0, 2.0 ** -17  # rounds to the smallest code, or to 0
    x[..., 256, :] = float("nan")
    x[..., 288, :] = -0.0
    x = x.to(torch.bfloat16)
    v = x.flip(3).contiguous()
    kv, scales = cmc.quantize_cache(x.to(cuda_device), v.to(cuda_device))
    codes, want = q8.quantize(to_f64(x), to_f64(v), np.ones((1, 320), dtype=bool))
    np.testing.assert_array_equal(bytes_of(scales), want)
    np.testing.assert_array_equal(bytes_of(kv), codes)


def test_quantize_bad_index(cuda_device):
    rng = np.random.default_rng(5)
    bank = rows_bf16(rng, 2, 1, 2, 40, 128)
    idx = np.arange(40, dtype=np.int32)[None].repeat(2, 0)
    idx[0, 3], idx[1, 7], idx[1, 39] = -1, 40, 2 ** 31 - 1
    ws = cmc.DecodeWorkspace(cmc.CmcDims(2, 1, 2, 2, 128, 40, 40, 1), cuda_device)
    count = torch.tensor([40, 39], device=cuda_device)
    kv, scales = cmc.quantize_cache(bank.to(cuda_device), bank.to(cuda_device),
                                    torch.from_numpy(idx).to(cuda_device), count=count, workspace=ws)
    assert ws.status() == cmc.DEVFLAG_BAD_INDEX
    live = np.ones((2, 40), dtype=bool)
    live[0, 3] = live[1, 7] = live[1, 39] = False
    x = np.stack([to_f64(bank)[b][:, :, np.clip(idx[b], 0, 39)] for b in range(2)])
    codes, want = q8.quantize(x, x, live)
    np.testing.assert_array_equal(bytes_of(scales), want)
    np.testing.assert_array_equal(bytes_of(kv), codes)
    # a bad index of a row that holds no token is not looked at
    cmc.quantize_cache(bank.to(cuda_device), bank.to(cuda_device), torch.from_numpy(idx).to(cuda_device),
                       count=torch.tensor([3, 7], device=cuda_device), workspace=ws)
    assert ws.status() == 0


def test_quantize_no_rows(cuda_device):
    bank = torch.zeros(2, 1, 1, 5, 64, dtype=torch.bfloat16, device=cuda_device)
    kv, scales = cmc.quantize_cache(bank, bank, torch.empty(2, 0, dtype=torch.int32, device=cuda_device))
    assert kv.shape == (2, 1, 1, 2, 0, 64) and scales.shape == (2, 1, 1, 2, 0)
    k, v = cmc.dequantize_cache(kv, scales) if kv.shape[4] else (kv, kv)
    assert k.numel() == v.numel() == 0


@pytest.mark.parametrize("B,L,H,N,d", SHAPES)
@pytest.mark.parametrize("by_index", [False, True])
def test_dequantize(cuda_device, B, L, H, N, d, by_index):
    rng = np.random.default_rng(N + d)
    codes = rng.integers(0, 256, (B, L, H, 2, N, d), dtype=np.uint8)  # every code, NaN among them
    scales = rng.integers(20, 240, (B, L, H, 2, q8.scale_bytes(N)), dtype=np.uint8)
    kv, s = to_dev(codes, scales, cuda_device)
    x = q8.values(codes, scales)
    idx = None
    if by_index:
        idx = rng.integers(0, N, (B, 2 * N + 1)).astype(np.int32)
        x = np.stack([x[b][..., idx[b], :] for b in range(B)])
        idx = torch.from_numpy(idx).to(cuda_device)
    k, v = cmc.dequantize_cache(kv, s, idx)
    np.testing.assert_array_equal(to_f64(k), x[:, :, :, 0])  # exact: four significant bits
    np.testing.assert_array_equal(to_f64(v), x[:, :, :, 1])


def test_dequantize_extreme_powers_and_bad_index(cuda_device):
    codes = np.full((1, 1, 1, 2, 96, 64), 0x38, dtype=np.uint8)  # 1.0
    codes[..., 0, 0] = 0x01                                    # 2^-9
    scales = np.zeros((1, 1, 1, 2, 4), dtype=np.uint8)
    scales[..., 1], scales[..., 2] = 254, 255
    kv, s = to_dev(codes, scales, cuda_device)
    k, v = cmc.dequantize_cache(kv, s)
    got = to_f64(k)[0, 0, 0]
    assert got[0, 0] == 0.0 and (got[1:32] == 2.0 ** -127).all()  # 2^-136 is below bf16's smallest
    assert (got[32:64] == 2.0 ** 127).all() and np.isnan(got[64:]).all()
    ws = cmc.DecodeWorkspace(cmc.CmcDims(1, 1, 1, 1, 64, 96, 3, 1), cuda_device)
    idx = torch.tensor([[1, 96, -5]], dtype=torch.int32, device=cuda_device)
    k, v = cmc.dequantize_cache(kv, s, idx, workspace=ws)
    assert ws.status() == cmc.DEVFLAG_BAD_INDEX
    assert (to_f64(v)[0, 0, 0, 1:] == 0).all() and (to_f64(v)[0, 0, 0, 0] == 2.0 ** -127).all()


def test_quantise_then_read_back_is_within_half_a_step(cuda_device):
    x = torch.rand(2, 2, 2, 200, 128, device=cuda_device).add(0.01).to(torch.bfloat16)
    k, v = cmc.dequantize_cache(*cmc.quantize_cache(x, x))
    assert torch.equal(k, v)
    # amax < 1.01 and values above 0.01 > 2^-15 amax: half a step of e4m3
    assert ((k.double() - x.double()).abs() / x.double()).max().item() <= 2.0 ** -4


def test_quantize_many_blocks(cuda_device):
    """More blocks than the grid has warps, whole and by index: sampled units against the oracle."""
    rng = np.random.default_rng(21)
    B, L, H, N, d = 6, 16, 8, 130, 128
    k, v = (torch.randn(B, L, H, N, d, device=cuda_device).to(torch.bfloat16) for _ in range(2))
    count = np.array([0, 1, 64, 129, 130, 500])
    idx = np.stack([rng.permutation(N) for _ in range(B)]).astype(np.int32)
    for index in (None, idx):
        kv, scales = cmc.quantize_cache(k, v, None if index is None else torch.from_numpy(index).to(cuda_device),
                                        count=torch.from_numpy(count).to(cuda_device))
        for _ in range(12):
            b, l, h = rng.integers(B), rng.integers(L), rng.integers(H)
            rows = np.arange(N) if index is None else index[b]
            x = [to_f64(t[b, l, h])[rows][None, None, None] for t in (k, v)]
            codes, want = q8.quantize(*x, (np.arange(N) < count[b])[None])
            np.testing.assert_array_equal(bytes_of(scales[b, l, h]), want[0, 0, 0])
            np.testing.assert_array_equal(bytes_of(kv[b, l, h]), codes[0, 0, 0])


def test_far_offsets(cuda_device):
    """A ring of more than 2^32 bytes: its last slots are appended to, attended over and read back."""
    W, d = (1 << 24) - 5, 128
    kv = torch.zeros(1, 1, 1, 2, W, d, dtype=torch.uint8, device=cuda_device).view(E4M3)
    scales = torch.full((1, 1, 1, 2, q8.scale_bytes(W)), 127, dtype=torch.uint8, device=cuda_device).view(E8M0)
    pos = torch.tensor([W - 1], device=cuda_device)
    q = torch.zeros(1, 1, 1, d, dtype=torch.bfloat16, device=cuda_device)
    q[..., 0] = 64.0
    key, value = torch.zeros(2, 1, 1, 1, d, dtype=torch.bfloat16, device=cuda_device)
    key[..., 0], value[..., :] = 30.0, 3.0
    got = cmc.decode_step_q8(q, None, None, kv, scales, pos, key, value)  # score 64 * 30 / sqrt(128) = 170
    assert (got == 3.0).all() and pos.item() == W
    key[..., 0], value[..., :] = 60.0, 5.0
    pos.fill_(2 * W - 2)
    cmc.window_append_q8(kv, scales, pos, key, value)
    got = cmc.two_tier_decode_attn_q8(q, None, None, kv, scales, pos)
    assert (got == 5.0).all()
    rows = torch.tensor([[W - 1, W - 2, W - 3, 0]], dtype=torch.int32, device=cuda_device)
    k, v = cmc.dequantize_cache(kv, scales, rows)
    assert k[0, 0, 0, :, 0].tolist() == [30.0, 60.0, 0.0, 0.0]
    assert v[0, 0, 0, :, d - 1].tolist() == [3.0, 5.0, 0.0, 0.0]


# ---- append ----

@pytest.mark.parametrize("B,L,H,W,d", [(1, 1, 1, 1, 64), (3, 1, 2, 7, 128), (2, 2, 2, 32, 64),
                                       (2, 1, 3, 33, 128), (4, 1, 1, 130, 128), (1, 40, 8, 64, 128)])
def test_append(cuda_device, B, L, H, W, d):
    """More tokens than the ring holds, from sequences at different places in it."""
    rng = np.random.default_rng(W)
    pos = np.array([0, W // 2, 3 * W + 1, 2 ** 33 + 5][:B], dtype=np.int64)
    codes, scales = cache(rng, B, L, H, W, d, np.arange(W)[None] < pos[:, None])
    kv, s = to_dev(codes, scales, cuda_device)
    p = torch.from_numpy(pos.copy()).to(cuda_device)
    steps = min(2 * W + 3, 70) if B * L * H < 100 else 4
    for t in range(steps):
        k_new, v_new = (rows_bf16(rng, B, L, H, d, spread=6.0) for _ in range(2))
        cmc.window_append_q8(kv, s, p, k_new.to(cuda_device), v_new.to(cuda_device))
        q8.append(codes, scales, pos, to_f64(k_new), to_f64(v_new))
        np.testing.assert_array_equal(bytes_of(s), scales, err_msg=f"step {t}")
        np.testing.assert_array_equal(bytes_of(kv), codes, err_msg=f"step {t}")
    np.testing.assert_array_equal(p.cpu().numpy(), pos)


def test_append_special_rows(cuda_device):
    """Zero, infinite and NaN rows, rows far above and far below the block, a negative position."""
    rng = np.random.default_rng(9)
    W, d = 40, 64
    codes, scales = cache(rng, 2, 1, 1, W, d)
    pos = np.array([W + 3, -1], dtype=np.int64)
    kv, s = to_dev(codes, scales, cuda_device)
    p = torch.from_numpy(pos.copy()).to(cuda_device)
    rows = [torch.zeros(d), torch.full((d,), float("nan")), torch.full((d,), -float("inf")),
            torch.full((d,), 3e38), torch.full((d,), 2.0 ** -130), torch.randn(d),
            torch.cat([torch.tensor([float("inf"), float("nan")]), torch.randn(d - 2) * 1e30])]
    for t in range(45):
        row = rows[t % len(rows)].to(torch.bfloat16)[None, None, None].repeat(2, 1, 1, 1)
        cmc.window_append_q8(kv, s, p, row.to(cuda_device), row.to(cuda_device))
        q8.append(codes, scales, pos, to_f64(row), to_f64(row))
        np.testing.assert_array_equal(bytes_of(s), scales, err_msg=f"step {t}")
        np.testing.assert_array_equal(bytes_of(kv), codes, err_msg=f"step {t}")
    assert p.tolist() == pos.tolist() == [W + 48, -1]


# ---- attention ----

def attn_bound(q, tier1, ring, pos, scale, out, mag, q_error=0.0):
    """How far an output may be off, from the roundings on the way to it.

    * The output is rounded to bf16: 2^-8 of it.
    * A probability is rounded to fp16: 2^-11 of it, and 2^-29 of the largest for those far below; the
      sum that divides is not rounded.  (The largest is that of the keys seen so far: at
      most 1 of the sum.)
    * A score is off by what fp16 leaves of the query (2^-30 of its largest element, times the key's
      sum of magnitudes; `q_error` of every product where the query was computed), by the
      roundings of d products' fp32 sum and of a few more products (2^-23 each), and 2^x by 2^-21.
      An error e of all scores changes the quotient by at most 2 e of the sum of p |v|, to first
      order: twice that is allowed where it is large."""
    B, L, Hq, d = q.shape
    bound = np.zeros_like(out)
    for b in range(B):
        n = max(0, min(int(pos[b]), ring.shape[4]))
        for l in range(L):
            for h in range(Hq):
                g = h // (Hq // ring.shape[2])
                K = np.concatenate([tier1[b, l, g, 0], ring[b, l, g, 0, :n]])
                V = np.concatenate([tier1[b, l, g, 1], ring[b, l, g, 1, :n]])
                if not len(K):
                    continue
                a = np.abs(q[b, l, h])
                e = scale * (2.0 ** -30 * a.max() * np.abs(K).sum(axis=1)
                             + ((d + 8) * 2.0 ** -23 + q_error) * (np.abs(K) @ a)).max()
                bound[b, l, h] = (2.0 ** -8 * np.abs(out[b, l, h])
                                  + (2.0 ** -11 + 2 * (e + 2.0 ** -21) * (1 + e)) * mag[b, l, h]
                                  + 2.0 ** -29 * np.abs(V).sum(axis=0))
    return bound


def check_attention(got, q, t1, ring, pos, scale=None, q_error=0.0, what=""):
    """got [B, L, Hq, d] (device) against the oracle over caches (codes, scales) of the host."""
    B, L, Hq, d = q.shape
    scale = 1 / np.sqrt(d) if scale is None else scale
    H = ring[0].shape[2]
    tier1 = q8.values(*t1) if t1 is not None else np.zeros((B, L, H, 2, 0, d))
    x = q8.values(*ring)
    out, mag = q8.attention(q, tier1, x, pos, scale)
    err = np.abs(to_f64(got) - out)
    bound = attn_bound(q, tier1, x, pos, scale, out, mag, q_error)
    assert np.isfinite(out).all() and (err <= bound).all(), (
        what, float((err / np.maximum(bound, 1e-300)).max()))
    if np.linalg.norm(out) > 0:
        # the output's rounding, half a step at most, is what counts; a dropped key among 300 is 4 %
        rel = np.linalg.norm(err) / np.linalg.norm(out)
        assert rel <= 2.0 ** -8 + 8 * q_error, (what, rel)


ATTN = [  # B, L, Hq, Hkv, d, k, W, pos
    (1, 1, 1, 1, 64, 0, 1, [1]),
    (1, 1, 8, 2, 64, 32, 128, [128]),
    (2, 1, 8, 1, 128, 1, 7, [3, 100]),
    (1, 2, 4, 2, 128, 31, 33, [20]),
    (3, 1, 4, 4, 64, 33, 130, [0, 129, 131]),
    (2, 2, 16, 4, 128, 127, 64, [2 ** 33 + 5, 64]),
    (2, 1, 16, 2, 128, 128, 257, [200, 1]),
    (1, 1, 16, 2, 64, 129, 31, [2]),
    (2, 1, 8, 8, 128, 300, 300, [299, 301]),
    (1, 1, 32, 8, 128, 700, 1100, [1100]),
    (40, 4, 8, 2, 64, 5, 40, list(range(1, 41))),
    (60, 2, 8, 4, 128, 40, 150, [150 + i for i in range(60)]),
]


ATTN += [  # more units than resident CTAs: whole ones, cut ones, runs over many sequences
    (200, 1, 8, 4, 128, 30, 130, [(7 * i) % 150 for i in range(200)]),
    (20, 16, 8, 4, 64, 0, 40, [3 * i - 5 for i in range(20)]),
    (700, 1, 1, 1, 64, 0, 33, [(i * 37) % 60 - 3 for i in range(700)]),
    (45, 1, 64, 8, 128, 70, 500, [(i * 131) % 700 for i in range(45)]),
    (500, 1, 8, 1, 64, 3, 300, [(i * 17) % 400 for i in range(500)]),
    # a warp takes several units, of sequences with nothing, a little and a full ring
    (700, 1, 4, 4, 128, 0, 40, [(i * 29) % 75 - 3 for i in range(700)]),
    (2600, 1, 2, 1, 64, 0, 33, [(i * 11) % 50 - 2 for i in range(2600)]),
    (7, 64, 8, 8, 64, 33, 70, [0, 1, 31, 64, 69, 70, 135]),
    (170, 1, 64, 8, 128, 5, 20, [i % 25 for i in range(170)]),
    (24, 8, 32, 8, 128, 30, 130, [0, -4, 260, 130, 129] + [(i * 37) % 150 for i in range(19)]),
    # several waves of whole units, the longest sequences first
    (64, 1, 8, 8, 128, 37, 1000, [(i * 131) % 1900 - 3 for i in range(64)]),
    (128, 6, 2, 1, 64, 0, 1060, [0, 5, 5, 1060, 1061, 3400] + [(i * 97) % 1800 for i in range(122)]),
    # clusters, three CTAs an SM: of two and of eight
    (44, 2, 8, 2, 64, 9, 1300, [(i * 131) % 1700 for i in range(44)]),
    (10, 1, 16, 4, 128, 1001, 2900, [1, 2, 40, 700, 1500, 2000, 2899, 2900, 2901, 9000]),
]


def problem(rng, B, L, Hq, H, d, k, W, pos):
    pos = np.array(pos, dtype=np.int64)
    ring = cache(rng, B, L, H, W, d, np.arange(W)[None] < pos[:, None])
    t1 = cache(rng, B, L, H, k, d) if k else None
    q = rows_bf16(rng, B, L, Hq, d, spread=1.0)
    return q, t1, ring, pos


def device_args(q, t1, ring, pos, dev):
    t = (None, None) if t1 is None else to_dev(*t1, dev)
    return [q.to(dev), *t, *to_dev(*ring, dev), torch.from_numpy(pos.copy()).to(dev)]


@pytest.mark.parametrize("B,L,Hq,H,d,k,W,pos", ATTN)
def test_attention(cuda_device, B, L, Hq, H, d, k, W, pos):
    rng = np.random.default_rng(W + k)
    q, t1, ring, pos = problem(rng, B, L, Hq, H, d, k, W, pos)
    args = device_args(q, t1, ring, pos, cuda_device)
    got = cmc.two_tier_decode_attn_q8(*args)
    check_attention(got, to_f64(q), t1, ring, pos)
    assert torch.equal(cmc.two_tier_decode_attn_q8(*args), got)  # and the same bits again
    # nothing but the output is written
    for a, b in zip(args, device_args(q, t1, ring, pos, cuda_device)):
        assert a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_attention_empty_and_negative(cuda_device):
    rng = np.random.default_rng(3)
    q, t1, ring, pos = problem(rng, 3, 1, 4, 2, 64, 0, 40, [0, -7, 4])
    args = device_args(q, t1, ring, pos, cuda_device)
    ws = cmc.DecodeWorkspace(cmc.CmcDims(3, 1, 4, 2, 64, 1, 0, 40), cuda_device, q8=True)
    got = cmc.two_tier_decode_attn_q8(*args, workspace=ws)
    assert (got[:2] == 0).all()
    assert ws.status() == cmc.DEVFLAG_BAD_POS
    check_attention(got, to_f64(q), t1, ring, pos)


def test_attention_scale_and_sharp_scores(cuda_device):
    """A given scale; scores of hundreds, where one key takes all."""
    rng = np.random.default_rng(4)
    q, t1, ring, pos = problem(rng, 2, 1, 8, 2, 128, 60, 200, [150, 500])
    q = (q.float() * 8).to(torch.bfloat16)
    for scale in (1.0, 0.01):
        got = cmc.two_tier_decode_attn_q8(*device_args(q, t1, ring, pos, cuda_device), scale=scale)
        check_attention(got, to_f64(q), t1, ring, pos, scale, what=str(scale))


def test_attention_blocks_of_very_different_size(cuda_device):
    """Blocks whose values differ by 2^60 and more, in either order, and tiny and huge queries."""
    rng = np.random.default_rng(6)
    for order in (1, -1):
        q, t1, ring, pos = problem(rng, 1, 1, 4, 1, 128, 256, 256, [256])
        for codes, scales in (t1, ring):
            step = np.arange(8)[::order] * 8
            scales[..., 1, :8] = (scales[..., 1, :8].astype(int) - 30 + step).astype(np.uint8)
        q[:, :, 0] = (q[:, :, 0].float() * 1e-20).to(torch.bfloat16)
        q[:, :, 1] = (q[:, :, 1].float() * 1e4).to(torch.bfloat16)
        q[:, :, 2] = 0.0
        got = cmc.two_tier_decode_attn_q8(*device_args(q, t1, ring, pos, cuda_device))
        check_attention(got, to_f64(q), t1, ring, pos, what=str(order))


def test_attention_nan_reaches_the_output_only_from_live_tokens(cuda_device):
    rng = np.random.default_rng(7)
    q, t1, ring, pos = problem(rng, 2, 1, 4, 2, 128, 40, 100, [70, 100])
    t1[0][0, 0, 1, 1, 5, 3] = 0x7F  # a NaN among Tier-1's values of sequence 0, head 1
    ring[0][1, 0, 0, 0, 99, 0] = 0xFF  # and among the ring's keys of sequence 1, head 0
    got = to_f64(cmc.two_tier_decode_attn_q8(*device_args(q, t1, ring, pos, cuda_device)))
    assert np.isnan(got[0, 0, 2:, 3]).all() and np.isnan(got[1, 0, :2]).all()
    bad = np.isnan(got)
    assert bad.sum() == 2 + 2 * 128


@pytest.mark.parametrize("graph", [False, True])
def test_attention_on_other_streams_and_captured(cuda_device, graph):
    """Two calls at once on two streams, and two captured ones replayed on two streams, each with
    the workspace that the call chooses."""
    rng = np.random.default_rng(8)
    probs = [problem(rng, 60, 1, 8, 4, 128, 40, 150, [150 + i + s for i in range(60)]) for s in range(2)]
    args = [device_args(*x, cuda_device) for x in probs]
    want = [cmc.two_tier_decode_attn_q8(*a).clone() for a in args]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(w) for w in want]
    torch.cuda.synchronize()
    runs = []
    for a, o, s in zip(args, outs, streams):
        def call(a=a, o=o):
            cmc.two_tier_decode_attn_q8(*a, out=o)
        if graph:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=streams[0]):
                call()
            call = g.replay
        runs.append((call, s))
    for _ in range(20):
        for call, s in runs:
            with torch.cuda.stream(s):
                call()
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)


# ---- the fused step ----

STEP = ATTN + [
    (5, 1, 8, 2, 128, 10, 33, [0, 31, 32, 33, 2 ** 33 + 5]),  # blocks' first slots, and a wrap
    (20, 10, 4, 2, 64, 0, 100, [7 * i for i in range(20)]),
]


@pytest.mark.parametrize("B,L,Hq,H,d,k,W,pos", STEP)
def test_step_is_append_then_attention(cuda_device, B, L, Hq, H, d, k, W, pos):
    """Three steps: ring, powers of two and pos bit for bit those of the append, the outputs those of
    attention over them."""
    rng = np.random.default_rng(W + k + 1)
    q, t1, ring, pos = problem(rng, B, L, Hq, H, d, k, W, pos)
    args = device_args(q, t1, ring, pos, cuda_device)
    codes, scales = (x.copy() for x in ring)
    for t in range(3):
        q, k_new, v_new = (rows_bf16(rng, B, L, h, d, spread=4.0 if h == H else 1.0) for h in (Hq, H, H))
        args[0] = q.to(cuda_device)
        got = cmc.decode_step_q8(*args, k_new.to(cuda_device), v_new.to(cuda_device))
        q8.append(codes, scales, pos, to_f64(k_new), to_f64(v_new))
        np.testing.assert_array_equal(bytes_of(args[4]), scales, err_msg=f"step {t}")
        np.testing.assert_array_equal(bytes_of(args[3]), codes, err_msg=f"step {t}")
        np.testing.assert_array_equal(args[5].cpu().numpy(), pos)
        check_attention(got, to_f64(q), t1, (codes, scales), pos, what=f"step {t}")


def test_step_negative_position(cuda_device):
    rng = np.random.default_rng(11)
    q, t1, ring, pos = problem(rng, 2, 2, 8, 2, 128, 30, 50, [-4, 20])
    args = device_args(q, t1, ring, pos, cuda_device)
    new = [rows_bf16(rng, 2, 2, 2, 128) for _ in range(2)]
    ws = cmc.DecodeWorkspace(cmc.CmcDims(2, 2, 8, 2, 128, 30, 30, 50), cuda_device, q8=True)
    got = cmc.decode_step_q8(*args, *(x.to(cuda_device) for x in new), workspace=ws)
    assert ws.status() == cmc.DEVFLAG_BAD_POS and (got[0] == 0).all()
    codes, scales = (x.copy() for x in ring)
    q8.append(codes, scales, pos, *(to_f64(x) for x in new))
    np.testing.assert_array_equal(bytes_of(args[3]), codes)
    np.testing.assert_array_equal(bytes_of(args[4]), scales)
    assert args[5].tolist() == pos.tolist() == [-4, 21]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("theta,offset,start", [(1e4, 0, 0), (5e5, 30, 130), (5e5, 2 ** 31, 2 ** 20 + 7)])
def test_step_with_rotary_embedding(cuda_device, d, theta, offset, start):
    rng = np.random.default_rng(d)
    B, L, Hq, H, k, W = 3, 2, 8, 2, 30, 130
    q, t1, ring, pos = problem(rng, B, L, Hq, H, d, k, W, [start, start + 40, start + 200])
    args = device_args(q, t1, ring, pos, cuda_device)
    for t in range(2):
        q, k_new, v_new = (rows_bf16(rng, B, L, h, d) for h in (Hq, H, H))
        args[0] = q.to(cuda_device)
        before = (bytes_of(args[3]).copy(), bytes_of(args[4]).copy())
        got = cmc.decode_step_q8(*args, k_new.to(cuda_device), v_new.to(cuda_device), rope_theta=theta,
                                 rope_offset=offset)
        rq, rk = np.zeros(q.shape), np.zeros(k_new.shape)
        for b in range(B):
            rq[b] = oracle.rope_rotate(to_f64(q)[b], float(offset + pos[b]), theta)
            rk[b] = oracle.rope_rotate(to_f64(k_new)[b], float(offset + pos[b]), theta)
        codes, scales = before
        q8.append(codes, scales, pos, rk, to_f64(v_new))
        got_codes = bytes_of(args[3])
        # The rotated key is within 2^-21 of its row's largest element (angles to 1e-7, fp32), so its
        # codes may be one step off where the exact value is that near a rounding border: rarely.
        same = got_codes == codes
        np.testing.assert_array_equal(got_codes[:, :, :, 1], codes[:, :, :, 1])
        assert (~same).sum() <= 4
        assert np.abs(got_codes.astype(int) - codes.astype(int)).max() <= 1
        np.testing.assert_array_equal(bytes_of(args[4]), scales)
        np.testing.assert_array_equal(args[5].cpu().numpy(), pos)
        # a rotated query element is off by 2^-21 of the head's largest (as the key) and rounded to eleven
        # significant bits
        check_attention(got, rq, t1, (got_codes, scales), pos, q_error=2.0 ** -11 + 2.0 ** -20,
                        what=f"step {t}")


@pytest.mark.parametrize("shape", [(1, 1, 8, 2, 64, 32, 128), (2, 1, 16, 2, 128, 400, 900),
                                   (60, 2, 8, 4, 128, 40, 150)])
def test_step_captured_and_replayed(cuda_device, shape):
    """A captured step, replayed, does what that many direct calls do, with the workspace that the
    call chooses; eager calls of the same shape on the same stream in between do not disturb it."""
    rng = np.random.default_rng(12)
    B = shape[0]
    q, t1, ring, pos = problem(rng, *shape, [50 + b for b in range(B)])
    new = [rows_bf16(rng, B, shape[1], shape[3], shape[4]).to(cuda_device) for _ in range(2)]
    one, two = (device_args(q, t1, ring, pos, cuda_device) for _ in range(2))
    out = torch.empty_like(one[0])
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        cmc.decode_step_q8(*one, *new, out=out, rope_theta=1e4)
    with torch.cuda.stream(stream):
        for _ in range(5):
            graph.replay()
            want = cmc.decode_step_q8(*two, *new, rope_theta=1e4)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    for a, b in zip(one[3:], two[3:]):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert one[5].tolist() == [55 + b for b in range(B)]


def test_steps_of_two_requests_on_two_streams(cuda_device):
    rng = np.random.default_rng(13)
    probs = [problem(rng, 4, 3, 8, 2, 128, 100, 300, [290 + s] * 4) for s in range(2)]
    new = [[rows_bf16(rng, 4, 3, 2, 128).to(cuda_device) for _ in range(2)] for _ in range(2)]
    serial = [device_args(*x, cuda_device) for x in probs]
    want = [[cmc.decode_step_q8(*a, *n).clone() for _ in range(15)] for a, n in zip(serial, new)]
    par = [device_args(*x, cuda_device) for x in probs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for t in range(15):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(cmc.decode_step_q8(*par[i], *new[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(got[i], want[i]))
        for a, b in zip(par[i][3:], serial[i][3:]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_whole_path(cuda_device):
    """A request as it is served: select, quantise the selected rows and the prefilled window, decode; and
    the same with the bank kept in 8 bits, whose rows are read back for the bf16 path."""
    rng = np.random.default_rng(14)
    B, L, Hq, H, d, N, k, W = 2, 2, 8, 2, 64, 200, 40, 70
    bank = [rows_bf16(rng, B, L, H, N, d, spread=0.5).to(cuda_device) for _ in range(2)]
    window = [rows_bf16(rng, B, L, H, W, d, spread=0.5).to(cuda_device) for _ in range(2)]
    pos = torch.tensor([30, W + 5], device=cuda_device)
    cmes, question = torch.randn(B, N, 32, device=cuda_device), torch.randn(B, 32, device=cuda_device)
    idx = cmc.score_select(question, cmes, k)
    t1 = cmc.quantize_cache(*bank, idx)
    ring = cmc.quantize_cache(*window, count=pos)
    bank8 = cmc.quantize_cache(*bank)
    d1 = cmc.dequantize_cache(*bank8, idx)
    ring16 = [x.clone() for x in cmc.dequantize_cache(*ring)]
    pos16 = pos.clone()
    for t in range(50):
        q, k_new, v_new = (rows_bf16(rng, B, L, h, d, spread=0.5).to(cuda_device) for h in (Hq, H, H))
        got = cmc.decode_step_q8(q, *t1, *ring, pos, k_new, v_new)
        n = [int(x) for x in pos]
        host = [(bytes_of(c), bytes_of(s)) for c, s in (t1, ring)]
        check_attention(got, to_f64(q), host[0], host[1], np.array(n), what=f"step {t}")
        near = cmc.decode_step(q, *d1, None, *ring16, pos16, k_new, v_new)
        # the two caches differ by roundings of single values to e4m3, 2^-4 of a value at most
        far = (near.double() - got.double()).norm() / near.double().norm()
        assert far <= 2.0 ** -3, (t, float(far))
    assert pos.tolist() == pos16.tolist() == [80, W + 55]


@pytest.mark.parametrize("shape", [(1, 1, 8, 2, 64, 32, 128), (60, 2, 8, 4, 128, 40, 150),
                                   (400, 1, 4, 4, 128, 3, 40)])
def test_step_timeout_is_reported(cuda_device, shape):
    """With every stage's wait made to run out, the launch ends, the workspace's status word says so, and
    the context stays usable."""
    rng = np.random.default_rng(15)
    B = shape[0]
    q, t1, ring, pos = problem(rng, *shape, [5] * B)
    new = [rows_bf16(rng, B, shape[1], shape[3], shape[4]).to(cuda_device) for _ in range(2)]
    args = device_args(q, t1, ring, pos, cuda_device)
    dims = cmc.CmcDims(*shape[:5], shape[5], shape[5], shape[6])
    ws = cmc.DecodeWorkspace(dims, cuda_device, q8=True)
    cmc.lib().cmc_test_stall_attention_waits(1)
    try:
        cmc.decode_step_q8(*args, *new, workspace=ws)
    finally:
        cmc.lib().cmc_test_stall_attention_waits(0)
    assert ws.status() & cmc.DEVFLAG_TIMEOUT
    ws.buf.zero_()
    args = device_args(q, t1, ring, pos, cuda_device)
    got = cmc.decode_step_q8(*args, *new, workspace=ws)
    assert ws.status() == 0
    codes, scales = (x.copy() for x in ring)
    q8.append(codes, scales, pos, *(to_f64(x) for x in new))
    check_attention(got, to_f64(q), t1, (codes, scales), pos)


def test_plan(cuda_device):
    """A cluster per unit, one CTA per unit, one warp per unit, and units that just miss one wave."""
    def plan(B, L, H, k, W):
        return cmc.decode_attn_q8_plan(cmc.CmcDims(B, L, 4 * H, H, 128, max(k, 1), k, W))
    assert plan(1, 1, 2, 32, 128) == 4        # five blocks a unit: a cluster of two
    assert plan(1, 1, 1, 0, 32) == 1          # one block
    assert plan(1, 1, 2, 2048, 2048) == 16    # the largest cluster
    assert plan(1, 32, 8, 128, 512) == 256
    assert plan(64, 1, 8, 30, 64) == 128      # 512 short units: a warp each, four a CTA
    assert plan(64, 1, 8, 256, 2048) == 512
    assert plan(22, 1, 8, 0, 61 * 32) == 352  # two CTAs a unit, three CTAs an SM
    assert plan(5, 1, 8, 2048, 2048) == 320   # eight, three CTAs an SM
    assert plan(7, 1, 8, 2048, 2048) == 224   # four, where eight would take two waves
    assert plan(13, 3, 8, 256, 2048) == 312   # one CTA a unit, three an SM
    assert plan(128, 1, 8, 256, 2048) == 1024 # several waves of whole units, by length
    assert plan(129, 1, 8, 256, 2048) == 258  # a warp a unit where there are too many to order
    assert plan(8, 32, 8, 30, 130) == 304     # short units, one after another


def test_empty_tier1_and_other_workspaces(cuda_device):
    """A Tier-1 of no rows is none; a workspace of the bf16 calls will do, and serves both in turn."""
    rng = np.random.default_rng(22)
    q, t1, ring, pos = problem(rng, 3, 1, 8, 2, 64, 0, 70, [9, 70, 200])
    args = device_args(q, t1, ring, pos, cuda_device)
    bank = torch.zeros(3, 1, 2, 5, 64, dtype=torch.bfloat16, device=cuda_device)
    args[1:3] = cmc.quantize_cache(bank, bank, torch.empty(3, 0, dtype=torch.int32, device=cuda_device))
    ws = cmc.DecodeWorkspace(cmc.CmcDims(3, 1, 8, 2, 64, 5, 5, 70), cuda_device)
    ring16 = [x.clone() for x in cmc.dequantize_cache(*args[3:5])]
    new = [rows_bf16(rng, 3, 1, 2, 64).to(cuda_device) for _ in range(2)]
    pos16 = args[5].clone()
    for _ in range(4):
        cmc.decode_step(args[0], bank, bank, None, *ring16, pos16, *new, workspace=ws)
        got = cmc.decode_step_q8(*args, *new, workspace=ws)
    assert ws.status() == 0 and torch.equal(pos16, args[5])
    check_attention(got, to_f64(q), None, (bytes_of(args[3]), bytes_of(args[4])), args[5].cpu().numpy())


def test_calls_with_another_device_current(cuda_device, monkeypatch):
    """A call makes its tensors' device the current one: seen from a current device of another number."""
    from paper_2609_25537_gb300 import cmc as module
    rng = np.random.default_rng(23)
    q, t1, ring, pos = problem(rng, 2, 1, 8, 2, 128, 40, 70, [9, 200])
    args = device_args(q, t1, ring, pos, cuda_device)
    want = cmc.two_tier_decode_attn_q8(*args)
    asked = []
    monkeypatch.setattr(module, "_current_device", lambda: asked.append(0) or cuda_device.index + 1)
    assert torch.equal(cmc.two_tier_decode_attn_q8(*args), want)
    k, v = cmc.dequantize_cache(*args[1:3])
    again = cmc.quantize_cache(k, v)
    row = torch.zeros(2, 1, 2, 128, dtype=torch.bfloat16, device=cuda_device)
    cmc.window_append_q8(args[3], args[4], args[5], row, row)
    cmc.decode_step_q8(*args, row, row)
    assert len(asked) == 5 and args[5].tolist() == [11, 202]
    assert torch.equal(again[0].view(torch.uint8), args[1].view(torch.uint8))


# ---- refusals of the binding ----

def test_binding_refusals(cuda_device):
    dev = cuda_device
    bank = torch.zeros(2, 1, 2, 40, 64, dtype=torch.bfloat16, device=dev)
    kv, scales = cmc.quantize_cache(bank, bank)
    pos = torch.zeros(2, dtype=torch.int64, device=dev)
    q = torch.zeros(2, 1, 4, 64, dtype=torch.bfloat16, device=dev)
    row = torch.zeros(2, 1, 2, 64, dtype=torch.bfloat16, device=dev)
    attn = cmc.two_tier_decode_attn_q8
    for exc, call in [
            (TypeError, lambda: cmc.quantize_cache(bank.float(), bank)),
            (ValueError, lambda: cmc.quantize_cache(bank, bank[:, :, :, :39].contiguous())),
            (ValueError, lambda: cmc.quantize_cache(bank.transpose(3, 4), bank)),
            (TypeError, lambda: cmc.quantize_cache(bank, bank, pos[:, None])),
            (TypeError, lambda: cmc.quantize_cache(bank, bank, count=pos.int())),
            (ValueError, lambda: cmc.quantize_cache(bank, bank, out_kv=kv[:1].contiguous())),
            (TypeError, lambda: cmc.dequantize_cache(kv.view(torch.uint8), scales)),
            (ValueError, lambda: cmc.dequantize_cache(kv, scales[..., :2].contiguous())),
            (ValueError, lambda: cmc.dequantize_cache(kv[:, :, :, :1].contiguous(), scales)),
            (ValueError, lambda: cmc.window_append_q8(kv, scales, pos[:1], row, row)),
            (ValueError, lambda: cmc.window_append_q8(kv, scales, pos, row[:, :, :1].contiguous(), row)),
            (ValueError, lambda: attn(q[:1].contiguous(), None, None, kv, scales, pos)),
            (TypeError, lambda: attn(q, kv, None, kv, scales, pos)),
            (ValueError, lambda: attn(q, kv[:1].contiguous(), scales[:1].contiguous(), kv, scales, pos)),
            (ValueError, lambda: attn(q, None, None, kv, scales, pos, out=q[:1].contiguous())),
            (ValueError, lambda: cmc.decode_step_q8(q, None, None, kv, scales, pos, row[:1].contiguous(), row)),
            (ValueError, lambda: cmc.decode_step_q8(q, None, None, kv, scales, pos, row, row, rope_theta=0.0)),
            (ValueError, lambda: attn(q[:, :, :3].contiguous(), None, None, kv, scales, pos)),  # 3 over 2 heads
    ]:
        with pytest.raises(exc):
            call()
    # no tensor where one has to be, after calls of the same shapes that were right
    for fn, good in ((cmc.quantize_cache, [bank, bank]), (cmc.dequantize_cache, [kv, scales]),
                     (cmc.window_append_q8, [kv, scales, pos, row, row]),
                     (attn, [q, kv.clone(), scales.clone(), kv, scales, pos]),
                     (cmc.decode_step_q8, [q, kv.clone(), scales.clone(), kv, scales, pos, row, row])):
        fn(*good)
        for i in range(len(good)):
            for bad in (None, [1, 2], good[i].cpu()):
                with pytest.raises((TypeError, ValueError)):
                    fn(*good[:i], bad, *good[i + 1:])
    small = cmc.DecodeWorkspace(cmc.CmcDims(1, 1, 2, 2, 64, 1, 0, 1), dev, q8=True)
    small.nbytes = 511
    with pytest.raises(cmc.CmcError):
        attn(q, None, None, kv, scales, pos, workspace=small)
