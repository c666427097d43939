"""fp64 oracle of the two-tier cache held in 8 bits (test infrastructure only).

Written from the format alone: codes are bytes looked up in a table of the 256
e4m3 values, rounding is a search among them, and a block's power of two is
found by trying exponents in turn.

  codes   uint8 [B, L, Hkv, 2, T, d]      keys, then values
  scales  uint8 [B, L, Hkv, 2, 4 ceil(T / 128)], byte c for 2^(c - 127), one a
          block of 32 tokens (the bytes past ceil(T / 32) are padding)
"""

from __future__ import annotations

import numpy as np

from .cmc_oracle import softmax_attention

BLOCK = 32


def _table() -> np.ndarray:
    """The value of every e4m3 byte: sign, four exponent bits (bias 7), three
    mantissa bits; exponent 0 is subnormal, 0x7F and 0xFF are NaN."""
    out = np.empty(256)
    for byte in range(256):
        e, m = (byte >> 3) & 15, byte & 7
        x = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        if byte & 127 == 127:
            x = float("nan")
        out[byte] = -x if byte & 128 else x
    return out


E4M3 = _table()


def round_e4m3(x: np.ndarray) -> np.ndarray:
    """Bytes of the nearest e4m3 values of x (fp64), ties to the even byte; NaN for what is
    not finite; magnitudes above 448 give 448."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(x)
    values = E4M3[:127]
    hi = np.clip(np.searchsorted(values, a), 0, 126)  # first value >= a
    lo = np.maximum(hi - 1, 0)
    up, down = values[hi] - a, a - values[lo]
    byte = np.where(up < down, hi, np.where(up > down, lo, np.where(hi % 2 == 0, hi, lo)))
    byte = np.where(a >= values[126], 126, byte)
    byte = np.where(np.isfinite(x), byte, 127)
    return (byte | np.where(np.signbit(x) & np.isfinite(x), 128, 0)).astype(np.uint8)


def power(c) -> float:
    return float("nan") if int(c) == 255 else 2.0 ** (int(c) - 127)


def block_byte(amax: float) -> int:
    """The smallest byte c with amax <= 448 * 2^(c - 127)."""
    c = 0
    while amax > 448.0 * power(c):
        c += 1
    return c


def _amax(x: np.ndarray) -> float:
    a = np.abs(x)
    a = a[np.isfinite(a)]
    return float(a.max()) if a.size else 0.0


def scale_bytes(T: int) -> int:
    return 4 * ((T + 127) // 128)


def quantize(k: np.ndarray, v: np.ndarray, live: np.ndarray):
    """Cache of fp64 rows k, v [B, L, Hkv, T, d]; live [B, T] says which hold a token."""
    B, L, H, T, d = k.shape
    codes = np.zeros((B, L, H, 2, T, d), dtype=np.uint8)
    scales = np.zeros((B, L, H, 2, scale_bytes(T)), dtype=np.uint8)
    for b in range(B):
        for l in range(L):
            for h in range(H):
                for w, x in enumerate((k, v)):
                    for j in range(0, T, BLOCK):
                        rows = np.where(live[b, j:j + BLOCK, None], x[b, l, h, j:j + BLOCK], 0.0)
                        c = block_byte(_amax(rows))
                        codes[b, l, h, w, j:j + BLOCK] = round_e4m3(rows * 2.0 ** (127 - c))
                        scales[b, l, h, w, j // BLOCK] = c
    return codes, scales


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """fp64 values [B, L, Hkv, 2, T, d] of a cache."""
    s = np.array([power(c) for c in range(256)])[scales]
    return E4M3[codes] * np.repeat(s, BLOCK, axis=-1)[..., :codes.shape[4], None]


def append(codes: np.ndarray, scales: np.ndarray, pos: np.ndarray, k_new: np.ndarray,
           v_new: np.ndarray) -> None:
    """One token (fp64 rows [B, L, Hkv, d]) per sequence, in place; negative positions are skipped."""
    B, L, H, _, W, d = codes.shape
    for b in range(B):
        if pos[b] < 0:
            continue
        slot, n = int(pos[b]) % W, min(int(pos[b]), W)
        first = slot // BLOCK * BLOCK
        others = [s for s in range(first, min(first + BLOCK, W)) if s < n and s != slot]
        for l in range(L):
            for h in range(H):
                for w, x in enumerate((k_new, v_new)):
                    row, old = x[b, l, h], int(scales[b, l, h, w, slot // BLOCK])
                    block = codes[b, l, h, w]
                    c = block_byte(_amax(row))
                    if slot == first:
                        c = max(c, block_byte(_amax(E4M3[block[others]] * power(old))))
                    else:
                        c = max(c, old)
                    if c != old:
                        block[others] = round_e4m3(E4M3[block[others]] * (power(old) / power(c)))
                    block[slot] = round_e4m3(row / power(c))
                    scales[b, l, h, w, slot // BLOCK] = c
        pos[b] += 1


def attention(q: np.ndarray, tier1: np.ndarray, ring: np.ndarray, pos: np.ndarray, scale: float):
    """softmax(scale q k) v in fp64 over the rows of tier1 [B, L, Hkv, 2, k, d] (values) and the
    first min(pos, W) slots of ring [B, L, Hkv, 2, W, d].  Returns the outputs [B, L, Hq, d] and,
    for error bounds, the same sums of |v|."""
    B, L, Hq, d = q.shape
    H, W = ring.shape[2], ring.shape[4]
    out, mag = np.zeros((B, L, Hq, d)), np.zeros((B, L, Hq, d))
    for b in range(B):
        if pos[b] < 0:
            continue
        n = min(int(pos[b]), W)
        for l in range(L):
            for h in range(Hq):
                g = h // (Hq // H)
                K = np.concatenate([tier1[b, l, g, 0], ring[b, l, g, 0, :n]])
                V = np.concatenate([tier1[b, l, g, 1], ring[b, l, g, 1, :n]])
                if len(K):
                    out[b, l, h] = softmax_attention(q[b, l, h], K, V, scale)
                    mag[b, l, h] = softmax_attention(q[b, l, h], K, np.abs(V), scale)
    return out, mag
