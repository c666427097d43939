"""fp64 oracle of the cache with weights: norm and rotation of heads, prefill of the ring, attention that
accumulates what each key receives, eviction by weight.

Written from the definitions in include/cmc.h; shares no code with the library.  Arrays are float64 but for
indices, counts and the rounding to bf16 that a stored key has."""

from __future__ import annotations

import decimal
import functools
import math

import numpy as np


def to_bf16(x):
    """Nearest bf16 value, ties to even, of finite values within its range."""
    x = np.asarray(x, dtype=np.float64)
    m, e = np.frexp(x)  # x = m 2^e, |m| in [0.5, 1): eight significant bits
    step = np.ldexp(1.0, np.maximum(e, -125) - 8)  # and bf16's smallest steps, 2^-133
    return np.rint(x / step) * step


@functools.lru_cache(maxsize=8)
def turns_of(theta, h):
    """theta^(-i/h) / (2 pi) of i = 0 .. h - 1, in units of 2^-128."""
    with decimal.localcontext() as c:
        c.prec = 60
        two_pi = 2 * decimal.Decimal("3.14159265358979323846264338327950288419716939937510582097494459")
        ln = decimal.Decimal(theta).ln()
        return [int((-ln * i / h).exp() / two_pi * (1 << 128) + decimal.Decimal("0.5")) for i in range(h)]


def heads(x, weight=None, eps=1e-6, theta=None, p=None):
    """x [..., H, d] with gains `weight` [..., d] (one for each leading index, None: no norm), turned at positions
    p [...] (integers) where theta is given."""
    y = np.asarray(x, dtype=np.float64).copy()
    d = y.shape[-1]
    if weight is not None:
        y = y / np.sqrt((y * y).mean(axis=-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)[..., None, :]
    if theta is not None:
        h = d // 2
        shape = np.shape(p)
        # the fractional turn, in integers: a position of 2^40 takes more digits of the frequency than a double has
        turns = turns_of(float(theta), h)
        each, place = np.unique(np.asarray(p, dtype=np.int64), return_inverse=True)
        a = np.array([[int(v) * f % (1 << 128) / (1 << 128) for f in turns] for v in each]).reshape(len(each), h)
        a = 2 * math.pi * a[place.reshape(shape)]
        c, s = np.cos(a)[..., None, :], np.sin(a)[..., None, :]
        y = np.concatenate([y[..., :h] * c - y[..., h:] * s, y[..., h:] * c + y[..., :h] * s], axis=-1)
    return y


def positions(pos, evicted, offset, T):
    """[B, T]: the positions of a call's tokens."""
    e = np.zeros_like(pos) if evicted is None else evicted
    return (offset + e + pos)[:, None] + np.arange(T)


def prefill(k, v, ring_k, ring_v, ring_weight, pos, count):
    """Appends the first count[b] of k, v [B, L, T, Hkv, d] (prepared) to the ring, in place, as that many
    single appends."""
    W = ring_k.shape[3]
    for b in range(pos.shape[0]):
        if pos[b] < 0:
            continue
        for t in range(int(count[b])):
            s = int(pos[b] % W)
            ring_k[b, :, :, s] = k[b, :, t]
            ring_v[b, :, :, s] = v[b, :, t]
            if ring_weight is not None:
                ring_weight[b, :, :, s] = 0.0
            pos[b] += 1


def attend(q, tier1, ring, pos, scale):
    """tier1, ring: (K, V, weight) with K, V [B, L, Hkv, T, d]; tier1 None: the ring alone.  Adds to the weights in place;
    returns the outputs, sum_j p_j |v_j| and, as (tier1, ring), what the weights grew by and the largest
    scale * sum |q||k| of each key."""
    B, L, Hq, d = q.shape
    Hkv, W = ring[0].shape[2], ring[0].shape[3]
    k = 0 if tier1 is None else tier1[0].shape[3]
    G = Hq // Hkv
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    grew = np.zeros((B, L, Hkv, k + W))
    size = np.zeros((B, L, Hkv))
    for b in range(B):
        if pos[b] < 0:
            continue
        n = int(min(pos[b], W))
        for l in range(L):
            for g in range(Hkv):
                K, V = ring[0][b, l, g, :n], ring[1][b, l, g, :n]
                if k:
                    K = np.concatenate([tier1[0][b, l, g], K])
                    V = np.concatenate([tier1[1][b, l, g], V])
                if K.shape[0] == 0:
                    continue
                for h in range(g * G, (g + 1) * G):
                    s = scale * (K @ q[b, l, h])
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    out[b, l, h] = w @ V
                    mag[b, l, h] = w @ np.abs(V)
                    grew[b, l, g, :k + n] += w
                    size[b, l, g] = max(size[b, l, g], scale * (np.abs(K) @ np.abs(q[b, l, h])).max())
    if k:
        tier1[2][...] += grew[..., :k]
    ring[2][...] += grew[..., k:]
    return out, mag, (grew[..., :k], grew[..., k:]), size


def evict(weight, keep, recent=0, pos=None):
    """The rows that each unit keeps of weight [B, L, Hkv, T] (float32, as stored), in order of age: int64 [B, L, Hkv, keep],
    then -1; and how many each sequence holds then.  A negative pos: none, and pos."""
    B, L, Hkv, T = weight.shape
    idx = np.full((B, L, Hkv, keep), -1, dtype=np.int64)
    held = np.zeros(B, dtype=np.int64)
    for b in range(B):
        p = T if pos is None else int(pos[b])
        if p < 0:
            held[b] = p
            continue
        n = min(p, T)
        rows = [(p - n + i) % T for i in range(n)] if p > T else list(range(n))
        m = min(n, keep)
        young = min(recent, m)
        held[b] = m
        for l in range(L):
            for g in range(Hkv):
                old = [(float(weight[b, l, g, r]), i) for i, r in enumerate(rows[:n - young])]
                old.sort(key=lambda x: (math.isnan(x[0]), 0.0 if math.isnan(x[0]) else -x[0], x[1]))
                stay = sorted(i for _, i in old[:m - young]) + list(range(n - young, n))
                idx[b, l, g, :m] = [rows[i] for i in stay]
    return idx, held
