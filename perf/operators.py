"""Performance cases of the two-tier cache held in 8 bits.

Five operators, each through the package's public functions or, where `own` is false, in plain
torch operations:

quantize  rows of a bf16 K/V bank (all of them, or those an index names) into an 8-bit cache
readback  an 8-bit cache (all of it, or the rows an index names) back to bf16
append    one token per sequence into an 8-bit ring
attend    decode attention over [Tier-1 | Tier-2], both in 8 bits
step      append and attend in one call, with rotary embedding where a case says so

The cache.  Codes are float8_e4m3fn [B, L, Hkv, 2, T, d] (keys, then values) with one power of two
for each block of 32 tokens, head, and of K and V: float8_e8m0fnu [B, L, Hkv, 2, S],
S = 4 ceil(T / 128), of which ceil(T / 32) are used.  A block's power of two is the smallest that
holds its largest finite value within 448, the largest code.
"""

import math

import torch

own = False

ROPE_THETA = 5.0e5  # Llama-3
DEV = "cuda"
BLOCK = 32


# ----------------------------------------------------------------------------
# The cases
# ----------------------------------------------------------------------------

def _rows(name, kind, B, L, Hkv, d, N, k, fill="full"):
    """quantize / readback: k of N rows by index; k = 0: all N in order."""
    return {"name": name, "kind": kind, "B": B, "L": L, "Hkv": Hkv, "d": d, "N": N, "k": k,
            "fill": fill}


def _decode(name, kind, B, L, Hkv, G, d, k, W, fill="full", rope=False):
    return {"name": name, "kind": kind, "B": B, "L": L, "Hkv": Hkv, "G": G, "d": d, "k": k,
            "W": W, "fill": fill, "rope": rope}


def listed():
    return [
        # a question's Tier-1 of a Llama-3-8B-shaped decoder: the 128 selected of 1,024 rows
        _rows("write_llama", "quantize", 1, 32, 8, 128, 1024, 128),
        # the local windows of the paper's efficiency runs (batch 8, 130 tokens), prefilled to
        # different degrees
        _rows("write_windows", "quantize", 8, 32, 8, 128, 130, 0, fill="ragged"),
        # a bank kept in 8 bits: the rows of one question for the bf16 path
        _rows("read_llama", "readback", 1, 32, 8, 128, 1024, 128),
        # the banks of a batch of long contexts, read back whole
        _rows("read_long", "readback", 8, 1, 8, 128, 16384, 0),
        # one token of a small decoder: call and launch latency
        _decode("append_tiny", "append", 1, 1, 2, 4, 64, 0, 128),
        # one token of every layer of a batch of 32
        _decode("append_b32", "append", 32, 32, 8, 4, 128, 0, 512),
        # a small decoder's window without Tier-1
        _decode("attend_tiny", "attend", 1, 1, 2, 4, 64, 0, 128),
        # one layer of a batch of 64 with long windows
        _decode("attend_b64", "attend", 64, 1, 8, 4, 128, 256, 2048, fill="ragged"),
        # a small decoder's step
        _decode("step_tiny", "step", 1, 1, 2, 4, 64, 32, 128),
        # the paper's efficiency runs with rotary embedding; sizes that are no multiples of a block
        _decode("step_paper_b8", "step", 8, 32, 8, 4, 128, 30, 130, fill="ragged", rope=True),
        # one step of one request of a Llama-3-8B-shaped decoder
        _decode("step_llama", "step", 1, 32, 8, 4, 128, 128, 512, rope=True),
        # one layer of a batch of long contexts
        _decode("step_long", "step", 8, 1, 8, 4, 128, 2048, 2048),
    ]


def _log(rng, lo, hi):
    """An integer between lo and hi, spread evenly over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_MOST_BYTES = 3.0e8  # of a drawn case: below the largest listed ones


def draw(rng):
    """Another case of the same ranges, odd sizes among them."""
    while True:
        kind = rng.choice(["quantize", "readback", "append", "attend", "attend", "step", "step"])
        B, L, Hkv = _log(rng, 1, 64), rng.choice([1, 1, 2, 32]), rng.choice([8, 8, 4, 2, 1])
        d = rng.choice([128, 128, 64])
        fill = rng.choice(["full", "ragged"])
        if kind in ("quantize", "readback"):
            N = _log(rng, 1, 16384)
            k = _log(rng, 1, N) if rng.random() < 0.5 else 0
            c = _rows("", kind, B, L, Hkv, d, N, k, fill=fill if kind == "quantize" else "full")
            if 4 * B * L * Hkv * N * d > 3e9:  # the bank that the rows come from
                continue
        else:
            k = _log(rng, 1, 4096) if kind != "append" and rng.random() < 0.9 else 0
            c = _decode("", kind, B, L, Hkv, rng.choice([4, 4, 8, 2, 1]), d, k, _log(rng, 1, 4096),
                        fill=fill, rope=kind == "step" and rng.random() < 0.5)
            if 2 * B * L * Hkv * (k + c["W"]) * d > _MOST_BYTES:
                continue
        c.pop("name")
        if work(c)["bytes"] <= _MOST_BYTES:
            return c


def _scale_bytes(T):
    return 4 * ((T + 127) // 128)


def _live(c, T):
    """Tokens of a ring of T slots, in the mean over the seeds (rows without one need not be read)."""
    return T if c["fill"] == "full" else T * (1 - 2.0 ** -4) / (4 * math.log(2.0))


def work(c):
    B, L, Hkv, d = c["B"], c["L"], c["Hkv"], c["d"]
    units = B * L * Hkv
    if c["kind"] in ("quantize", "readback"):
        n = c["k"] or c["N"]
        codes = units * 2 * (n * d + -(-n // BLOCK))
        return {"bytes": codes + units * 4 * _live(c, n) * d + (4 * B * n if c["k"] else 0),
                "flops": units * 2 * n * d}
    row = units * 2 * d
    if c["kind"] == "append":  # the new row in bf16, its codes, the block's power of two, pos
        return {"bytes": 3 * row + units * 4 + 16 * B, "flops": 2 * row}
    n = c["k"] + _live(c, c["W"])
    heads = B * L * c["G"] * Hkv
    nbytes = units * 2 * (n * d + n / BLOCK) + heads * 4 * d + 8 * B
    if c["kind"] == "step":
        nbytes += 3 * row + units * 4 + 8 * B
    return {"bytes": nbytes, "flops": 4 * heads * n * d}


# ----------------------------------------------------------------------------
# The cache format in plain torch operations (32 bits)
# ----------------------------------------------------------------------------

def _block_code(amax):
    """The byte of the power of two of a block whose largest finite magnitude is `amax` (fp32):
    the smallest c >= 0 with amax <= 448 * 2^(c - 127), from amax's exponent and mantissa."""
    bits = amax.view(torch.int32)
    c = (bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000).to(torch.int32)
    return c.clamp_(min=0)


def _pow2(c):
    """2^(c - 127) for bytes c as fp32."""
    return c.to(torch.uint8).view(torch.float8_e8m0fnu).to(torch.float32)


def _codes(x, c):
    """The codes of x under the powers of two with bytes c (broadcast): an infinity is stored as NaN."""
    y = x * _pow2(254 - c)
    return torch.where(torch.isfinite(x), y, float("nan")).to(torch.float8_e4m3fn)


def _blocks(x, T):
    """[..., T, d] padded with zeros to [..., blocks, 32, d]."""
    pad = -T % BLOCK
    x = torch.cat([x, x.new_zeros(x.shape[:-2] + (pad, x.shape[-1]))], dim=-2) if pad else x
    return x.reshape(x.shape[:-2] + (-1, BLOCK, x.shape[-1]))


def _finite(x):
    return torch.where(torch.isfinite(x), x, 0.0)


def _quantize(k, v, live):
    """The cache of rows k, v [B, L, Hkv, T, d]; `live` [B, T] (None: all) says which hold a token."""
    B, L, Hkv, T, d = k.shape
    x = torch.stack([k, v], dim=3).to(torch.float32)  # [B, L, Hkv, 2, T, d]
    if live is not None:
        x = torch.where(live[:, None, None, None, :, None], x, 0.0)
    xb = _blocks(x, T)
    c = _block_code(_finite(xb).abs().amax(dim=(-1, -2)))
    kv = _codes(xb, c[..., None, None]).reshape(B, L, Hkv, 2, -1, d)[..., :T, :].contiguous()
    scales = torch.zeros((B, L, Hkv, 2, _scale_bytes(T)), dtype=torch.uint8, device=k.device)
    scales[..., :c.shape[-1]] = c.to(torch.uint8)
    return kv, scales.view(torch.float8_e8m0fnu)


def _values(kv, scales):
    """The values of a whole cache, fp32 [B, L, Hkv, 2, T, d]."""
    T = kv.shape[4]
    s = scales.to(torch.float32).repeat_interleave(BLOCK, dim=-1)[..., :T]
    return kv.to(torch.float32) * s[..., None]


def _append(s, k_new, v_new):
    """One token per sequence into s's ring, in place; k_new, v_new in fp32."""
    ring, scales, pos = s["ring_kv"], s["ring_scales"], s["pos"]
    B, W = pos.shape[0], ring.shape[4]
    b = torch.arange(B, device=pos.device)
    slot = pos % W
    blk = slot // BLOCK
    rows = blk[:, None] * BLOCK + torch.arange(BLOCK, device=pos.device)  # [B, 32]
    other = (rows < pos.clamp(max=W)[:, None]) & (rows != slot[:, None])
    at = torch.where(other, rows, slot[:, None])  # the other rows point at the new token's
    codes = ring.view(torch.uint8)[b[:, None], :, :, :, at]  # [B, 32, L, Hkv, 2, d]
    codes = codes.view(torch.float8_e4m3fn).to(torch.float32)
    c_old = scales.view(torch.uint8)[b, :, :, :, blk].to(torch.int32)  # [B, L, Hkv, 2]
    new = torch.stack([k_new, v_new], dim=3)  # [B, L, Hkv, 2, d]
    amax = _finite(new).abs().amax(dim=-1)
    held = torch.where(other[:, :, None, None, None, None], codes, 0.0)
    held = (_finite(held).abs().amax(dim=(1, -1))) * _pow2(c_old)
    first = (slot % BLOCK == 0)[:, None, None, None]
    c = torch.where(first, _block_code(torch.maximum(amax, held)),
                    torch.maximum(_block_code(amax), c_old))
    moved = codes * _pow2((127 + c_old - c).clamp(0, 254))[:, None, ..., None]
    put = torch.where(other[:, :, None, None, None, None], moved.to(torch.float8_e4m3fn).to(torch.float32),
                      _codes(new, c[..., None]).to(torch.float32)[:, None])
    ring.view(torch.uint8)[b[:, None], :, :, :, at] = put.to(torch.float8_e4m3fn).view(torch.uint8)
    scales.view(torch.uint8)[b, :, :, :, blk] = c.to(torch.uint8)
    pos += 1


def _rotate(x, p):
    """Rotary embedding of x [B, L, H, d] at positions p [B] (half-split pairs), angles in 64 bits."""
    h = x.shape[-1] // 2
    f = torch.exp2(torch.arange(h, device=x.device, dtype=torch.float64) * (-math.log2(ROPE_THETA) / h))
    a = (p.to(torch.float64)[:, None] * f)[:, None, None, :]
    cos, sin = a.cos().to(torch.float32), a.sin().to(torch.float32)
    lo, hi = x[..., :h], x[..., h:]
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1)


def _attend(q, t1_kv, t1_scales, ring_kv, ring_scales, count):
    """softmax(q k / sqrt(d)) v over the rows of Tier-1 and the first count[b] slots of the ring."""
    B, L, Hq, d = q.shape
    Hkv, W = ring_kv.shape[2], ring_kv.shape[4]
    x = _values(ring_kv, ring_scales)
    dead = (torch.arange(W, device=q.device) >= count[:, None])[:, None, None, :]  # [B, 1, 1, W]
    x.masked_fill_(dead[:, :, :, None, :, None], 0.0)
    if t1_kv is not None:
        x = torch.cat([_values(t1_kv, t1_scales), x], dim=4)
        dead = torch.cat([dead.new_zeros((B, 1, 1, t1_kv.shape[4])), dead], dim=-1)
    s = torch.matmul(q.reshape(B, L, Hkv, -1, d), x[:, :, :, 0].transpose(-1, -2)) / math.sqrt(d)
    s = s.masked_fill(dead[..., None, :], float("-inf"))
    m = s.amax(dim=-1, keepdim=True)
    p = torch.exp(s - torch.where(m == float("-inf"), 0.0, m))
    o = torch.matmul(p, x[:, :, :, 1]) / p.sum(dim=-1, keepdim=True).clamp(min=1e-30)
    return o.reshape(B, L, Hq, d).to(torch.bfloat16)


# ----------------------------------------------------------------------------
# Inputs (plain torch, from the seed alone)
# ----------------------------------------------------------------------------

def _gen(seed, *more):
    s = int(seed) & 0x7FFFFFFF
    for m in more:
        s = (s * 1000003 + int(m) + 12345) & 0x7FFFFFFFFFFF
    return torch.Generator(device=DEV).manual_seed(s)


def _kv(g, B, L, Hkv, T, d):
    """K and V rows as a decoder leaves them: heads of different magnitude, a few channels of
    the keys larger than the others."""
    out = []
    for which in range(2):
        x = torch.empty((B, L, Hkv, T, d), dtype=torch.bfloat16, device=DEV)
        size = torch.exp2(torch.randn((1, L, Hkv, 1, 1), generator=g, device=DEV))
        gain = torch.ones(d, device=DEV)
        if which == 0:
            size = size.clamp(max=1.0)
            gain[torch.randperm(d, generator=g, device=DEV)[:3]] = 4.0
        for b in range(B):
            x[b] = (torch.randn((L, Hkv, T, d), generator=g, device=DEV) * gain * size[0]).to(torch.bfloat16)
        out.append(x)
    return out


def _count(c, g, T):
    """Tokens seen by each sequence's ring of T slots: some way past full, or filled to between a
    sixteenth and all of it."""
    if c["fill"] == "full":
        return torch.randint(T, 4 * T + 1, (c["B"],), generator=g, device=DEV)
    f = torch.rand((c["B"],), generator=g, device=DEV, dtype=torch.float64)
    return torch.exp2(f * 4 - 4).mul(T).ceil().to(torch.int64)


def _index(c, g):
    return (torch.rand((c["B"], c["N"]), generator=g, device=DEV).topk(c["k"], dim=1).indices
            .sort(dim=1).values.to(torch.int32))


def prepare(case, seed):
    c = case
    g = _gen(seed)
    B, L, Hkv, d = c["B"], c["L"], c["Hkv"], c["d"]
    s = {"case": c}
    if c["kind"] in ("quantize", "readback"):
        s["idx"] = _index(c, g) if c["k"] else None
        k, v = _kv(g, B, L, Hkv, c["N"], d)
        if c["kind"] == "quantize":
            s["k"], s["v"] = k, v
            s["count"] = _count(c, g, c["k"] or c["N"]) if c["fill"] == "ragged" else None
        else:
            s["kv"], s["scales"] = _quantize(k, v, None)
        return s
    W = c["W"]
    s["pos"] = _count(c, g, W)
    live = torch.arange(W, device=DEV) < s["pos"][:, None]
    s["ring_kv"], s["ring_scales"] = _quantize(*_kv(g, B, L, Hkv, W, d), live)
    if c["kind"] != "attend":
        k, v = _kv(g, B, L, Hkv, 1, d)
        s["k_new"], s["v_new"] = k[:, :, :, 0].contiguous(), v[:, :, :, 0].contiguous()
    if c["kind"] != "append":
        s["t1_kv"] = s["t1_scales"] = None
        if c["k"]:
            s["t1_kv"], s["t1_scales"] = _quantize(*_kv(g, B, L, Hkv, c["k"], d), None)
        s["q"] = (torch.randn((B, L, Hkv * c["G"], d), generator=g, device=DEV) * 1.5).to(torch.bfloat16)
    return s


# ----------------------------------------------------------------------------
# One pass
# ----------------------------------------------------------------------------

def _run_own(s):
    import paper_2609_25537_gb300 as cmc
    c = s["case"]
    kind = c["kind"]
    if kind == "quantize":
        return cmc.quantize_cache(s["k"], s["v"], s["idx"], count=s["count"])
    if kind == "readback":
        return cmc.dequantize_cache(s["kv"], s["scales"], s["idx"])
    if kind == "append":
        cmc.window_append_q8(s["ring_kv"], s["ring_scales"], s["pos"], s["k_new"], s["v_new"])
        return s["ring_kv"], s["ring_scales"], s["pos"]
    if kind == "attend":
        return cmc.two_tier_decode_attn_q8(s["q"], s["t1_kv"], s["t1_scales"], s["ring_kv"],
                                           s["ring_scales"], s["pos"])
    out = cmc.decode_step_q8(s["q"], s["t1_kv"], s["t1_scales"], s["ring_kv"], s["ring_scales"],
                             s["pos"], s["k_new"], s["v_new"],
                             rope_theta=ROPE_THETA if c["rope"] else None, rope_offset=c["k"])
    return out, s["ring_kv"], s["ring_scales"], s["pos"]


def _run_plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "quantize":
        k, v, idx = s["k"], s["v"], s["idx"]
        if idx is not None:
            b = torch.arange(c["B"], device=k.device)[:, None]
            k, v = (x[b, :, :, idx.long()].permute(0, 2, 3, 1, 4) for x in (k, v))
        live = None
        if s["count"] is not None:
            live = torch.arange(k.shape[3], device=k.device) < s["count"][:, None]
        return _quantize(k, v, live)
    if kind == "readback":
        kv, scales, idx = s["kv"], s["scales"], s["idx"]
        if idx is None:
            x = _values(kv, scales)
        else:
            b, i = torch.arange(c["B"], device=kv.device)[:, None], idx.long()
            x = kv.view(torch.uint8)[b, :, :, :, i].view(torch.float8_e4m3fn).to(torch.float32)
            x = x * scales.view(torch.uint8)[b, :, :, :, i // BLOCK].view(torch.float8_e8m0fnu).to(torch.float32)[..., None]
            x = x.permute(0, 2, 3, 4, 1, 5)
        return x[:, :, :, 0].to(torch.bfloat16).contiguous(), x[:, :, :, 1].to(torch.bfloat16).contiguous()
    if kind == "append":
        _append(s, s["k_new"].to(torch.float32), s["v_new"].to(torch.float32))
        return s["ring_kv"], s["ring_scales"], s["pos"]
    q, W = s["q"].to(torch.float32), c["W"]
    if kind == "attend":
        return _attend(q, s["t1_kv"], s["t1_scales"], s["ring_kv"], s["ring_scales"], s["pos"].clamp(max=W))
    k_new = s["k_new"].to(torch.float32)
    if c["rope"]:
        p = s["pos"] + c["k"]
        q, k_new = _rotate(q, p), _rotate(k_new, p)
    _append(s, k_new, s["v_new"].to(torch.float32))
    out = _attend(q, s["t1_kv"], s["t1_scales"], s["ring_kv"], s["ring_scales"], s["pos"].clamp(max=W))
    return out, s["ring_kv"], s["ring_scales"], s["pos"]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ----------------------------------------------------------------------------
# 64 bits, from the definition
# ----------------------------------------------------------------------------

def _two_to(E):
    """2^E for whole E from -1022 to 1023 in 64 bits, exactly (exp2 may be off in its last bit)."""
    return ((E.to(torch.int64) + 1023) << 52).view(torch.float64)


def _power_of(amax):
    """The exponent E of a block whose largest magnitude is amax (64 bits): the smallest E >= -127
    with amax <= 448 * 2^E."""
    m, e = torch.frexp(amax)  # amax = m 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
    E = e - 9 + (m > 0.875).to(e.dtype)
    return torch.where(amax > 0, E, -127).clamp(min=-127)


def _nearest(y):
    """The nearest e4m3 value of y (64 bits, within 448), ties to the even significand: steps of an
    eighth of the power of two below y, and of 2^-9 under 2^-6."""
    e = torch.frexp(y)[1] - 1
    step = _two_to(torch.where(y == 0, -6, e).clamp(min=-6) - 3)
    return torch.round(y / step) * step  # half to even


def _exact_quantize(x, live):
    """Codes' values and powers of two of rows x (64 bits, [B, L, Hkv, T, d]), block by block."""
    B, L, Hkv, T, d = x.shape
    kv = torch.zeros_like(x)
    scales = torch.full((B, L, Hkv, _scale_bytes(T)), -127, device=x.device)
    x = torch.where(live[:, None, None, :, None], x, 0.0)
    for j in range(-(-T // BLOCK)):
        part = x[:, :, :, j * BLOCK:(j + 1) * BLOCK]
        E = _power_of(part.abs().flatten(3).max(dim=3).values)
        kv[:, :, :, j * BLOCK:(j + 1) * BLOCK] = _nearest(part * _two_to(-E)[..., None, None])
        scales[..., j] = E
    return kv, _two_to(scales)


def _exact_values(kv, scales):
    """A cache's values in 64 bits: K and V, [B, L, Hkv, T, d] each."""
    codes = kv.to(torch.float64, copy=True)
    for j in range(-(-kv.shape[4] // BLOCK)):
        codes[..., j * BLOCK:(j + 1) * BLOCK, :] *= scales[..., j].to(torch.float64)[..., None, None]
    return codes[:, :, :, 0], codes[:, :, :, 1]


def _exact_append(s, new):
    """The ring's codes' values, powers of two and pos after the append of `new` [B, L, Hkv, 2, d]."""
    W = s["ring_kv"].shape[4]
    codes = s["ring_kv"].to(torch.float64, copy=True)
    power = torch.frexp(s["ring_scales"].to(torch.float64))[1] - 1
    for b, n in enumerate(s["pos"].tolist()):
        slot = n % W
        first = slot - slot % BLOCK
        last = min(first + BLOCK, W, max(slot + 1, n))  # behind it no slot holds a token yet
        rows = codes[b, :, :, :, first:last]
        E0 = power[b, :, :, :, slot // BLOCK]
        rows[..., slot - first, :] = 0.0
        top = new[b].abs().amax(dim=-1)
        if slot == first:
            E = _power_of(torch.maximum(top, rows.abs().amax(dim=(-1, -2)) * _two_to(E0)))
        else:
            E = torch.maximum(_power_of(top), E0)
        rows = _nearest(rows * _two_to(E0 - E)[..., None, None])
        rows[..., slot - first, :] = _nearest(new[b] * _two_to(-E)[..., None])
        codes[b, :, :, :, first:last] = rows
        power[b, :, :, :, slot // BLOCK] = E
    return codes, _two_to(power), s["pos"] + 1


def _exact_attend(c, q, tiers, count):
    """Attention in 64 bits, one sequence and KV head at a time over all layers; `tiers`: (K, V) pairs, the
    last one the ring's."""
    B, L, Hq, d = q.shape
    G = c["G"]
    out = torch.zeros((B, L, Hq, d), dtype=torch.float64, device=q.device)
    for b in range(B):
        n = int(count[b])
        for g in range(c["Hkv"]):
            K = torch.cat([t[0][b, :, g] for t in tiers[:-1]] + [tiers[-1][0][b, :, g, :n]], dim=1)
            V = torch.cat([t[1][b, :, g] for t in tiers[:-1]] + [tiers[-1][1][b, :, g, :n]], dim=1)
            w = torch.softmax(q[b, :, g * G:(g + 1) * G] @ K.transpose(1, 2) / math.sqrt(d), dim=-1)
            out[b, :, g * G:(g + 1) * G] = w @ V
    return out


def _exact_rotate(x, p):
    h = x.shape[-1] // 2
    y = x.clone()
    for i in range(h):
        a = p.to(torch.float64) * ROPE_THETA ** (-i / h)
        co, si = torch.cos(a)[:, None, None], torch.sin(a)[:, None, None]
        y[..., i] = x[..., i] * co - x[..., i + h] * si
        y[..., i + h] = x[..., i + h] * co + x[..., i] * si
    return y


def exact(case, seed):
    c, s = case, prepare(case, seed)
    kind = c["kind"]
    if kind == "quantize":
        n = c["k"] or c["N"]
        live = torch.ones((c["B"], n), dtype=torch.bool, device=DEV)
        if s["count"] is not None:
            live = torch.arange(n, device=DEV)[None] < s["count"][:, None]
        kv, scales = [], []
        for x in (s["k"], s["v"]):
            if s["idx"] is not None:
                x = torch.stack([x[b].index_select(2, s["idx"][b].long()) for b in range(c["B"])])
            a, p = _exact_quantize(x.to(torch.float64), live)
            kv.append(a)
            scales.append(p)
        return torch.stack(kv, dim=3), torch.stack(scales, dim=3)
    if kind == "readback":
        k, v = _exact_values(s["kv"], s["scales"])
        if s["idx"] is not None:
            k, v = (torch.stack([x[b].index_select(2, s["idx"][b].long()) for b in range(c["B"])])
                    for x in (k, v))
        return k.contiguous(), v.contiguous()
    if kind != "attend":
        k_new, v_new = s["k_new"].to(torch.float64), s["v_new"].to(torch.float64)
        if c["rope"]:
            k_new = _exact_rotate(k_new, s["pos"] + c["k"])
        ring, powers, pos = _exact_append(s, torch.stack([k_new, v_new], dim=3))
        if kind == "append":
            return ring, powers, pos
    else:
        ring, powers, pos = s["ring_kv"], s["ring_scales"], s["pos"]
    q = s["q"].to(torch.float64)
    if c["rope"]:
        q = _exact_rotate(q, s["pos"] + c["k"])
    tiers = [_exact_values(ring, powers)]
    if c["k"]:
        tiers.insert(0, _exact_values(s["t1_kv"], s["t1_scales"]))
    out = _exact_attend(c, q, tiers, pos.clamp(max=c["W"]))
    if kind == "attend":
        return out
    # a rotated key's values next to a rounding border fall on either side of it in 32 bits, so the
    # ring after a step with rotary embedding has no exact codes
    return (out, None, None, pos) if c["rope"] else (out, ring, powers, pos)
