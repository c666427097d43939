"""Performance cases of a two-tier cache whose tokens are kept by the attention that they received.

Five operators, each through the package's public functions or, where `own` is false, in plain
torch operations:

norm     RMS norm of every query and key head and rotary embedding, of many tokens or of one
prefill  the same for a prompt's tokens, whose keys and values go to the Tier-2 ring
attend   decode attention over [Tier-1 | Tier-2] that adds each key's probabilities to its weight
step     append and attend in one call, with norm and rotary embedding where a case says so
evict    the heaviest and the youngest tokens of a cache, moved together in order of age

A key's weight is the sum of the probabilities that all queries of its KV head have given it, fp32
[B, L, Hkv, rows] beside the bf16 rows [B, L, Hkv, rows, d].  Positions: token t of a call is at
rope_offset + evicted[b] + pos[b] + t, where pos[b] counts the tokens that the ring was given and
evicted[b] those that were taken out of it again.
"""

import math

import torch

own = False

ROPE_THETA = 5.0e5  # Llama-3
EPS = 1e-6
DEV = "cuda"


# ----------------------------------------------------------------------------
# The cases
# ----------------------------------------------------------------------------

def _tokens(name, kind, B, L, Hkv, G, d, T, W=0, fill="full", norm=True, packed=True):
    """norm / prefill: T tokens of each of B sequences and L layers; packed: q, k and v are parts of
    one projection's output."""
    return {"name": name, "kind": kind, "B": B, "L": L, "Hkv": Hkv, "G": G, "d": d, "T": T, "W": W,
            "fill": fill, "norm": norm, "packed": packed}


def _decode(name, kind, B, L, Hkv, G, d, k, W, fill="full", norm=False, rope=False):
    return {"name": name, "kind": kind, "B": B, "L": L, "Hkv": Hkv, "G": G, "d": d, "k": k, "W": W,
            "fill": fill, "norm": norm, "rope": rope}


def _evict(name, B, L, Hkv, d, T, keep, recent, fill):
    """fill: "rows" (all T rows hold tokens), "ring" (a ring that has wrapped), "ragged" (rings filled
    to different degrees)."""
    return {"name": name, "kind": "evict", "B": B, "L": L, "Hkv": Hkv, "d": d, "T": T, "keep": keep,
            "recent": recent, "fill": fill}


def listed():
    return [
        # one token of a small decoder's layer: call and launch latency
        _tokens("norm_tiny", "norm", 1, 1, 2, 4, 64, 1, packed=False),
        # one layer's projections of a batch of prompts
        _tokens("norm_b8", "norm", 8, 1, 8, 4, 128, 1024),
        # the local windows of the paper's efficiency runs (batch 8, 130 tokens), of different
        # lengths; Llama-3 has no norm on queries and keys
        _tokens("prefill_paper_b8", "prefill", 8, 32, 8, 4, 128, 130, 130, fill="ragged", norm=False),
        # prompts longer than the window: their last 2,048 tokens stay
        _tokens("prefill_long", "prefill", 8, 1, 8, 4, 128, 4096, 2048),
        # a small decoder's attention
        _decode("attend_tiny", "attend", 1, 1, 2, 4, 64, 32, 128),
        # one layer of a batch of 64 with long windows
        _decode("attend_b64", "attend", 64, 1, 8, 4, 128, 256, 2048, fill="ragged"),
        # the paper's efficiency runs; sizes that are no multiples of a block
        _decode("step_paper_b8", "step", 8, 32, 8, 4, 128, 30, 130, fill="ragged", rope=True),
        # one step of one request of a Llama-3-8B-shaped decoder, with norms
        _decode("step_llama", "step", 1, 32, 8, 4, 128, 128, 512, norm=True, rope=True),
        # one layer of a batch of long contexts
        _decode("step_long", "step", 8, 1, 8, 4, 128, 2048, 2048),
        # a small decoder's ring that is full
        _evict("evict_tiny", 1, 1, 2, 64, 128, 64, 16, "ring"),
        # the rings of all layers of a Llama-3-8B-shaped decoder, cut to a half
        _evict("evict_llama", 1, 32, 8, 128, 512, 256, 64, "ring"),
        # one layer's Tier-1 banks of long contexts, cut to what a budget of 2,048 rows allows
        _evict("evict_bank", 8, 1, 8, 128, 16384, 2048, 0, "rows"),
    ]


def _log(rng, lo, hi):
    """An integer between lo and hi, spread evenly over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_MOST_BYTES = 3.0e8  # of a drawn case: below the largest listed one


def draw(rng):
    """Another case of the same ranges, odd sizes among them."""
    while True:
        kind = rng.choice(["norm", "prefill", "attend", "attend", "step", "step", "evict", "evict"])
        B, L, Hkv = _log(rng, 1, 64), rng.choice([1, 1, 2, 32]), rng.choice([8, 8, 4, 2, 1])
        d, G = rng.choice([128, 128, 64]), rng.choice([4, 4, 8, 2, 1])
        fill = rng.choice(["full", "ragged"])
        norm = rng.random() < 0.5
        if kind in ("norm", "prefill"):
            T = 1 if rng.random() < 0.2 else _log(rng, 1, 4096)
            c = _tokens("", kind, B, L, Hkv, G, d, T, _log(rng, 1, 4096) if kind == "prefill" else 0,
                        fill if kind == "prefill" else "full", norm, rng.random() < 0.5)
            held = 2 * B * L * d * Hkv * (T * (G + 2) + 2 * c["W"])
        elif kind == "evict":
            T = _log(rng, 1, 16384)
            keep = _log(rng, 1, T)
            c = _evict("", B, L, Hkv, d, T, keep, rng.choice([0, rng.randint(0, keep)]),
                       rng.choice(["rows", "ring", "ragged"]))
            held = 4 * B * L * Hkv * T * d
        else:
            k = _log(rng, 1, 4096) if rng.random() < 0.9 else 0
            c = _decode("", kind, B, L, Hkv, G, d, k, _log(rng, 1, 4096), fill,
                        norm and kind == "step", kind == "step" and rng.random() < 0.6)
            held = 4 * B * L * Hkv * (k + c["W"]) * d
        c.pop("name")
        if held < 1e9 and work(c)["bytes"] <= _MOST_BYTES:
            return c


def _held(c, T, most=None):
    """min(tokens that a sequence holds of T, most) in the mean over the seeds: all T, or T 2^-f
    with f even between 0 and 4."""
    most = T if most is None else min(T, most)
    if c["fill"] != "ragged":
        return most
    a = min(math.log2(T / most), 4.0)  # f below a: more than `most`
    return most * a / 4 + (T * 2.0 ** -a - T / 16) / (4 * math.log(2.0))


def work(c):
    B, L, Hkv, d = c["B"], c["L"], c["Hkv"], c["d"]
    units = B * L * Hkv
    row = units * 2 * d  # a bf16 row of each
    if c["kind"] == "norm":
        n = c["T"] * (c["G"] + 1)
        return {"bytes": 2 * n * row, "flops": 5 * n * row}
    if c["kind"] == "prefill":
        n, w = _held(c, c["T"]), _held(c, c["T"], c["W"])
        return {"bytes": 2 * n * c["G"] * row + 4 * w * row + 4 * w * units + 16 * B,
                "flops": 5 * (n * c["G"] + w) * row}
    if c["kind"] == "evict":
        n, m = _held(c, c["T"]), _held(c, c["T"], c["keep"])
        return {"bytes": units * (4 * n + 8 * m) + 4 * m * row + 16 * B, "flops": units * n}
    n = c["k"] + _held(c, c["W"])
    nbytes = 2 * n * row + 8 * n * units + 2 * c["G"] * row + 8 * B
    if c["kind"] == "step":
        nbytes += 4 * row + 8 * B
    return {"bytes": nbytes, "flops": 4 * c["G"] * units * n * d}


# ----------------------------------------------------------------------------
# Inputs (plain torch, from the seed alone)
# ----------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) & 0x7FFFFFFF)


def _rows(g, B, L, Hkv, T, d, keys):
    """K or V rows as a decoder leaves them: heads of different magnitude, a few channels of the keys
    larger than the others."""
    size = torch.exp2(torch.randn((1, L, Hkv, 1, 1), generator=g, device=DEV))
    gain = torch.ones(d, device=DEV)
    if keys:
        size = size.clamp(max=1.0)
        gain[torch.randperm(d, generator=g, device=DEV)[:3]] = 4.0
    x = torch.empty((B, L, Hkv, T, d), dtype=torch.bfloat16, device=DEV)
    for b in range(B):
        x[b] = (torch.randn((L, Hkv, T, d), generator=g, device=DEV) * gain * size[0]).to(torch.bfloat16)
    return x


def _received(g, *shape):
    """Weights that tokens have gathered: most little, a few much, and some none at all."""
    x = torch.exp(torch.randn(shape, generator=g, device=DEV) * 2.0 - 3.0)
    return torch.where(torch.rand(shape, generator=g, device=DEV) < 0.05, 0.0, x)


def _count(c, g, T):
    """Tokens of each sequence, of T: all, or between a sixteenth and all of them."""
    if c["fill"] != "ragged":
        return torch.full((c["B"],), T, dtype=torch.int64, device=DEV)
    f = torch.rand((c["B"],), generator=g, device=DEV, dtype=torch.float64)
    return torch.exp2(f * 4 - 4).mul(T).ceil().to(torch.int64)


def _norms(c, g):
    """The norms' gains of each layer."""
    if not c["norm"]:
        return None, None
    return tuple(1.0 + 0.3 * torch.randn((c["L"], c["d"]), generator=g, device=DEV) for _ in range(2))


def prepare(case, seed):
    c = case
    g = _gen(seed)
    B, L, Hkv, d = c["B"], c["L"], c["Hkv"], c["d"]
    s = {"case": c}
    if c["kind"] == "evict":
        T, keep = c["T"], c["keep"]
        s["k"], s["v"] = _rows(g, B, L, Hkv, T, d, True), _rows(g, B, L, Hkv, T, d, False)
        s["weight"] = _received(g, B, L, Hkv, T)
        s["pos"] = {"rows": None, "ragged": _count(c, g, T),
                    "ring": torch.randint(T, 4 * T + 1, (B,), generator=g, device=DEV)}[c["fill"]]
        s["evicted"] = torch.randint(0, 1000, (B,), generator=g, device=DEV)
        s["out_k"], s["out_v"] = (torch.zeros((B, L, Hkv, keep, d), dtype=torch.bfloat16, device=DEV)
                                  for _ in range(2))
        s["out_weight"] = torch.zeros((B, L, Hkv, keep), device=DEV)
        return s
    s["q_weight"], s["k_weight"] = _norms(c, g)
    s["evicted"] = torch.randint(0, 1000, (B,), generator=g, device=DEV)
    Hq = Hkv * c["G"]
    if c["kind"] in ("norm", "prefill"):
        T, W = c["T"], c["W"]
        x = torch.empty((B, L, T, Hq + 2 * Hkv, d), dtype=torch.bfloat16, device=DEV)
        for b in range(B):
            x[b] = (torch.randn(x.shape[1:], generator=g, device=DEV) * 1.5).to(torch.bfloat16)
        parts = x.split([Hq, Hkv, Hkv], dim=3)
        s["q"], s["k"], s["v"] = parts if c["packed"] else [p.contiguous() for p in parts]
        s["pos"] = torch.randint(0, 4000, (B,), generator=g, device=DEV)
        if c["kind"] == "prefill":
            s["ring_k"], s["ring_v"] = (torch.zeros((B, L, Hkv, W, d), dtype=torch.bfloat16, device=DEV)
                                        for _ in range(2))
            s["ring_weight"] = _received(g, B, L, Hkv, W)
            s["count"] = _count(c, g, T) if c["fill"] == "ragged" else None
            s["out_q"] = torch.zeros((B, L, T, Hq, d), dtype=torch.bfloat16, device=DEV)
        return s
    W, k = c["W"], c["k"]
    s["pos"] = (torch.randint(W, 4 * W + 1, (B,), generator=g, device=DEV) if c["fill"] == "full"
                else _count(c, g, W))
    s["ring_k"], s["ring_v"] = _rows(g, B, L, Hkv, W, d, True), _rows(g, B, L, Hkv, W, d, False)
    s["ring_weight"] = _received(g, B, L, Hkv, W)
    s["t1_k"] = s["t1_v"] = s["t1_weight"] = None
    if k:
        s["t1_k"], s["t1_v"] = _rows(g, B, L, Hkv, k, d, True), _rows(g, B, L, Hkv, k, d, False)
        s["t1_weight"] = _received(g, B, L, Hkv, k)
    s["q"] = (torch.randn((B, L, Hq, d), generator=g, device=DEV) * 1.5).to(torch.bfloat16)
    if c["kind"] == "step":
        s["k_new"], s["v_new"] = (_rows(g, B, L, Hkv, 1, d, keys)[:, :, :, 0].contiguous()
                                  for keys in (True, False))
    return s


# ----------------------------------------------------------------------------
# One pass
# ----------------------------------------------------------------------------

def _run_own(s):
    import paper_2609_25537_gb300 as cmc
    c = s["case"]
    kind = c["kind"]
    if kind == "evict":
        return cmc.evict_cache(s["k"], s["v"], s["weight"], c["keep"], pos=s["pos"],
                               recent=c["recent"], evicted=s["evicted"], out_k=s["out_k"],
                               out_v=s["out_v"], out_weight=s["out_weight"]) + (s["evicted"],)
    with_norm = {"q_weight": s["q_weight"], "k_weight": s["k_weight"], "eps": EPS}
    if kind == "norm":
        return cmc.qk_norm_rope(s["q"], s["k"], s["pos"], rope_theta=ROPE_THETA, rope_offset=7,
                                evicted=s["evicted"], **with_norm)
    if kind == "prefill":
        q = cmc.window_prefill(s["q"], s["k"], s["v"], s["ring_k"], s["ring_v"], s["pos"],
                               ring_weight=s["ring_weight"], count=s["count"], rope_theta=ROPE_THETA,
                               rope_offset=7, evicted=s["evicted"], out_q=s["out_q"], **with_norm)
        return q, s["ring_k"], s["ring_v"], s["ring_weight"], s["pos"]
    caches = (s["t1_k"], s["t1_v"], s["t1_weight"], s["ring_k"], s["ring_v"], s["ring_weight"], s["pos"])
    if kind == "attend":
        return cmc.two_tier_decode_attn_weighted(s["q"], *caches), s["t1_weight"], s["ring_weight"]
    out = cmc.decode_step_weighted(s["q"], *caches, s["k_new"], s["v_new"],
                                   rope_theta=ROPE_THETA if c["rope"] else None, rope_offset=c["k"],
                                   evicted=s["evicted"], **with_norm)
    return (out,) + caches[2:]


def _norm_rotate(x, w, p):
    """x [B, L, T, H, d] in fp32: RMS norm with gains w [L, d] and rotary embedding at positions
    p [B, T] (half-split pairs; angles in 64 bits), each where it is given."""
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * w[:, None, None]
    if p is None:
        return x
    h = x.shape[-1] // 2
    f = torch.exp2(torch.arange(h, device=x.device, dtype=torch.float64) * (-math.log2(ROPE_THETA) / h))
    a = (p.to(torch.float64)[..., None] * f)[:, None, :, None]
    cos, sin = a.cos().to(torch.float32), a.sin().to(torch.float32)
    lo, hi = x[..., :h], x[..., h:]
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1)


def _attend(s, q):
    """softmax(q k / sqrt(d)) v over the rows of Tier-1 and the occupied slots of the ring; the
    probabilities are added to the weights."""
    c = s["case"]
    B, L, Hq, d = q.shape
    Hkv, W = c["Hkv"], c["W"]
    dead = (torch.arange(W, device=q.device) >= s["pos"].clamp(max=W)[:, None])[:, None, None, :]
    k = s["ring_k"].to(torch.float32).masked_fill_(dead[..., None], 0.0)
    v = s["ring_v"].to(torch.float32).masked_fill_(dead[..., None], 0.0)
    if c["k"]:
        k = torch.cat([s["t1_k"].to(torch.float32), k], dim=3)
        v = torch.cat([s["t1_v"].to(torch.float32), v], dim=3)
        dead = torch.cat([dead.new_zeros((B, 1, 1, c["k"])), dead], dim=-1)
    x = torch.matmul(q.reshape(B, L, Hkv, -1, d), k.transpose(-1, -2)) / math.sqrt(d)
    x = x.masked_fill(dead[..., None, :], float("-inf"))
    m = x.amax(dim=-1, keepdim=True)
    x = torch.exp(x - torch.where(m == float("-inf"), 0.0, m))
    x = x / x.sum(dim=-1, keepdim=True).clamp(min=1e-30)
    given = x.sum(dim=3)
    if c["k"]:
        s["t1_weight"] += given[..., :c["k"]]
    s["ring_weight"] += given[..., c["k"]:]
    return torch.matmul(x, v).reshape(B, L, Hq, d).to(torch.bfloat16)


def _evict_plain(s):
    c = s["case"]
    T, keep = c["T"], c["keep"]
    pos = s["pos"] if s["pos"] is not None else torch.full((c["B"],), T, dtype=torch.int64, device=DEV)
    n = pos.clamp(max=T)
    m = n.clamp(max=keep)
    age = torch.arange(T, device=DEV)
    row = (torch.where(pos > T, pos % T, 0)[:, None] + age) % T  # [B, T]: the i-th oldest token's row
    row = row[:, None, None].expand(s["weight"].shape)
    x = torch.gather(s["weight"], 3, row)
    young = (age >= (n - m.clamp(max=c["recent"]))[:, None])[:, None, None]
    x = torch.where(young, float("inf"), x)
    x = torch.where((age >= n[:, None])[:, None, None], float("-inf"), x)
    first = torch.sort(x, dim=-1, descending=True, stable=True).indices[..., :keep]
    live = torch.arange(keep, device=DEV) < m[:, None, None, None]
    first = torch.sort(torch.where(live, first, T), dim=-1).values
    row = torch.gather(row, 3, first.clamp(max=T - 1))
    s["out_weight"].copy_(torch.where(live, torch.gather(s["weight"], 3, row), s["out_weight"]))
    for to, x in ((s["out_k"], s["k"]), (s["out_v"], s["v"])):
        x = torch.gather(x, 3, row[..., None].expand(to.shape))
        to.copy_(torch.where(live[..., None], x, to))
    s["evicted"] += pos - m
    return (s["out_k"], s["out_v"], s["out_weight"], torch.where(live, row, -1).to(torch.int32), m,
            s["evicted"])


def _run_plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "evict":
        return _evict_plain(s)
    if kind in ("norm", "prefill"):
        T = c["T"]
        t = torch.arange(T, device=DEV)
        p = (7 + s["evicted"] + s["pos"])[:, None] + t
        q = _norm_rotate(s["q"].to(torch.float32), s["q_weight"], p).to(torch.bfloat16)
        k = _norm_rotate(s["k"].to(torch.float32), s["k_weight"], p).to(torch.bfloat16)
        if kind == "norm":
            return q, k
        W = c["W"]
        n = s["count"] if s["count"] is not None else torch.full((c["B"],), T, dtype=torch.int64, device=DEV)
        live = t < n[:, None]
        s["out_q"].copy_(torch.where(live[:, None, :, None, None], q, s["out_q"]))
        # the slot's last token: the largest t < n with (pos + t) mod W = slot
        slot = torch.arange(W, device=DEV)
        last = n[:, None] - 1 - (s["pos"][:, None] + n[:, None] - 1 - slot) % W
        put = (last >= 0)[:, None, None, :, None]
        b = torch.arange(c["B"], device=DEV)[:, None]
        for ring, x in ((s["ring_k"], k), (s["ring_v"], s["v"])):
            x = x[b, :, last.clamp(min=0)].permute(0, 2, 3, 1, 4)  # [B, W, L, Hkv, d] before
            ring.copy_(torch.where(put, x, ring))
        s["ring_weight"].masked_fill_(put[..., 0], 0.0)
        s["pos"] += n
        return s["out_q"], s["ring_k"], s["ring_v"], s["ring_weight"], s["pos"]
    q = s["q"].to(torch.float32)
    if kind == "attend":
        return _attend(s, q), s["t1_weight"], s["ring_weight"]
    p = (c["k"] + s["evicted"] + s["pos"])[:, None] if c["rope"] else None
    q = _norm_rotate(q[:, :, None], s["q_weight"], p)[:, :, 0]
    k_new = _norm_rotate(s["k_new"].to(torch.float32)[:, :, None], s["k_weight"], p)[:, :, 0]
    b = torch.arange(c["B"], device=DEV)
    slot = s["pos"] % c["W"]
    s["ring_k"][b, :, :, slot] = k_new.to(torch.bfloat16)
    s["ring_v"][b, :, :, slot] = s["v_new"]
    s["ring_weight"][b, :, :, slot] = 0.0
    s["pos"] += 1
    return _attend(s, q), s["t1_weight"], s["ring_k"], s["ring_v"], s["ring_weight"], s["pos"]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ----------------------------------------------------------------------------
# 64 bits, from the definition
# ----------------------------------------------------------------------------

def _exact_heads(x, w, p):
    """Norm and rotary embedding of x [B, L, T, H, d], pair by pair."""
    y = x.to(torch.float64)
    if w is not None:
        ms = torch.linalg.vector_norm(y, dim=-1, keepdim=True) ** 2 / x.shape[-1]
        y = y / torch.sqrt(ms + EPS) * w.to(torch.float64)[None, :, None, None, :]
    if p is None:
        return y
    h = x.shape[-1] // 2
    out = torch.empty_like(y)
    for i in range(h):
        turn = torch.polar(torch.ones(p.shape, dtype=torch.float64, device=DEV),
                           p.to(torch.float64) * ROPE_THETA ** (-i / h))[:, None, :, None]
        z = torch.complex(y[..., i], y[..., i + h]) * turn
        out[..., i], out[..., i + h] = z.real, z.imag
    return out


def _exact_attend(c, q, tiers, count):
    """Outputs and the weights' increments in 64 bits, one sequence and KV head at a time over all
    layers; `tiers`: (K, V) pairs, the last one the ring's."""
    B, L, Hq, d = q.shape
    G = c["G"]
    out = torch.zeros((B, L, Hq, d), dtype=torch.float64, device=DEV)
    given = torch.zeros((B, L, c["Hkv"], c["k"] + c["W"]), dtype=torch.float64, device=DEV)
    for b in range(B):
        n = int(count[b])
        for g in range(c["Hkv"]):
            K, V = (torch.cat([t[i][b, :, g] for t in tiers[:-1]] + [tiers[-1][i][b, :, g, :n]], dim=1)
                    .to(torch.float64) for i in range(2))
            w = torch.softmax(q[b, :, g * G:(g + 1) * G] @ K.transpose(1, 2) / math.sqrt(d), dim=-1)
            out[b, :, g * G:(g + 1) * G] = w @ V
            given[b, :, g, :c["k"] + n] = w.sum(dim=1)
    return out, given


def _exact_evict(c, s):
    """One unit at a time: a token's rank is the number of those that are kept before it."""
    B, L, Hkv, T, d = s["k"].shape
    keep = c["keep"]
    out = [s[x].to(torch.float64) for x in ("out_k", "out_v", "out_weight")]
    idx = torch.full((B, L, Hkv, keep), -1, dtype=torch.int64, device=DEV)
    pos = [T] * B if s["pos"] is None else s["pos"].tolist()
    left = []
    for b in range(B):
        n = min(pos[b], T)
        rows = [i % T for i in range(pos[b] - n, pos[b])] if pos[b] > T else list(range(n))
        rows = torch.tensor(rows, device=DEV)
        m = min(n, keep)
        young = min(c["recent"], m)
        left.append(m)
        old = n - young
        for x in range(L * Hkv):
            u = (b, x // Hkv, x % Hkv)
            w = s["weight"][u][rows[:old]].to(torch.float64)
            i = torch.arange(old, device=DEV)
            rank = torch.zeros(old, dtype=torch.int64, device=DEV)
            for j in range(0, old, 4096):
                part = w[j:j + 4096, None]
                rank += (part > w).sum(dim=0) + ((part == w) & (i[j:j + 4096, None] < i)).sum(dim=0)
            stay = rows[torch.cat([i[rank < m - young], torch.arange(old, n, device=DEV)])]
            for to, name in zip(out, ("k", "v", "weight")):
                to[u][:m] = s[name][u][stay].to(torch.float64)
            idx[u][:m] = stay
    left = torch.tensor(left, device=DEV)
    return (*out, idx.to(torch.int32), left, s["evicted"] + torch.tensor(pos, device=DEV) - left)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    kind = c["kind"]
    if kind == "evict":
        return _exact_evict(c, s)
    if kind in ("norm", "prefill"):
        first = 7 + s["evicted"] + s["pos"]
        p = first[:, None] + torch.arange(c["T"], device=DEV)[None]
        q, k = _exact_heads(s["q"], s["q_weight"], p), _exact_heads(s["k"], s["k_weight"], p)
        if kind == "norm":
            return q, k
        out, W = s["out_q"].to(torch.float64), c["W"]
        ring_k, ring_v, weight = (s[x].to(torch.float64) for x in ("ring_k", "ring_v", "ring_weight"))
        n = [c["T"]] * c["B"] if s["count"] is None else s["count"].tolist()
        for b, start in enumerate(s["pos"].tolist()):
            out[b, :, :n[b]] = q[b, :, :n[b]]
            t = torch.arange(max(0, n[b] - W), n[b], device=DEV)
            slot = (start + t) % W
            ring_k[b, :, :, slot] = k[b, :, t].transpose(1, 2)
            ring_v[b, :, :, slot] = s["v"][b, :, t].transpose(1, 2).to(torch.float64)
            weight[b, :, :, slot] = 0.0
        return out, ring_k, ring_v, weight, s["pos"] + torch.tensor(n, device=DEV)
    q, pos = s["q"].to(torch.float64), s["pos"]
    ring = [s["ring_k"].to(torch.float64), s["ring_v"].to(torch.float64)]
    ring_weight = s["ring_weight"].to(torch.float64)
    if kind == "step":
        p = (c["k"] + s["evicted"] + pos)[:, None] if c["rope"] else None
        q = _exact_heads(q[:, :, None], s["q_weight"], p)[:, :, 0]
        k_new = _exact_heads(s["k_new"][:, :, None], s["k_weight"], p)[:, :, 0]
        for b, n in enumerate(pos.tolist()):
            ring[0][b, :, :, n % c["W"]] = k_new[b]
            ring[1][b, :, :, n % c["W"]] = s["v_new"][b].to(torch.float64)
            ring_weight[b, :, :, n % c["W"]] = 0.0
        pos = pos + 1
    stored = (ring[0].to(torch.bfloat16), ring[1])  # the new token attends to itself as it is stored
    tiers = ([(s["t1_k"], s["t1_v"])] if c["k"] else []) + [stored]
    out, given = _exact_attend(c, q, tiers, pos.clamp(max=c["W"]))
    t1_weight = s["t1_weight"].to(torch.float64) + given[..., :c["k"]] if c["k"] else None
    ring_weight = ring_weight + given[..., c["k"]:]
    if kind == "attend":
        return out, t1_weight, ring_weight
    return out, t1_weight, *ring, ring_weight, pos
