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


def step_inputs(dev, case, form, seed):
    """Arguments of a step of one form, and its queries as the formula prepares them."""
    B, L, H, G, d, k, W, _ = case
    q, t1, ring, pos, g = attention_problem(dev, case, seed, poison=False)
    q.view(B, L, H, G, d)[:] = q.view(B, L, H, G, d)[:, :, :, :1].clone()  # the heads of a KV head alike
    new = [randn(g, B, L, H, d), randn(g, B, L, H, d)]
    opts, qw, p = {}, None, None
    if form in ("norm", "both"):
        qw, kw = (1 + 0.5 * torch.randn(L, d, generator=g, device=dev) for _ in range(2))
        opts.update(q_weight=qw, k_weight=kw, eps=1e-5)
    if form in ("rope", "both"):
        opts.update(rope_theta=THETA, rope_offset=0)
        p = ow.positions(f64(pos), None, 0, 1)
    return q, t1, ring, pos, new, opts, f64(q) if form == "plain" else prepared_queries(q, qw, 1e-5, p)


@pytest.mark.parametrize("form", ["plain", "norm", "rope", "both"])
@pytest.mark.parametrize("G, d", [(1, 64), (4, 128), (8, 64)])
@pytest.mark.parametrize("unit", ["a CTA", "a cluster", "a warp"])
def test_keys_of_a_step_that_are_not_finite(cuda_device, unit, G, d, form):
    """A key whose score is minus infinity counts nothing, whatever norm and rotation make of the query; one of plus infinity
    or NaN gives NaN in its KV head's outputs and weights, and leaves the others as they were."""
    B, H, k = PLACES[unit]
    case = (B, 1, H, G, d, k, 70, [0, 69, 70, 30, 500])
    q, t1, ring, pos, new, opts, qq = step_inputs(cuda_device, case, form, 41)
    start = [x.clone() for x in (*t1, *ring, pos)]

    def run(change):
        x = [y.clone() for y in start]
        change(x)
        out = cmc.decode_step_weighted(q, *x, *new, **opts)
        return out, x

    want, clean = run(lambda x: None)
    # sequences 0 (position 0, where a rotation leaves the query as it is) and 1, a few elements of the query each
    spots = [(b, row, i) for b in (0, 1) for row, i in zip(range(5, 13), range(3, d, d // 8))]

    def infinite(sign):
        def change(x):
            for b, row, i in spots:
                x[0][b, 0, 0, row, i] = sign * float("inf") * (1 if qq[b, 0, 0, i] > 0 else -1)
        return change
    out, x = run(infinite(-1.0))
    assert not out.isnan().any() and not x[2].isnan().any() and not x[5].isnan().any()
    rows = f64(start[0])
    for b, row, i in spots:  # as good as no key: a score of -200
        rows[b, 0, 0, row] = -200 * math.sqrt(d) * qq[b, 0, 0] / (qq[b, 0, 0] ** 2).sum()
        assert x[2][b, 0, 0, row] == start[2][b, 0, 0, row]
    before = [rows] + [f64(y) for y in start[1:3]]
    left = [f64(y) for y in x[3:6]]
    w = f64(start[5])
    n = f64(start[6])
    for b in range(B):
        w[b, :, :, int(n[b] % 70)] = 0.0
    check_attention(out, x[2], x[5], qq, before, left[:2] + [w], n + 1, 1 / math.sqrt(d), prepared=form != "plain")

    def nan(x):
        for b in (0, 1):
            x[0][b, 0, 0, 7, 11] = float("nan")
    for change in (infinite(1.0), nan):
        out, x = run(change)
        for b in (0, 1):
            assert out[b, 0, :G].isnan().all() and x[2][b, 0, 0].isnan().all()
            live = min(int(x[6][b]), 70)
            assert x[5][b, 0, 0, :live].isnan().all() and not x[5][b, 0, 0, live:].isnan().any()
            assert torch.equal(out[b, 0, G:], want[b, 0, G:]) and torch.equal(x[2][b, 0, 1:], clean[2][b, 0, 1:])
            assert torch.equal(x[5][b, 0, 1:], clean[5][b, 0, 1:])
        assert torch.equal(out[2:], want[2:]) and torch.equal(x[2][2:], clean[2][2:]) and torch.equal(x[5][2:], clean[5][2:])


def test_eviction_refuses_outputs_that_meet(cuda_device):
    k = torch.zeros(2, 1, 2, 10, 64, dtype=torch.bfloat16, device=cuda_device)
    v, w = k.clone(), torch.zeros(2, 1, 2, 10, device=cuda_device)
    pos = torch.full((2,), 10, device=cuda_device)
    a, b, c = k[..., :6, :].contiguous(), v[..., :6, :].contiguous(), w[..., :6].contiguous()
    for kw in (dict(out_k=a, out_v=a, out_weight=c), dict(out_k=k, out_v=v, out_weight=k.view(torch.float32).view(-1)[:40].view(2, 1, 2, 10)),
               dict(evicted=pos), dict(out_pos=c.view(torch.int64).view(-1)[:2], out_k=a, out_v=b, out_weight=c)):
        with pytest.raises(cmc.CmcError, match="RANGE"):
            cmc.evict_cache(k, v, w, 5, pos=pos, **kw)
    # K that is V too: moved together in place
    k.copy_(torch.arange(10, device=cuda_device, dtype=torch.bfloat16)[:, None].expand(k.shape))
    w[..., [1, 4, 5, 8]] = 1.0
    cmc.evict_cache(k, k, w, 4, pos=pos, out_k=k, out_v=k, out_weight=w, out_pos=pos)
    assert pos.tolist() == [4, 4] and k[0, 0, 0, :4, 0].tolist() == [1.0, 4.0, 5.0, 8.0]


@pytest.mark.parametrize("unit", list(PLACES))
@pytest.mark.parametrize("prepared", [False, True])
def test_outputs_in_the_queries_place(cuda_device, unit, prepared):
    """The one overlap that is allowed, in every variant; others are refused and change nothing."""
    B, H, k = PLACES[unit]
    form = "both" if prepared else "plain"
    q, t1, ring, pos, new, opts, _ = step_inputs(cuda_device, (B, 1, H, 4, 64, k, 70, list(range(70))), form, 42)
    state = [x.clone() for x in (*t1, *ring, pos)]
    want = cmc.decode_step_weighted(q, *state, *new, **opts)
    args = [*t1, *ring, pos]
    before = [x.clone() for x in args]
    inside = ring[0].view(-1)[:q.numel()].view(q.shape)
    for change in (dict(out=inside), dict(out=t1[1].view(-1)[:q.numel()].view(q.shape))):
        with pytest.raises(cmc.CmcError, match="RANGE"):
            cmc.decode_step_weighted(q, *args, *new, **opts, **change)
    for x, y in zip(args, before):
        assert torch.equal(x, y)
    got = cmc.decode_step_weighted(q, *args, *new, out=q, **opts)
    assert got is q and torch.equal(got, want)
    for x, y in zip(args, state):
        assert torch.equal(x, y)


@pytest.mark.parametrize("form", ["norm", "rope", "both"])
@pytest.mark.parametrize("d", [64, 128])
def test_a_token_has_the_same_key_prefilled_and_stepped(cuda_device, d, form):
    """Bit for bit, in each variant of the step, and as qk_norm_rope gives it."""
    for B, H, k in PLACES.values():
        q, t1, ring, pos, g = attention_problem(cuda_device, (B, 3, H, 1, d, k, 70, [0, 3, 10 ** 6, 69, 2 ** 33]), 43, poison=False)
        k_new, v_new = randn(g, B, 3, H, d, scale=2.0), randn(g, B, 3, H, d)
        opts = {}
        if form in ("norm", "both"):
            opts.update(q_weight=1 + torch.randn(3, d, generator=g, device=cuda_device), k_weight=1 + torch.randn(3, d, generator=g, device=cuda_device))
        if form in ("rope", "both"):
            opts.update(rope_theta=THETA, rope_offset=k)
        other = [x.clone() for x in (ring[0], ring[1], pos)]
        _, key = cmc.qk_norm_rope(q, k_new, pos, **opts)
        cmc.window_prefill(None, k_new, v_new, *other, **opts)
        cmc.decode_step_weighted(q, *t1, *ring, pos, k_new, v_new, **opts)
        for x, y in zip(other, (ring[0], ring[1], pos)):
            assert torch.equal(x, y)
        slot = ((pos - 1) % 70).tolist()
        assert torch.equal(key, torch.stack([ring[0][b, :, :, s] for b, s in enumerate(slot)]))


@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-6, 1e3])
@pytest.mark.parametrize("d", [64, 128])
def test_norms_of_rows_of_any_magnitude(cuda_device, d, eps):
    """Rows whose squares fp32 does not hold, from bf16's smallest values to its largest, alone and next to small elements; the
    same bits from all three calls."""
    g = gen(cuda_device, 44)
    B, T, H = 3, 40, 7
    x = torch.randn(B, 1, T, H, d, generator=g, device=cuda_device, dtype=torch.float64).clamp(-3.9, 3.9)
    size = torch.randint(-133, 126, (B, 1, T, H, 1), generator=g, device=cuda_device)
    size[0, 0, :16, 0, 0] = torch.tensor([-133, -132, -127, -126, -100, -64, -63, -62, -48, -45, 58, 59, 63, 64, 120, 125], device=cuda_device)
    size[1, :, :, 0] = size[1, :, :, 0].clamp(min=-60)
    x = x * torch.exp2(size.double())
    x[1, :, :, 0] *= torch.exp2(-60.0 * torch.rand(T, d, generator=g, device=cuda_device).double())  # elements far apart
    x[2, :, 3, 1], x[2, :, 4, 1] = 3.3895313892515355e38, -9.183549615799121e-41  # the largest and the smallest
    x[2, :, 5, 1] = 0.0
    x[2, :, 5, 1, 7] = 3.3895313892515355e38
    x = x.to(torch.bfloat16)
    assert x.isfinite().all()
    pos = torch.tensor([0, 5, 10 ** 6], device=cuda_device)
    kw = 1 + 0.5 * torch.rand(1, d, generator=g, device=cuda_device)
    opts = dict(q_weight=kw, k_weight=kw, eps=eps)
    heads = f64(x)
    if eps == 0.0:  # rows without a value have no norm
        assert (heads != 0).any(-1).all()
    for rope in ({}, dict(rope_theta=THETA)):
        p = ow.positions(f64(pos), None, 0, T) if rope else None
        oq, ok = cmc.qk_norm_rope(x, x, pos, **opts, **rope)
        check_heads(ok, heads, kw, p, "norm", eps=eps)
        assert torch.equal(oq, ok)
        place = [x.clone(), x.clone()]
        cmc.qk_norm_rope(*place, pos, out_q=place[0], out_k=place[1], **opts, **rope)
        assert torch.equal(place[0], ok) and torch.equal(place[1], ok)
        place = x.clone()
        cmc.window_prefill(place, x, x, *(torch.zeros(B, 1, H, T, d, dtype=torch.bfloat16, device=cuda_device) for _ in range(2)),
                           pos.clone(), out_q=place, **opts, **rope)
        assert torch.equal(place, oq)
        ring = [torch.zeros(B, 1, H, T, d, dtype=torch.bfloat16, device=cuda_device) for _ in range(2)]
        at = pos.clone()
        cmc.window_prefill(None, x, x, *ring, at, **opts, **rope)
        for b in range(B):
            slots = (pos[b] + torch.arange(T, device=cuda_device)) % T
            assert torch.equal(ring[0][b, :, :, slots], ok[b].transpose(1, 2)) and torch.equal(ring[1][b, :, :, slots], x[b].transpose(1, 2))
        w = torch.zeros(B, 1, H, T, device=cuda_device)
        ring = [torch.zeros_like(y) for y in ring]
        at = pos.clone()
        for t in range(T):
            row = x[:, :, t].contiguous()
            cmc.decode_step_weighted(row, None, None, None, *ring, w, at, row, torch.zeros_like(row), **opts, **rope)
        for b in range(B):
            slots = (pos[b] + torch.arange(T, device=cuda_device)) % T
            assert torch.equal(ring[0][b, :, :, slots], ok[b].transpose(1, 2))
    # a norm of the queries alone: keys and values of any magnitude are left as they are
    oq, ok = cmc.qk_norm_rope(x, x, pos, q_weight=kw, eps=eps)
    check_heads(oq, heads, kw, None, "queries", eps=eps)
    assert torch.equal(ok, x)


@pytest.mark.parametrize("unit", list(PLACES))
@pytest.mark.parametrize("G, d", [(1, 64), (4, 128), (8, 64)])
def test_finite_scores_of_any_size(cuda_device, unit, G, d):
    """Scores of 2^33 and more, exact in fp32: all goes to the largest, a half each to two that are equal."""
    B, H, k = PLACES[unit]
    g = gen(cuda_device, 45)
    q = torch.zeros(B, 1, H * G, d, dtype=torch.bfloat16, device=cuda_device)
    q[..., 9] = 2.0 ** 20
    q[..., 9] *= torch.tensor([1.0, -1.0, 1.0, 2.0 ** 30], device=cuda_device).repeat(H * G)[:H * G]
    size = torch.randint(-200, 200, (B, 1, H, k + 70), generator=g, device=cuda_device)
    size[..., 3], size[..., k - 4] = 250, -250
    size[:, :, :, k + 8] = size[:, :, :, 3]  # (slots 0 to 9 of the ring are occupied)
    keys = torch.zeros(B, 1, H, k + 70, d, dtype=torch.bfloat16, device=cuda_device)
    keys[..., 9] = size * 2.0 ** 20
    values = torch.randint(-60, 60, keys.shape, generator=g, device=cuda_device).to(torch.bfloat16)
    w = torch.rand(B, 1, H, k + 70, generator=g, device=cuda_device).round(decimals=1)
    pos = torch.full((B,), 10, device=cuda_device)
    parts = [[x[:, :, :, :k].contiguous(), x[:, :, :, k:].contiguous()] for x in (keys, values, w)]
    out = cmc.two_tier_decode_attn_weighted(q, *(x[0] for x in parts), *(x[1] for x in parts), pos)
    up = ((values[:, :, :, 3].float() + values[:, :, :, k + 8].float()) / 2).to(torch.bfloat16)
    down = values[:, :, :, k - 4]
    sign = q[..., 9].view(B, 1, H, G, 1) > 0
    assert torch.equal(out.view(B, 1, H, G, d), torch.where(sign, up[:, :, :, None], down[:, :, :, None]))
    given = torch.zeros_like(w)
    given[..., 3] = given[..., k + 8] = 0.5 * sign.sum((3, 4))
    given[..., k - 4] = (~sign).sum((3, 4))
    assert torch.equal(torch.cat([parts[2][0], parts[2][1]], dim=-1), w + given)


def long_units(dev, W, seed, B=1, H=160, poison=True):
    """Units whose products go to the workspace (G = 8, d = 64: more than 9,216 keys, and more CTAs than an SM each)."""
    case = (B, 1, H, 8, 64, 40, W, [W + 5])
    dims = cmc.CmcDims(B, 1, 8 * H, H, 64, 40, 40, W)
    assert cmc.decode_attn_weighted_plan(dims) > torch.cuda.get_device_properties(dev).multi_processor_count
    assert cmc.decode_attn_weighted_workspace_size(dims) > 36 * B * H * W
    return attention_problem(dev, case, seed, poison)[:4], dims


def test_workspaces_of_long_units_do_not_pile_up(cuda_device):
    """One for each batch size and stream, as large as the longest has asked for; its flags are those of all calls."""
    stream = torch.cuda.Stream()
    cmc.weighted_cache_status()
    with torch.cuda.stream(stream):
        before = torch.cuda.memory_allocated()
        for W in (10240, 9500, 9984, 10200, 9300):
            (q, t1, ring, pos), dims = long_units(cuda_device, W, 46, H=24)
            pos.fill_(-1 if W == 9984 else W)
            cmc.two_tier_decode_attn_weighted(q, *t1, *ring, pos)
            size = cmc.decode_attn_weighted_workspace_size(dims)
            most = max(size, most) if W != 10240 else size
            del q, t1, ring, pos
        stream.synchronize()
        assert torch.cuda.memory_allocated() - before <= most + (1 << 20)
        # a larger one after a flag, and the right results in it
        (q, t1, ring, pos), dims = long_units(cuda_device, 10400, 47, H=24)
        given = [x.clone() for x in (*t1, *ring)]
        out = cmc.two_tier_decode_attn_weighted(q, *t1, *ring, pos)
        ws = cmc.DecodeWorkspace(dims, cuda_device, weighted=True)
        want = cmc.two_tier_decode_attn_weighted(q, *given, pos, workspace=ws)
        assert torch.equal(out, want) and torch.equal(t1[2], given[2]) and torch.equal(ring[2], given[5])
    assert cmc.weighted_cache_status() == cmc.DEVFLAG_BAD_POS and cmc.weighted_cache_status() == 0


def test_a_captured_call_finds_anything_behind_its_counters(cuda_device):
    """Its own workspace: the flags and counters are zeroed at every replay, the products' place holds what was there."""
    (q, t1, ring, pos), dims = long_units(cuda_device, 9300, 48, H=24)
    state = [x.clone() for x in (*t1, *ring, pos)]
    new = [torch.ones(1, 1, 24, 64, dtype=torch.bfloat16, device=cuda_device) for _ in range(2)]
    want = cmc.decode_step_weighted(q, *state, *new)
    out = torch.empty_like(q)
    start = [x.clone() for x in (*t1, *ring, pos)]
    args = [*t1, *ring, pos]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        for _ in range(2):
            bad = torch.full((cmc.decode_attn_weighted_workspace_size(dims) // 4,), float("nan"), device=cuda_device)
            del bad
        cmc.decode_step_weighted(q, *args, *new, out=out)
    for _ in range(3):
        for x, y in zip(args, start):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        for x, y in zip(args, state):
            assert torch.equal(x, y)


# B, L, Hkv, G, d, k, W, positions: units too long for shared memory, on more CTAs than SMs (of which a unit takes eight), so that their
# products and weights go to the workspace; the last two on so many that the longest sequences start first
LONG = {"G 8": (9, 1, 4, 8, 64, 300, 9000, [8999, -1, 0, 40, 9000, 9001, 5000, 31, 2 ** 33 + 7]),
        "G 4": (5, 1, 4, 4, 128, 33, 18432, [18431, -7, 18500, 100, 0]),
        "G 2": (3, 7, 1, 2, 64, 0, 30721, [30720, 11, 30721]), "G 1": (5, 1, 4, 1, 64, 46000, 100, [99, 0, 100, -1, 65]),
        "G 8, ordered": (16, 2, 2, 8, 128, 40, 9200, [9199, 17, 9200, -1, 4000]), "G 4, ordered": (60, 1, 1, 4, 64, 18000, 500, [499, 0, -3, 500, 77])}


@pytest.mark.parametrize("prepared", [False, True])
@pytest.mark.parametrize("name", list(LONG))
def test_steps_of_units_whose_products_go_to_the_workspace(cuda_device, name, prepared):
    case = LONG[name]
    B, L, H, G, d, k, W, positions = case
    sms = torch.cuda.get_device_properties(cuda_device).multi_processor_count
    dims = cmc.CmcDims(B, L, H * G, H, d, max(k, 1), k, W)
    ctas = cmc.decode_attn_weighted_plan(dims)
    assert ctas == 8 * B * L * H and ctas > sms * (3 if "ordered" in name else 1)
    head = int(cmc.lib().cmc_cache_workspace_size(B))
    assert cmc.decode_attn_weighted_workspace_size(dims) >= head + 4 * (G + 1) * B * L * H * (k + W)
    ws = cmc.DecodeWorkspace(dims, cuda_device, weighted=True)
    ws.buf[head:] = 255  # NaN: nothing is read there that the call has not written
    check_step(cuda_device, case, prepared, 49, workspace=ws)
    assert ws.status() == (cmc.DEVFLAG_BAD_POS if min(positions) < 0 else 0) and not ws.buf[256:head].any()
