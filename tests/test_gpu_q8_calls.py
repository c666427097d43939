"""The binding of the cache in 8 bits: arguments at the ends of their ranges, caches without a row, workspaces that
a call chooses itself, waits that run out."""

import numpy as np
import pytest
import torch

import paper_2609_25537_gb300 as cmc
from oracle import q8
from test_gpu_q8_range import check
from _gpu_helpers import to_f64

pytestmark = pytest.mark.gpu


def test_rotary_offsets_beyond_64_bits_are_refused(cuda_device):
    """As any offset outside [0, 2^32], in both decode steps; nothing is written."""
    bank = torch.ones(1, 1, 2, 40, 64, dtype=torch.bfloat16, device=cuda_device)
    q, row = bank[:, :, :, 0].repeat(1, 1, 2, 1), bank[:, :, :, 0].contiguous()
    pos = torch.tensor([3], device=cuda_device)
    ring = [bank.clone(), bank.clone()]
    ring8 = cmc.quantize_cache(bank, bank)
    for offset in (-1, 2 ** 32 + 1, 2 ** 63, 2 ** 64, 2 ** 64 + 5, -2 ** 64 + 7):
        with pytest.raises(cmc.CmcError, match="RANGE"):
            cmc.decode_step(q, bank, bank, None, *ring, pos, row, row, rope_theta=1e4, rope_offset=offset)
        with pytest.raises(cmc.CmcError, match="RANGE"):
            cmc.decode_step_q8(q, None, None, *ring8, pos, row, row, rope_theta=1e4, rope_offset=offset)
    assert pos.item() == 3 and torch.equal(ring[0], bank)
    cmc.decode_step_q8(q, None, None, *ring8, pos, row, row, rope_theta=1e4, rope_offset=2 ** 32)
    assert pos.item() == 4


def test_a_cache_without_rows_is_read_back(cuda_device):
    """As any other: whole, by an index of no rows, and quantised again; but no row can be taken from it."""
    bank = torch.zeros(2, 1, 3, 5, 64, dtype=torch.bfloat16, device=cuda_device)
    none = torch.empty(2, 0, dtype=torch.int32, device=cuda_device)
    kv, scales = cmc.quantize_cache(bank, bank, none)
    assert kv.shape == (2, 1, 3, 2, 0, 64) and scales.shape == (2, 1, 3, 2, 0)
    for idx in (None, none):
        k, v = cmc.dequantize_cache(kv, scales, idx)
        assert k.shape == v.shape == (2, 1, 3, 0, 64) and k.dtype == torch.bfloat16
        again, powers = cmc.quantize_cache(k, v, idx)
        assert again.shape == kv.shape and powers.shape == scales.shape
    one = torch.zeros(2, 1, dtype=torch.int32, device=cuda_device)
    for call in (lambda: cmc.dequantize_cache(kv, scales, one), lambda: cmc.quantize_cache(k, v, one)):
        with pytest.raises(cmc.CmcError, match="SHAPE"):
            call()


# form: B, L, Hkv, G, d, k, W, grid
STALLED = {
    "cluster": (1, 1, 8, 4, 128, 2048, 2048, 64),
    "cta": (29, 1, 8, 4, 128, 256, 512, 232),
    "three CTAs an SM": (39, 1, 8, 4, 128, 256, 512, 312),
    "longest first": (64, 1, 8, 2, 128, 32, 480, 512),
    "a warp a unit": (150, 1, 8, 2, 128, 64, 256, 300),
    "several units a warp": (8, 32, 8, 4, 128, 30, 130, 304),
}


class stalled:
    """Within it every stage's wait runs out."""

    def __enter__(self):
        cmc.lib().cmc_test_stall_attention_waits(1)

    def __exit__(self, *_):
        cmc.lib().cmc_test_stall_attention_waits(0)


def step_problem(dev, B, L, H, G, d, k, W, seed):
    g = torch.Generator(device=dev).manual_seed(seed)

    def rand(*shape):
        return torch.randn(shape, generator=g, device=dev).to(torch.bfloat16)
    t1 = cmc.quantize_cache(rand(B, L, H, k, d), rand(B, L, H, k, d))
    ring = cmc.quantize_cache(rand(B, L, H, W, d), rand(B, L, H, W, d))
    pos = W + torch.arange(B, device=dev) * 7
    return [rand(B, L, G * H, d), *t1, *ring, pos, rand(B, L, H, d), rand(B, L, H, d)]


@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("form", STALLED)
def test_a_step_after_one_that_timed_out(cuda_device, form, given):
    """The counters of the workspace are zero again, every position was advanced once, and the next step with
    the same workspace, given or the call's own, is right without its being cleared."""
    B, L, H, G, d, k, W, grid = STALLED[form]
    dims = cmc.CmcDims(B, L, G * H, H, d, k, k, W)
    assert cmc.decode_attn_q8_plan(dims) == grid
    args = step_problem(cuda_device, B, L, H, G, d, k, W, 1)
    before = [x.clone() for x in args]
    ws = cmc.DecodeWorkspace(dims, cuda_device, q8=True) if given else None
    cmc.decode_step_q8(*args, workspace=ws)  # the call's own exists from here on
    for x, y in zip(args, before):
        x.copy_(y)
    torch.cuda.synchronize()
    with stalled():
        cmc.decode_step_q8(*args, workspace=ws)
        torch.cuda.synchronize()
    assert torch.equal(args[5], before[5] + 1)
    if given:
        assert ws.status() & cmc.DEVFLAG_TIMEOUT
        assert not ws.buf.any()
    for x, y in zip(args, before):
        x.copy_(y)
    got = cmc.decode_step_q8(*args, workspace=ws)
    torch.cuda.synchronize()
    ring, t1 = ([x.view(torch.uint8).cpu().numpy() for x in before[i:i + 2]] for i in (3, 1))
    pos = before[5].cpu().numpy()
    q8.append(*ring, pos, *(to_f64(x) for x in before[6:]))
    assert np.array_equal(args[5].cpu().numpy(), pos)
    for x, y in zip(args[3:5], ring):
        np.testing.assert_array_equal(x.view(torch.uint8).cpu().numpy(), y)
    if L == 1:
        check(got, before[0].cpu(), t1, ring, range(3), form)
    if given:
        assert ws.status() == 0


def test_flags_of_calls_without_a_workspace(cuda_device):
    """Of all of a device, on any stream and of any batch size, until they are cleared."""
    cmc.decode_q8_status()
    assert cmc.decode_q8_status(cuda_device) == 0
    one, two = (step_problem(cuda_device, B, 1, 2, 2, 64, 32, 64, 2) for B in (1, 3))
    one[5].fill_(-4)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        cmc.two_tier_decode_attn_q8(*one[:6])
    with stalled():
        cmc.decode_step_q8(*two)
        torch.cuda.synchronize()
    both = cmc.DEVFLAG_BAD_POS | cmc.DEVFLAG_TIMEOUT
    assert cmc.decode_q8_status("cuda", clear=False) == both
    assert cmc.decode_q8_status() == both
    assert cmc.decode_q8_status() == 0
    cmc.decode_step_q8(*two)
    assert cmc.decode_q8_status() == 0


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N,by_index", [(70, False), (70, True), (3000, False)])
def test_quantising_reports_a_wait_that_ran_out(cuda_device, d, N, by_index):
    """With one stage a warp and with two (more blocks than one wave takes); the next call is right."""
    bank = torch.randn(4, 4, 8, N, d, device=cuda_device).to(torch.bfloat16)
    idx = torch.arange(N - 1, -1, -1, dtype=torch.int32, device=cuda_device).repeat(4, 1) if by_index else None
    want = [x.clone().view(torch.uint8) for x in cmc.quantize_cache(bank, bank, idx)]
    ws = cmc.DecodeWorkspace(cmc.CmcDims(4, 1, 8, 8, d, 1, 0, 1), cuda_device, q8=True)
    torch.cuda.synchronize()
    with stalled():
        cmc.quantize_cache(bank, bank, idx, workspace=ws)
        flags = ws.status()
    assert flags == cmc.DEVFLAG_TIMEOUT
    for x, y in zip(cmc.quantize_cache(bank, bank, idx, workspace=ws), want):
        assert torch.equal(x.view(torch.uint8), y)
    assert ws.status() == 0


def test_a_workspace_elsewhere_is_refused(cuda_device):
    """On the host, whose memory a kernel cannot count on reaching; nothing is written."""
    q, *t1, kv, scales, pos, k_new, v_new = step_problem(cuda_device, 2, 1, 2, 2, 64, 32, 64, 3)
    before = [x.clone() for x in (kv, scales, pos)]
    ws = cmc.DecodeWorkspace(cmc.CmcDims(2, 1, 4, 2, 64, 32, 32, 64), torch.device("cpu"))
    first = torch.zeros(2, 1, dtype=torch.int32, device=cuda_device)
    bank = torch.zeros(2, 1, 2, 5, 64, dtype=torch.bfloat16, device=cuda_device)
    for call in (lambda: cmc.quantize_cache(bank, bank, workspace=ws),
                 lambda: cmc.dequantize_cache(kv, scales, workspace=ws),
                 lambda: cmc.two_tier_decode_attn_q8(q, *t1, kv, scales, pos, workspace=ws),
                 lambda: cmc.decode_step_q8(q, *t1, kv, scales, pos, k_new, v_new, workspace=ws),
                 # and in the calls over a bf16 cache
                 lambda: cmc.tier1_gather(bank, bank, first, workspace=ws),
                 lambda: cmc.two_tier_decode_attn(q, bank, bank, None, bank, bank, pos, workspace=ws),
                 lambda: cmc.decode_step(q, bank, bank, None, bank, bank, pos, k_new, v_new, workspace=ws)):
        with pytest.raises(ValueError, match="workspace is on cpu"):
            call()
    torch.cuda.synchronize()
    for x, y in zip((kv, scales, pos), before):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    assert not ws.buf.any()
