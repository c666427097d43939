"""The binding of the cache in 8 bits: arguments at the ends of their ranges, caches without a row, workspaces that
a call chooses itself, waits that run out."""

import pytest
import torch

import paper_2609_25537_gb300 as cmc

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
