"""Sizes of a 4-bit cache that 64 bits do not hold are refused, not cut off."""
import ctypes

import pytest

import paper_2402_14808_amd as ra
from paper_2402_14808_amd import binding
from test_abi import _params


def _size(**kw):
    block, total = ctypes.c_size_t(), ctypes.c_size_t()
    st = ra.load().relay_attn_fp4_cache_bytes(ctypes.byref(_params(**kw)), ctypes.byref(block), ctypes.byref(total))
    return st, block.value, total.value


@pytest.mark.parametrize("heads,blocks,bs,d", [(2**31 - 1, 2**31 - 1, 1 << 24, 128), (1 << 30, 1 << 30, 8, 64), (1 << 28, 1 << 20, 1 << 15, 128),
                                               (8, 1 << 31 >> 1, 1 << 24, 128), (1 << 16, 1 << 20, 1 << 20, 64), (1, 0, 16, 128)])
def test_sizes_around_64_bits(heads, blocks, bs, d):
    block = bs * (d // 2 + d // 32)
    want = block * heads * blocks
    st, one, all_ = _size(num_kv_heads=heads, num_blocks=blocks, block_size=bs, head_dim=d)
    if want < 2**64:
        assert (st, one, all_) == (binding.RA_OK, block, want)
    else:
        assert st == binding.RA_ERR_UNSUPPORTED
