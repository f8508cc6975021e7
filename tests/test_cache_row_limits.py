"""Tokens with more pieces than a workgroup counts are refused (their number passed 32 bits, and the launch divided by it)."""
import ctypes

import pytest

import paper_2402_14808_amd as ra
from paper_2402_14808_amd import binding
from test_abi import FAKE, _params
from test_fp4_abi import _rows

V = ctypes.c_void_p


def _bf16(p, k_new=FAKE):
    return ra.load().relay_attn_cache_append(ctypes.byref(p), V(k_new), V(FAKE), 128, 128, None, 1, V(FAKE), V(FAKE), V(FAKE), V(FAKE), None)


@pytest.mark.parametrize("heads,d", [(1 << 28, 128), (1 << 27, 128), ((1 << 26) + 1, 128), (1 << 28, 64)])
def test_rows_of_too_many_heads(heads, d):
    p = _params(batch=1, num_q_heads=heads, num_kv_heads=heads, head_dim=d)
    assert _bf16(p) == binding.RA_ERR_UNSUPPORTED
    for name in ("relay_attn_cache_append_fp4", "relay_attn_cache_read_fp4"):
        assert _rows(name, p, n=1, st=0, sh=d, slots=FAKE) == binding.RA_ERR_UNSUPPORTED


def test_the_most_heads_are_not_refused_for_their_number():
    p = _params(batch=1, num_q_heads=1 << 26, num_kv_heads=1 << 26)          # (an address that is refused behind it)
    assert _bf16(p, k_new=FAKE + 2) == binding.RA_ERR_INVALID_ARG
    assert _rows("relay_attn_cache_append_fp4", p, a=FAKE + 2, n=1, st=0, slots=FAKE) == binding.RA_ERR_INVALID_ARG
