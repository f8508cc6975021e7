"""Refusals of the calls around the 4-bit cache and the block tables: on the host, before any HIP call."""
import ctypes

import pytest
import torch

import paper_2402_14808_amd as ra
from paper_2402_14808_amd import binding
from test_abi import FAKE, _params

V = ctypes.c_void_p
BAD, NOT_HERE, OK = binding.RA_ERR_INVALID_ARG, binding.RA_ERR_UNSUPPORTED, binding.RA_OK


def _rows(name, p, a=FAKE, b=FAKE, st=2 * 128, sh=128, cu=FAKE, n=9, slots=None, kc=FAKE, vc=FAKE, bt=FAKE, cl=FAKE):
    return getattr(ra.load(), name)(ctypes.byref(p) if p else None, V(a), V(b), st, sh, V(cu), n, V(slots), V(kc), V(vc),
                                    V(bt), V(cl), None)


@pytest.mark.parametrize("name", ["relay_attn_cache_append_fp4", "relay_attn_cache_read_fp4"])
def test_rows_in_and_out_refuse(name):
    p = _params()
    assert _rows(name, None) == BAD
    for kw in (dict(a=None), dict(b=None), dict(kc=None), dict(vc=None), dict(bt=None), dict(cl=None), dict(a=FAKE + 2),
               dict(b=FAKE + 8), dict(kc=FAKE + 4), dict(vc=FAKE + 1), dict(st=-8), dict(st=12), dict(sh=4), dict(sh=64),
               dict(n=-1), dict(cu=None), dict(slots=FAKE, a=None)):
        assert _rows(name, p, **kw) == BAD, kw
    for kw in (dict(block_size=4, max_blocks_per_seq=128), dict(block_size=1, max_blocks_per_seq=128), dict(head_dim=96), dict(num_q_heads=18)):
        assert _rows(name, _params(**kw)) == NOT_HERE, kw
    assert _rows(name, _params(batch=0), n=3) == BAD
    assert _rows(name, p, n=0) == OK
    assert _rows(name, p, n=0, a=None, kc=None, bt=None) == OK


def test_read_refuses_rows_on_top_of_each_other():
    for st, sh in ((0, 128), (64, 128), (128, 128), (248, 128), (128, 8 * 128 + 120)):      # 9 tokens of 2 heads of 128
        assert _rows("relay_attn_cache_read_fp4", _params(), st=st, sh=sh) == BAD, (st, sh)


def test_rows_want_to_know_how_many_blocks_there_are():
    for name in ("relay_attn_cache_append_fp4", "relay_attn_cache_read_fp4"):
        assert _rows(name, _params(num_blocks=0)) == BAD
        assert _rows(name, _params(num_blocks=0), slots=FAKE) == BAD
        assert _rows(name, _params(block_size=1 << 25, max_blocks_per_seq=4)) == NOT_HERE


def _attend(p, prefill, q=FAKE, ks=FAKE, vs=FAKE, kc=FAKE, vc=FAKE, bt=FAKE, cl=FAKE, out=FAKE, ws=FAKE, ws_bytes=1 << 40,
            cu=FAKE, n=9, most=5):
    lib = ra.load()
    args = [V(ks), V(vs), V(kc), V(vc), V(bt), V(cl), V(out), None, V(ws), ws_bytes, None]
    pp = ctypes.byref(p) if p else None
    return lib.relay_attn_prefill_fp4(pp, V(q), V(cu), n, most, *args) if prefill else lib.relay_attn_decode_fp4(pp, V(q), *args)


@pytest.mark.parametrize("prefill", [False, True])
def test_attention_refuses_what_the_bf16_calls_refuse_and_small_blocks(prefill):
    p = _params()
    assert _attend(None, prefill) == BAD
    for kw in (dict(q=None), dict(ks=None), dict(vs=None), dict(kc=None), dict(vc=None), dict(bt=None), dict(cl=None),
               dict(out=None), dict(q=FAKE + 2), dict(kc=FAKE + 8), dict(ws=None), dict(ws=FAKE + 16)):
        assert _attend(p, prefill, **kw) == BAD, kw
    assert _attend(p, prefill, ws_bytes=0) == binding.RA_ERR_WORKSPACE_TOO_SMALL
    for bs in (1, 2, 4):
        assert _attend(_params(block_size=bs, max_blocks_per_seq=128), prefill) == NOT_HERE
    assert _attend(_params(block_size=1 << 25, max_blocks_per_seq=4), prefill) == NOT_HERE
    assert _attend(_params(reserved0=7), prefill) == BAD
    if prefill:
        assert _attend(p, True, cu=None) == BAD and _attend(p, True, most=1) == BAD and _attend(p, True, n=-1) == BAD
        assert _attend(p, True, n=0, most=0) == OK
    else:
        assert _attend(_params(batch=0), False) == OK


def test_cache_bytes():
    assert ra.fp4_cache_shape(10, 8, 16, 128) == (10, 8, 16 * 68)
    assert ra.fp4_cache_shape(0, 1, 8, 64) == (0, 1, 8 * 34)
    block, total = ctypes.c_size_t(), ctypes.c_size_t()
    call = lambda p, a=ctypes.byref(block), b=ctypes.byref(total): ra.load().relay_attn_fp4_cache_bytes(p, a, b)  # noqa: E731
    assert call(ctypes.byref(_params(num_blocks=2**31 - 1, num_kv_heads=8))) == OK
    assert total.value == block.value * 8 * (2**31 - 1)
    assert call(None) == BAD and call(ctypes.byref(_params()), None) == BAD
    assert call(ctypes.byref(_params(num_kv_heads=0))) == BAD and call(ctypes.byref(_params(block_size=12))) == BAD
    assert call(ctypes.byref(_params(head_dim=96))) == NOT_HERE and call(ctypes.byref(_params(block_size=4))) == NOT_HERE
    with pytest.raises(ra.RelayAttnError):
        ra.fp4_cache_shape(1, 1, 4, 128)


def test_make_params_reads_the_block_size_off_a_4_bit_cache():
    q = torch.zeros((3, 8, 128), dtype=torch.bfloat16)
    k = torch.zeros(ra.fp4_cache_shape(5, 2, 32, 128), dtype=torch.uint8)
    p = ra.make_params(q, q, None, k, torch.zeros((3, 4), dtype=torch.int32), batch=3, softmax_scale=1.0)
    assert (p.block_size, p.num_blocks, p.num_kv_heads) == (32, 5, 2)


def _tables(p, old=FAKE, new=FAKE + 256, pin=FAKE + 512, pout=FAKE + 1024, free=FAKE, bt=FAKE, cl=FAKE + 2048, cu=None, slots=FAKE,
            n=5):
    return ra.load().relay_attn_update_tables(ctypes.byref(p) if p else None, V(old), V(new), V(pin), V(pout), V(free), V(bt),
                                              V(cl), V(cu), V(slots), n, None)


def test_update_tables_refuses():
    p = _params()
    assert _tables(None) == BAD
    for kw in (dict(old=None), dict(new=None), dict(pin=None), dict(pout=None), dict(free=None), dict(bt=None), dict(cl=None),
               dict(slots=None), dict(n=-1), dict(pout=FAKE + 512), dict(cl=FAKE), dict(cl=FAKE + 256)):
        assert _tables(p, **kw) == BAD, kw
    for kw in (dict(batch=-1), dict(num_blocks=-1), dict(max_blocks_per_seq=-1), dict(block_size=0), dict(block_size=12),
               dict(reserved0=1), dict(block_size=1 << 20, max_blocks_per_seq=1 << 12)):
        assert _tables(_params(**kw)) == BAD, kw
    assert _tables(_params(num_blocks=1 << 28)) == NOT_HERE                       # 2^32 positions
    assert _tables(_params(batch=1 << 20, max_blocks_per_seq=1 << 12)) == NOT_HERE
