"""Which form a call over a 4-bit cache takes, and with which numbers: the launches that its host side would make."""
import dataclasses

import numpy as np
import pytest

import fp4_launches as L
import launch_record as R
import test_gpu_fp4 as T
import test_gpu_fp4_graph as G
import test_gpu_no_number as N
import workloads as W
from test_fp4_workspace import shape


def _launches(cfg, seed, prompts, **kw):
    """Of the batch that make_case draws."""
    case = W.make_case(cfg, seed, prefill=prompts, extra_context=prompts)
    return _of(cfg, case.context_lens, case.cu_seqlens_q if prompts else None, case.k_cache.shape[0], **kw)


def _of(cfg, lens, cu, held, bound=None, num_blocks=None, width=None, **tuning):
    p = shape(batch=cfg.batch, num_q_heads=cfg.num_q_heads, num_kv_heads=cfg.num_kv_heads, head_dim=cfg.head_dim, sys_len=cfg.sys_len,
              block_size=cfg.block_size, num_blocks=held if num_blocks is None else num_blocks, max_blocks_per_seq=width or -(-int(max(lens)) // cfg.block_size),
              max_context_len=int(max(lens)) if bound is None else bound, **tuning)
    return L.decode(p) if cu is None else L.prefill(p, int(cu[-1]), int(np.diff(cu).max()))


def _even(cfg, **kw):
    """Of a prompt phase with lengths spread evenly over the ranges of `cfg`."""
    counts = np.linspace(cfg.q_lo, cfg.q_hi, cfg.batch).astype(int)
    lens = np.linspace(cfg.ctx_lo, cfg.ctx_hi, cfg.batch).astype(int) + counts
    return _of(cfg, lens, np.cumsum([0] + list(counts)), int(sum(-(-lens // cfg.block_size)) * 11 // 10), **kw)


def _form(launches):
    first = launches[0]
    assert first["launch"] == "direct_fp4" or first["fp4"] == 1
    if first["launch"] == "rows":
        return "whole" if first["whole"] else "many rows"
    if first["launch"] == "direct_fp4":
        return "one launch"
    assert [x["launch"] for x in launches] == ["tiles", "fuse"]
    return "few" if first["prompts"] else "many-rows system" if first["rows_sys"] else "streamed"


# What the GPU tests of these shapes exercise.
@pytest.mark.parametrize("form,want", zip(N.FORMS, ["one launch", "streamed", "streamed", "many-rows system", "streamed", "whole",
                                                    "many rows", "few"]))
def test_the_forms_that_are_tested_for_no_numbers_are_those_named(form, want):
    cfg, prompts, kw = N.FORMS[form]
    for seed in (1201, 1202, 1203):
        assert _form(_launches(cfg, seed, prompts, **kw)) == want


@pytest.mark.parametrize("name,want", zip(G.SHAPES, ["few", "few", "whole", "many rows"]))
def test_the_forms_that_are_captured_are_those_named(name, want):
    cfg, counts, longest = G.SHAPES[name]
    width = -(-longest // cfg.block_size)
    assert _form(_of(cfg, [longest], np.cumsum([0] + counts), cfg.batch * width + 3, width=width)) == want


def test_both_forms_of_few_new_tokens_are_tested():
    forms = [_form(_launches(cfg, 945, True)) for cfg in T.FEW]
    assert forms == ["few", "few", "many rows", "few", "few", "many rows", "few"]
    loose = [_form(_launches(cfg, 945, True, bound=0, width=400)) for cfg in T.FEW]
    assert loose == forms


def test_decode_tests_cover_one_launch_and_two():
    assert {_form(_launches(cfg, 911, False)) for cfg in T.DECODE} == {"one launch", "streamed", "many-rows system"}
    assert {_form(_launches(cfg, 911, False, ctx_part_tokens=128)) for cfg in T.DECODE} == {"streamed", "many-rows system"}


SHORT = T._cfg(batch=16, num_q_heads=40, num_kv_heads=40, q_lo=8, q_hi=27, ctx_lo=32, ctx_hi=137, sys_len=0)
LONG = dataclasses.replace(SHORT, ctx_lo=3000, ctx_hi=5000, q_hi=8)
BRIEF = dataclasses.replace(SHORT, num_q_heads=8, num_kv_heads=8)


def test_few_new_tokens_are_streamed_where_contexts_are_known_to_be_a_good_part():
    assert [_form(_even(cfg)) for cfg in (SHORT, LONG, BRIEF)] == ["few", "few", "many rows"]
    # a cache for many more, under a bound that the caller gives: still known
    assert [_form(_even(cfg, num_blocks=1 << 17)) for cfg in (SHORT, LONG, BRIEF)] == ["few", "few", "many rows"]
    # the tables' capacity as the bound, and a cache about as large as its contents
    assert [_form(_even(cfg, bound=0, width=475)) for cfg in (SHORT, LONG, BRIEF)] == ["few", "few", "many rows"]
    # neither says anything: not where the spans that are planned for the capacity are long
    for num_blocks in (1 << 17, 0):                              # a server's whole memory; not filled in
        assert [_form(_even(cfg, bound=0, width=475, num_blocks=num_blocks)) for cfg in (SHORT, LONG, BRIEF)] == ["many rows"] * 3
        two = dataclasses.replace(LONG, batch=2, num_q_heads=8, num_kv_heads=8)
        launches = _even(two, bound=0, width=475, num_blocks=num_blocks)
        assert _form(launches) == "few" and launches[0]["floor"] <= 8


def test_more_rows_than_a_wavefront_takes_or_a_cut_by_hand_go_the_other_way():
    assert _form(_even(dataclasses.replace(LONG, q_lo=33, q_hi=33))) in ("many rows", "whole")
    assert _form(_even(dataclasses.replace(LONG, q_lo=32, q_hi=32))) == "few"
    assert _form(_even(LONG, sys_chunk_tokens=64)) == "many rows"


def test_a_system_tile_weighs_three_context_tiles_of_a_decode_step_and_one_of_few_new_tokens():
    p = shape(batch=64, num_q_heads=40, num_kv_heads=40, head_dim=128, sys_len=1024, num_blocks=6400, max_blocks_per_seq=160,
              max_context_len=2500)
    four_bits, bf16 = L.decode(p)[0], R.decode(p)[0]
    assert four_bits["light"] > 0 and four_bits["chunk"] == bf16["chunk"]
    tiles = -(-four_bits["chunk"] // 32)
    assert four_bits["sys_wg_tiles"] == 3 * tiles and four_bits["sys_tiles"] == 3 * 40 * 2 * 32
    few = L.prefill(shape(), 160, 8)[0]
    assert few["light"] > 0 and few["sys_wg_tiles"] == -(-few["chunk"] // 32) and few["sys_tiles"] == 8 * 20 * 19
    assert {x["exact"] for x in (four_bits, few)} == {0} and L.decode(shape(out_is_fp32=1, batch=64))[0]["exact"] == 1
