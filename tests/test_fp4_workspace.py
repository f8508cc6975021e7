"""What the calls over a 4-bit cache ask for beyond the others is asked for by their own size, and all of them live within the
size that they are given."""
import pytest
import torch

import fp4_launches as L
import launch_record as R
import paper_2402_14808_amd as ra


def shape(**kw):
    p = ra.RAParams()
    given = dict(batch=32, num_q_heads=32, num_kv_heads=8, head_dim=64, sys_len=600, block_size=16, num_blocks=3000, max_blocks_per_seq=140,
                 max_context_len=2200, softmax_scale=0.1)
    given.update(kw)
    for name, value in given.items():
        setattr(p, name, value)
    p.q_stride_token = p.o_stride_token = p.num_q_heads * p.head_dim
    p.q_stride_head = p.o_stride_head = p.sys_stride_head = p.head_dim
    p.sys_stride_token = p.num_kv_heads * p.head_dim
    return p


# shape, new tokens, most of a request, megabytes that hold every call over a bfloat16 cache (14.64 and 10.57)
CASES = [(dict(), 160, 8, 15), (dict(batch=8, head_dim=128, num_blocks=1000), 32, 6, 11)]


def _used(launches, p):
    fuse = [x for x in launches if x["launch"] == "fuse"]
    return sum(x["partials"] * x["rows"] * (p.head_dim + 1) * 4 for x in fuse)


@pytest.mark.parametrize("kw,total_q,most,megabytes", CASES)
def test_a_bf16_prompt_phase_pays_for_its_own_forms_only(kw, total_q, most, megabytes):
    p = shape(**kw)
    size = L.workspace_bytes(p, total_q, fp4=False)
    assert size == R.workspace_bytes(p, total_q) == ra.relay_attn_workspace_bytes(p, total_q) <= megabytes * 10**6
    assert R.prefill(p, total_q, most, workspace=size) == R.prefill(p, total_q, most, workspace=1 << 40)


@pytest.mark.parametrize("kw,total_q,most,megabytes", CASES)
def test_few_new_tokens_over_a_4_bit_cache_fit_either_size(kw, total_q, most, megabytes):
    p = shape(**kw)
    small, full = L.workspace_bytes(p, total_q, fp4=False), L.workspace_bytes(p, total_q)
    assert full > small and full == ra.relay_attn_workspace_bytes_fp4(p, total_q)
    assert L.prefill(p, total_q, most, workspace=full) == L.prefill(p, total_q, most, workspace=1 << 40)
    for size in (small, full):
        assert 0 < _used(L.prefill(p, total_q, most, workspace=size), p) <= size


@pytest.mark.parametrize("total_q", [0, 32, 32 * 9, 5000])
def test_other_calls_ask_for_the_same(total_q):
    p = shape()
    assert L.workspace_bytes(p, total_q) == L.workspace_bytes(p, total_q, fp4=False)
    assert L.workspace_bytes(shape(head_dim=96), total_q) == 0 and L.workspace_bytes(shape(batch=0), 0) > 0


def test_parameters_know_which_cache_they_were_made_from():
    q, tables = torch.zeros((160, 32, 64), dtype=torch.bfloat16), torch.zeros((32, 140), dtype=torch.int32)
    made = [ra.make_params(q, q, None, k, tables, batch=32, softmax_scale=0.1, max_context_len=2200)
            for k in (torch.zeros((300, 8, 16, 64), dtype=torch.bfloat16), torch.zeros(ra.fp4_cache_shape(300, 8, 16, 64), dtype=torch.uint8))]
    sizes = [ra.relay_attn_workspace_bytes(p, 160) for p in made]
    assert sizes == [L.workspace_bytes(made[0], 160, fp4=False), L.workspace_bytes(made[1], 160)]
    assert sizes[1] >= sizes[0]
