"""A cache of one kind handed to a call for the other kind is refused before anything is launched."""
import pytest
import torch

import paper_2402_14808_amd as ra
from paper_2402_14808_amd import binding

Q = torch.zeros((3, 4, 64), dtype=torch.bfloat16)
NEW = torch.zeros((3, 2, 64), dtype=torch.bfloat16)
INT = torch.zeros((3, 4), dtype=torch.int32)
SPACE = torch.zeros(256, dtype=torch.uint8)
BF16 = torch.zeros((5, 2, 16, 64), dtype=torch.bfloat16)
FP4 = torch.zeros(ra.fp4_cache_shape(5, 2, 16, 64), dtype=torch.uint8)

PAGED = (INT, INT, Q, None, SPACE)         # block tables, lengths, output, log-sum-exps, workspace
CALLS = {
    "relay_attn_decode": lambda p, k, v: (p, Q, None, None, k, v, *PAGED),
    "relay_attn_decode_append": lambda p, k, v: (p, Q, NEW, NEW, None, None, k, v, *PAGED),
    "relay_attn_debug_timeline": lambda p, k, v: (p, Q, None, 3, 1, None, None, k, v, *PAGED, torch.zeros(4, dtype=torch.int64)),
    "relay_attn_decode_static": lambda p, k, v: (p, Q, None, None, k, v, *PAGED[:4]),
    "relay_attn_debug_decode_phases": lambda p, k, v: (p, 1, Q, None, None, k, v, *PAGED),
    "relay_attn_prefill": lambda p, k, v: (p, Q, INT, 3, 1, None, None, k, v, *PAGED),
    "relay_attn_prefill_multi": lambda p, k, v: (p, [(None, None, 0, 3)], [3], Q, INT, 3, 1, k, v, *PAGED),
    "paged_attn_decode_naive": lambda p, k, v: (p, Q, k, v, *PAGED),
    "relay_attn_cache_append": lambda p, k, v: (p, NEW, NEW, None, 3, k, v, INT, INT),
    "relay_attn_decode_multi": lambda p, k, v: (p, [(None, None, 0, 3)], Q, k, v, *PAGED),
    "relay_attn_decode_grouped": lambda p, k, v: (p, [(None, None, 3)], INT, INT, Q, k, v, *PAGED),
    "relay_attn_cache_append_fp4": lambda p, k, v: (p, NEW, NEW, None, 3, k, v, INT, INT),
    "relay_attn_cache_read_fp4": lambda p, k, v: (p, NEW, NEW, None, 3, k, v, INT, INT),
    "relay_attn_decode_fp4": lambda p, k, v: (p, Q, None, None, k, v, *PAGED),
    "relay_attn_prefill_fp4": lambda p, k, v: (p, Q, INT, 3, 1, None, None, k, v, *PAGED),
}


@pytest.mark.parametrize("name", CALLS)
def test_a_cache_of_the_other_kind_is_refused(name):
    right, wrong = (FP4, BF16) if name.endswith("_fp4") else (BF16, FP4)
    for k, v in ((wrong, wrong), (wrong, right), (right, wrong)):
        for of in (BF16, FP4):
            p = ra.make_params(Q, Q, None, of, INT, batch=3, softmax_scale=1.0)
            with pytest.raises(ra.RelayAttnError) as e:
                getattr(ra, name)(*CALLS[name](p, k, v))
            assert e.value.status == binding.RA_ERR_INVALID_ARG and name in str(e.value)


def test_every_call_that_takes_a_cache_is_here():
    calls = [getattr(ra, name) for name in ra.__all__]
    assert {f.__name__ for f in calls if "v_cache" in getattr(getattr(f, "__code__", None), "co_varnames", ())} == set(CALLS)
