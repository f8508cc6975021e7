"""Results that are no number, in every form a call can run in: a row whose query or whose keys hold one gives none, in its
output and in its log-sum-exp, and no other row changes."""
import sys
from dataclasses import replace

import numpy as np
import pytest
import torch

import fp4_util as F
import oracle
import workloads as W
from gpu_util import DeviceCase
from test_gpu_fp4 import Fp4Case, _cfg

pytestmark = pytest.mark.gpu

# name -> (shape of the batch, prompt phase, what else the call is given)
FORMS = {
    "decode, one launch": (_cfg(batch=4, ctx_lo=0, ctx_hi=200), False, {}),
    "decode, two launches": (_cfg(batch=4, ctx_lo=0, ctx_hi=200), False, dict(ctx_part_tokens=128)),
    "decode, two launches, 64-wide heads": (_cfg(batch=4, ctx_lo=0, ctx_hi=200, head_dim=64), False, dict(ctx_part_tokens=128)),
    "decode, many rows": (_cfg(batch=40, num_q_heads=32, num_kv_heads=4, sys_len=1100, ctx_lo=0, ctx_hi=90), False, {}),
    "decode, many partials a row": (_cfg(batch=2, ctx_lo=2500, ctx_hi=3000, sys_len=600), False,
                                    dict(ctx_part_tokens=128, sys_chunk_tokens=32)),
    "prompts, one launch": (_cfg(batch=4, q_lo=40, q_hi=60, ctx_lo=0, ctx_hi=50), True, {}),
    "prompts, two launches": (_cfg(batch=4, q_lo=40, q_hi=60, ctx_lo=0, ctx_hi=50), True, dict(ctx_part_tokens=128, sys_chunk_tokens=64)),
    "prompts, few new tokens": (_cfg(batch=9, q_lo=1, q_hi=8, num_q_heads=8, num_kv_heads=2, ctx_lo=1020, ctx_hi=1070), True, {}),
}


def _say(msg):
    print("[case] " + msg, flush=True)
    sys.stdout.flush()


class Call:
    """One form over one kind of cache; the same case on both."""

    def __init__(self, form, cache, seed, edit=lambda case: case):
        cfg, self.prompts, self.kw = FORMS[form]
        case = edit(W.make_case(cfg, seed, prefill=self.prompts, extra_context=self.prompts))
        _say("%s, %s cache: %s" % (form, cache, cfg))
        self.fp4 = cache == "fp4"
        self.on = Fp4Case(case) if self.fp4 else DeviceCase(case)
        self.case = self.on.case

    def run(self):
        if self.fp4:
            return self.on.run(self.prompts, **self.kw)
        return self.on.prefill(**self.kw) if self.prompts else self.on.decode(**self.kw)

    def tolerances(self, case):
        """Of outputs and log-sum-exps in 32 bits (the bf16 calls hold the weights in two bfloat16 parts, 2^-17 of each)."""
        vmax = max(np.abs(case.v_sys).max(initial=0.0), np.abs(np.nan_to_num(case.v_cache)).max())
        out, lse, _ = F.bounds(replace(case, k_cache=np.nan_to_num(case.k_cache), v_cache=np.nan_to_num(case.v_cache)), False)
        return out + (0 if self.fp4 else 2 * vmax * 2.0 ** -17), lse

    def want(self, case):
        args = (case.k_sys, case.v_sys, case.k_cache, case.v_cache, case.block_tables, case.context_lens, case.scale)
        if self.prompts:
            return oracle.prefill_attention(case.q, case.cu_seqlens_q, *args)[:2]
        return oracle.decode_attention(case.q, *args)[:2]


def _compare(call, got, want, bad, case, both_off=1):
    """Rows `bad` are no numbers in output and log-sum-exp, the others are those of `want`."""
    tol, ltol = call.tolerances(case)
    assert np.isnan(got[0][bad]).all() and np.isnan(got[1][bad]).all()
    assert np.abs(got[0][~bad] - want[0][~bad]).max() <= both_off * tol
    empty = np.isneginf(want[1])
    assert np.array_equal(np.isneginf(got[1])[~bad], empty[~bad])
    assert np.abs(got[1][~bad & ~empty] - want[1][~bad & ~empty]).max() <= both_off * ltol


@pytest.mark.parametrize("cache", ["fp4", "bf16"])
@pytest.mark.parametrize("form", FORMS)
def test_a_query_that_is_no_number(form, cache):
    """The row of a request whose context is empty among them: what it sees of the system prompt is no number either."""
    call = Call(form, cache, 1201)
    rows = [1, call.on.q.shape[0] - 1]
    if not call.prompts and call.case.context_lens.min() < 2000:
        call.on.__dict__["context_lens" if cache == "bf16" else "lens"][1] = 0
    clean = call.run()
    bad = np.zeros(clean[0].shape[:2], dtype=bool)
    bad[rows, 5] = True
    call.on.q[rows, 5, 17] = float("nan")
    _compare(call, call.run(), clean, bad, call.case, both_off=2)       # (running maxima may move at other places)


@pytest.mark.parametrize("cache", ["fp4", "bf16"])
@pytest.mark.parametrize("form", FORMS)
def test_a_system_key_that_is_no_number(form, cache):
    """Every row of its kv head sees it."""
    call = Call(form, cache, 1202)
    clean = call.run()
    call.on.k_sys[70, 1, 9] = float("nan")
    group = call.case.cfg.num_q_heads // call.case.cfg.num_kv_heads
    bad = np.zeros(clean[0].shape[:2], dtype=bool)
    bad[:, group:2 * group] = True
    _compare(call, call.run(), clean, bad, call.case, both_off=2)


@pytest.mark.parametrize("cache", ["fp4", "bf16"])
@pytest.mark.parametrize("sys_len", [None, 1])
@pytest.mark.parametrize("form", FORMS)
def test_a_system_key_whose_scores_overflow(form, sys_len, cache):
    """The largest value of a 4-bit cache in a key that was made part of a system prompt.  A query of +2 there scores beyond what
    32 bits hold and has no result; one of -2 scores minus infinity and has that of a prompt without the position, also where
    that leaves nothing of the prompt."""
    at = 0 if sys_len == 1 else 70

    def spoil(case):
        n = case.k_sys.shape[0] if sys_len is None else sys_len
        case = replace(case, cfg=replace(case.cfg, sys_len=n), k_sys=case.k_sys[:n].copy(), v_sys=case.v_sys[:n], q=case.q.copy())
        case.k_sys[at, :, 3] = 6 * 2.0 ** 125
        case.q[..., 3] = -2
        case.q[:, 5, 3] = 2
        return case

    call = Call(form, cache, 1203, spoil)
    keep = np.arange(call.case.k_sys.shape[0]) != at
    case = replace(call.case, cfg=replace(call.case.cfg, sys_len=int(keep.sum())), k_sys=call.case.k_sys[keep], v_sys=call.case.v_sys[keep])
    want = call.want(case)
    bad = np.zeros(want[0].shape[:2], dtype=bool)
    bad[:, 5] = True
    _compare(call, call.run(), want, bad, case)
