"""The 4-bit context cache on the GPU: append and read-out against the format's definition, attention against the
64-bit oracle on the values the cache holds, and the calls of a step one behind the other."""
import sys
from dataclasses import replace

import numpy as np
import pytest
import torch

import fp4_util as F
import oracle
import paper_2402_14808_amd as ra
import workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _say(msg):
    print("[case] " + msg, flush=True)
    sys.stdout.flush()


def _bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(torch.bfloat16)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _cfg(**kw):
    base = dict(name="f", batch=5, num_q_heads=8, num_kv_heads=4, head_dim=128, sys_len=150, ctx_lo=1, ctx_hi=200,
                block_size=16, q_lo=1, q_hi=40)
    base.update(kw)
    return W.AttnConfig(**base)


class Fp4Case:
    """An AttnCase with its context caches in the 4-bit format, on the GPU."""

    def __init__(self, case):
        self.case, kb, vb = F.to_fp4(case)
        self.q, self.k_sys, self.v_sys = (_bf16(x) for x in (case.q, case.k_sys, case.v_sys))
        self.k, self.v = torch.from_numpy(kb).to(DEV), torch.from_numpy(vb).to(DEV)
        self.tables, self.lens, self.cu = _i32(case.block_tables), _i32(case.context_lens), _i32(case.cu_seqlens_q)

    def run(self, prefill=False, fp32_out=True, max_context_len=None, q=None, **tuning):
        c, q = self.case, self.q if q is None else q
        n, hq, d = q.shape
        out = torch.full((n, hq, d), float("nan"), device=DEV, dtype=torch.float32 if fp32_out else torch.bfloat16)
        lse = torch.full((n, hq), float("nan"), device=DEV)
        mcl = int(c.context_lens.max()) if max_context_len is None else max_context_len
        p = ra.make_params(q, out, self.k_sys, self.k, self.tables, batch=c.cfg.batch, softmax_scale=c.scale,
                           max_context_len=mcl, **tuning)
        assert p.block_size == c.cfg.block_size
        ws = torch.full((ra.relay_attn_workspace_bytes(p, n),), 0xFF, dtype=torch.uint8, device=DEV)
        if prefill:
            ra.relay_attn_prefill_fp4(p, q, self.cu, n, int(np.diff(c.cu_seqlens_q).max()), self.k_sys, self.v_sys, self.k,
                                      self.v, self.tables, self.lens, out, lse, ws)
        else:
            ra.relay_attn_decode_fp4(p, q, self.k_sys, self.v_sys, self.k, self.v, self.tables, self.lens, out, lse, ws)
        torch.cuda.synchronize()
        return out.float().cpu().numpy(), lse.cpu().numpy()

    def want(self, prefill=False):
        c = self.case
        if prefill:
            return oracle.prefill_attention(c.q, c.cu_seqlens_q, c.k_sys, c.v_sys, c.k_cache, c.v_cache, c.block_tables,
                                            c.context_lens, c.scale)[:2]
        return oracle.decode_attention(c.q, c.k_sys, c.v_sys, c.k_cache, c.v_cache, c.block_tables, c.context_lens,
                                       c.scale)[:2]

    def check(self, prefill=False, fp32_out=True, **kw):
        got, lse = self.run(prefill, fp32_out, **kw)
        want, wlse = self.want(prefill)
        tol, ltol, rel = F.bounds(self.case, not fp32_out)
        empty = np.isneginf(wlse)
        assert np.array_equal(np.isneginf(lse), empty)
        err, lerr = np.abs(got - want).max(), np.abs(lse[~empty] - wlse[~empty]).max(initial=0.0)
        off = np.linalg.norm(got - want) / max(np.linalg.norm(want), 1e-30)
        _say("max-abs err %.3e of %.3e, lse err %.3e of %.3e, norm %.3e of %.3e" % (err, tol, lerr, ltol, off, rel))
        assert np.isfinite(got).all() and err <= tol and lerr <= ltol and off <= rel
        assert not got[empty].any()


# ---- rows in and out --------------------------------------------------------------------------------------------

def _every_bf16(d):
    """Rows whose blocks of 32 hold every bfloat16 there is, next to neighbours that make its block's scale."""
    bits = np.arange(65536, dtype=np.uint32)
    x = (bits << 16).view(np.float32).reshape(-1, 32)
    rng = np.random.Generator(np.random.PCG64(5))
    mixed = W.bf16_round(rng.standard_normal((2048, 32), dtype=np.float32) * 2.0 ** rng.integers(-20, 20, (2048, 1)))
    edge = np.repeat(np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 6.96875, 7.0, 7.96875, 0.2490234375],
                              dtype=np.float32), 32).reshape(-1, 32)
    edge[:, 1] = np.array([6, 6.5, 7, 4], dtype=np.float32).repeat(3)
    edge[:, 2] = -edge[:, 0]
    zero = np.zeros((4, 32), dtype=np.float32)
    zero[1, 3], zero[2, 4], zero[3] = -0.0, 1e-40, -(2.0 ** -133)
    every = np.concatenate([x, mixed, edge, zero])
    pad = -len(every) % (2 * (d // 32))
    return np.concatenate([every, np.zeros((pad, 32), np.float32)]).reshape(-1, 2, d)        # [tokens, 2 heads, d]


@pytest.mark.parametrize("d,bs", [(128, 16), (64, 8), (128, 64)])
def test_append_rounds_every_bf16_and_reads_back_what_it_stored(d, bs):
    rows = _every_bf16(d)
    n, hkv = rows.shape[:2]
    k_new, v_new = _bf16(rows), _bf16(rows[::-1])
    rows = k_new.double().cpu().numpy()
    blocks = -(-n // bs)
    k, v = (torch.full(ra.fp4_cache_shape(blocks + 1, hkv, bs, d), 0xAB, dtype=torch.uint8, device=DEV) for _ in range(2))
    order = np.random.Generator(np.random.PCG64(3)).permutation(blocks * bs)[:n].astype(np.int32) + bs
    slots = _i32(order)
    p = ra.make_params(k_new, k_new, None, k, torch.zeros((1, 1), dtype=torch.int32), batch=1, softmax_scale=1.0)
    ra.relay_attn_cache_append_fp4(p, k_new, v_new, None, n, k, v, None, None, slot_map=slots)
    k_out, v_out = torch.full_like(k_new, 7.0), torch.full_like(v_new, 7.0)
    ra.relay_attn_cache_read_fp4(p, k_out, v_out, None, n, k, v, None, None, slot_map=slots)
    torch.cuda.synchronize()
    for cache, src, out in ((k, rows, k_out), (v, rows[::-1], v_out)):
        code, scale = F.round_rows(src)
        got_code, got_scale = F.unpack(cache.cpu().numpy(), bs, d)
        at = (order // bs, slice(None), order % bs)
        assert np.array_equal(got_scale[at], scale)
        assert np.array_equal(got_code[at], code)
        assert np.array_equal(out.double().cpu().numpy(), F.values(code, scale))
        rest = np.ones((blocks + 1, bs), dtype=bool)
        rest[order // bs, order % bs] = False
        assert (got_scale.transpose(0, 2, 1, 3)[rest] == 0xAB).all()
        assert np.isin(got_code.transpose(0, 2, 1, 3)[rest], (0xA, 0xB)).all()


@pytest.mark.parametrize("cfg,seed,prefill", [
    (_cfg(), 901, False),
    (_cfg(head_dim=64, block_size=8, num_kv_heads=2), 902, False),
    (_cfg(), 903, True),
    (_cfg(block_size=32, q_hi=9, ctx_hi=30, num_kv_heads=1, num_q_heads=1), 904, True),
    (_cfg(batch=140, q_hi=20, ctx_hi=60), 905, True),
    (_cfg(batch=2, q_lo=600, q_hi=900, num_kv_heads=8, num_q_heads=8), 906, True),
])
def test_append_by_lengths_lands_where_the_bf16_cache_has_it(cfg, seed, prefill):
    case = W.make_case(cfg, seed, prefill=prefill, extra_context=prefill, poison_tails=False)
    _say("%s" % (cfg,))
    rng = np.random.Generator(np.random.PCG64(seed + 1000))
    n, hkv, d, bs = int(case.cu_seqlens_q[-1]), cfg.num_kv_heads, cfg.head_dim, cfg.block_size
    wide = W.bf16_round(rng.standard_normal((n, 3 * hkv, d), dtype=np.float32))     # a fused projection's output
    wide_d = _bf16(wide)
    k_new, v_new = wide_d[:, hkv:2 * hkv], wide_d[:, 2 * hkv:]
    fc = Fp4Case(case)
    before_k, before_v = fc.k.cpu().numpy(), fc.v.cpu().numpy()
    p = ra.make_params(fc.q, fc.q, None, fc.k, fc.tables, batch=cfg.batch, softmax_scale=1.0)
    cu = fc.cu if prefill else None
    ra.relay_attn_cache_append_fp4(p, k_new, v_new, cu, n, fc.k, fc.v, fc.tables, fc.lens)
    out = torch.zeros((n, 2 * hkv, d), dtype=torch.bfloat16, device=DEV)            # strided on the way out too
    ra.relay_attn_cache_read_fp4(p, out[:, :hkv], out[:, hkv:], cu, n, fc.k, fc.v, fc.tables, fc.lens)
    torch.cuda.synchronize()
    for before, after, new, mine in ((before_k, fc.k, wide[:, hkv:2 * hkv], out[:, :hkv]),
                                     (before_v, fc.v, wide[:, 2 * hkv:], out[:, hkv:])):
        code, scale = F.unpack(before, bs, d)
        code, scale = code.copy(), scale.copy()
        new_code, new_scale = F.round_rows(new)
        for i in range(cfg.batch):
            a, b = int(case.cu_seqlens_q[i]), int(case.cu_seqlens_q[i + 1])
            for j in range(b - a):
                pos = int(case.context_lens[i]) - (b - a) + j
                code[case.block_tables[i, pos // bs], :, pos % bs] = new_code[a + j]
                scale[case.block_tables[i, pos // bs], :, pos % bs] = new_scale[a + j]
        assert np.array_equal(after.cpu().numpy(), F.pack(code, scale))
        assert np.array_equal(mine.double().cpu().numpy(), F.values(new_code, new_scale))


def test_slots_out_of_range_leave_cache_and_rows_alone():
    n, hkv, d, bs, blocks = 9, 3, 64, 16, 4
    x = torch.randn(n, hkv, d, device=DEV).to(torch.bfloat16)
    k, v = (torch.full(ra.fp4_cache_shape(blocks, hkv, bs, d), 0x11, dtype=torch.uint8, device=DEV) for _ in range(2))
    slots = _i32([-1, blocks * bs, 2**31 - 1, -2**31, 5, blocks * bs - 1, -7, 0, blocks * bs + 1])
    p = ra.make_params(x, x, None, k, torch.zeros((1, 1), dtype=torch.int32), batch=1, softmax_scale=1.0)
    ra.relay_attn_cache_append_fp4(p, x, x, None, n, k, v, None, None, slot_map=slots)
    out = torch.full_like(x, 9.0)
    ra.relay_attn_cache_read_fp4(p, out, torch.full_like(x, 9.0), None, n, k, v, None, None, slot_map=slots)
    torch.cuda.synchronize()
    code, scale = F.round_rows(x.double().cpu().numpy())
    want = F.values(code, scale)
    written = [4, 5, 7]
    got = out.double().cpu().numpy()
    assert np.array_equal(got[written], want[written])
    assert (np.delete(got, written, 0) == 9.0).all()
    raw_code, raw_scale = F.unpack(k.cpu().numpy(), bs, d)
    touched = np.zeros((blocks, bs), dtype=bool)
    touched[[0, blocks - 1, 0], [5, bs - 1, 0]] = True
    assert (raw_scale.transpose(0, 2, 1, 3)[~touched] == 0x11).all() and (raw_code.transpose(0, 2, 1, 3)[~touched] == 1).all()


# ---- attention ---------------------------------------------------------------------------------------------------

DECODE = [
    _cfg(),
    _cfg(num_kv_heads=8),                                       # one query head per kv head
    _cfg(num_q_heads=8, num_kv_heads=1, block_size=8),
    _cfg(num_q_heads=7, num_kv_heads=1, sys_len=0),
    _cfg(head_dim=64, block_size=8, sys_len=33),
    _cfg(head_dim=64, num_q_heads=6, num_kv_heads=2, block_size=64, ctx_hi=500),
    _cfg(batch=1, ctx_lo=1, ctx_hi=1, sys_len=0),
    _cfg(batch=1, ctx_lo=1, ctx_hi=1, sys_len=1, head_dim=64),
    _cfg(batch=70, ctx_lo=0, ctx_hi=40, sys_len=64, block_size=32),
    _cfg(batch=2, ctx_lo=2900, ctx_hi=3100, block_size=128, sys_len=700),
    _cfg(batch=40, num_q_heads=32, num_kv_heads=4, sys_len=1100, ctx_lo=10, ctx_hi=90),   # many stacked rows
]


@pytest.mark.parametrize("cfg", DECODE, ids=[str(i) for i in range(len(DECODE))])
@pytest.mark.parametrize("fp32_out", [True, False], ids=["fp32", "bf16"])
def test_decode_matches_oracle(cfg, fp32_out):
    _say("%s" % (cfg,))
    fc = Fp4Case(W.make_case(cfg, 911))
    fc.check(fp32_out=fp32_out)
    fc.check(fp32_out=fp32_out, ctx_part_tokens=128)             # two launches whatever the size
    if cfg.sys_len:
        fc.check(fp32_out=fp32_out, sys_chunk_tokens=64)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bs", [8, 16, 32])
def test_decode_at_every_length_around_tiles_and_blocks(d, bs):
    lens = [0, 1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 39, 40, 63, 64, 65, 95, 96, 97, 127, 128, 129, 160, 161, 255, 256, 257]
    cfg = _cfg(batch=len(lens), head_dim=d, block_size=bs, num_q_heads=4, num_kv_heads=2, sys_len=0, ctx_hi=257)
    rng = np.random.Generator(np.random.PCG64(7))
    ctx = [[W.bf16_round(rng.standard_normal((c, 2, d), dtype=np.float32)) for c in lens] for _ in range(2)]
    empty = np.zeros((0, 2, d), dtype=np.float32)
    q = W.bf16_round(rng.standard_normal((len(lens), 4, d), dtype=np.float32))
    fc = Fp4Case(W.from_dense(cfg, q, empty, empty, *ctx))
    fc.check()                                                   # the request of length 0: zero row, lse -inf
    fc.check(max_context_len=0)                                  # bounded by the table's capacity
    fc.check(ctx_part_tokens=128)


@pytest.mark.parametrize("kw", [dict(sys_chunk_tokens=64), dict(ctx_part_tokens=256), dict(max_context_len=0)])
def test_decode_cut_by_hand_or_under_a_loose_bound(kw):
    case = W.make_case(_cfg(batch=3, ctx_lo=300, ctx_hi=2000, sys_len=500), 921)
    wide = np.full((3, 400), W.POISON_BLOCK, dtype=np.int32)
    wide[:, :case.block_tables.shape[1]] = case.block_tables
    Fp4Case(replace(case, block_tables=wide)).check(**kw)


def test_decode_of_a_strided_query_and_extreme_scales():
    case = W.make_case(_cfg(num_q_heads=12, num_kv_heads=4), 931)
    fc = Fp4Case(case)
    wide = torch.zeros((case.cfg.batch, 20, 136), dtype=torch.bfloat16, device=DEV)
    wide[:, 3:15, :128] = fc.q
    fc.check(q=wide[:, 3:15, :128])
    for scale, part in [(s, part) for s in (-0.05, 0.0, 3.0) for part in (0, 128)]:       # one launch, and two
        _say("scale %g, part %d" % (scale, part))
        out, lse = _run_scaled(fc, scale, part)
        c = fc.case
        want, wlse = oracle.decode_attention(c.q, c.k_sys, c.v_sys, c.k_cache, c.v_cache, c.block_tables, c.context_lens,
                                             scale)[:2]
        tol, ltol, rel = F.bounds(c, False, scale)
        assert np.abs(out - want).max() <= tol and np.abs(lse - wlse).max() <= ltol
        assert np.linalg.norm(out - want) <= rel * np.linalg.norm(want)


def _run_scaled(fc, scale, part):
    c = fc.case
    wide = torch.full((fc.q.shape[0], fc.q.shape[1] + 2, fc.q.shape[2] + 8), 7.0, device=DEV)   # rows of a wider output
    out, lse = wide[:, 1:-1, :-8], torch.empty(fc.q.shape[:2], device=DEV)
    p = ra.make_params(fc.q, out, fc.k_sys, fc.k, fc.tables, batch=c.cfg.batch, softmax_scale=scale, ctx_part_tokens=part)
    ws = torch.empty(ra.relay_attn_workspace_bytes(p, c.cfg.batch), dtype=torch.uint8, device=DEV)
    ra.relay_attn_decode_fp4(p, fc.q, fc.k_sys, fc.v_sys, fc.k, fc.v, fc.tables, fc.lens, out, lse, ws)
    torch.cuda.synchronize()
    assert (wide[:, 0] == 7).all() and (wide[:, -1] == 7).all() and (wide[:, :, -8:] == 7).all()
    return out.cpu().numpy(), lse.cpu().numpy()


PROMPT = [
    _cfg(),
    _cfg(head_dim=64, num_q_heads=8, num_kv_heads=2, sys_len=95, block_size=8),
    _cfg(sys_len=0, q_hi=130, num_q_heads=4),
    _cfg(batch=1, q_lo=1, q_hi=1, sys_len=0, ctx_lo=0, ctx_hi=0),
    _cfg(batch=40, q_lo=1, q_hi=6, sys_len=1030, num_q_heads=8, num_kv_heads=1),
    _cfg(batch=3, q_lo=200, q_hi=300, num_q_heads=2, num_kv_heads=1, ctx_hi=900, block_size=64),
    _cfg(batch=2, q_lo=1, q_hi=3, ctx_lo=4000, ctx_hi=5000, block_size=32, head_dim=64, sys_len=0),
    _cfg(batch=8, q_lo=64, q_hi=100, num_q_heads=16, num_kv_heads=16, head_dim=64, sys_len=300),
]


@pytest.mark.parametrize("cfg", PROMPT, ids=[str(i) for i in range(len(PROMPT))])
@pytest.mark.parametrize("extra", [True, False], ids=["behind a context", "alone"])
def test_prompt_phase_matches_oracle(cfg, extra):
    _say("%s extra=%s" % (cfg, extra))
    fc = Fp4Case(W.make_case(cfg, 941, prefill=True, extra_context=extra))
    fc.check(prefill=True)
    fc.check(prefill=True, fp32_out=False)
    fc.check(prefill=True, ctx_part_tokens=128, sys_chunk_tokens=128)       # two launches whatever the size


FEW = [
    _cfg(batch=9, num_q_heads=32, num_kv_heads=4, q_lo=1, q_hi=4, ctx_lo=0, ctx_hi=2300),         # up to 32 rows, groups of 8
    _cfg(batch=9, num_q_heads=8, num_kv_heads=2, q_lo=1, q_hi=8, ctx_lo=1020, ctx_hi=1070, block_size=8),
    _cfg(batch=9, num_q_heads=8, num_kv_heads=2, q_lo=1, q_hi=8, ctx_lo=20, ctx_hi=70, block_size=8),     # the other form
    _cfg(batch=40, num_q_heads=6, num_kv_heads=2, q_lo=1, q_hi=10, ctx_lo=0, ctx_hi=900, head_dim=64, sys_len=0),
    _cfg(batch=3, num_q_heads=2, num_kv_heads=2, q_lo=17, q_hi=32, ctx_lo=1300, ctx_hi=1400, block_size=64),
    _cfg(batch=70, num_q_heads=16, num_kv_heads=2, q_lo=1, q_hi=4, ctx_lo=1, ctx_hi=200, sys_len=1500, head_dim=64),
    _cfg(batch=1, num_q_heads=8, num_kv_heads=1, q_lo=3, q_hi=3, ctx_lo=3000, ctx_hi=3000, sys_len=33, block_size=32),
]


@pytest.mark.parametrize("cfg", FEW, ids=[str(i) for i in range(len(FEW))])
@pytest.mark.parametrize("fp32_out", [True, False], ids=["fp32", "bf16"])
def test_prompt_phase_of_few_new_tokens(cfg, fp32_out):
    _say("%s" % (cfg,))
    fc = Fp4Case(W.make_case(cfg, 945, prefill=True, extra_context=True))
    fc.check(prefill=True, fp32_out=fp32_out)
    wide = np.full((cfg.batch, 400), W.POISON_BLOCK, dtype=np.int32)     # a loose bound
    wide[:, :fc.case.block_tables.shape[1]] = fc.case.block_tables
    fc.tables = _i32(wide)
    fc.check(prefill=True, fp32_out=fp32_out, max_context_len=0)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("few", [True, False])
def test_prompt_phase_with_requests_that_bring_nothing(d, few):
    """Requests without new tokens in the middle and at both ends, contexts that end anywhere in a tile, one token or many."""
    most = 8 if few else 21
    counts = [0, 1, most, 0, 0, 3, 1, 7, 0]
    lens = [40, 1, 33 + most, 0, 500, 64, 31, 7, 9000]          # (the last makes the contexts long in the mean)
    cfg = _cfg(batch=len(lens), head_dim=d, num_q_heads=8, num_kv_heads=2, sys_len=45, ctx_hi=500)
    rng = np.random.Generator(np.random.PCG64(11))
    ctx = [[W.bf16_round(rng.standard_normal((c, 2, d), dtype=np.float32)) for c in lens] for _ in range(2)]
    k_sys, v_sys = (W.bf16_round(rng.standard_normal((45, 2, d), dtype=np.float32)) for _ in range(2))
    q = W.bf16_round(rng.standard_normal((sum(counts), 8, d), dtype=np.float32))
    cu = np.cumsum([0] + counts).astype(np.int32)
    Fp4Case(W.from_dense(cfg, q, k_sys, v_sys, *ctx, cu_seqlens_q=cu)).check(prefill=True)


def test_an_infinity_spoils_the_results_that_see_it_and_no_other():
    """A key and a value of infinity and NaN in the middle of a prompt: rows in front of it are those of a clean cache."""
    cfg = _cfg(batch=2, q_lo=40, q_hi=40, sys_len=70)
    case = W.make_case(cfg, 951, prefill=True)
    rng = np.random.Generator(np.random.PCG64(952))
    n = int(case.cu_seqlens_q[-1])
    k_new, v_new = (_bf16(rng.standard_normal((n, cfg.num_kv_heads, cfg.head_dim), dtype=np.float32)) for _ in range(2))
    held = replace(case, **{name: F.values(*F.round_rows(x.double().cpu().numpy())) for name, x in (("k_cache", k_new), ("v_cache", v_new))})
    results = []
    for spoil in (False, True):
        fc = Fp4Case(case)
        if spoil:
            k_new[25, :, 3], v_new[25, :, 9] = float("inf"), float("nan")
        p = ra.make_params(fc.q, fc.q, None, fc.k, fc.tables, batch=2, softmax_scale=1.0)
        ra.relay_attn_cache_append_fp4(p, k_new, v_new, fc.cu, n, fc.k, fc.v, fc.tables, fc.lens)
        results.append(fc.run(prefill=True))
    clean = np.r_[0:25, 40:80]
    tol, ltol, _ = F.bounds(held, False)                        # (the running maxima may move at other places: both sides' error)
    assert np.abs(results[0][0][clean] - results[1][0][clean]).max() <= 2 * tol
    assert np.abs(results[0][1][clean] - results[1][1][clean]).max() <= 2 * ltol
    assert not np.array_equal(results[0][0][25:40], results[1][0][25:40])


@pytest.mark.parametrize("kw", [{}, dict(ctx_part_tokens=128)])
@pytest.mark.parametrize("prefill", [False, True])
def test_a_query_that_is_no_number_gives_none_and_leaves_the_others(prefill, kw):
    case = W.make_case(_cfg(batch=4, ctx_lo=40, ctx_hi=300, q_lo=2, q_hi=9), 955, prefill=prefill, extra_context=prefill)
    fc = Fp4Case(case)
    bad = 2
    q = fc.q.clone()
    q[bad, 5, 17] = float("nan")
    clean, lse = fc.run(prefill, **kw)
    got, _ = fc.run(prefill, q=q, **kw)
    rest = np.ones(got.shape[:2], dtype=bool)
    rest[bad, 5] = False
    assert np.isnan(got[bad, 5]).all()
    tol, _, _ = F.bounds(fc.case, False)                        # (running maxima are moved by groups of rows)
    assert np.abs(got[rest] - clean[rest]).max() <= 2 * tol


def test_a_step_whose_pool_runs_dry():
    """Requests that are not served keep their length, their new tokens have no slots, and the others are served in full."""
    rng = np.random.Generator(np.random.PCG64(957))
    B, hq, hkv, d, bs, s, blocks = 5, 8, 2, 64, 8, 30, 12
    counts = [17, 30, 5, 40, 8]                                  # 3 + 4 + 1 + 5 blocks of 12: the fourth is not served, nor the last
    served = [True, True, True, False, False]
    new = lambda *shape: W.bf16_round(rng.standard_normal(shape, dtype=np.float32))  # noqa: E731
    k_sys, v_sys, n = new(s, hkv, d), new(s, hkv, d), sum(counts)
    q, kn, vn = new(n, hq, d), new(n, hkv, d), new(n, hkv, d)
    k, v = (torch.full(ra.fp4_cache_shape(blocks, hkv, bs, d), 0xFF, dtype=torch.uint8, device=DEV) for _ in range(2))
    tables = torch.full((B, 6), W.POISON_BLOCK, dtype=torch.int32, device=DEV)
    free, pool, pool_out = _i32(rng.permutation(blocks)), _i32([blocks, 0]), _i32([0, 0])
    held, cu, slots = _i32([-1] * B), _i32([-1] * (B + 1)), _i32([-7] * n)
    ra.relay_attn_update_tables(ra.make_table_params(tables, num_blocks=blocks, block_size=bs), _i32([0] * B), _i32(counts), pool,
                                pool_out, free, tables, held, cu, slots)
    out, lse = torch.full((n, hq, d), float("nan"), device=DEV), torch.empty((n, hq), device=DEV)
    ks, vs = _bf16(k_sys), _bf16(v_sys)
    p = ra.make_params(_bf16(q), out, ks, k, tables, batch=B, softmax_scale=d ** -0.5)
    ws = torch.full((ra.relay_attn_workspace_bytes(p, n),), 0xFF, dtype=torch.uint8, device=DEV)
    ra.relay_attn_cache_append_fp4(p, _bf16(kn), _bf16(vn), None, n, k, v, None, None, slot_map=slots)
    ra.relay_attn_prefill_fp4(p, _bf16(q), cu, n, max(counts), ks, vs, k, v, tables, held, out, lse, ws)
    torch.cuda.synchronize()
    assert held.tolist() == [c if ok else 0 for c, ok in zip(counts, served)] and pool_out.tolist() == [4, 2]
    at = np.cumsum([0] + counts)
    assert cu.tolist() == at.tolist()
    rows = [[F.values(*F.round_rows(x[at[i]:at[i + 1]])).astype(np.float32) for i in range(3)] for x in (kn, vn)]
    cfg = _cfg(batch=3, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, block_size=bs, sys_len=s)
    m = int(at[3])
    case = W.from_dense(cfg, q[:m], k_sys, v_sys, *rows, cu_seqlens_q=at[:4].astype(np.int32), poison_tails=False)
    want, _, _ = oracle.prefill_attention(q[:m], case.cu_seqlens_q, k_sys, v_sys, case.k_cache, case.v_cache, case.block_tables,
                                          case.context_lens, case.scale)
    got = out.cpu().numpy()
    assert np.abs(got[:m] - want).max() <= F.bounds(case, False)[0]
    assert (slots[m:] == -1).all() and np.isfinite(got[m:]).all()   # the others see the system prompt alone


def test_a_cache_beyond_four_gigabytes():
    """Blocks at the far end of a cache whose byte offsets pass 32 bits."""
    d, bs, hkv, hq = 128, 64, 8, 8
    case = W.make_case(_cfg(batch=3, num_q_heads=hq, num_kv_heads=hkv, block_size=bs, ctx_lo=100, ctx_hi=300), 961)
    fc = Fp4Case(case)
    block = fc.k.shape[1] * fc.k.shape[2]
    total = 2**32 // block + 2 + fc.k.shape[0]
    far = total - fc.k.shape[0]
    assert far * block > 2**32
    near = [fc.k, fc.v]
    fc.k, fc.v = (torch.empty((total, *x.shape[1:]), dtype=torch.uint8, device=DEV) for x in near)
    fc.k[far:], fc.v[far:] = near
    used = fc.tables < 2**30
    fc.tables = torch.where(used, fc.tables + far, fc.tables)
    fc.check()
    rows = torch.empty((int(case.context_lens[0]), hkv, d), dtype=torch.bfloat16, device=DEV)
    p = ra.make_params(fc.q, fc.q, None, fc.k, fc.tables, batch=1, softmax_scale=1.0)
    again = torch.empty_like(rows)
    ra.relay_attn_cache_read_fp4(p, rows, again, _i32([0, len(rows)]), len(rows), fc.k, fc.v, fc.tables, fc.lens)
    torch.cuda.synchronize()
    want, _ = W.logical_context(fc.case, 0)
    assert np.array_equal(rows.float().cpu().numpy(), want)


def test_a_context_becomes_a_system_prompt():
    """The whole context of a request, read out into a system cache in the recommended layout, is seen by the others of its
    batch as if they had it in front of their own."""
    cfg = _cfg(batch=3, sys_len=0, ctx_lo=77, ctx_hi=200, num_q_heads=4, num_kv_heads=4)
    fc = Fp4Case(W.make_case(cfg, 991))
    n, hkv, d = int(fc.case.context_lens[0]), 4, 128
    k_sys, v_sys = (ra.system_cache_view(torch.full((ra.relay_attn_system_cache_layout(n, hkv, d)[2] // 2,), float("nan"),
                                                    dtype=torch.bfloat16, device=DEV), n, hkv, d) for _ in range(2))
    p = ra.make_params(fc.q, fc.q, None, fc.k, fc.tables, batch=1, softmax_scale=1.0)
    ra.relay_attn_cache_read_fp4(p, k_sys, v_sys, _i32([0, n]), n, fc.k, fc.v, fc.tables, fc.lens)
    torch.cuda.synchronize()
    k, v = W.logical_context(fc.case, 0)
    assert np.array_equal(k_sys.float().cpu().numpy(), k) and np.array_equal(v_sys.float().cpu().numpy(), v)
    fc.k_sys, fc.v_sys = k_sys, v_sys
    fc.case = replace(fc.case, cfg=replace(cfg, sys_len=n), k_sys=k, v_sys=v)
    fc.check()


def test_a_block_that_holds_a_whole_context():
    fc = Fp4Case(W.make_case(_cfg(batch=3, block_size=4096, ctx_lo=1500, ctx_hi=3900, num_q_heads=4, num_kv_heads=2), 993))
    fc.check()
    fc.check(ctx_part_tokens=256)
    few = Fp4Case(W.make_case(_cfg(batch=2, block_size=2048, ctx_lo=1500, ctx_hi=1700, num_q_heads=4, num_kv_heads=2, q_lo=3,
                                   q_hi=9, head_dim=64), 994, prefill=True, extra_context=True))
    few.check(prefill=True)


def test_block_placement_and_stream_do_not_change_a_bit():
    case = W.make_case(_cfg(batch=4, ctx_lo=50, ctx_hi=400), 971)
    first = Fp4Case(case).run()
    fc = Fp4Case(W.repage(case, 972))
    second = fc.run()
    with torch.cuda.stream(torch.cuda.Stream()):
        third = fc.run()
    for other in (second, third):
        assert np.array_equal(first[0], other[0]) and np.array_equal(first[1], other[1])


# ---- a step as a serving loop makes it ---------------------------------------------------------------------------

def test_serving_steps_captured_in_a_graph_and_replayed():
    """Tables, append, prompt phase and then generation steps with a shared system prompt, the generation step a graph;
    every step against the oracle on the values that the cache holds by the format's definition."""
    rng = np.random.Generator(np.random.PCG64(981))
    B, hq, hkv, d, bs, s = 4, 8, 2, 128, 16, 90
    width, blocks = 12, 40
    new = lambda *shape: W.bf16_round(rng.standard_normal(shape, dtype=np.float32))  # noqa: E731
    k_sys, v_sys = new(s, hkv, d), new(s, hkv, d)
    prompt = [17, 1, 40, 33]
    k, v = (torch.full(ra.fp4_cache_shape(blocks, hkv, bs, d), 0xFF, dtype=torch.uint8, device=DEV) for _ in range(2))
    tables = torch.full((B, width), W.POISON_BLOCK, dtype=torch.int32, device=DEV)
    free, pools = _i32(rng.permutation(blocks)), [_i32([blocks, 0]), _i32([0, 0])]
    old, lens = _i32([0] * B), _i32(prompt)
    held, cu = torch.zeros_like(lens), torch.zeros(B + 1, dtype=torch.int32, device=DEV)
    tp = ra.make_table_params(tables, num_blocks=blocks, block_size=bs)
    ks, vs = _bf16(k_sys), _bf16(v_sys)
    history = [[[], []] for _ in range(B)]                      # what the cache should hold, per request: k rows, v rows

    def remember(k_new, v_new, counts):
        at = 0
        for i, m in enumerate(counts):
            for rows, x in zip(history[i], (k_new, v_new)):
                rows.extend(F.values(*F.round_rows(x[at:at + m])))
            at += m

    def check(q, counts, out, lse):
        cfg = _cfg(batch=B, num_q_heads=hq, num_kv_heads=hkv, block_size=bs, ctx_hi=width * bs, sys_len=s)
        case = W.from_dense(cfg, q, k_sys, v_sys, *[[np.array(history[i][x], dtype=np.float32) for i in range(B)] for x in (0, 1)],
                            cu_seqlens_q=np.cumsum([0] + counts).astype(np.int32), poison_tails=False)
        want, wlse, _ = oracle.prefill_attention(q, case.cu_seqlens_q, k_sys, v_sys, case.k_cache, case.v_cache,
                                                 case.block_tables, case.context_lens, case.scale)
        tol, ltol, _ = F.bounds(case, False)
        assert np.abs(out.cpu().numpy() - want).max() <= tol and np.abs(lse.cpu().numpy() - wlse).max() <= ltol

    # the prompts
    n = sum(prompt)
    slots = torch.zeros(n, dtype=torch.int32, device=DEV)
    q, kn, vn = new(n, hq, d), new(n, hkv, d), new(n, hkv, d)
    out, lse = torch.empty((n, hq, d), device=DEV), torch.empty((n, hq), device=DEV)
    ra.relay_attn_update_tables(tp, old, lens, pools[0], pools[1], free, tables, held, cu, slots)
    p = ra.make_params(_bf16(q), out, ks, k, tables, batch=B, softmax_scale=d ** -0.5)
    ws = torch.empty(ra.relay_attn_workspace_bytes(p, n), dtype=torch.uint8, device=DEV)
    ra.relay_attn_cache_append_fp4(p, _bf16(kn), _bf16(vn), None, n, k, v, None, None, slot_map=slots)
    ra.relay_attn_prefill_fp4(p, _bf16(q), cu, n, max(prompt), ks, vs, k, v, tables, held, out, lse, ws)
    torch.cuda.synchronize()
    assert pools[1].tolist() == [blocks - sum(-(-m // bs) for m in prompt), 0]
    remember(kn, vn, prompt)
    check(q, prompt, out, lse)

    # generation: one token each, the same graph every step
    qd, kd, vd = (torch.zeros((B, h, d), dtype=torch.bfloat16, device=DEV) for h in (hq, hkv, hkv))
    slots = torch.zeros(B, dtype=torch.int32, device=DEV)
    out, lse = torch.empty((B, hq, d), device=DEV), torch.empty((B, hq), device=DEV)
    p = ra.make_params(qd, out, ks, k, tables, batch=B, softmax_scale=d ** -0.5)
    ws = torch.empty(ra.relay_attn_workspace_bytes(p, B), dtype=torch.uint8, device=DEV)
    pools[0].copy_(pools[1])
    old.copy_(held)
    lens.copy_(old + 1)

    def step():
        ra.relay_attn_update_tables(tp, old, lens, pools[0], pools[1], free, tables, held, cu, slots)
        ra.relay_attn_cache_append_fp4(p, kd, vd, None, B, k, v, None, None, slot_map=slots)
        ra.relay_attn_decode_fp4(p, qd, ks, vs, k, v, tables, held, out, lse, ws)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(20):
        q, kn, vn = new(B, hq, d), new(B, hkv, d), new(B, hkv, d)
        for dst, src in ((qd, q), (kd, kn), (vd, vn)):
            dst.copy_(_bf16(src))
        graph.replay()
        torch.cuda.synchronize()
        remember(kn, vn, [1] * B)
        check(q, [1] * B, out, lse)
        replayed = out.clone()
        step()                                                   # the same step outside the graph, bit for bit
        torch.cuda.synchronize()
        assert torch.equal(out, replayed)
        pools[0].copy_(pools[1])
        old.copy_(held)
        lens.copy_(old + 1)
    used = sum(-(-(m + 20) // bs) for m in prompt)
    assert pools[1].tolist() == [blocks - used, 0]
