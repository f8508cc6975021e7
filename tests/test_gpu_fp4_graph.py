"""The calls of a 4-bit cache in a captured graph, replayed with other lengths, tables and values, and two streams at once: the
same bits as the calls made one by one."""
import numpy as np
import pytest
import torch

import paper_2402_14808_amd as ra
import workloads as W
from test_gpu_fp4 import _bf16, _cfg, _i32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Prompts:
    """append by lengths, prompt phase and read-out of what was appended, over buffers that stay where they are."""

    def __init__(self, cfg, counts, longest):
        self.cfg, self.counts, self.longest = cfg, counts, longest
        self.n, d, hkv, hq = sum(counts), cfg.head_dim, cfg.num_kv_heads, cfg.num_q_heads
        self.width = -(-longest // cfg.block_size)
        self.blocks = cfg.batch * self.width + 3
        self.k, self.v = (torch.full(ra.fp4_cache_shape(self.blocks, hkv, cfg.block_size, d), 0x33, dtype=torch.uint8, device=DEV) for _ in range(2))
        self.q = torch.zeros((self.n, hq, d), dtype=torch.bfloat16, device=DEV)
        self.k_new, self.v_new, self.k_out, self.v_out = (torch.zeros((self.n, hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(4))
        self.k_sys, self.v_sys = (torch.zeros((cfg.sys_len, hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        self.tables = torch.zeros((cfg.batch, self.width), dtype=torch.int32, device=DEV)
        self.lens = torch.zeros(cfg.batch, dtype=torch.int32, device=DEV)
        self.cu = _i32(np.cumsum([0] + counts))
        self.out, self.lse = torch.zeros((self.n, hq, d), device=DEV), torch.zeros((self.n, hq), device=DEV)
        self.p = ra.make_params(self.q, self.out, self.k_sys, self.k, self.tables, batch=cfg.batch, softmax_scale=cfg.scale, max_context_len=longest)
        self.ws = torch.full((ra.relay_attn_workspace_bytes(self.p, self.n),), 0xFF, dtype=torch.uint8, device=DEV)

    def fill(self, seed):
        rng = np.random.Generator(np.random.PCG64(seed))
        for x in (self.q, self.k_new, self.v_new, self.k_sys, self.v_sys):
            x.copy_(_bf16(W.bf16_round(rng.standard_normal(tuple(x.shape), dtype=np.float32))))
        self.lens.copy_(_i32([rng.integers(max(m, 1), self.longest + 1) for m in self.counts]))
        self.tables.copy_(_i32(rng.permutation(self.blocks)[:self.tables.numel()].reshape(self.tables.shape)))

    def calls(self):
        where = (self.k, self.v, self.tables, self.lens)
        ra.relay_attn_cache_append_fp4(self.p, self.k_new, self.v_new, self.cu, self.n, *where)
        ra.relay_attn_prefill_fp4(self.p, self.q, self.cu, self.n, max(self.counts), self.k_sys, self.v_sys, *where, self.out, self.lse, self.ws)
        ra.relay_attn_cache_read_fp4(self.p, self.k_out, self.v_out, self.cu, self.n, *where)

    def results(self):
        return [x.clone() for x in (self.out, self.lse, self.k_out, self.v_out, self.k, self.v)]


SHAPES = {
    "few": (_cfg(batch=9, num_q_heads=8, num_kv_heads=2, sys_len=70), [3, 1, 8, 0, 5, 2, 7, 1, 4], 2300),
    "few, 64-wide heads": (_cfg(batch=5, num_q_heads=8, num_kv_heads=4, head_dim=64, sys_len=300, block_size=8), [3, 1, 8, 0, 5], 3000),
    "whole": (_cfg(batch=3, sys_len=90), [60, 33, 80], 90),
    "many rows": (_cfg(batch=6, sys_len=1500), [2, 3, 1, 4, 2, 20], 60),
}


@pytest.mark.parametrize("name", SHAPES)
def test_replays_are_the_calls_made_one_by_one(name):
    s = Prompts(*SHAPES[name])
    s.fill(1600)
    s.calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.calls()
    for turn in range(4):
        s.fill(1601 + turn)
        before = [x.clone() for x in (s.k, s.v)]
        graph.replay()
        torch.cuda.synchronize()
        replayed = s.results()
        for x, was in zip((s.k, s.v), before):
            x.copy_(was)
        for x in (s.out, s.lse, s.k_out, s.v_out):
            x.fill_(float("nan"))
        s.calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, s.results()))
        assert all(torch.isfinite(x.float()).all() for x in replayed[:4])


def test_two_streams_at_once():
    """Each with a workspace and buffers of its own."""
    steps = [Prompts(*SHAPES["few"]), Prompts(*SHAPES["many rows"])]
    alone = []
    for i, s in enumerate(steps):
        s.fill(1700 + i)
        s.calls()
        torch.cuda.synchronize()
        alone.append(s.results())
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(5):
        for s, stream in zip(steps, streams):
            with torch.cuda.stream(stream):
                s.calls()
    torch.cuda.synchronize()
    for s, want in zip(steps, alone):
        assert all(torch.equal(a, b) for a, b in zip(s.results(), want))
