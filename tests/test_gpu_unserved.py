"""A scheduler step whose pool runs dry for requests that have rows in the cache: the cache write that follows leaves those rows
as they are."""
import numpy as np
import pytest
import torch

import fp4_util as F
import paper_2402_14808_amd as ra
import workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BS, HKV, D, WIDTH = 8, 2, 64, 8
OLD = [20, 33, 9, 16, 40, 24, 3]
NEW = [21, 45, 9, 17, 60, 30, 0]           # the last ends and gives a block back; 0 + 1 + 0 + 1 + 3 + 1 are asked for


def _i32(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


class Step:
    def __init__(self, spare):
        rng = np.random.Generator(np.random.PCG64(1301))
        held = [-(-n // BS) for n in OLD]
        self.blocks = sum(held) + spare
        ids, at = rng.permutation(self.blocks), 0
        rows = np.full((len(OLD), WIDTH), W.POISON_BLOCK, dtype=np.int32)
        for row, n in zip(rows, held):
            row[:n] = ids[at:at + n]
            at += n
        self.before = rows
        self.old, self.tables = _i32(OLD), torch.from_numpy(rows).to(DEV)
        self.free = _i32(list(ids[at:]) + [W.POISON_BLOCK] * at)
        self.pool, self.pool_out = _i32([spare, 0]), _i32([-1, -1])
        self.counts = [max(0, b - a) for a, b in zip(OLD, NEW)]
        self.rng = rng

    def update(self, new):
        lens, cu = _i32([-1] * len(OLD)), _i32([-1] * (len(OLD) + 1))
        slots = _i32([-7] * sum(self.counts))
        ra.relay_attn_update_tables(ra.make_table_params(self.tables, num_blocks=self.blocks, block_size=BS), self.old, new,
                                    self.pool, self.pool_out, self.free, self.tables, lens, cu, slots)
        torch.cuda.synchronize()
        return lens, cu, slots

    def places(self, lens):
        """(block, offset) of the new tokens of the requests that are served, in order, and those tokens."""
        tables, at, places, tokens = self.tables.cpu().numpy(), 0, [], []
        for i, m in enumerate(self.counts):
            if int(lens[i]) == NEW[i]:
                places += [(int(tables[i, p // BS]), p % BS) for p in range(OLD[i], NEW[i])]
                tokens += range(at, at + m)
            at += m
        return places, tokens

    def rows(self, n):
        return torch.from_numpy(W.bf16_round(self.rng.standard_normal((n, HKV, D), dtype=np.float32))).to(DEV, torch.bfloat16)


# blocks that are free before the step (one comes back in it), and who is served with them
SUPPLY = {0: [1, 1, 1, 0, 0, 0, 1], 1: [1, 1, 1, 1, 0, 0, 1], 3: [1, 1, 1, 1, 0, 0, 1], 5: [1] * 7}


@pytest.mark.parametrize("spare", SUPPLY)
def test_append_by_slots_leaves_the_rows_of_requests_that_are_not_served(spare):
    step = Step(spare)
    lens, _, slots = step.update(_i32(NEW))
    assert [int(n) for n in lens] == [b if ok else a for a, b, ok in zip(OLD, NEW, SUPPLY[spare])]
    k, v = (torch.full(ra.fp4_cache_shape(step.blocks, HKV, BS, D), 0x2A, dtype=torch.uint8, device=DEV) for _ in range(2))
    k_new, v_new = step.rows(sum(step.counts)), step.rows(sum(step.counts))
    p = ra.make_params(k_new, k_new, None, k, step.tables, batch=len(OLD), softmax_scale=1.0)
    ra.relay_attn_cache_append_fp4(p, k_new, v_new, None, len(k_new), k, v, None, None, slot_map=slots)
    torch.cuda.synchronize()
    places, tokens = step.places(lens)
    for cache, new in ((k, k_new), (v, v_new)):
        code, scale = F.unpack(np.full(tuple(cache.shape), 0x2A, dtype=np.uint8), BS, D)
        code, scale = code.copy(), scale.copy()
        new_code, new_scale = F.round_rows(new.double().cpu().numpy())
        for (block, off), t in zip(places, tokens):
            code[block, :, off], scale[block, :, off] = new_code[t], new_scale[t]
        assert np.array_equal(cache.cpu().numpy(), F.pack(code, scale))


@pytest.mark.parametrize("spare", SUPPLY)
@pytest.mark.parametrize("fp4", [False, True], ids=["bf16", "fp4"])
def test_append_by_lengths_of_a_second_call_leaves_them_too(spare, fp4):
    step = Step(spare)
    lens, _, _ = step.update(_i32(NEW))
    first = [x.clone() for x in (step.tables, step.free, step.pool_out)]
    again, cu, _ = step.update(lens)
    assert torch.equal(again, lens) and torch.equal(step.tables, first[0]) and torch.equal(step.free, first[1])
    assert step.pool_out.tolist() == [int(first[2][0]), 0]
    places, tokens = step.places(lens)
    assert cu.tolist() == np.cumsum([0] + [m if ok else 0 for m, ok in zip(step.counts, SUPPLY[spare])]).tolist()
    k_new, v_new = (step.rows(sum(step.counts))[tokens] for _ in range(2))
    if fp4:
        k, v = (torch.full(ra.fp4_cache_shape(step.blocks, HKV, BS, D), 0x2A, dtype=torch.uint8, device=DEV) for _ in range(2))
        call = ra.relay_attn_cache_append_fp4
    else:
        k, v = (torch.full((step.blocks, HKV, BS, D), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        call = ra.relay_attn_cache_append
    p = ra.make_params(k_new, k_new, None, k, step.tables, batch=len(OLD), softmax_scale=1.0)
    call(p, k_new, v_new, cu, len(tokens), k, v, step.tables, again)
    torch.cuda.synchronize()
    for cache, new in ((k, k_new), (v, v_new)):
        if fp4:
            code, scale = (x.copy() for x in F.unpack(np.full(tuple(cache.shape), 0x2A, dtype=np.uint8), BS, D))
            new_code, new_scale = F.round_rows(new.double().cpu().numpy())
            for j, (block, off) in enumerate(places):
                code[block, :, off], scale[block, :, off] = new_code[j], new_scale[j]
            assert np.array_equal(cache.cpu().numpy(), F.pack(code, scale))
        else:
            want = torch.full_like(cache, 7.0)
            for j, (block, off) in enumerate(places):
                want[block, :, off] = new[j]
            assert torch.equal(cache, want)
