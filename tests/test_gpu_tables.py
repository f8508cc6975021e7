"""relay_attn_update_tables against a scheduler that goes through the requests one by one."""
import sys

import numpy as np
import pytest
import torch

import paper_2402_14808_amd as ra

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NOT_USED = 0x7FFFFFF0


def _say(msg):
    print("[case] " + msg, flush=True)
    sys.stdout.flush()


def one_by_one(old, new, tables, free, height, bs, n_slots):
    """(tables, lengths, running sums, slots, [height, not served], stack) after the step."""
    tables, free = tables.copy(), free.copy()
    cap = tables.shape[1] * bs
    old = [min(max(int(x), 0), cap) for x in old]
    new = [max(int(x), 0) for x in new]
    blocks = lambda x: -(-x // bs)  # noqa: E731
    stack = [int(x) for x in free[:height]]
    for i, (a, b) in enumerate(zip(old, new)):
        if b <= cap:
            stack += [int(x) for x in tables[i, blocks(b):blocks(a)]]
    top, asked, lens, sums, slots, left_out = len(stack), 0, [], [0], [], 0
    for i, (a, b) in enumerate(zip(old, new)):
        need = max(0, blocks(b) - blocks(a)) if b <= cap else 0
        asked += need
        served = b <= cap and (need == 0 or asked <= top)
        if served:
            for j in range(need):
                tables[i, blocks(a) + j] = stack.pop()
        left_out += not served
        lens.append(b if served else a)
        sums.append(sums[-1] + max(0, b - a))
        slots += [int(tables[i, p // bs]) * bs + p % bs if served else -1 for p in range(a, max(a, b))][:max(0, n_slots - len(slots))]
    for k in range(height, len(stack)):
        free[k] = stack[k]
    return tables, lens, sums, slots + [-1] * (n_slots - len(slots)), [len(stack), left_out], free


def _case(rng, batch, bs, width, spare, grow, shrink=0.2, end=0.1, top_len=None):
    cap = width * bs
    top_len = cap if top_len is None else top_len
    old = rng.integers(0, top_len + 1, batch)
    new = np.minimum(old + rng.integers(0, grow + 1, batch), cap)
    kind = rng.random(batch)
    new = np.where(kind < shrink, np.maximum(old - rng.integers(0, grow + 1, batch), 0), new)
    new = np.where(kind > 1 - end, 0, new)
    held = -(-old // bs)
    total = int(held.sum()) + spare
    ids = rng.permutation(total).astype(np.int32)
    tables = np.full((batch, width), NOT_USED, dtype=np.int32)
    at = 0
    for i, h in enumerate(held):
        tables[i, :h] = ids[at:at + h]
        at += int(h)
    free = np.full(total, NOT_USED, dtype=np.int32)
    free[:spare] = ids[at:]
    return old.astype(np.int32), new.astype(np.int32), tables, free, spare


def _run(old, new, tables, free, height, bs, n_slots, sums=True):
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)  # noqa: E731
    t, f = dev(tables), dev(free)
    pool_in, pool_out = dev([height, 0]), dev([-5, -5])
    lens = torch.full((len(old),), -9, dtype=torch.int32, device=DEV)
    cu = torch.full((len(old) + 1,), -9, dtype=torch.int32, device=DEV) if sums else None
    slots = torch.full((n_slots,), -9, dtype=torch.int32, device=DEV) if n_slots else None
    p = ra.make_table_params(t, num_blocks=len(free), block_size=bs)
    o, n = dev(old), dev(new)
    results = []
    for _ in range(2):                                  # the second call works on what the first left: the same again
        ra.relay_attn_update_tables(p, o, n, pool_in, pool_out, f, t, lens, cu, slots)
        torch.cuda.synchronize()
        results.append([x.cpu().numpy().copy() if x is not None else None for x in (t, lens, cu, slots, pool_out, f)])
    for a, b in zip(*results):
        assert (a is None and b is None) or np.array_equal(a, b)
    return results[0]


def _check(old, new, tables, free, height, bs, n_slots=None, sums=True):
    total = int(sum(max(0, max(int(b), 0) - min(max(int(a), 0), tables.shape[1] * bs)) for a, b in zip(old, new)))
    n_slots = total if n_slots is None else n_slots
    want = one_by_one(old, new, tables, free, height, bs, n_slots)
    got = _run(old, new, tables, free, height, bs, n_slots, sums)
    for name, a, b in zip(("tables", "lengths", "sums", "slots", "pool", "stack"), got, want):
        if a is not None:
            assert np.array_equal(a, np.asarray(b, dtype=np.int32)), name


@pytest.mark.parametrize("batch,bs,width,grow", [(1, 16, 4, 5), (3, 1, 9, 2), (64, 16, 20, 40), (255, 8, 6, 9), (256, 16, 5, 16),
                                                (257, 32, 5, 70), (700, 16, 9, 33), (2500, 16, 7, 20)])
@pytest.mark.parametrize("supply", ["plenty", "scarce", "none"])
def test_any_mix_of_growing_shrinking_and_ending_requests(batch, bs, width, grow, supply):
    rng = np.random.Generator(np.random.PCG64(batch * 31 + bs))
    want = batch * (grow // bs + 2)
    spare = {"plenty": want, "scarce": want // 6, "none": 0}[supply]
    _say("batch %d block %d width %d grow %d spare %d" % (batch, bs, width, grow, spare))
    _check(*_case(rng, batch, bs, width, spare, grow), bs)


def test_long_prompts_and_more_or_fewer_slots_than_tokens():
    rng = np.random.Generator(np.random.PCG64(77))
    case = _case(rng, 5, 16, 900, 5000, 14000, shrink=0.0, end=0.0, top_len=100)
    total = int((case[1] - case[0]).sum())
    for n_slots in (total, total + 1500, 1000, 0):
        _check(*case, 16, n_slots=n_slots)
    _check(*case, 16, sums=False)


def test_everyone_ends_and_a_pool_of_every_block():
    rng = np.random.Generator(np.random.PCG64(78))
    old, _, tables, free, height = _case(rng, 40, 16, 8, 3, 10)
    _check(old, np.zeros_like(old), tables, free, height, 16)
    _check(np.zeros_like(old), np.zeros_like(old), tables, free, height, 16)


def test_lengths_that_do_not_fit_or_are_negative():
    rng = np.random.Generator(np.random.PCG64(79))
    old, new, tables, free, height = _case(rng, 30, 16, 8, 200, 40, top_len=100)
    new = np.minimum(new + 1, 128)
    new[[3, 11, 29]] = [129, 5000, 2**30]               # beyond the row's 128 positions
    new[[5, 6]] = [-4, -2**31]
    old[7], tables[7] = -3, NOT_USED
    _check(old, new, tables, free, height, 16, n_slots=3000)


def test_a_height_that_is_no_height_and_an_empty_batch():
    rng = np.random.Generator(np.random.PCG64(80))
    old, new, tables, free, height = _case(rng, 12, 16, 8, 50, 40)
    none = _run(old, new, tables, free, -7, 16, 10)
    assert np.array_equal(none[0], one_by_one(old, new, tables, free, 0, 16, 10)[0])
    empty = _run(old[:0], new[:0], tables[:0], free, height, 16, 4)
    assert empty[4].tolist() == [height, 0] and empty[2].tolist() == [0] and empty[3].tolist() == [-1] * 4
