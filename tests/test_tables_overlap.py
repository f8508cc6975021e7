"""relay_attn_update_tables: an array that is written on top of another one is refused, before any launch."""
import ctypes

import pytest

from paper_2402_14808_amd import binding
from test_abi import _params
import fp4_launches as L

V = ctypes.c_void_p
BATCH, WIDTH, BLOCKS, SLOTS = 4, 8, 64, 5
# name, numbers of 32 bits; in the order of the arguments
ARRAYS = [("old_lens", BATCH), ("new_lens", BATCH), ("pool_in", 2), ("pool_out", 2), ("free_blocks", BLOCKS), ("block_tables", BATCH * WIDTH),
          ("context_lens", BATCH), ("cu_seqlens_q", BATCH + 1), ("slot_map", SLOTS)]
READ = ("old_lens", "new_lens", "pool_in")


def _call(at, batch=BATCH):
    p = _params(batch=batch, num_blocks=BLOCKS, max_blocks_per_seq=WIDTH)
    status = L.library().relay_attn_update_tables(ctypes.byref(p), *[V(at[name]) for name, _ in ARRAYS], SLOTS, None)
    launched = L.library().take_launches()
    assert (launched != b"[]") == (status == binding.RA_OK)
    return status


def _side_by_side():
    at, address = {}, 1 << 20
    for name, n in ARRAYS:
        at[name] = address
        address += 4 * n
    return at


def test_arrays_side_by_side_are_fine():
    assert _call(_side_by_side()) == binding.RA_OK
    assert _call({**_side_by_side(), "cu_seqlens_q": None}) == binding.RA_OK
    at = _side_by_side()
    assert _call({**at, "new_lens": at["old_lens"]}) == binding.RA_OK                       # only read
    assert _call({**at, "old_lens": at["context_lens"], "new_lens": at["context_lens"]}, batch=0) == binding.RA_OK      # nothing there


@pytest.mark.parametrize("written", [name for name, _ in ARRAYS if name not in READ])
@pytest.mark.parametrize("other", [name for name, _ in ARRAYS])
def test_one_on_top_of_another(written, other):
    if written == other:
        return
    size = dict(ARRAYS)
    at = _side_by_side()
    for address in (at[other], at[other] + 4 * (size[other] - 1), at[other] - 4 * (size[written] - 1)):      # first, last number shared
        moved = {**{name: a + (1 << 24) for name, a in at.items()}, other: at[other], written: address}
        assert _call(moved) == binding.RA_ERR_INVALID_ARG, (written, other)
    for address in (at[other] + 4 * size[other], at[other] - 4 * size[written]):                             # beside it
        moved = {**{name: a + (1 << 24) for name, a in at.items()}, other: at[other], written: address}
        assert _call(moved) == binding.RA_OK, (written, other)
