"""A batch padded to a fixed number of tokens: those behind the last request's have no place in a cache, and read-out leaves their
rows as they were."""
import numpy as np
import pytest
import torch

import fp4_util as F
import paper_2402_14808_amd as ra
import workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _i32(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


# new tokens and lengths of the requests; block-table slots behind the ones in use name a block that holds rows of its own
CASES = [([3, 5], [11, 16]), ([4, 0, 2], [4, 9, 8]), ([0, 0], [5, 7]), ([1] * 64, [9] * 64), ([2] * 70, [15] * 70)]


@pytest.mark.parametrize("counts,lens", CASES, ids=[str(i) for i in range(len(CASES))])
@pytest.mark.parametrize("fp4", [False, True], ids=["bf16", "fp4"])
def test_tokens_of_no_request(counts, lens, fp4):
    rng = np.random.Generator(np.random.PCG64(1501))
    bs, hkv, d, width, batch, pad = 8, 2, 64, 5, len(counts), 21
    blocks = 2 * batch + 1
    ids = rng.permutation(blocks)
    tables = np.full((batch, width), ids[-1], dtype=np.int32)
    tables[:, 0], tables[:, 1] = ids[:batch], np.where(np.array(lens) > bs, ids[batch:-1], ids[-1])
    cu = np.cumsum([0] + counts)
    n = int(cu[-1])
    k_new, v_new = (torch.from_numpy(W.bf16_round(rng.standard_normal((n + pad, hkv, d), dtype=np.float32))).to(DEV, torch.bfloat16)
                    for _ in range(2))
    if fp4:
        k, v = (torch.full(ra.fp4_cache_shape(blocks, hkv, bs, d), 0x2A, dtype=torch.uint8, device=DEV) for _ in range(2))
    else:
        k, v = (torch.full((blocks, hkv, bs, d), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    p = ra.make_params(k_new, k_new, None, k, torch.from_numpy(tables), batch=batch, softmax_scale=1.0)
    where = (_i32(cu.tolist()), n + pad, k, v, torch.from_numpy(tables).to(DEV), _i32(lens))
    (ra.relay_attn_cache_append_fp4 if fp4 else ra.relay_attn_cache_append)(p, k_new, v_new, *where)
    places = [(tables[i, q // bs], q % bs) for i, m in enumerate(counts) for q in range(lens[i] - m, lens[i])]
    torch.cuda.synchronize()
    for cache, new in ((k, k_new), (v, v_new)):
        if fp4:
            code, scale = (x.copy() for x in F.unpack(np.full(tuple(cache.shape), 0x2A, dtype=np.uint8), bs, d))
            new_code, new_scale = F.round_rows(new.double().cpu().numpy())
            for t, (block, off) in enumerate(places):
                code[block, :, off], scale[block, :, off] = new_code[t], new_scale[t]
            assert np.array_equal(cache.cpu().numpy(), F.pack(code, scale))
        else:
            want = torch.full_like(cache, 7.0)
            for t, (block, off) in enumerate(places):
                want[int(block), :, off] = new[t]
            assert torch.equal(cache, want)
    if fp4:
        out = torch.full((2, n + pad, hkv, d), 3.0, dtype=torch.bfloat16, device=DEV)
        ra.relay_attn_cache_read_fp4(p, out[0], out[1], *where)
        torch.cuda.synchronize()
        assert (out[:, n:] == 3.0).all() and (n == 0 or not (out[:, :n] == 3.0).all())
