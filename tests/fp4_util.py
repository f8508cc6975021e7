"""The 4-bit cache format in numpy, written from its definition, and attention cases over it.

Values are looked up among the numbers the format has; nothing here is shared with the library."""
from __future__ import annotations

from dataclasses import replace

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def round_rows(x):
    """x [..., d] (float64 holding bfloat16 values): codes [..., d] uint8, scale bytes [..., d / 32] uint8."""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    mag = np.where(np.isnan(blocks), np.inf, np.abs(blocks))
    top = mag.max(-1)
    with np.errstate(divide="ignore", invalid="ignore"):
        low = np.floor(np.log2(np.where((top > 0) & np.isfinite(top), top, 1.0)))
        e = low - 2 + (top >= 1.75 * 2.0 ** low)
        e = np.where(top == 0, -127, np.where(np.isinf(top), 125, np.clip(e, -127, 125))).astype(np.int64)
        y = mag / (2.0 ** e)[..., None]
    y = np.minimum(y, 1e9)
    dist = np.abs(y[..., None] - GRID)
    near = dist == dist.min(-1, keepdims=True)
    # of two equally near, the even code; behind the last, the last
    code = np.where(near[..., ::2].any(-1), 2 * near[..., ::2].argmax(-1), near.argmax(-1))
    code = np.where(y >= 6, 7, code)
    sign = np.signbit(blocks)
    code = (code + 8 * sign).astype(np.uint8).reshape(x.shape)
    return code, (e + 127).astype(np.uint8)


def values(code, scale):
    """codes [..., d], scale bytes [..., d / 32] -> float64 [..., d]."""
    v = GRID[code & 7] * np.where(code & 8, -1.0, 1.0)
    v = v.reshape(*v.shape[:-1], -1, 32) * (2.0 ** (scale.astype(np.float64) - 127))[..., None]
    return v.reshape(code.shape)


def pack(code, scale):
    """codes [num_blocks, Hkv, block_size, d], scales [num_blocks, Hkv, block_size, d / 32] -> the cache's bytes."""
    nb, hkv, bs, d = code.shape
    out = np.empty((nb, hkv, bs * (d // 2 + d // 32)), dtype=np.uint8)
    out[..., :bs * d // 2] = (code[..., 0::2] | code[..., 1::2] << 4).reshape(nb, hkv, -1)
    out[..., bs * d // 2:] = scale.transpose(0, 1, 3, 2).reshape(nb, hkv, -1)
    return out


def unpack(cache, bs, d):
    nb, hkv, _ = cache.shape
    raw = cache[..., :bs * d // 2].reshape(nb, hkv, bs, d // 2)
    code = np.stack((raw & 15, raw >> 4), -1).reshape(nb, hkv, bs, d)
    return code, cache[..., bs * d // 2:].reshape(nb, hkv, d // 32, bs).transpose(0, 1, 3, 2)


def to_fp4(case):
    """(case whose context caches hold what the format makes of them, k bytes, v bytes).  What the tables do not use, whole
    blocks and the tails of last ones, is 0xff throughout: codes of -6 under a power of two that does not exist."""
    bs = case.cfg.block_size
    used = np.zeros((case.k_cache.shape[0], bs), dtype=bool)
    for i, c in enumerate(case.context_lens):
        for p in range(int(c)):
            used[case.block_tables[i, p // bs], p % bs] = True
    out = []
    for cache in (case.k_cache, case.v_cache):
        clean = np.where(used[:, None, :, None], cache, 0.0)
        code, scale = round_rows(clean)
        held = values(code, scale)
        code[~np.broadcast_to(used[:, None], code.shape[:3])] = 0xF
        scale[~np.broadcast_to(used[:, None], scale.shape[:3])] = 0xFF
        out.append((held.astype(np.float32), pack(code, scale)))
    (k, kb), (v, vb) = out
    return replace(case, k_cache=k, v_cache=v), kb, vb


def bounds(case, bf16_out, scale=None):
    """How far an output, a log-sum-exp, and the outputs' 2-norm relative to their own may be off.
      scores   a sum of d exact products in 32 bits: each addition is off by 2^-24 of a partial sum, which is at most |q| |k|
               (`smax` with the scale); sqrt(d) of them add up at random, eight standard deviations of that; the
               exponential and the scale's own product add 2^-22 of the exponent
      weights  split into two bfloat16 parts for a bfloat16 output, half a step of the second being 2^-17 of the weight, and
               into three for an fp32 one, 2^-26
      output   a mean of values of at most `vmax` with those weights, whose relative errors count twice (in the sum above
               and the sum below); half a step, 2^-8 of it, where it is stored in bfloat16
      norm     the errors of the weights do not add up coherently: one standard deviation of them, twice
      sums     what is left at a scale of zero, where all scores are equal: each of n additions of a sum over n positions is off
               by at most 2^-24 of a partial sum, at random sqrt(n) 2^-24 of the sum; then the reciprocal, its product, the
               weight in the merge and the stored fp32 result are rounded once each, 4 * 2^-24
    """
    d = case.cfg.head_dim
    keys = np.concatenate([np.nan_to_num(case.k_sys).reshape(-1, d), case.k_cache.reshape(-1, d)]).astype(np.float64)
    vmax = max(np.abs(np.nan_to_num(case.v_sys)).max(initial=0.0), np.abs(case.v_cache).max())
    smax = abs(case.scale if scale is None else scale) * (np.linalg.norm(case.q.reshape(-1, d).astype(np.float64), axis=-1).max() *
                                                          np.linalg.norm(keys, axis=-1).max())
    score = (8 * d ** 0.5 * 2.0 ** -24 + 2.0 ** -22) * smax
    weight = 2.0 ** (-17 if bf16_out else -26)
    sums = ((case.cfg.sys_len + int(case.context_lens.max())) ** 0.5 + 4) * 2.0 ** -24
    out = vmax * (2 * score + 2 * weight + sums)
    norm = 2 * (weight + d ** 0.5 * 2.0 ** -24 * smax) + sums
    return out + (vmax * 2.0 ** -8 if bf16_out else 0.0), score + 2.0 ** -16, norm + (2.0 ** -8 if bf16_out else 0.0)
