// What the host entry points share: the checks of ra_params.
#pragma once
#include "../../include/relay_attn.h"

#include <stdint.h>

#include "ra_kernels.h"

namespace ra {

// Block sizes of a 4-bit cache: its kernels take eight positions of a block at a time, and count bytes of a block in 31 bits.
constexpr int kFp4LeastBlock = 8, kFp4MostBlock = 1 << 24;
inline bool fp4_block_size(int32_t block_size) { return block_size >= kFp4LeastBlock && block_size <= kFp4MostBlock; }

// Rows that a call moves: a workgroup counts the 16-byte pieces of a token (of all kv heads) in 31 bits, with room for a round.
inline bool token_pieces_fit(const ra_params *p) { return (int64_t)p->num_kv_heads * (p->head_dim / 8) <= 1 << 30; }

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline ra_status check_params(const ra_params *p, int32_t total_q) {
    if (!p) return RA_ERR_INVALID_ARG;
    if (p->batch < 0 || total_q < 0 || p->num_q_heads < 1 || p->num_kv_heads < 1 ||
        p->sys_len < 0 || p->block_size < 1 || p->num_blocks < 0 || p->max_blocks_per_seq < 0 ||
        p->max_context_len < 0 || p->sys_chunk_tokens < 0 || p->ctx_part_tokens < 0 ||
        p->reserved0 != 0)
        return RA_ERR_INVALID_ARG;
    if (p->num_q_heads % p->num_kv_heads != 0) return RA_ERR_INVALID_ARG;
    if ((p->block_size & (p->block_size - 1)) != 0) return RA_ERR_INVALID_ARG;
    if (!(p->softmax_scale == p->softmax_scale)) return RA_ERR_INVALID_ARG;  // NaN
    if (p->out_is_fp32 != 0 && p->out_is_fp32 != 1) return RA_ERR_INVALID_ARG;
    const int64_t strides[] = {p->q_stride_token, p->q_stride_head, p->o_stride_token,
                               p->o_stride_head, p->sys_stride_token, p->sys_stride_head};
    for (int64_t s : strides)
        if (s < 0 || (s % 8) != 0) return RA_ERR_INVALID_ARG;
    if (p->sys_chunk_tokens % 32 != 0 || p->ctx_part_tokens % 128 != 0) return RA_ERR_INVALID_ARG;
    if ((int64_t)p->max_blocks_per_seq * p->block_size > INT32_MAX) return RA_ERR_INVALID_ARG;
    if (p->max_context_len > (int64_t)p->max_blocks_per_seq * p->block_size)
        return RA_ERR_INVALID_ARG;
    if (p->head_dim != 64 && p->head_dim != 128) return RA_ERR_UNSUPPORTED;
    const int g = p->num_q_heads / p->num_kv_heads;
    if (g < 1 || g > 8) return RA_ERR_UNSUPPORTED;
    if ((int64_t)total_q * p->num_q_heads > (1 << 28)) return RA_ERR_UNSUPPORTED;
    return RA_OK;
}

// Attention over a 4-bit context cache: the plans and launches of the bf16 calls (relay_attn.hip), with the kernels
// that those do not have handed in.  cu_seqlens_q null: a decode step.
struct Fp4Calls {
    hipError_t (*decode_direct)(const DirectArgs &, const DirectOne &, int head_dim, hipStream_t);
};
ra_status attend_fp4(const ra_params *p, const void *q, const int32_t *cu_seqlens_q, int32_t total_q, int32_t max_q_len,
                     const void *k_sys, const void *v_sys, const void *k_cache, const void *v_cache,
                     const int32_t *block_tables, const int32_t *context_lens, void *out, float *lse_out,
                     void *workspace, size_t workspace_bytes, void *hip_stream, const Fp4Calls &calls);

}  // namespace ra
