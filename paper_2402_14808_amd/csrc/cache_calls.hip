// Host side of the calls around the 4-bit context cache and the block tables (include/relay_attn.h): argument checks before
// any HIP call, then the launches.  Attention over the cache shares the plans of the bf16 calls (relay_attn.hip).
#include "../../include/relay_attn.h"

#include <hip/hip_runtime.h>

#include "ra_host.h"
#include "ra_kernels.h"

using ra::aligned16;
using ra::check_params;
using ra::fp4_block_size;

namespace {

// Rows of the 4-bit cache: written from k / v, or read out into them.
ra_status fp4_rows(const ra_params *p, void *k, void *v, int64_t stride_token, int64_t stride_head,
                   const int32_t *cu_seqlens_q, int32_t total_q, const int32_t *slot_map, void *k_cache, void *v_cache,
                   const int32_t *block_tables, const int32_t *context_lens, void *hip_stream, bool read) {
    const ra_status st = check_params(p, total_q);
    if (st != RA_OK) return st;
    if (!fp4_block_size(p->block_size) || !ra::token_pieces_fit(p)) return RA_ERR_UNSUPPORTED;
    if (stride_token < 0 || stride_head < 0 || stride_token % 8 || stride_head % 8) return RA_ERR_INVALID_ARG;
    if (!slot_map && !cu_seqlens_q && total_q != p->batch) return RA_ERR_INVALID_ARG;
    if (total_q == 0) return RA_OK;
    if (!k || !v || !k_cache || !v_cache) return RA_ERR_INVALID_ARG;
    if (p->num_blocks < 1) return RA_ERR_INVALID_ARG;        // (no place would be in range)
    if (!slot_map && (p->batch < 1 || !block_tables || !context_lens)) return RA_ERR_INVALID_ARG;
    if (!aligned16(k) || !aligned16(v) || !aligned16(k_cache) || !aligned16(v_cache)) return RA_ERR_INVALID_ARG;
    if (stride_head < p->head_dim && p->num_kv_heads > 1) return RA_ERR_INVALID_ARG;
    // Rows that are written may not overlap: tokens behind all heads of a token, or heads behind all tokens of a head.
    if (read && total_q > 1 && stride_token < (p->num_kv_heads - 1) * stride_head + p->head_dim &&
        (stride_token < p->head_dim || stride_head < (total_q - 1) * stride_token + p->head_dim))
        return RA_ERR_INVALID_ARG;
    ra::Fp4RowsArgs a{};
    a.k_rows = static_cast<uint16_t *>(k);
    a.v_rows = static_cast<uint16_t *>(v);
    a.k_cache = static_cast<uint8_t *>(k_cache);
    a.v_cache = static_cast<uint8_t *>(v_cache);
    a.slot_map = slot_map;
    a.block_tables = block_tables;
    a.context_lens = context_lens;
    a.cu_seqlens_q = cu_seqlens_q;
    a.stride_token = stride_token;
    a.stride_head = stride_head;
    a.n_slots = (int64_t)p->num_blocks * p->block_size;
    a.batch = p->batch;
    a.n_tokens = total_q;
    a.Hkv = p->num_kv_heads;
    while ((1 << a.block_size_log2) < p->block_size) ++a.block_size_log2;
    a.max_blocks_per_seq = p->max_blocks_per_seq;
    return ra::launch_fp4_rows(a, p->head_dim, read, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? RA_OK
                                                                                                       : RA_ERR_HIP;
}

struct Range {                                            // of 32-bit numbers; null: none
    const int32_t *first;
    int64_t n;
    bool meets(const Range &o) const {
        const uintptr_t a = reinterpret_cast<uintptr_t>(first), b = reinterpret_cast<uintptr_t>(o.first);
        return first && o.first && n > 0 && o.n > 0 && a < b + 4 * (uintptr_t)o.n && b < a + 4 * (uintptr_t)n;
    }
};

constexpr ra::Fp4Calls kFp4Calls{ra::launch_decode_direct_fp4};

}  // namespace

extern "C" {

ra_status relay_attn_fp4_cache_bytes(const ra_params *p, size_t *block_bytes_out, size_t *bytes_out) {
    if (!p || !block_bytes_out || !bytes_out) return RA_ERR_INVALID_ARG;
    if (p->num_kv_heads < 1 || p->num_blocks < 0 || p->block_size < 1 || (p->block_size & (p->block_size - 1)) != 0)
        return RA_ERR_INVALID_ARG;
    if ((p->head_dim != 64 && p->head_dim != 128) || !fp4_block_size(p->block_size)) return RA_ERR_UNSUPPORTED;
    *block_bytes_out = (size_t)p->block_size * (p->head_dim / 2 + p->head_dim / 32);
    // (a size that is cut off to 64 bits would be taken for a small one)
    const size_t rows = (size_t)p->num_kv_heads * (size_t)p->num_blocks;       // below 2^62
    if (__builtin_mul_overflow(*block_bytes_out, rows, bytes_out)) return RA_ERR_UNSUPPORTED;
    return RA_OK;
}

ra_status relay_attn_cache_append_fp4(const ra_params *p, const void *k_new, const void *v_new,
                                      int64_t new_stride_token, int64_t new_stride_head,
                                      const int32_t *cu_seqlens_q, int32_t total_q, const int32_t *slot_map,
                                      void *k_cache, void *v_cache, const int32_t *block_tables,
                                      const int32_t *context_lens, void *hip_stream) {
    return fp4_rows(p, const_cast<void *>(k_new), const_cast<void *>(v_new), new_stride_token, new_stride_head,
                    cu_seqlens_q, total_q, slot_map, k_cache, v_cache, block_tables, context_lens, hip_stream, false);
}

ra_status relay_attn_cache_read_fp4(const ra_params *p, void *k_out, void *v_out, int64_t out_stride_token,
                                    int64_t out_stride_head, const int32_t *cu_seqlens_q, int32_t total_q,
                                    const int32_t *slot_map, const void *k_cache, const void *v_cache,
                                    const int32_t *block_tables, const int32_t *context_lens, void *hip_stream) {
    return fp4_rows(p, k_out, v_out, out_stride_token, out_stride_head, cu_seqlens_q, total_q, slot_map,
                    const_cast<void *>(k_cache), const_cast<void *>(v_cache), block_tables, context_lens, hip_stream,
                    true);
}

ra_status relay_attn_decode_fp4(const ra_params *p, const void *q, const void *k_sys, const void *v_sys,
                                const void *k_cache, const void *v_cache, const int32_t *block_tables,
                                const int32_t *context_lens, void *out, float *lse_out, void *workspace,
                                size_t workspace_bytes, void *hip_stream) {
    if (!p) return RA_ERR_INVALID_ARG;
    return ra::attend_fp4(p, q, nullptr, p->batch, 1, k_sys, v_sys, k_cache, v_cache, block_tables, context_lens, out,
                          lse_out, workspace, workspace_bytes, hip_stream, kFp4Calls);
}

ra_status relay_attn_prefill_fp4(const ra_params *p, const void *q, const int32_t *cu_seqlens_q, int32_t total_q,
                                 int32_t max_q_len, const void *k_sys, const void *v_sys, const void *k_cache,
                                 const void *v_cache, const int32_t *block_tables, const int32_t *context_lens,
                                 void *out, float *lse_out, void *workspace, size_t workspace_bytes,
                                 void *hip_stream) {
    if (!p || max_q_len < 0 || total_q < 0) return RA_ERR_INVALID_ARG;
    if (total_q > 0 && (!cu_seqlens_q || p->batch < 1)) return RA_ERR_INVALID_ARG;
    if ((int64_t)max_q_len * p->batch < total_q) return RA_ERR_INVALID_ARG;
    return ra::attend_fp4(p, q, cu_seqlens_q, total_q, max_q_len, k_sys, v_sys, k_cache, v_cache, block_tables,
                          context_lens, out, lse_out, workspace, workspace_bytes, hip_stream, kFp4Calls);
}

ra_status relay_attn_update_tables(const ra_params *p, const int32_t *old_lens, const int32_t *new_lens,
                                   const int32_t *pool_in, int32_t *pool_out, int32_t *free_blocks,
                                   int32_t *block_tables, int32_t *context_lens, int32_t *cu_seqlens_q,
                                   int32_t *slot_map, int32_t num_slots, void *hip_stream) {
    if (!p || num_slots < 0) return RA_ERR_INVALID_ARG;
    if (p->batch < 0 || p->num_blocks < 0 || p->max_blocks_per_seq < 0 || p->block_size < 1 ||
        (p->block_size & (p->block_size - 1)) != 0 || p->reserved0 != 0)
        return RA_ERR_INVALID_ARG;
    if ((int64_t)p->max_blocks_per_seq * p->block_size > INT32_MAX) return RA_ERR_INVALID_ARG;
    if (!pool_in || !pool_out || pool_in == pool_out || (num_slots > 0 && !slot_map)) return RA_ERR_INVALID_ARG;
    if (p->num_blocks > 0 && !free_blocks) return RA_ERR_INVALID_ARG;
    if (p->batch > 0 && (!old_lens || !new_lens || !context_lens || (!block_tables && p->max_blocks_per_seq > 0)))
        return RA_ERR_INVALID_ARG;
    if (p->batch > 0 && (context_lens == old_lens || context_lens == new_lens)) return RA_ERR_INVALID_ARG;
    // heights of the stack and positions of the cache are 32-bit numbers
    if ((int64_t)p->batch * p->max_blocks_per_seq + p->num_blocks > INT32_MAX ||
        (int64_t)p->num_blocks * p->block_size > INT32_MAX)
        return RA_ERR_UNSUPPORTED;
    // Every workgroup reads all lengths and the pool's height while others write: nothing written may lie on anything else.
    const Range arrays[] = {{pool_out, 2},    {context_lens, p->batch}, {cu_seqlens_q, (int64_t)p->batch + 1}, {slot_map, num_slots},
                            {free_blocks, p->num_blocks}, {block_tables, (int64_t)p->batch * p->max_blocks_per_seq},
                            {pool_in, 2},     {old_lens, p->batch},     {new_lens, p->batch}};
    constexpr int kWritten = 6;
    for (int i = 0; i < kWritten; ++i)
        for (int j = i + 1; j < (int)(sizeof(arrays) / sizeof(arrays[0])); ++j)
            if (arrays[i].meets(arrays[j])) return RA_ERR_INVALID_ARG;
    ra::TableArgs a{};
    a.old_lens = old_lens;
    a.new_lens = new_lens;
    a.pool_in = pool_in;
    a.pool_out = pool_out;
    a.free_blocks = free_blocks;
    a.block_tables = block_tables;
    a.context_lens = context_lens;
    a.cu_seqlens_q = cu_seqlens_q;
    a.slot_map = slot_map;
    a.n_slots = num_slots;
    a.batch = p->batch;
    a.num_blocks = p->num_blocks;
    while ((1 << a.block_size_log2) < p->block_size) ++a.block_size_log2;
    a.max_blocks_per_seq = p->max_blocks_per_seq;
    return ra::launch_update_tables(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? RA_OK : RA_ERR_HIP;
}

}  // extern "C"
