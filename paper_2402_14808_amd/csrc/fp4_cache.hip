// Rows into the 4-bit context cache, and out of it (the format: fp4.h).
//
// Append rounds the new keys/values: for each block of 32 values the largest magnitude a, the power of two
// 2^e that brings it to at most a grid step of 6, and 32 codes.  A thread takes 8 values (16 bytes), the four threads of a block
// find its maximum by two data-parallel moves on the bfloat16 bits (as whole numbers: magnitudes order alike), so
// nothing is rounded before the one rounding to codes.  Read-out is the way back, exact.
// Bound: HBM for many tokens (2 bytes a value on one side, 17/32 on the other), the chain arguments -> place -> block id ->
// row for a step's few (3.1 and 2.6 us a launch).  4608 tokens of 40 heads, in and out again, 120 MB each: 60.3 us with ordinary
// loads and stores of the bfloat16 side, 52.9 with non-temporal ones (4.5 TB/s; a large copy reaches 4.8).
#include "fp4.h"
#include "ra_kernels.h"
#include "token_place.h"

namespace ra {

constexpr int kRowsMaxTokens = 16;

// The largest of the 8 magnitudes of a thread, then of the four threads of its block.
__device__ __forceinline__ uint32_t block_top(const u32x4 x) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max(x[i] & 0x7fffu, (x[i] >> 16) & 0x7fffu));
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xf, 0xf, true));   // quad_perm [1,0,3,2]
    return max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xf, 0xf, true));  // quad_perm [2,3,0,1]
}

template <int D, bool READ>
__global__ __launch_bounds__(kThreads) void fp4_rows_kernel(const Fp4RowsArgs a, const int tpw) {
    __shared__ int64_t sm_slot[kRowsMaxTokens];          // position in the cache: block * block_size + offset, or -1
    constexpr int CPR = D / 8;                            // pieces of 8 values per row
    const int bsl = a.block_size_log2, bmask = (1 << bsl) - 1;
    const int token0 = (int)blockIdx.x * tpw;
    const int per_token = a.Hkv * CPR;
    const int n = min(tpw, a.n_tokens - token0) * per_token;
    const int64_t block_bytes = Fp4<D>::block_bytes(bsl);
    constexpr int U = 4;
    u32x4 k[U], v[U];
    auto row_of = [&](int i, int &t, int &g, int &chunk) {
        t = i / per_token;
        const int in_token = i - t * per_token;
        g = in_token / CPR, chunk = in_token % CPR;
        return (int64_t)(token0 + t) * a.stride_token + (int64_t)g * a.stride_head + chunk * 8;
    };
    auto read_new = [&](int i0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * kThreads;
            if (i >= n) continue;
            int t, g, chunk;
            const int64_t src = row_of(i, t, g, chunk);
            k[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(a.k_rows + src));
            v[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(a.v_rows + src));
        }
    };
    if constexpr (!READ) read_new(threadIdx.x);
    if (threadIdx.x < kWave) {
        const int lane = (int)threadIdx.x;
        const int token = token0 + lane;
        const bool mine = lane < tpw && token < a.n_tokens;
        int64_t slot = -1;
        if (a.slot_map) {
            if (mine) slot = a.slot_map[token];
        } else {
            int req, pos;
            place_of_token(a.cu_seqlens_q, a.context_lens, a.batch, token0, tpw, lane, req, pos);
            if (mine) {
                if (!a.cu_seqlens_q) pos = a.context_lens[req] - 1;
                if (pos >= 0 && (pos >> bsl) < a.max_blocks_per_seq)           // (malformed lengths: no row)
                    slot = ((int64_t)a.block_tables[(int64_t)req * a.max_blocks_per_seq + (pos >> bsl)] << bsl) + (pos & bmask);
            }
        }
        if (lane < tpw) sm_slot[lane] = slot >= 0 && slot < a.n_slots ? slot : -1;
    }
    __syncthreads();
    for (int i0 = threadIdx.x; i0 < n; i0 += U * kThreads) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * kThreads;
            if (i >= n) continue;                         // (the four threads of a block together)
            int t, g, chunk;
            const int64_t row = row_of(i, t, g, chunk);
            const int64_t slot = sm_slot[t];
            if (slot < 0) continue;
            const int64_t block = ((slot >> bsl) * a.Hkv + g) * block_bytes;
            const int off = (int)slot & bmask;
            const int64_t code_at = block + off * Fp4<D>::ROW + chunk * 4;
            const int64_t scale_at = block + ((int64_t)Fp4<D>::ROW << bsl) + ((chunk >> 2) << bsl) + off;
            if constexpr (READ) {
                const uint32_t kc = *reinterpret_cast<const uint32_t *>(a.k_cache + code_at);
                const uint32_t vc = *reinterpret_cast<const uint32_t *>(a.v_cache + code_at);
                const float ks = fp4_scale(a.k_cache[scale_at]), vs = fp4_scale(a.v_cache[scale_at]);
                __builtin_nontemporal_store(fp4_octet(kc, ks), reinterpret_cast<u32x4 *>(a.k_rows + row));
                __builtin_nontemporal_store(fp4_octet(vc, vs), reinterpret_cast<u32x4 *>(a.v_rows + row));
            } else {
                const uint32_t kb = fp4_scale_byte(block_top(k[u])), vb = fp4_scale_byte(block_top(v[u]));
                *reinterpret_cast<uint32_t *>(a.k_cache + code_at) = fp4_encode(k[u], fp4_scale(kb));
                *reinterpret_cast<uint32_t *>(a.v_cache + code_at) = fp4_encode(v[u], fp4_scale(vb));
                if ((chunk & 3) == 0) {
                    a.k_cache[scale_at] = (uint8_t)kb;
                    a.v_cache[scale_at] = (uint8_t)vb;
                }
            }
        }
        if constexpr (!READ) read_new(i0 + U * kThreads);
    }
}

hipError_t launch_fp4_rows(const Fp4RowsArgs &a, int head_dim, bool read, hipStream_t stream) {
    if (a.n_tokens == 0) return hipSuccess;
    // about 1024 of the pieces per workgroup (one round of U = 4), fewer where that would leave compute units idle
    const int per_token = a.Hkv * (head_dim / 8);
    int tpw = 1024 / per_token;
    if (tpw > a.n_tokens / 512) tpw = a.n_tokens / 512;
    if (tpw > kRowsMaxTokens) tpw = kRowsMaxTokens;
    if (tpw < 1) tpw = 1;
    const dim3 grid((unsigned)((a.n_tokens + tpw - 1) / tpw)), block(kThreads);
    if (head_dim == 128 && read) hipLaunchKernelGGL((fp4_rows_kernel<128, true>), grid, block, 0, stream, a, tpw);
    else if (head_dim == 128) hipLaunchKernelGGL((fp4_rows_kernel<128, false>), grid, block, 0, stream, a, tpw);
    else if (head_dim == 64 && read) hipLaunchKernelGGL((fp4_rows_kernel<64, true>), grid, block, 0, stream, a, tpw);
    else if (head_dim == 64) hipLaunchKernelGGL((fp4_rows_kernel<64, false>), grid, block, 0, stream, a, tpw);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace ra
