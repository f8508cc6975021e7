// A span of one request's 4-bit context for the query heads of one kv head: the context part of a decode step, one
// wavefront per span (Eq. 7, second term; the format: fp4.h).
//
// A tile is 32 positions.  Both products run on v_mfma_f32_16x16x32_bf16 with the values converted on the way from the
// registers the loads landed in: nothing passes through LDS.  What makes that possible is that the contraction index of a
// matrix product may be numbered at will as long as both operands agree:
//   S^T = K Q^T   Row m of product u (0, 1) is position 8 (m / 4) + 4 u + m % 4 of the tile.  Lane (m, h) holds a quarter
//                 of that position's channels, D/4 from h D/4 on: 16 (d = 64: 8) bytes of codes, one load, one scale
//                 (32 channels or half of them).  Word n of it is the operand of step n as it stands.
//   O^T += V^T P^T  S^T leaves lane (col, h) with positions 8 h .. 8 h + 7 of query head `col`, which is what the operand
//                 P^T wants of it.  So V^T's operand is 8 positions of a channel per lane: lane (i, h) loads the
//                 word of channels 8 i .. 8 i + 7 of its 8 positions, converts two codes at a time and swaps
//                 halves between two positions (v_perm_b32); product n gets channel 8 i + n.
// The rows' powers of two are part of the conversions, so both operands are exact, and P is split into a high
// and a low bfloat16 part as in the bf16 kernels.
// Bound: HBM.  A tile is 4.25 KiB (d = 128) and some 200 vector instructions.
#pragma once
#include "fp4.h"
#include "ra_kernels.h"

#include <type_traits>

namespace ra {

// The value of lane ^ 16, as max_with_other_half does it for lane ^ 32.
__device__ __forceinline__ float max_with_other_row(float x) {
    const uint32_t bits = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane16_swap(bits, bits, false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_with_other_row(float x) {
    const uint32_t bits = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane16_swap(bits, bits, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

constexpr float kFp4LazyLog2 = 8.0f;              // see kLazyLog2 in rows_item.h

// Positions [key_begin, key_end) (key_begin a multiple of 32) of request `req`, kv head g, into partial `part_index`.
// `tbl`: kMaxPartBlocks entries of LDS that belong to the wavefront.
template <int D>
__device__ __forceinline__ void fp4_attend(const TileArgs &a, const int req, const int g, const int key_begin,
                                           int key_end, const int part_index, const int lane, int32_t *tbl) {
    constexpr int KW = D / 32;                    // code words of a lane's part of a K row; steps of S^T
    constexpr int NT = D / 16;                    // products of O^T
    constexpr int ROW = Fp4<D>::ROW;
    const int col = lane & 15, h = lane >> 4;
    const int bsl = a.block_size_log2, bmask = (1 << bsl) - 1;
    const int64_t block_bytes = Fp4<D>::block_bytes(bsl);
    const int scales_at = ROW << bsl;

    // block ids of the span
    const int first_blk = key_begin >> bsl;
    {
        int nblk = key_end > key_begin ? ((key_end - 1) >> bsl) - first_blk + 1 : 0;
        // (never binding: the host sized the spans for the table and context_lens for the row)
        nblk = min(nblk, min(kMaxPartBlocks, a.max_blocks_per_seq - first_blk));
        key_end = min(key_end, (first_blk + nblk) << bsl);
        const int32_t *bt = a.block_tables + (int64_t)req * a.max_blocks_per_seq + first_blk;
        for (int j = lane; j < nblk; j += kWave) tbl[j] = bt[j];
    }

    // Q^T: channels h D/4 + 8 n .. + 7 of head `col`.  A negative scale goes into its sign; a zero one becomes
    // 1e-30 (see rows_item.h).
    const bool flip = a.scale_log2 < 0.f;
    const float scale = fmaxf(fabsf(a.scale_log2), 1e-30f);
    const float lazy_raw = kFp4LazyLog2 / scale;
    bf16x8 qf[KW];
#pragma unroll
    for (int n = 0; n < KW; ++n) {
        u32x4 w = {0, 0, 0, 0};
        if (col < a.G)
            w = *reinterpret_cast<const u32x4 *>(a.q + (int64_t)req * a.q_stride_token +
                                                 (int64_t)(g * a.G + col) * a.q_stride_head + h * (D / 4) + 8 * n);
        if (flip) w ^= u32x4{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
        qf[n] = __builtin_bit_cast(bf16x8, w);
    }

    const uint8_t *k_cache = reinterpret_cast<const uint8_t *>(a.k_cache);
    const uint8_t *v_cache = reinterpret_cast<const uint8_t *>(a.v_cache);
    const int oct = D == 128 ? col : col & 7;     // V: the word of a row that this lane takes
    const int k_group = h * (D / 4) / 32, v_group = oct / 4;

    struct Tile {
        uint32_t k[2][KW], k_scale[2], v[8];
        u32x2 v_scale;                            // of positions 8 h .. 8 h + 7, a byte each
    };
    auto block_of = [&](int key) { return ((int64_t)tbl[(key >> bsl) - first_blk] * a.Hkv + g) * block_bytes; };
    auto load = [&](int tile0, Tile &t) {
        // Rows behind the end re-load the last one; V words come eight positions at a time, which lie in one block
        // (block_size >= 8), so that the ones behind the end there are read, and count for nothing.
        const int last = key_end - 1;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int key = min(tile0 + 8 * (col >> 2) + 4 * u + (col & 3), last);
            const uint8_t *block = k_cache + block_of(key);
            const int off = key & bmask;
            const uint8_t *src = block + off * ROW + h * (KW * 4);
            if constexpr (KW == 4) {
                const u32x4 w = *reinterpret_cast<const u32x4 *>(src);
#pragma unroll
                for (int n = 0; n < KW; ++n) t.k[u][n] = w[n];
            } else {
                const u32x2 w = *reinterpret_cast<const u32x2 *>(src);
#pragma unroll
                for (int n = 0; n < KW; ++n) t.k[u][n] = w[n];
            }
            t.k_scale[u] = block[scales_at + (k_group << bsl) + off];
        }
        const int key = min(tile0 + 8 * h, last & ~7);
        const uint8_t *block = v_cache + block_of(key);
        const int off = key & bmask;
        const uint8_t *src = block + off * ROW + oct * 4;
#pragma unroll
        for (int j = 0; j < 8; ++j) t.v[j] = *reinterpret_cast<const uint32_t *>(src + j * ROW);
        t.v_scale = *reinterpret_cast<const u32x2 *>(block + scales_at + (v_group << bsl) + off);
    };

    f32x4 acc[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, msc = 0.f, l_run = 0.f;

    auto compute = [&](int tile0, const Tile &t) {
        f32x4 s[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            s[u] = f32x4{0.f, 0.f, 0.f, 0.f};
            const float ks = fp4_scale(t.k_scale[u]);
#pragma unroll
            for (int n = 0; n < KW; ++n)
                s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fp4_octet(t.k[u][n], ks)), qf[n],
                                                               s[u], 0, 0, 0);
        }
        u32x2 v_scale = t.v_scale;
        if (tile0 + 32 > key_end) {               // ragged last tile: no weight and a harmless power of two behind the end
            const int mine = min(max(key_end - (tile0 + 8 * h), 0), 8);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[u][r] = 4 * u + r < mine ? s[u][r] : -INFINITY;
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const int bytes = min(max(mine - 4 * w, 0), 4);
                const uint32_t word = v_scale[w];
                v_scale[w] = bytes == 4 ? word : word & ((1u << (8 * bytes)) - 1u);
            }
        }
        float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                         fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        // The maximum that the sums are expressed against moves when a column outgrew it by the margin or sees its
        // first key; only then do the four lanes of a column have to agree on it.
        if (__builtin_amdgcn_ballot_w64(mx > m_run + lazy_raw) != 0) {
            mx = max_with_other_half(max_with_other_row(mx));
            const float m_new = fmaxf(m_run, mx);
            const float msc_new = m_new == -INFINITY ? 0.f : m_new * scale;
            const float corr = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(msc - msc_new);
            l_run *= corr;
#pragma unroll
            for (int n = 0; n < NT; ++n) acc[n] *= corr;
            m_run = m_new;
            msc = msc_new;
        }
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float p0 = __builtin_amdgcn_exp2f(fmaf(s[i / 2][2 * (i & 1)], scale, -msc));
            const float p1 = __builtin_amdgcn_exp2f(fmaf(s[i / 2][2 * (i & 1) + 1], scale, -msc));
            l_run += p0 + p1;
            hi[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{p0, p1}), bf16x2));
            lo[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{p0 - bf16_lo(hi[i]), p1 - bf16_hi(hi[i])}), bf16x2));
        }
        const bf16x8 ph = __builtin_bit_cast(bf16x8, (u32x4{hi[0], hi[1], hi[2], hi[3]}));
        const bf16x8 pl = __builtin_bit_cast(bf16x8, (u32x4{lo[0], lo[1], lo[2], lo[3]}));

        float vs[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) vs[j] = fp4_scale((v_scale[j / 4] >> (8 * (j & 3))) & 0xffu);
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = D == 128 ? t.v[j] : t.v[j] >> (16 * (col >> 3));
        auto products = [&](auto byte_tag) {      // channels 2 BYTE and 2 BYTE + 1 of each lane's word
            constexpr int BYTE = decltype(byte_tag)::value;
            u32x4 even, odd;
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const uint32_t x = fp4_pair<BYTE>(w[2 * p], vs[2 * p]), y = fp4_pair<BYTE>(w[2 * p + 1], vs[2 * p + 1]);
                even[p] = __builtin_amdgcn_perm(y, x, 0x05040100u);
                odd[p] = __builtin_amdgcn_perm(y, x, 0x07060302u);
            }
            const bf16x8 ve = __builtin_bit_cast(bf16x8, even), vo = __builtin_bit_cast(bf16x8, odd);
            acc[2 * BYTE] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ve, ph, acc[2 * BYTE], 0, 0, 0);
            acc[2 * BYTE + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vo, ph, acc[2 * BYTE + 1], 0, 0, 0);
            acc[2 * BYTE] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ve, pl, acc[2 * BYTE], 0, 0, 0);
            acc[2 * BYTE + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vo, pl, acc[2 * BYTE + 1], 0, 0, 0);
        };
        products(std::integral_constant<int, 0>{});
        products(std::integral_constant<int, 1>{});
        if constexpr (D == 128) {
            products(std::integral_constant<int, 2>{});
            products(std::integral_constant<int, 3>{});
        }
    };

    // three tiles on their way while one is worked off
    Tile ring[4];
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (key_begin + 32 * i < key_end) load(key_begin + 32 * i, ring[i]);
    for (int tile0 = key_begin; tile0 < key_end;) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (tile0 + 96 < key_end) load(tile0 + 96, ring[(i + 3) & 3]);
            compute(tile0, ring[i]);
            tile0 += 32;
            if (tile0 >= key_end) break;
        }
    }

    l_run = sum_with_other_half(sum_with_other_row(l_run));
    if (col < a.G) {
        const float inv = l_run > 0.f ? 1.f / l_run : 0.f;
        const int64_t prow = (int64_t)part_index * a.rows + (int64_t)req * a.Hq + g * a.G + col;
        float *dst = a.part_o + prow * D;
#pragma unroll
        for (int r = 0; r < 4; ++r) {             // row 4 h + r of product n is channel 8 (4 h + r) + n, see above
            const int i = 4 * h + r;
            float *to = dst + (D == 128 ? 8 * i : 8 * (i & 7) + 4 * (i >> 3));
            // (d = 64: lanes 8 .. 15 of a group take the upper half of the words)
#pragma unroll
            for (int n = 0; n < NT; n += 4) {
                *reinterpret_cast<f32x4 *>(to + n) =
                    f32x4{acc[n][r] * inv, acc[n + 1][r] * inv, acc[n + 2][r] * inv, acc[n + 3][r] * inv};
            }
        }
        if (h == 0) a.part_lse[prow] = l_run > 0.f ? msc + log2f(l_run) : -INFINITY;
    }
}

}  // namespace ra
