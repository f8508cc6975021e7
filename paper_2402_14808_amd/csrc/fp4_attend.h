// A span of one request's 4-bit context for the query rows of one kv head: the context part of a decode step, or of a prompt
// phase that brings few new tokens, one wavefront per span (Eq. 7, second term; the format: fp4.h).
//
// A tile is 32 positions.  Both products run on v_mfma_f32_16x16x32_bf16 with the values converted on the way from the
// registers the loads landed in.  What makes that possible is that the contraction index of a
// matrix product may be numbered at will as long as both operands agree:
//   S^T = K Q^T   Row m of product u (0, 1) is position 8 (m / 4) + 4 u + m % 4 of the tile.  Lane (m, h) holds a quarter
//                 of that position's channels, D/4 from h D/4 on: 16 (d = 64: 8) bytes of codes, one load, one scale
//                 (32 channels or half of them).  Word n of it is the operand of step n as it stands.
//   O^T += V^T P^T  S^T leaves lane (col, h) with positions 8 h .. 8 h + 7 of query head `col`, which is what the operand
//                 P^T wants of it.  So V^T's operand is 8 positions of a channel per lane: lane (i, h) takes the
//                 word of channels 8 i .. 8 i + 7 of its 8 positions, converts two codes at a time and swaps
//                 halves between two positions (v_perm_b32); product n gets channel 8 i + n.  The words come through the
//                 wavefront's own LDS: loaded as they are needed, 4 bytes a lane, they held the loads of a launch to 5.4
//                 TB/s (d = 128) and 4.0 (64), 16 bytes a lane to 6.2 and more.
// A decode step has up to 8 rows, the query heads of the kv head; in the prompt phase row n is new token n / G and head n % G of
// them, in one or two groups (CG) of 16 that share what a tile costs to load and convert.
// The rows' powers of two are part of the conversions, so both operands are exact.  P is split into a high and a low bfloat16
// part as in the bf16 kernels, 2^-17 of a weight, and for an fp32 output (EX) into three, so that what is left, 2^-26, is below
// the sums' own rounding.
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

// Positions [key_begin, key_end) (key_begin a multiple of 32) of request `req`, kv head g, into partial `part_index`, for its
// rows: the packed tokens from `token0` on, the first of which sees the positions below first_end, each further one a
// position more (a decode step: one token, and all of them).
// `lds`: Fp4Lds<D>::BYTES bytes that belong to the wavefront, aligned to 16.
constexpr int kFp4TableEntries = kMaxPartBlocks + 32 / 8;
template <int D>
struct Fp4Lds {                                   // of the two tiles in turn
    static constexpr int TABLE = kFp4TableEntries * 8;
    static constexpr int V_TILE = 36 * Fp4<D>::ROW;             // rows, each eight of them one row further: no bank conflicts
    static constexpr int S_TILE = 2 * Fp4<D>::GROUPS * 32;      // scales [K, V][group][position]
    static constexpr int V_AT = TABLE, S_AT = V_AT + 2 * V_TILE;
    static constexpr int K_AT = S_AT + 2 * S_TILE, BYTES = K_AT + (D == 64 ? 2 * V_TILE : 0);   // K rows, d = 64
};
template <int D, int CG, bool EX>
__device__ __forceinline__ void fp4_attend(const TileArgs &a, const int req, const int g, const int token0, const int rows,
                                           const int first_end, const int key_begin, int key_end, const int part_index,
                                           const int lane, unsigned char *lds) {
    constexpr int KW = D / 32;                    // code words of a lane's part of a K row; steps of S^T
    constexpr int NT = D / 16;                    // products of O^T
    constexpr int ROW = Fp4<D>::ROW;
    const int col = lane & 15, h = lane >> 4;
    const int bsl = a.block_size_log2, bmask = (1 << bsl) - 1;
    const int scales_at = ROW << bsl;
    using L = Fp4Lds<D>;
    int64_t *tbl = reinterpret_cast<int64_t *>(lds);

    // Where the blocks of the span begin, in bytes.  Behind the last one it is named again, so that a tile that ends in
    // it finds an address for its missing rows.
    const int first_blk = key_begin >> bsl;
    {
        int nblk = key_end > key_begin ? ((key_end - 1) >> bsl) - first_blk + 1 : 0;
        // (never binding: the host sized the spans for the table and context_lens for the row)
        nblk = min(nblk, min(kMaxPartBlocks, a.max_blocks_per_seq - first_blk));
        key_end = min(key_end, (first_blk + nblk) << bsl);
        const int32_t *bt = a.block_tables + (int64_t)req * a.max_blocks_per_seq + first_blk;
        if (nblk > 0)
            for (int j = lane; j < nblk + 32 / 8; j += kWave)
                tbl[j] = ((int64_t)bt[min(j, nblk - 1)] * a.Hkv + g) * Fp4<D>::block_bytes(bsl);
    }

    // Q^T: channels h D/4 + 8 n .. + 7 of head `col`.  A negative scale goes into its sign; a zero one becomes
    // 1e-30 (see rows_item.h).
    const bool flip = a.scale_log2 < 0.f;
    const float scale = fmaxf(fabsf(a.scale_log2), 1e-30f);
    const float lazy_raw = kFp4LazyLog2 / scale;
    bf16x8 qf[CG][KW];
    int row_end[CG], row_of[CG];                  // positions that a lane's row sees; its output row
#pragma unroll
    for (int c = 0; c < CG; ++c) {
        const int n = 16 * c + col, j = CG > 1 ? n / a.G : 0;
        const int token = token0 + j, hq = g * a.G + n - j * a.G;
        row_end[c] = CG > 1 ? min(key_end, first_end + j) : key_end;
        row_of[c] = n < rows ? token * a.Hq + hq : -1;
#pragma unroll
        for (int k = 0; k < KW; ++k) {
            u32x4 w = {0, 0, 0, 0};
            if (n < rows)
                w = *reinterpret_cast<const u32x4 *>(a.q + (int64_t)token * a.q_stride_token + (int64_t)hq * a.q_stride_head +
                                                     h * (D / 4) + 8 * k);
            if (flip) w ^= u32x4{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
            qf[c][k] = __builtin_bit_cast(bf16x8, w);
        }
    }
    // below this, no row misses a position
    const int all_see = CG > 1 ? min(key_end, first_end) : key_end;

    // d = 128: a lane loads quarter h of positions kp and kp + 4 of K, which it multiplies, and of V.  d = 64: half of position
    // lane / 2 of each, 16 bytes as well, and K takes the way through LDS too (a quarter each, 8 bytes a lane, held the loads of a
    // launch to 5.2 TB/s).  Eight positions that begin at a multiple of eight lie in one block.  Then four scales: of K in the
    // lower lanes and of V in the upper ones (d = 64 has half as many, and takes them twice).  Rows behind the end are loaded
    // like the others, whatever they hold: scores and powers of two are put right below.
    const int oct = D == 128 ? col : col & 7;     // V: the word of a row that this lane multiplies
    const int kp = 8 * (col >> 2) + (col & 3);
    const int lp = D == 128 ? kp : lane >> 1, lq = D == 128 ? h : lane & 1;      // position and 16 bytes of it that this lane loads
    const int sl = D == 128 ? lane : lane & 31;   // scales: cache, group, positions 4 (sl % 8) ..
    const int s_group = (sl >> 3) & (Fp4<D>::GROUPS - 1), s_pos = 4 * (sl & 7);
    const bool s_is_v = sl >= 8 * Fp4<D>::GROUPS;
    const int lane_at = (lp & bmask) * ROW + lq * 16, lane_scales_at = (s_group << bsl) + (s_pos & bmask);
    const uint8_t *k_codes = reinterpret_cast<const uint8_t *>(a.k_cache), *v_codes = reinterpret_cast<const uint8_t *>(a.v_cache);
    const uint8_t *scale_bytes = (s_is_v ? v_codes : k_codes) + scales_at;
    const int64_t *code_tbl = tbl + (lp >> bsl), *scale_tbl = tbl + (s_pos >> bsl);
    uint32_t *const s_put = reinterpret_cast<uint32_t *>(lds + L::S_AT + 4 * sl);
    unsigned char *const v_put = lds + L::V_AT + lp * ROW + (lp >> 3) * ROW + lq * 16;
    const unsigned char *const v_get = lds + L::V_AT + 9 * h * ROW + oct * 4;
    [[maybe_unused]] const unsigned char *const k_get = lds + L::K_AT + kp * ROW + (kp >> 3) * ROW + h * 8;
    const unsigned char *const ks_get = lds + L::S_AT + (h * (D / 4) / 32) * 32 + (kp & ~7);
    const unsigned char *const vs_get = lds + L::S_AT + (Fp4<D>::GROUPS + oct / 4) * 32 + 8 * h;

    constexpr int LOADS = D / 64;                 // of K, and of V, a tile
    struct Tile {
        u32x4 k[LOADS], v[LOADS];
        uint32_t scales;
    };
    const int last_tile = key_begin + ((key_end - key_begin - 1) & ~31);
    auto load = [&](int tile0, Tile &t) {
        // As many loads each time: the waits count them.  Behind the last tile all lanes take the same few bytes of it (as
        // a whole tile, up to four of those a span were fetched again, non-temporal as they are).
        const int none = tile0 > last_tile ? 0 : -1;
        tile0 = min(tile0, last_tile);
        const int blk = (tile0 >> bsl) - first_blk, off = tile0 & bmask;
        const int64_t at = code_tbl[blk] + (off * ROW + (lane_at & none)), scales_of = scale_tbl[blk] + (off + (lane_scales_at & none));
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {         // (rows are read once: non-temporal)
            t.k[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(k_codes + at + 4 * u * ROW));
            t.v[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(v_codes + at + 4 * u * ROW));
        }
        t.scales = *reinterpret_cast<const uint32_t *>(scale_bytes + scales_of);
    };
    auto through_lds = [&](const Tile (&t)[2]) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            s_put[x * (L::S_TILE / 4)] = t[x].scales;
            if constexpr (D == 64) *reinterpret_cast<u32x4 *>(v_put + (L::K_AT - L::V_AT) + x * L::V_TILE) = t[x].k[0];
#pragma unroll
            for (int u = 0; u < LOADS; ++u) *reinterpret_cast<u32x4 *>(v_put + x * L::V_TILE + 4 * u * ROW) = t[x].v[u];
        }
    };
    auto k_words = [&](const Tile (&t)[2], int i, uint32_t (&w)[KW]) {   // of product i % 2 of tile i / 2
        if constexpr (D == 64) {
            const u32x2 x = *reinterpret_cast<const u32x2 *>(k_get + (i / 2) * L::V_TILE + 4 * (i & 1) * ROW);
#pragma unroll
            for (int n = 0; n < KW; ++n) w[n] = x[n];
        } else {
#pragma unroll
            for (int n = 0; n < KW; ++n) w[n] = t[i / 2].k[(i & 1) & (LOADS - 1)][n];
        }
    };

    f32x4 acc[CG][NT];
    float m_run[CG], msc[CG], l_run[CG];
#pragma unroll
    for (int c = 0; c < CG; ++c) {
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[c][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        m_run[c] = -INFINITY, msc[c] = 0.f, l_run[c] = 0.f;
    }

    auto compute = [&](int tile0, const Tile (&t)[2]) {       // two tiles: their chains of products are independent
        through_lds(t);
        u32x2 v_scale[2];
        f32x4 s[CG][4];                           // s[..][2 x + u]: product u of tile x
        float ks[4];
        uint32_t kw[4][KW];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            k_words(t, i, kw[i]);
#pragma unroll
            for (int c = 0; c < CG; ++c) s[c][i] = f32x4{0.f, 0.f, 0.f, 0.f};
            // byte kp % 4 of the word to bits 23 .. 30 (the conversions read no other)
            const uint32_t word = *reinterpret_cast<const uint32_t *>(ks_get + (i / 2) * L::S_TILE + 4 * (i & 1));
            ks[i] = __uint_as_float(__builtin_amdgcn_alignbit(word, word, (8 * (col & 3) + 9) & 31));
        }
#pragma unroll
        for (int n = 0; n < KW; ++n)              // (the four chains in turn: a product that waits for the one before it stalls)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bf16x8 kf = __builtin_bit_cast(bf16x8, fp4_octet(kw[i][n], ks[i]));
                s[0][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[0][n], s[0][i], 0, 0, 0);
                if (CG > 1) s[CG - 1][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[CG - 1][n], s[CG - 1][i], 0, 0, 0);
            }
#pragma unroll
        for (int x = 0; x < 2; ++x) v_scale[x] = *reinterpret_cast<const u32x2 *>(vs_get + x * L::S_TILE);
        if (tile0 + 64 > all_see) {               // no weight behind the last position that a row sees
#pragma unroll
            for (int c = 0; c < CG; ++c)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int mine = row_end[c] - (tile0 + 32 * x + 8 * h);
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[c][2 * x + u][r] = 4 * u + r < mine ? s[c][2 * x + u][r] : -INFINITY;
                }
        }
        if (tile0 + 64 > key_end) {               // ragged end: a harmless power of two behind it
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const int bytes = min(max(key_end - (tile0 + 32 * x + 8 * h) - 4 * w, 0), 4);
                    const uint32_t word = v_scale[x][w];
                    v_scale[x][w] = bytes == 4 ? word : word & ((1u << (8 * bytes)) - 1u);
                }
        }
        // The maximum that the sums are expressed against moves when a column outgrew it by the margin or sees its
        // first key; only then do the four lanes of a column have to agree on it.
#pragma unroll
        for (int c = 0; c < CG; ++c) {
            float mx = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i) mx = fmaxf(mx, fmaxf(fmaxf(s[c][i][0], s[c][i][1]), fmaxf(s[c][i][2], s[c][i][3])));
            if (__builtin_amdgcn_ballot_w64(mx > m_run[c] + lazy_raw) != 0) {
                mx = max_with_other_half(max_with_other_row(mx));
                const float m_new = fmaxf(m_run[c], mx);
                const float msc_new = m_new == -INFINITY ? 0.f : m_new * scale;
                const float corr = m_run[c] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(msc[c] - msc_new);
                l_run[c] *= corr;
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[c][n] *= corr;
                m_run[c] = m_new;
                msc[c] = msc_new;
            }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            bf16x8 ph[CG], pl[CG], pt[CG];
#pragma unroll
            for (int c = 0; c < CG; ++c) {
                uint32_t hi[4], lo[4], third[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float p0 = __builtin_amdgcn_exp2f(fmaf(s[c][2 * x + i / 2][2 * (i & 1)], scale, -msc[c]));
                    const float p1 = __builtin_amdgcn_exp2f(fmaf(s[c][2 * x + i / 2][2 * (i & 1) + 1], scale, -msc[c]));
                    l_run[c] += p0 + p1;
                    hi[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{p0, p1}), bf16x2));
                    const float r0 = p0 - bf16_lo(hi[i]), r1 = p1 - bf16_hi(hi[i]);
                    lo[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{r0, r1}), bf16x2));
                    if constexpr (EX)
                        third[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{r0 - bf16_lo(lo[i]), r1 - bf16_hi(lo[i])}), bf16x2));
                }
                if constexpr (EX) pt[c] = __builtin_bit_cast(bf16x8, (u32x4{third[0], third[1], third[2], third[3]}));
                ph[c] = __builtin_bit_cast(bf16x8, (u32x4{hi[0], hi[1], hi[2], hi[3]}));
                pl[c] = __builtin_bit_cast(bf16x8, (u32x4{lo[0], lo[1], lo[2], lo[3]}));
            }
            float vs[8];
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t word = v_scale[x][j / 4];
                vs[j] = __uint_as_float((j & 3) == 3 ? word >> 1 : word << (23 - 8 * (j & 3)));
                const uint32_t v = *reinterpret_cast<const uint32_t *>(v_get + x * L::V_TILE + j * ROW);
                w[j] = D == 128 ? v : v >> (16 * (col >> 3));
            }
            auto products = [&](auto byte_tag) {  // channels 2 BYTE and 2 BYTE + 1 of each lane's word
                constexpr int BYTE = decltype(byte_tag)::value;
                u32x4 even, odd;
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    const uint32_t y0 = fp4_pair<BYTE>(w[2 * p], vs[2 * p]), y1 = fp4_pair<BYTE>(w[2 * p + 1], vs[2 * p + 1]);
                    even[p] = __builtin_amdgcn_perm(y1, y0, 0x05040100u);
                    odd[p] = __builtin_amdgcn_perm(y1, y0, 0x07060302u);
                }
                const bf16x8 ve = __builtin_bit_cast(bf16x8, even), vo = __builtin_bit_cast(bf16x8, odd);
#pragma unroll
                for (int c = 0; c < CG; ++c) {
                    f32x4 &e = acc[c][2 * BYTE], &o = acc[c][2 * BYTE + 1];
                    e = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ve, ph[c], e, 0, 0, 0);
                    o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vo, ph[c], o, 0, 0, 0);
                    e = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ve, pl[c], e, 0, 0, 0);
                    o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vo, pl[c], o, 0, 0, 0);
                    if constexpr (EX) {
                        e = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ve, pt[c], e, 0, 0, 0);
                        o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vo, pt[c], o, 0, 0, 0);
                    }
                }
            };
            products(std::integral_constant<int, 0>{});
            products(std::integral_constant<int, 1>{});
            if constexpr (D == 128) {
                products(std::integral_constant<int, 2>{});
                products(std::integral_constant<int, 3>{});
            }
        }
    };

    // Two tiles on their way while two are worked off.  (Loads are made and counted on every path, so that the waits of
    // the loop are for the tiles in turn and not for all that is on its way; a loop that is left in its middle counts as
    // paths that come back without them.)
    Tile even[2], odd[2];
    auto load2 = [&](int tile0, Tile (&t)[2]) {
        load(tile0, t[0]);
        load(tile0 + 32, t[1]);
        __builtin_amdgcn_sched_barrier(0);
    };
    if (key_begin < key_end) {
        load2(key_begin, even);
        for (int tile0 = key_begin; tile0 < key_end; tile0 += 128) {
            load2(tile0 + 64, odd);
            compute(tile0, even);
            load2(tile0 + 128, even);
            if (tile0 + 64 < key_end) compute(tile0 + 64, odd);
        }
    }

#pragma unroll
    for (int c = 0; c < CG; ++c) {
        const float l = sum_with_other_half(sum_with_other_row(l_run[c]));
        if (row_of[c] < 0) continue;
        const float inv = l > 0.f ? 1.f / l : 0.f;
        const int64_t prow = (int64_t)part_index * a.rows + row_of[c];
        float *dst = a.part_o + prow * D;
#pragma unroll
        for (int r = 0; r < 4; ++r) {             // row 4 h + r of product n is channel 8 (4 h + r) + n, see above
            const int i = 4 * h + r;
            float *to = dst + (D == 128 ? 8 * i : 8 * (i & 7) + 4 * (i >> 3));
            // (d = 64: lanes 8 .. 15 of a group take the upper half of the words)
#pragma unroll
            for (int n = 0; n < NT; n += 4)
                *reinterpret_cast<f32x4 *>(to + n) =
                    f32x4{acc[c][n][r] * inv, acc[c][n + 1][r] * inv, acc[c][n + 2][r] * inv, acc[c][n + 3][r] * inv};
        }
        // (a sum that is no number, of a query or a score that is none, must not look like an empty partial)
        if (h == 0) a.part_lse[prow] = l == 0.f ? -INFINITY : msc[c] + log2f(l);
    }
}

}  // namespace ra
