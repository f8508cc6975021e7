// Block tables, lengths, bounds and slots of a step's new tokens from request lengths (relay_attn_update_tables).
//
// With had_i = ceil(old_i / block_size), want_i = ceil(new_i / block_size) a request needs max(0, want_i - had_i) blocks or
// gives back max(0, had_i - want_i).  The pool is a stack: the blocks given back go on top in (request, column) order, and
// block k that is taken, in the same order, is the k-th from the top.  So every place is a prefix sum over the requests
// away, and no two workgroups have to meet: each sums the lengths of all requests for itself (they are few, and in L2
// after the first) and then does its share of the requests, or of the tokens.  Nothing that one workgroup writes is
// read by another: taken blocks come from the stack below `held` or from table columns that only shrinking requests have,
// and the stack is written between `held` and its new height, which is empty when any of the blocks below are taken.
// Bound: the launch and a chain of trips to memory, not bytes: lengths, then the block of a place, which for one that was just
// given back is a search through the sums and a trip to its table.  4.0 us for 64 requests of a token each; 15 us for 1500 of which
// some end, some give back and the others bring up to 700 tokens (6 of them without any change of a table: summing 1500 lengths).
#include "ra_device.h"
#include "ra_kernels.h"

namespace ra {

namespace {
template <int T>
constexpr int kTableSlots = T == 1024 ? 4 : 1;

struct Step {                    // what one request asks for
    int had, want, need, back, old_len, new_len;
    bool fits;                   // its table row is long enough
};
__device__ __forceinline__ Step step_of(const TableArgs &a, int r) {
    Step s;
    const int bsl = a.block_size_log2, round = (1 << bsl) - 1, cap = a.max_blocks_per_seq << bsl;
    s.old_len = min(max(a.old_lens[r], 0), cap);
    s.new_len = max(a.new_lens[r], 0);
    s.fits = s.new_len <= cap;
    s.had = (s.old_len + round) >> bsl;
    s.want = s.fits ? (s.new_len + round) >> bsl : s.had;
    s.need = max(s.want - s.had, 0);
    s.back = max(s.had - s.want, 0);
    return s;
}
__device__ __forceinline__ int64_t tokens_of(const Step &s) { return max((int64_t)s.new_len - s.old_len, (int64_t)0); }

// Sums of the requests before each of the T runs of `per` consecutive requests, and of all.
template <int T>
struct Sums {
    int need[T], back[T];
    int64_t tokens[T];
    int all_need, all_back, taken, unserved;
    int64_t all_tokens;
};
}  // namespace

template <int T>
__global__ __launch_bounds__(T) void update_tables_kernel(const TableArgs a, const int request_groups) {
    constexpr int WAVES = T / kWave;
    // Consecutive tokens per thread: with many requests the search for a token's is worth sharing; with few each token wants a
    // thread of its own (64 requests of a token each: 4.0 us, 5.0 with four).
    constexpr int kSlots = kTableSlots<T>;
    __shared__ Sums<T> sm;
    __shared__ int sm_wave[2][WAVES];
    __shared__ int64_t sm_wave_tokens[WAVES];
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int bsl = a.block_size_log2;
    const int per = (a.batch + T - 1) / T;
    const int held = min(max(a.pool_in[0], 0), a.num_blocks);
    if (tid == 0) sm.taken = 0, sm.unserved = 0;

    // ---- sums over the requests, a run of `per` of them per thread
    const int r0 = min(tid * per, a.batch), r1 = min(r0 + per, a.batch);
    int need = 0, back = 0;
    int64_t tokens = 0;
    Step mine{};                                  // the first of the run: with up to T requests, the only one
    if (r0 < r1) mine = step_of(a, r0);
    for (int r = r0; r < r1; ++r) {
        const Step s = r == r0 ? mine : step_of(a, r);
        need += s.need, back += s.back, tokens += tokens_of(s);
    }
    int need_to = need, back_to = back;
    int64_t tokens_to = tokens;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int n = __shfl_up(need_to, d), b = __shfl_up(back_to, d);
        const int64_t t = __shfl_up((long long)tokens_to, d);
        if (lane >= d) need_to += n, back_to += b, tokens_to += t;
    }
    if (lane == kWave - 1) sm_wave[0][wave] = need_to, sm_wave[1][wave] = back_to, sm_wave_tokens[wave] = tokens_to;
    __syncthreads();
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) need_to += sm_wave[0][w], back_to += sm_wave[1][w], tokens_to += sm_wave_tokens[w];
    }
    sm.need[tid] = need_to - need, sm.back[tid] = back_to - back, sm.tokens[tid] = tokens_to - tokens;
    if (tid == T - 1) sm.all_need = need_to, sm.all_back = back_to, sm.all_tokens = tokens_to;
    __syncthreads();
    const int top = held + sm.all_back;

    // Served are the requests whose need and everything asked for in front of it the pool holds (or that need no
    // block); the blocks that leave are those of the last of them.
    auto served = [&](const Step &s, int through) { return s.fits && (s.need == 0 || through <= top); };
    int taken = 0, unserved = 0;
    for (int r = r0, through = need_to - need; r < r1; ++r) {
        const Step s = r == r0 ? mine : step_of(a, r);
        through += s.need;
        if (!served(s, through)) ++unserved;
        else if (s.need > 0) taken = through;
    }
    if (taken > 0) atomicMax(&sm.taken, taken);
    if (unserved > 0) atomicAdd(&sm.unserved, unserved);
    __syncthreads();
    const int left = top - sm.taken;

    // Block at height `at` of the stack with the given-back blocks on top; -1 where there is none.
    auto block_at = [&](int at) -> int {
        if (at < 0 || at >= top) return -1;
        if (at < held) return a.free_blocks[at];
        const int rank = at - held;
        int lo = 0, hi = T - 1;            // the last run that begins at or below `rank`
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (sm.back[mid] <= rank) lo = mid; else hi = mid - 1;
        }
        int before = sm.back[lo];
        for (int r = lo * per; r < min((lo + 1) * per, a.batch); ++r) {
            const Step s = step_of(a, r);
            if (rank < before + s.back) return a.block_tables[(int64_t)r * a.max_blocks_per_seq + s.want + (rank - before)];
            before += s.back;
        }
        return -1;                                // (not reached)
    };

    if ((int)blockIdx.x < request_groups) {
        if (blockIdx.x == 0 && tid == 0) {
            a.pool_out[0] = min(left, a.num_blocks);
            a.pool_out[1] = sm.unserved;
            if (a.cu_seqlens_q) a.cu_seqlens_q[a.batch] = (int32_t)sm.all_tokens;
        }
        // ---- requests, one wavefront each
        for (int r = (int)blockIdx.x * WAVES + wave; r < a.batch; r += request_groups * WAVES) {
            const int run = r / per;
            int need_before = 0, back_before = 0;
            int64_t tokens_before = 0;
            for (int i = run * per + lane; i < r; i += kWave) {
                const Step s = step_of(a, i);
                need_before += s.need, back_before += s.back, tokens_before += tokens_of(s);
            }
#pragma unroll
            for (int off = 1; off < kWave; off <<= 1) {
                need_before += __shfl_xor(need_before, off);
                back_before += __shfl_xor(back_before, off);
                tokens_before += __shfl_xor((long long)tokens_before, off);
            }
            need_before += sm.need[run], back_before += sm.back[run], tokens_before += sm.tokens[run];
            const Step s = step_of(a, r);
            const bool ok = served(s, need_before + s.need);
            int32_t *row = a.block_tables + (int64_t)r * a.max_blocks_per_seq;
            if (ok) {
                for (int j = lane; j < s.need; j += kWave) row[s.had + j] = block_at(top - 1 - (need_before + j));
            }
            for (int j = lane; j < s.back; j += kWave) {
                const int at = held + back_before + j;
                if (at < left && at < a.num_blocks) a.free_blocks[at] = row[s.want + j];
            }
            if (lane == 0) {
                a.context_lens[r] = ok ? s.new_len : s.old_len;
                if (a.cu_seqlens_q) a.cu_seqlens_q[r] = (int32_t)tokens_before;
            }
        }
        return;
    }

    // ---- slots of the new tokens: one search per thread, then on from request to request
    const int64_t first = ((int64_t)((int)blockIdx.x - request_groups) * T + tid) * kSlots;
    if (first >= a.n_slots) return;
    int32_t slot[kSlots];
#pragma unroll
    for (int k = 0; k < kSlots; ++k) slot[k] = -1;
    if (first < sm.all_tokens) {
        int lo = 0, hi = T - 1;                   // the last run that begins at or before the token
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (sm.tokens[mid] <= first) lo = mid; else hi = mid - 1;
        }
        int64_t before = sm.tokens[lo];
        int need_before = sm.need[lo], r = lo * per;
        Step s = step_of(a, r);
        int last_col = -1, id = -1;               // block of the token in front
#pragma unroll
        for (int k = 0; k < kSlots; ++k) {
            const int64_t t = first + k;
            if (t >= sm.all_tokens) break;
            while (t >= before + tokens_of(s)) {  // (ends: t is below the sum over all requests)
                before += tokens_of(s);
                need_before += s.need;
                s = step_of(a, ++r);
                last_col = -1;
            }
            if (!served(s, need_before + s.need)) continue;
            const int pos = s.old_len + (int)(t - before), col = pos >> bsl;
            if (col != last_col)
                id = col < s.had ? a.block_tables[(int64_t)r * a.max_blocks_per_seq + col]
                                 : block_at(top - 1 - (need_before + col - s.had));
            last_col = col;
            if (id >= 0 && id < a.num_blocks) slot[k] = (id << bsl) + (pos & ((1 << bsl) - 1));
        }
    }
    if constexpr (kSlots == 4) {
        if (first + kSlots <= a.n_slots && (reinterpret_cast<uintptr_t>(a.slot_map) & 15u) == 0) {
            *reinterpret_cast<u32x4 *>(a.slot_map + first) =
                u32x4{(uint32_t)slot[0], (uint32_t)slot[1], (uint32_t)slot[2], (uint32_t)slot[3]};
            return;
        }
    }
#pragma unroll
    for (int k = 0; k < kSlots; ++k)
        if (first + k < a.n_slots) a.slot_map[first + k] = slot[k];
}

template <int T>
static void launch_tables(const TableArgs &a, hipStream_t stream) {
    constexpr int WAVES = T / kWave, kSlots = kTableSlots<T>;
    int request_groups = (a.batch + WAVES - 1) / WAVES;
    if (request_groups > 256) request_groups = 256;
    if (request_groups < 1) request_groups = 1;            // (an empty batch hands its pool on)
    const int64_t slot_groups = ((int64_t)a.n_slots + T * kSlots - 1) / (T * kSlots);
    hipLaunchKernelGGL((update_tables_kernel<T>), dim3((unsigned)(request_groups + slot_groups)), dim3(T), 0, stream, a,
                       request_groups);
}

hipError_t launch_update_tables(const TableArgs &a, hipStream_t stream) {
    // A thread goes through its run of requests one after the other, and a token through the run that it is in: 1500 requests of
    // up to 700 new tokens took 26 us with 256 threads (runs of six) and take 15 with 1024.  Few requests start sooner in a small
    // workgroup.
    if (a.batch > 512) launch_tables<1024>(a, stream);
    else launch_tables<256>(a, stream);
    return hipGetLastError();
}

}  // namespace ra
