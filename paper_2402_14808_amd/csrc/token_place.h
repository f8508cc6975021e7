// Where the packed new tokens of a step belong: request and context position of each, found by the lanes of
// one wavefront together (the cache writes and the read-out).
#pragma once
#include "ra_device.h"

namespace ra {

// Lane l of a whole wavefront: request and context position (below 0: none) of token token0 + l, for the first `tpw` lanes.  Without
// cu_seqlens_q token i is request i, and the position is left to the caller (0 here).
// The lanes hold the bounds and lengths of 64 requests at a time, so that a token's place is one trip
// to its block id away once they are here (searched first and asked for then, the lengths were a
// trip of their own).
__device__ __forceinline__ void place_of_token(const int32_t *cu_seqlens_q, const int32_t *context_lens, int batch,
                                               int token0, int tpw, int lane, int &req, int &pos) {
    const int token = token0 + lane;
    req = token;
    pos = 0;
    if (cu_seqlens_q) {
        bool found = false;
        req = batch - 1;
        for (int base = 0; base < batch; base += kWave) {
            const int r = base + lane;
            const bool any = r < batch;
            const int first = any ? cu_seqlens_q[r] : 0, end = any ? cu_seqlens_q[r + 1] : INT_MAX;
            const int len = any ? context_lens[r] : 0;
            int owner = kWave;                        // requests of these that end at or before the token
            for (int t = 0; t < tpw; ++t) {
                const int ended = __builtin_popcountll(__builtin_amdgcn_ballot_w64(end <= token0 + t));
                if (lane == t) owner = ended;
            }
            // (a token behind the last request's, in a padded batch, has no place: counted on from that request it lay
            // beyond its context, in a block whose table slot is not in use)
            const bool last = base + kWave >= batch;
            const int from = min(owner, min(batch - base, kWave) - 1);
            const int f = __shfl(first, from), e = __shfl(end, from), l = __shfl(len, from);
            if (!found && (owner < kWave || last)) {
                found = true;
                req = base + from;
                pos = token < e ? l - (e - f) + (token - f) : -1;
            }
        }
    }
}

}  // namespace ra
