// Launches of the one-launch decode step over a bf16 cache (the kernel: direct_kernel.h).
#include "direct_kernel.h"

namespace ra {

template <int D, bool MULTI>
static void launch_direct(const DirectArgs &a, const typename DirectPrefixes<MULTI>::type &pfx, hipStream_t stream) {
    const dim3 grid((unsigned)a.Hkv, (unsigned)a.G, (unsigned)a.n_tokens), block(kDirectThreads);
    if constexpr (!MULTI) {                       // (no entry point appends with several prefixes)
        if (a.k_new) {
            hipLaunchKernelGGL((decode_direct_kernel<D, false, true>), grid, block, 0, stream, a, pfx);
            return;
        }
    }
    hipLaunchKernelGGL((decode_direct_kernel<D, MULTI, false>), grid, block, 0, stream, a, pfx);
}

hipError_t launch_decode_direct(const DirectArgs &a, const DirectOne *one, const DirectMany *many, int head_dim,
                                hipStream_t stream) {
    if (a.n_tokens == 0) return hipSuccess;
    if (a.n_tokens > 65535 || (!one && !many) || (!one && a.k_new)) return hipErrorInvalidValue;
    if (head_dim == 128 && one) launch_direct<128, false>(a, *one, stream);
    else if (head_dim == 128) launch_direct<128, true>(a, *many, stream);
    else if (head_dim == 64 && one) launch_direct<64, false>(a, *one, stream);
    else if (head_dim == 64) launch_direct<64, true>(a, *many, stream);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace ra
