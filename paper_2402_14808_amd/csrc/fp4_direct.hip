// Launch of the one-launch decode step over a 4-bit cache (the kernel: direct_kernel.h).
#include "direct_kernel.h"

namespace ra {

hipError_t launch_decode_direct_fp4(const DirectArgs &a, const DirectOne &one, int head_dim, hipStream_t stream) {
    if (a.n_tokens == 0) return hipSuccess;
    if (a.n_tokens > 65535 || a.k_new) return hipErrorInvalidValue;
    const dim3 grid((unsigned)a.Hkv, (unsigned)a.G, (unsigned)a.n_tokens), block(kDirectThreads);
    if (head_dim == 128) hipLaunchKernelGGL((decode_direct_kernel<128, false, false, true>), grid, block, 0, stream, a, one);
    else if (head_dim == 64) hipLaunchKernelGGL((decode_direct_kernel<64, false, false, true>), grid, block, 0, stream, a, one);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace ra
