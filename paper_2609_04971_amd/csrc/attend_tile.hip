// Attention of many query rows for gfx950: the launches of the tile kernels (attend_tile.h) on
// bf16 caches, and of the sums of their weights on bf16 and fp32 ones.
#include "attend_tile.h"

namespace bkv {

hipError_t launch_attend_tile(const attend::Args& a, const attend::Segment& sg, hipStream_t s) {
    using namespace attend;
    const long long items = (long long)sg.units * sg.nrb * sg.ns;
    if (items == 0) return hipSuccess;
    if (a.D == 128)
        hipLaunchKernelGGL(tile_kernel<Bf16<128>>, dim3((unsigned)items), dim3(kThreads), 0, s, a, sg);
    else
        hipLaunchKernelGGL(tile_kernel<Bf16<64>>, dim3((unsigned)items), dim3(kThreads), 0, s, a, sg);
    return hipGetLastError();
}

hipError_t launch_attend_tile_mass(const attend::Args& a, int dtype, float* part, int parts, hipStream_t s) {
    using namespace attend;
    const dim3 grid((unsigned)mass_blocks(a, parts)), block(kThreads);
    if (dtype == BKV_BF16 && a.D == 128)
        hipLaunchKernelGGL(tile_mass_kernel<Bf16<128>>, grid, block, 0, s, a, part, parts);
    else if (dtype == BKV_BF16)
        hipLaunchKernelGGL(tile_mass_kernel<Bf16<64>>, grid, block, 0, s, a, part, parts);
    else if (a.D == 128)
        hipLaunchKernelGGL(tile_mass_kernel<F32<128>>, grid, block, 0, s, a, part, parts);
    else
        hipLaunchKernelGGL(tile_mass_kernel<F32<64>>, grid, block, 0, s, a, part, parts);
    return hipGetLastError();
}

}  // namespace bkv
