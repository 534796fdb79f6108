// Attention of many query rows for gfx950: the launches of the tile kernels (attend_tile.h) on
// bf16 caches, and of the sums of their weights on bf16 and fp32 ones.
#include "attend_tile.h"

namespace bkv {

hipError_t launch_attend_tile(const attend::Args& a, const attend::Segment& sg, hipStream_t s) {
    using namespace attend;
    return a.D == 128 ? tile<Bf16<128>>(a, sg, s) : tile<Bf16<64>>(a, sg, s);
}

hipError_t launch_attend_tile_mass(const attend::Args& a, int dtype, float* part, int parts, hipStream_t s) {
    using namespace attend;
    if (dtype == BKV_BF16) return a.D == 128 ? tile_mass<Bf16<128>>(a, part, parts, s) : tile_mass<Bf16<64>>(a, part, parts, s);
    return a.D == 128 ? tile_mass<F32<128>>(a, part, parts, s) : tile_mass<F32<64>>(a, part, parts, s);
}

}  // namespace bkv
