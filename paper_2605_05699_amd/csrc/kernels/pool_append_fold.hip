// Append to a pool: the folded forms of the write path (d = 128 and 256).
#include "../pool_append.h"

namespace {
template <int D, class WRITE>
pool_append_kernel_t kernel() { return srft_pool_append_kernel<D, D, WRITE>; }
template <int BITS>
pool_append_kernel_t pick(int d, int gm, bool fold4_q) {
    if (d == 128) return gm == kGroupWide ? kernel<128, pool_write_fold<128, BITS, true>>() : kernel<128, pool_write_fold<128, BITS, false>>();
    if (d != 256) return nullptr;
    if (!fold4_q) return kernel<256, pool_write_fold<256, BITS, true>>();
    if (gm == kGroup16) return kernel<256, pool_write_fold4<BITS, kGroup16>>();
    return gm == kGroupWide ? kernel<256, pool_write_fold4<BITS, kGroupWide>>() : kernel<256, pool_write_fold4<BITS, kGroup32>>();
}
}  // namespace

pool_append_kernel_t srft_pick_pool_append_fold(int d, int bits, int gm, bool fold4_q) {
    return bits == 8 ? pick<8>(d, gm, fold4_q) : pick<4>(d, gm, fold4_q);
}
