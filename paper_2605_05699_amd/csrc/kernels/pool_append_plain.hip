// Append to a pool: the plain form of the write path.
#include "../pool_append.h"

namespace {
template <int D, int S, int GM, int BITS>
pool_append_kernel_t kernel() { return srft_pool_append_kernel<D, 2 * D / S, pool_write_plain<D, S, GM, BITS>>; }
template <int D>
pool_append_kernel_t pick(int bits, int gm) {
    constexpr int S = D == 64 ? 2 : 1;
    if (bits == 8) return gm == kGroup16 ? kernel<D, S, kGroup16, 8>() : gm == kGroupWide ? kernel<D, S, kGroupWide, 8>() : kernel<D, S, kGroup32, 8>();
    return gm == kGroup16 ? kernel<D, S, kGroup16, 4>() : gm == kGroupWide ? kernel<D, S, kGroupWide, 4>() : kernel<D, S, kGroup32, 4>();
}
pool_append_kernel_t dispatch(int d, int bits, int gm) { SRFT_DISPATCH_D(d, pick, bits, gm) }
}  // namespace

pool_append_kernel_t srft_pick_pool_append_plain(int d, int bits, int gm) { return dispatch(d, bits, gm); }
