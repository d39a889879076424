// Attention over a pool for few rows a key head, 8-bit codes; the merge of either.
#include "../pool_decode.h"

namespace {
template <int D> pool_attention_kernel_t pick(int cb, int gm) { return pool_pick_decode<D, 8>(cb, gm); }
pool_attention_kernel_t dispatch(int d, int cb, int gm) { SRFT_DISPATCH_D(d, pick, cb, gm) }
template <int D> pool_attention_kernel_t pick_merge(int cb) {
    if constexpr (D <= 128)
        if (cb == 2) return srft_pool_decode_merge_kernel<D, 2>;
    return srft_pool_decode_merge_kernel<D, 1>;
}
pool_attention_kernel_t dispatch_merge(int d, int cb) { SRFT_DISPATCH_D(d, pick_merge, cb) }
}  // namespace

pool_attention_kernel_t srft_pick_pool_decode_b8(int d, int cb, int gm) { return dispatch(d, cb, gm); }
pool_attention_kernel_t srft_pick_pool_decode_merge(int d, int cb) { return dispatch_merge(d, cb); }
