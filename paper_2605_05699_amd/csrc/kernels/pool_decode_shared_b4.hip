// Attention over a pool for few rows a key head, 4-bit codes, sequences with pages in common.
#include "../pool_decode.h"

namespace {
template <int D> pool_attention_kernel_t pick(int cb, int gm) { return pool_pick_decode<D, 4, kPoolShared>(cb, gm); }
pool_attention_kernel_t dispatch(int d, int cb, int gm) { SRFT_DISPATCH_D(d, pick, cb, gm) }
}  // namespace

pool_attention_kernel_t srft_pick_pool_decode_shared_b4(int d, int cb, int gm) { return dispatch(d, cb, gm); }
