// Attention over a pool for many rows a key head, of the last tokens and the first ones.
#include "../pool_chunk.h"

namespace {
template <int D> pool_attention_kernel_t pick(int bits) { return pool_pick_chunk<D, kPoolSliding>(bits); }
pool_attention_kernel_t dispatch(int d, int bits) { SRFT_DISPATCH_D(d, pick, bits) }
}  // namespace

pool_attention_kernel_t srft_pick_pool_chunk_sliding(int d, int bits) { return dispatch(d, bits); }
