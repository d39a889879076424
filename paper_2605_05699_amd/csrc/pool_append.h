// pool_append.h -- the kernel that quantizes the pages which an append fills, out of the write path's tiles.
//
// The rows of a filled page lie in the sequence's window and among the new tokens; their record goes to a page of the caller's.  Both
// addresses come from the list that the kernel in front of this one has written (pool.hip), one entry per page, and a tile of 32 rows
// lies in one page, so that they are uniform: scalar loads.  K and V are in one launch, half of the workgroups each.
#ifndef SRFT_POOL_APPEND_H
#define SRFT_POOL_APPEND_H
#include "pool.h"
#include "quantize_fold4_tiles.h"
#include "quantize_fold_tiles.h"
#include "quantize_tiles.h"

template <int D, int S, int GM, int BITS>
struct pool_write_plain {
    static __device__ __forceinline__ void run(const uint4* frag, float unscale, int n_vec, uint2* codes, float* scales, int gw,
                                               const srft_rows_pool& rows, int place, int blocks) {
        srft_quantize_tiles<D, S, kOutCodes, GM, BITS, srft_flush_staged(D, 1LL << 40)>(frag, nullptr, n_vec, codes, scales, nullptr, unscale,
                                                                                       unscale / (BITS == 8 ? 127.0f : 7.0f), gw, place, blocks, rows);
    }
};
template <int D, int BITS, bool WIDE>
struct pool_write_fold {
    static __device__ __forceinline__ void run(const uint4* frag, float unscale, int n_vec, uint2* codes, float* scales, int gw,
                                               const srft_rows_pool& rows, int place, int blocks) {
        srft_quantize_fold_tiles<D, BITS, WIDE>(frag, nullptr, n_vec, codes, scales, unscale, unscale / (BITS == 8 ? 127.0f : 7.0f), gw, place,
                                                blocks, n_vec / kTileVecs, nullptr, rows);
    }
};
template <int BITS, int GM>
struct pool_write_fold4 {
    static __device__ __forceinline__ void run(const uint4* frag, float, int n_vec, uint2* codes, float* scales, int, const srft_rows_pool& rows,
                                               int place, int blocks) {
        srft_quantize_fold4_tiles<BITS, GM>(frag, nullptr, n_vec, codes, scales, 1.0f / (BITS == 8 ? 127.0f : 7.0f), place, blocks,
                                            n_vec / kTileVecs, nullptr, rows);
    }
};

template <int D, int NT, class WRITE>
__global__ void __launch_bounds__(NT, NT == D && D >= 128 ? 2 : 1) srft_pool_append_kernel(const pool_append_args a) {
    const bool v = blockIdx.x & 1;
    const int place = blockIdx.x >> 1, blocks = gridDim.x >> 1;
    const int tiles = *(const __attribute__((address_space(4))) int*)a.list * (a.heads << a.s.log_R >> 5);
    if (place >= tiles) return;                              // (uniform)
    const srft_rows_pool rows{(const uint4*)(v ? a.v : a.k), (const uint4*)(v ? a.vb.window_f16_dev : a.kb.window_f16_dev),
                              (const i32x4*)(a.list + 4), (v ? a.v_token : a.k_token) / 16, (v ? a.v_head : a.k_head) / 16, a.heads, a.s.log_R,
                              a.tiles_magic};
    WRITE::run(v ? a.v_table : a.k_table, v ? a.v_unscale : a.k_unscale, tiles * kTileVecs, (uint2*)(v ? a.vb.codes_dev : a.kb.codes_dev),
               v ? a.vb.scales_dev : a.kb.scales_dev, a.gw, rows, place, blocks);
}

#endif  // SRFT_POOL_APPEND_H
