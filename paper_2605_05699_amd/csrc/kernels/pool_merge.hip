// Attention over a pool, the end: the sums of rows whose keys went to several workgroups are added in the order of the keys and
// finished; rows of sequences without a tile are zero.  One wavefront per 32 rows of a key head; those that their scan has finished have
// nothing to do here.
#include "../pool_attention.h"

namespace {

template <int D, bool CHUNK>
__global__ void __launch_bounds__(64) srft_pool_merge_kernel(const pool_attention_args a) {
    constexpr int BLOCKS = CHUNK ? kPoolChunkWaves<D> : 1, ROWS = kPoolBlock * BLOCKS, KEYS = CHUNK ? kPoolChunkKeys<D> : kPoolDecodeKeys;
    const int lane = threadIdx.x, of = (int)(blockIdx.x / (unsigned)a.merge_blocks), at = (int)blockIdx.x - of * a.merge_blocks;
    const int seq = of / a.heads, head = of - seq * a.heads, rt = at / BLOCKS, block = at - rt * BLOCKS;
    const pool_seq q = pool_seq_of(a.s, seq);
    if (q.n_new == 0 || pool_is_decode(q, a.group) == CHUNK || rt * ROWS + block * kPoolBlock >= q.n_new * a.group) return;
    const int* const before = CHUNK ? a.chunk_before : a.decode_before;
    const int total = before[a.s.n_seq];
    const int tiles = pool_tiles(CHUNK ? pool_seen(q, a.group, ROWS, rt) : q.length, q.full, KEYS);
    const pool_row row = pool_row_of(q, head, a.group, rt * ROWS + block * kPoolBlock + (lane & 31));
    char* const dst = row.there ? a.out + row.token * a.out_token + row.head * a.out_head : nullptr;
    if (tiles == 0) {
        if (dst)
            for (int i = lane >> 5; i < D / 8; i += 2) reinterpret_cast<uint4*>(dst)[i] = make_uint4(0, 0, 0, 0);
        return;
    }
    int first = before[seq];
    if constexpr (CHUNK) {
        const int n = (q.n_new * a.group + ROWS - 1) / ROWS;
        first += head * pool_chunk_units(q, a.group, ROWS, KEYS, n) + pool_chunk_units(q, a.group, ROWS, KEYS, rt);
    } else {
        first += head * tiles;
    }
    const pool_shares shares(total, CHUNK ? a.chunk_grid : a.decode_grid, CHUNK ? 1 : kPoolDecodeWaves);
    const int w0 = shares.owner(first), w1 = shares.owner(first + tiles - 1);
    if (w0 == w1) return;
    pool_block<D> b;
    b.clear();
    for (int w = w0; w <= w1; ++w) {
        const long long slot = 2LL * w + (w == w0 && shares.begin(w) != first ? 1 : 0);
        b.add((CHUNK ? a.chunk_parts : a.decode_parts) + (slot * BLOCKS + block) * kPoolPart<D>, lane);
    }
    pool_finish<D>(b, a.out_table, a.out_unscale, dst, a.bf16, lane);
}

template <int D> pool_attention_kernel_t pick(bool chunk) { return chunk ? srft_pool_merge_kernel<D, true> : srft_pool_merge_kernel<D, false>; }
pool_attention_kernel_t dispatch(int d, bool chunk) { SRFT_DISPATCH_D(d, pick, chunk) }

}  // namespace

pool_attention_kernel_t srft_pick_pool_merge(int d, bool chunk) { return dispatch(d, chunk); }
