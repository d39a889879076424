// Attention over a pool, the end: the sums of rows whose keys went to several workgroups are added in the order of the keys and
// finished; rows of sequences without a tile are zero.  The first a.decode_merges workgroups take the rows of the scan for few rows
// (pool_decode_merge), the others those of chunks, in one launch: apart, the first took 17 us beside the 29 of the others (d = 256).
// Chunks: one workgroup of four wavefronts per 32 rows of a key head, of the blocks of 256 rows that there are (by the longest sequence for each, 255 decode steps beside a
// prompt of 4096 tokens, 64 query heads, were a million workgroups, nearly all of them empty: 1376 us, now 36), each with every fourth
// run of 32 positions of the sums and then of the outputs (one wavefront per 32 rows read every part, and the matrix, one after
// the other: 104 us at d = 256, 28 at d = 128).  Bound by the chain of loads where parts are few (a first round for the maxima alone: 6.9 us,
// now 5.5, for a step of 4 sequences), by the parts' bytes where they are many (23 us for 67 MB at d = 128; more of them in flight is slower).  Rows that their scan has finished have nothing to do here.
#include "../pool_decode.h"

namespace {

template <int D>
__device__ __forceinline__ void chunk_merge(const pool_attention_args& a, unsigned workgroup, uint4* ops, float (*tops)[32]) {
    constexpr int BLOCKS = kPoolChunkWaves, ROWS = kPoolBlock * BLOCKS, KEYS = kPoolChunkKeys<D>, G = D / 32, T = D / 16, OWN = (G + kPoolTeam - 1) / kPoolTeam, AHEAD = 2;
    // ops: [k-step][hi, lo][lane]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int of = (int)(workgroup / BLOCKS), block = (int)workgroup - of * BLOCKS, at = of / a.heads, head = of - at * a.heads;
    if (at >= a.blocks_before[a.s.n_seq]) return;
    const int seq = a.s.n_seq == 1 ? 0 : __builtin_amdgcn_readfirstlane(pool_sequence_of(a.blocks_before, a.s.n_seq, at)), rt = at - a.blocks_before[seq];
    const pool_seq q = pool_seq_of(a.s, seq);
    const int r0 = rt * ROWS + block * kPoolBlock;
    if (r0 >= q.n_new * a.group) return;
    const int tiles = pool_tiles(pool_seen(q, a.group, ROWS, rt), q.full, KEYS);
    const pool_row row = pool_row_of(q, head, a.group, r0 + (lane & 31));
    char* const dst = row.there ? a.out + row.token * a.out_token + row.head * a.out_head : nullptr;
    if (tiles == 0) {
        if (dst)
            for (int i = 2 * wave + half; i < D / 8; i += 2 * kPoolTeam) reinterpret_cast<uint4*>(dst)[i] = make_uint4(0, 0, 0, 0);
        return;
    }
    const int* const before = a.chunk_before;
    const int units = before[a.s.n_seq];
    if (units == 0) return;                                  // (too many of them: see kPoolMostUnits)
    const int first = before[seq] + head * pool_chunk_units(q, a.group, ROWS, KEYS, (q.n_new * a.group + ROWS - 1) / ROWS) +
                      pool_chunk_units(q, a.group, ROWS, KEYS, rt);
    const pool_shares shares(units, a.chunk_grid, 1);
    const int w0 = shares.owner(first), w1 = shares.owner(first + tiles - 1);
    if (w0 == w1) return;
    const int behind = shares.begin(w0) != first ? 1 : 0;    // the first part's workgroup began with other rows
    const auto part = [&](int w) __attribute__((always_inline)) {
        return a.chunk_parts + ((2LL * w + (w == w0 ? behind : 0)) * BLOCKS + block) * kPoolPart<D>;
    };
    float t_all = kPoolLowest, den = 0.0f;
    int e_all = kPoolNoExponent;
    floatx16 sums[OWN];
#pragma unroll
    for (int i = 0; i < OWN; ++i) sums[i] = floatx16{0};
    for (int v = w0; v <= w1; v += AHEAD) {
        floatx4 x[AHEAD][OWN][4];
        pool_part_head h[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const float* const p = part(min(v + k, w1));
            h[k].load(p + 32 * D, lane);
#pragma unroll
            for (int i = 0; i < OWN; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) x[k][i][j] = reinterpret_cast<const floatx4*>(p)[(4 * min(wave + kPoolTeam * i, G - 1) + j) * 64 + lane];
        }
        const float before = pool_join(t_all, den, e_all, h, v, w1);
#pragma unroll
        for (int i = 0; i < OWN; ++i) sums[i] *= before;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
#pragma unroll
            for (int i = 0; i < OWN; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int m = 0; m < 4; ++m) sums[i][4 * j + m] = fmaf(x[k][i][j][m], h[k].factor, sums[i][4 * j + m]);
    }
    // ---- as pool_finish, the operands through LDS
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < OWN; ++i)
        if (wave + kPoolTeam * i < G)
#pragma unroll
            for (int v = 0; v < 16; ++v) m = fmaxf(m, fabsf(sums[i][v]));
    m = other_half_max(m);
    tops[wave][lane & 31] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kPoolTeam; ++w) m = fmaxf(m, tops[w][lane & 31]);
    const int e = max((int)((__float_as_uint(m) >> 23) & 0xFF) - 127, -100);
    const float up = pool_power(14 - e);
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const int b = wave + kPoolTeam * i;
        if (b < G)                                           // uniform
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                half8 hi, lo;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float x = sums[i][8 * k + j] * up;
                    hi[j] = (_Float16)x;
                    lo[j] = (_Float16)(x - (float)hi[j]);
                }
                ops[((2 * b + k) * 2 + 0) * 64 + lane] = __builtin_bit_cast(uint4, hi);
                ops[((2 * b + k) * 2 + 1) * 64 + lane] = __builtin_bit_cast(uint4, lo);
            }
    }
    __syncthreads();
    const float down = (den > 0.0f ? 1.0f / den : 0.0f) * a.out_unscale, p0 = pool_power(e - 14), p1 = pool_power(e_all);
    for (int j = wave; j < G; j += kPoolTeam) {
        floatx16 acc{0};
#pragma unroll
        for (int k = 0; k < T; ++k) {
            const half8 ah = __builtin_bit_cast(half8, a.out_table[((j * T + k) * 2 + 0) * 64 + lane]), al = __builtin_bit_cast(half8, a.out_table[((j * T + k) * 2 + 1) * 64 + lane]);
            const half8 bh = __builtin_bit_cast(half8, ops[(2 * k + 0) * 64 + lane]), bl = __builtin_bit_cast(half8, ops[(2 * k + 1) * 64 + lane]);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bh, acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(al, bh, acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bl, acc, 0, 0, 0);
        }
        pool_store16(acc, down, p0, p1, dst, 32 * j + 16 * half, a.bf16);
    }
}

template <int D, int CB>
__global__ void __launch_bounds__(64 * kPoolTeam) srft_pool_merge_kernel(const pool_attention_args a) {
    constexpr int OPS = D / 16 * 2 * 64;
    __shared__ __align__(16) unsigned char lds[std::max(kPoolFinishBytes<D>, OPS * 16 + kPoolTeam * 32 * 4)];
    const unsigned workgroup = blockIdx.y * gridDim.x + blockIdx.x;          // (what follows is uniform)
    if (workgroup >= a.merges) return;
    if (workgroup < (unsigned)a.decode_merges)
        pool_decode_merge<D, CB>(a, workgroup, lds);
    else
        chunk_merge<D>(a, workgroup - a.decode_merges, reinterpret_cast<uint4*>(lds), reinterpret_cast<float (*)[32]>(lds + OPS * 16));
}

template <int D> pool_attention_kernel_t pick(int cb) {
    if constexpr (D <= 128)
        if (cb == 2) return srft_pool_merge_kernel<D, 2>;
    return srft_pool_merge_kernel<D, 1>;
}
pool_attention_kernel_t dispatch(int d, int cb) { SRFT_DISPATCH_D(d, pick, cb) }

}  // namespace

pool_attention_kernel_t srft_pick_pool_merge(int d, int cb) { return dispatch(d, cb); }
