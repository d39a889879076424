// Attention over a pool, before the keys: the queries' transform, the windows' tokens in the rotated domain, and the units of work.
//
// Three products of rows with a D x D matrix, on the matrix cores with the matrix as fp16 hi + lo: q' = R_k^T q, w = W_k k and w = W_v v.
// A workgroup has D / 32 wavefronts, each with 32 rows of the matrix in registers, as on the write path; a tile is 32 rows.  The results
// are stored as fp16 under a power of two per row (the exponent of its largest value), in the order of positions.
// Workgroups: 0 counts the units of work; 1 .. q_grid take the query tiles in turn; the others a tile of a window each (most of
// them, where pages are small, have no token in it).
#include "../pool_attention.h"

namespace {

template <int BITS>
constexpr int position_channel(int e) { return BITS == 8 ? (e & 4) + ((e & 1) << 1) + ((e & 2) >> 1) : e / 2 + 4 * (e % 2); }

// units of work in front of each sequence, by one workgroup
template <int D>
__device__ __forceinline__ void count_units(const pool_attention_args& a) {
    constexpr int NT = 2 * D, KEYS = kPoolChunkKeys<D>, ROWS = kPoolBlock * kPoolChunkWaves<D>;
    const pool_seqs& s = a.s;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    // the sequences' own units first, then their sums in place
    for (int b = wave; b < s.n_seq; b += NT / 64) {
        const pool_seq q = pool_seq_of(s, b);
        const bool decode = pool_is_decode(q, a.group);
        const int chunk = decode || q.n_new == 0 ? 0 : a.heads * pool_chunk_units(q, a.group, ROWS, KEYS, (q.n_new * a.group + ROWS - 1) / ROWS);
        if (lane == 0) {
            a.decode_before[b + 1] = decode && q.n_new > 0 ? a.heads * pool_tiles(q.length, q.full, kPoolDecodeKeys) : 0;
            a.chunk_before[b + 1] = chunk;
        }
    }
    __syncthreads();
    for (int which = wave; which < 2; which += NT / 64) {
        int* const at = which == 0 ? a.decode_before : a.chunk_before;
        int sum = 0;
        if (lane == 0) at[0] = 0;
        for (int b0 = 1; b0 <= s.n_seq; b0 += 64) {
            int x = b0 + lane <= s.n_seq ? at[b0 + lane] : 0;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int other = __shfl_up(x, d);
                if (lane >= d) x += other;
            }
            if (b0 + lane <= s.n_seq) at[b0 + lane] = sum + x;
            sum += __shfl(x, 63);
        }
    }
}

template <int D, int BITS>
__global__ void __launch_bounds__(2 * D) srft_pool_rotate_kernel(const pool_attention_args a) {
    constexpr int G = D / 32, T = D / 16, U = D / 8, ROW = U + 1, NT = 2 * D;
    __shared__ uint4 tile_lds[kTileVecs * ROW];
    __shared__ float row_max[G][kTileVecs];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, half = lane >> 5;
    if (blockIdx.x == 0) {
        count_units<D>(a);
        return;
    }
    const bool queries = (int)blockIdx.x <= a.q_grid;
    const int page_tiles = a.heads << a.s.log_R >> 5, R = 1 << a.s.log_R;
    int seq = 0, v = 0, window = 0, tail = 0, first_row = 0;
    if (!queries) {
        const int i = (int)blockIdx.x - 1 - a.q_grid, t = i % page_tiles;
        v = i / page_tiles & 1;
        seq = i / page_tiles >> 1;
        const pool_seq q = pool_seq_of(a.s, seq);
        tail = q.length - q.full;
        window = a.s.windows[2 * seq + 1];
        first_row = 32 * t;
        // (rows of pages of 32 tokens and more: a tile is in one head, from slot first_row % R on)
        if (tail == 0 || q.n_new == 0 || (R >= 32 && (first_row & (R - 1)) >= tail) || !pool_there(window, a.s.n_windows)) return;
    }
    const uint4* const table = queries ? a.q_table : v ? a.v_table : a.k_table;
    half8 ahi[T], alo[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        ahi[t] = __builtin_bit_cast(half8, table[((wave * T + t) * 2 + 0) * 64 + lane]);
        alo[t] = __builtin_bit_cast(half8, table[((wave * T + t) * 2 + 1) * 64 + lane]);
    }
    const int q_heads = a.heads * a.group, n_rows = a.s.n_new * q_heads;
    const int last_tile = queries ? a.q_tiles : 1;
    for (int tile = queries ? (int)blockIdx.x - 1 : 0; tile < last_tile; tile += queries ? a.q_grid : 1) {
#pragma unroll
        for (int i = 0; i < kTileVecs * U / NT; ++i) {
            const int u = tid + i * NT, r = u / U, c = u % U;
            const uint4* src;
            if (queries) {
                const int row = min(tile * kTileVecs + r, n_rows - 1), token = row / q_heads, head = row - token * q_heads;
                src = reinterpret_cast<const uint4*>(a.q + token * a.q_token + head * a.q_head);
            } else {
                src = reinterpret_cast<const uint4*>(v ? a.vb.window_f16_dev : a.kb.window_f16_dev) +
                      ((long long)window * (a.heads << a.s.log_R) + first_row + r) * U;
            }
            tile_lds[r * ROW + c] = src[c];
        }
        __syncthreads();
        half8 x[T];
        int shift = 0;                                       // of a bf16 row: its values were multiplied by 2^shift
#pragma unroll
        for (int t = 0; t < T; ++t) x[t] = __builtin_bit_cast(half8, tile_lds[col * ROW + 2 * t + half]);
        if (queries && a.bf16) {                             // uniform; exact: eight bits in fp16 under a power of two per row
            float m = 0.0f;
#pragma unroll
            for (int t = 0; t < T; ++t) {
                const uint4 w = __builtin_bit_cast(uint4, x[t]);
                for (uint32_t y : {w.x, w.y, w.z, w.w}) m = fmaxf(m, fmaxf(fabsf(__uint_as_float(y << 16)), fabsf(__uint_as_float(y & 0xFFFF0000u))));
            }
            m = other_half_max(m);
            shift = 14 - max((int)((__float_as_uint(m) >> 23) & 0xFF) - 127, -100);
            const float f = pool_power(shift);
#pragma unroll
            for (int t = 0; t < T; ++t) {
                const uint4 w = __builtin_bit_cast(uint4, x[t]);
                const uint32_t y[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[t][2 * i] = (_Float16)(__uint_as_float(y[i] << 16) * f);
                    x[t][2 * i + 1] = (_Float16)(__uint_as_float(y[i] & 0xFFFF0000u) * f);
                }
            }
        }
        floatx16 acc{0};
#pragma unroll
        for (int t = 0; t < T; ++t) {
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ahi[t], x[t], acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(alo[t], x[t], acc, 0, 0, 0);
        }
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(acc[i]));
        m = other_half_max(m);
        row_max[wave][col] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < G; ++w) m = fmaxf(m, row_max[w][col]);
        // (the maximum of the matrix's scaled product; 2^14 .. 2^15 afterwards)
        const int e = max((int)((__float_as_uint(m) >> 23) & 0xFF) - 127, -100);
        const float up = pool_power(14 - e) * (queries ? a.sign : 1.0f);
        uint32_t o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {                        // positions 2 i, 2 i + 1 of the lane's 16 channels
            const int c0 = 8 * (2 * i / 8) + position_channel<BITS>(2 * i % 8), c1 = 8 * (2 * i / 8) + position_channel<BITS>(2 * i % 8 + 1);
            const half2v h = {(_Float16)(acc[c0] * up), (_Float16)(acc[c1] * up)};
            o[i] = __builtin_bit_cast(uint32_t, h);
        }
        const int r = (queries ? tile * kTileVecs : first_row) + col;
        if (!queries || r < n_rows) {
            const long long row = queries ? r : ((long long)(v * a.s.n_seq + seq) * (a.heads << a.s.log_R)) + r;
            uint4* const dst = reinterpret_cast<uint4*>((queries ? a.q_rows : a.tail_rows) + row * D) + 4 * wave + 2 * half;
            dst[0] = make_uint4(o[0], o[1], o[2], o[3]);
            dst[1] = make_uint4(o[4], o[5], o[6], o[7]);
            if (wave == 0 && half == 0) {
                const float unscale = queries ? a.q_unscale * a.exponent : v ? a.v_unscale : a.k_unscale;
                (queries ? a.q_factor : a.tail_factor)[row] = unscale * pool_power(e - 14) * pool_power(-shift);
            }
        }
        __syncthreads();                                     // (the tile and the maxima have been read)
    }
}

template <int D> pool_attention_kernel_t pick(int bits) { return bits == 8 ? srft_pool_rotate_kernel<D, 8> : srft_pool_rotate_kernel<D, 4>; }
pool_attention_kernel_t dispatch(int d, int bits) { SRFT_DISPATCH_D(d, pick, bits) }

}  // namespace

pool_attention_kernel_t srft_pick_pool_rotate(int d, int bits) { return dispatch(d, bits); }
