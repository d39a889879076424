// Attention over a pool, before the keys: the queries' transform, the windows' tokens in the rotated domain, and the units of work.
//
// Three products of rows with a D x D matrix, on the matrix cores with the matrix as fp16 hi + lo: q' = R_k^T q, w = W_k k and w = W_v v.
// A workgroup has D / 32 wavefronts, each with 32 rows of the matrix, in registers; a pass is 32 rows.  The results are stored as fp16 under
// a power of two per row (the exponent of its largest value), in the order of positions; of the queries also what that rounding leaves,
// where rows may go to pool_decode.
// Bound by the rows' bytes where there are many (65,536 of d = 128: 12.4 us, 34 MB), else by the chain from the matrix (4 D^2 bytes, 256 KB at
// d = 256, asked for before the rows) to the stores: 4.7 us for 4096 rows, 8.5 at d = 256.  Read as it is used, by passes of four tiles of
// rows to make up for that, the matrix came out of the L2 for every pass: 15.4 us for the 65,536 rows, 18.4 for 4000 of d = 256.
// Workgroups: 0 counts the units of work; 1 .. q_grid take the passes of the queries in turn; the others a part of a window each.
#include "../pool_attention.h"

namespace {

template <int BITS>
constexpr int position_channel(int e) { return BITS == 8 ? (e & 4) + ((e & 1) << 1) + ((e & 2) >> 1) : e / 2 + 4 * (e % 2); }

// units of work in front of each sequence, by one workgroup
template <int D>
__device__ __forceinline__ void count_units(const pool_attention_args& a) {
    constexpr int NT = 2 * D, KEYS = kPoolChunkKeys<D>, ROWS = kPoolBlock * kPoolChunkWaves;
    const pool_seqs& s = a.s;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    // the sequences' own units first, then their sums in place
    for (int b = wave; b < s.n_seq; b += NT / 64) {
        const pool_seq q = pool_seq_of(s, b);
        const bool decode = pool_is_decode(q, a.group, a.decode_rows);
        const int chunk = decode || q.n_new == 0 ? 0 : a.heads * pool_chunk_units(q, a.group, ROWS, KEYS, (q.n_new * a.group + ROWS - 1) / ROWS);
        if (lane == 0) {
            if (a.blocks_before) a.blocks_before[b + 1] = decode ? 0 : (q.n_new * a.group + ROWS - 1) / ROWS;
            a.decode_before[b + 1] = decode ? a.heads * ((q.n_new * a.group + a.decode_block - 1) / a.decode_block) * pool_tiles(q.length, q.full, a.decode_keys) : 0;
            a.chunk_before[b + 1] = chunk;
        }
    }
    __syncthreads();
    for (int which = wave; which < (a.blocks_before ? 3 : 2); which += NT / 64) {
        int* const at = which == 0 ? a.decode_before : which == 1 ? a.chunk_before : a.blocks_before;
        unsigned sum = 0;
        if (lane == 0) at[0] = 0;
        for (int b0 = 1; b0 <= s.n_seq; b0 += 64) {
            const int b = b0 + lane;
            unsigned x = b <= s.n_seq ? at[b] : 0;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const unsigned other = __shfl_up(x, d);
                if (lane >= d) x = min(x + other, kPoolMostUnits);
            }
            const unsigned before = min(sum + x, kPoolMostUnits);
            if (b <= s.n_seq) at[b] = b == s.n_seq && before == kPoolMostUnits ? 0 : (int)before;
            sum = min(sum + (unsigned)__shfl(x, 63), kPoolMostUnits);
        }
    }
}

template <int D, int BITS>
__global__ void __launch_bounds__(2 * D) srft_pool_rotate_kernel(const pool_attention_args a) {
    constexpr int G = D / 32, T = D / 16, U = D / 8, ROW = U + 1, NT = 2 * D, ROWS = kTileVecs;
    __shared__ uint4 rows_lds[ROWS * ROW];
    __shared__ float row_max[G][ROWS];
    __shared__ int shifts[ROWS];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, half = lane >> 5;
    if (blockIdx.x == 0) {
        count_units<D>(a);
        return;
    }
    const bool queries = (int)blockIdx.x <= a.q_grid;
    const int page_rows = a.heads << a.s.log_R, passes = page_rows / ROWS, R = 1 << a.s.log_R;
    int seq = 0, v = 0, window = 0, tail = 0, first_row = 0;
    if (!queries) {
        const int i = (int)blockIdx.x - 1 - a.q_grid, t = i % passes;
        v = i / passes & 1;
        seq = i / passes >> 1;
        const pool_seq q = pool_seq_of(a.s, seq);
        tail = q.length - q.full;
        window = a.s.windows[2 * seq + 1];
        first_row = ROWS * t;
        // (pages of ROWS tokens and more: a pass is in one head, from slot first_row % R on)
        if (tail == 0 || q.n_new == 0 || (R >= ROWS && (first_row & (R - 1)) >= tail) || !pool_there(window, a.s.n_windows)) return;
    }
    const uint4* const table = (queries ? a.q_table : v ? a.v_table : a.k_table) + wave * T * 2 * 64 + lane;
    half8 ahi[T], alo[T];                                    // the matrix stays in registers over the passes of a workgroup
#pragma unroll
    for (int t = 0; t < T; ++t) {
        ahi[t] = __builtin_bit_cast(half8, table[(2 * t + 0) * 64]);
        alo[t] = __builtin_bit_cast(half8, table[(2 * t + 1) * 64]);
    }
    const int q_heads = a.heads * a.group, n_rows = queries ? a.s.n_new * q_heads : page_rows;
    const int last_pass = queries ? a.q_tiles : 1;
    for (int pass = queries ? (int)blockIdx.x - 1 : 0; pass < last_pass; pass += queries ? a.q_grid : 1) {
        const int row0 = queries ? pass * ROWS : first_row;
#pragma unroll
        for (int i = 0; i < ROWS * U / NT; ++i) {
            const int u = tid + i * NT, r = u / U, c = u % U, row = min(row0 + r, n_rows - 1);
            const uint4* src;
            bool held = true;
            if (queries) {
                const int token = row / q_heads, head = row - token * q_heads;
                src = reinterpret_cast<const uint4*>(a.q + token * a.q_token + head * a.q_head);
            } else {
                src = reinterpret_cast<const uint4*>(v ? a.vb.window_f16_dev : a.kb.window_f16_dev) + ((long long)window * page_rows + row) * U;
                held = (row & (R - 1)) < tail;               // (slots behind the last token hold anything: zeros)
            }
            rows_lds[r * ROW + c] = held ? src[c] : make_uint4(0, 0, 0, 0);
        }
        for (int r = tid; r < ROWS; r += NT) shifts[r] = 0;
        __syncthreads();
        if (queries && a.bf16) {                             // uniform; exact: eight bits in fp16 under a power of two per row
            for (int r = tid >> 5; r < ROWS; r += NT / 32) {             // half a wavefront a row
                uint4 w = rows_lds[r * ROW + min(tid & 31, U - 1)];
                uint32_t y[4] = {w.x, w.y, w.z, w.w};
                float m = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) m = fmaxf(m, fmaxf(fabsf(__uint_as_float(y[i] << 16)), fabsf(__uint_as_float(y[i] & 0xFFFF0000u))));
#pragma unroll
                for (int d = 1; d < 32; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
                const int shift = 14 - max((int)((__float_as_uint(m) >> 23) & 0xFF) - 127, -100);
                const float f = pool_power(shift);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const half2v h = {(_Float16)(__uint_as_float(y[i] << 16) * f), (_Float16)(__uint_as_float(y[i] & 0xFFFF0000u) * f)};
                    y[i] = __builtin_bit_cast(uint32_t, h);
                }
                if ((tid & 31) < U) rows_lds[r * ROW + (tid & 31)] = make_uint4(y[0], y[1], y[2], y[3]);
                if ((tid & 31) == 0) shifts[r] = shift;
            }
            __syncthreads();
        }
        floatx16 acc{0};
#pragma unroll
        for (int t = 0; t < T; ++t) {
            const half8 x = __builtin_bit_cast(half8, rows_lds[col * ROW + 2 * t + half]);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ahi[t], x, acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(alo[t], x, acc, 0, 0, 0);
        }
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(acc[i]));
        row_max[wave][col] = other_half_max(m);
        __syncthreads();
        m = 0.0f;
#pragma unroll
        for (int w = 0; w < G; ++w) m = fmaxf(m, row_max[w][col]);
        // (the maximum of the matrix's scaled product; 2^14 .. 2^15 afterwards)
        const int e = max((int)((__float_as_uint(m) >> 23) & 0xFF) - 127, -100);
        const float up = pool_power(14 - e) * (queries ? a.sign : 1.0f);
        uint32_t o[8], low[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {                    // positions 2 i, 2 i + 1 of the lane's 16 channels
            const int c0 = 8 * (2 * i / 8) + position_channel<BITS>(2 * i % 8), c1 = 8 * (2 * i / 8) + position_channel<BITS>(2 * i % 8 + 1);
            const half2v h = {(_Float16)(acc[c0] * up), (_Float16)(acc[c1] * up)};
            o[i] = __builtin_bit_cast(uint32_t, h);
            const half2v l = {(_Float16)(acc[c0] * up - (float)h[0]), (_Float16)(acc[c1] * up - (float)h[1])};
            low[i] = __builtin_bit_cast(uint32_t, l);
        }
        const int r = row0 + col;
        if (r < n_rows) {
            const long long row = queries ? r : (long long)(v * a.s.n_seq + seq) * page_rows + r;
            uint4* const dst = reinterpret_cast<uint4*>((queries ? a.q_rows : a.tail_rows) + row * D) + 4 * wave + 2 * half;
            dst[0] = make_uint4(o[0], o[1], o[2], o[3]);
            dst[1] = make_uint4(o[4], o[5], o[6], o[7]);
            if (queries && a.q_rows_low) {               // uniform
                uint4* const dst_low = reinterpret_cast<uint4*>(a.q_rows_low + row * D) + 4 * wave + 2 * half;
                dst_low[0] = make_uint4(low[0], low[1], low[2], low[3]);
                dst_low[1] = make_uint4(low[4], low[5], low[6], low[7]);
            } else if (v) {
                const int h = r >> a.s.log_R, slot = r & (R - 1);
                unsigned short* const columns = a.tail_columns + (((long long)seq * a.heads + h) * D + 32 * wave + 16 * half << a.s.log_R) + slot;
#pragma unroll
                for (int i = 0; i < 16; ++i) columns[i << a.s.log_R] = __builtin_bit_cast(unsigned short, (_Float16)(acc[i] * up));
            }
            if (wave == 0 && half == 0) {
                const float unscale = queries ? a.q_unscale * a.exponent : v ? a.v_unscale : a.k_unscale;
                (queries ? a.q_factor : a.tail_factor)[row] = unscale * pool_power(e - 14) * pool_power(-shifts[col]);
            }
        }
        __syncthreads();                                     // (the rows and their maxima have been read)
    }
}

template <int D> pool_attention_kernel_t pick(int bits) { return bits == 8 ? srft_pool_rotate_kernel<D, 8> : srft_pool_rotate_kernel<D, 4>; }
pool_attention_kernel_t dispatch(int d, int bits) { SRFT_DISPATCH_D(d, pick, bits) }

}  // namespace

pool_attention_kernel_t srft_pick_pool_rotate(int d, int bits) { return dispatch(d, bits); }
