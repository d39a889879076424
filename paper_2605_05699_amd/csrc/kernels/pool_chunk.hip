// Attention over a pool for many rows a key head (a chunk of a prompt): 256 rows (tokens x query heads of the group) a workgroup.
//
// Bound by the vector instructions of the softmax and of the decoding, beside the matrix instructions.  A tile of keys is
// decoded once for all the workgroup's rows, by all its wavefronts, into LDS (two buffers: the next tile is decoded while this one is
// used, one barrier a tile); each of the eight wavefronts takes 32 rows through it with the scheme of pool_decode.hip: keys on the
// rows of the score product, so that scores, weights and the running softmax of a row stay in one lane and its neighbour across the
// wavefront, and weights go into the second product as they are.
//
// A tile's exponent (of K's scales and of V's) has to be known before it is decoded.  Its scales are loaded with its codes two tiles ahead;
// each wavefront brings its largest one to LDS at the end of the tile in between, one atomic maximum, in a ring of four.
#include "../pool_attention.h"

namespace {

template <int D, int BITS>
__global__ void __launch_bounds__(64 * kPoolChunkWaves<D>, 2) srft_pool_chunk_kernel(const pool_attention_args a) {
    constexpr int W = kPoolChunkWaves<D>, NT = 64 * W, KEYS = kPoolChunkKeys<D>, ROWS = kPoolBlock * W, KB = KEYS / 32;
    constexpr int T = D / 16, CB = D * BITS / 8;
    constexpr int KROW = 2 * D + 16, VROW = 2 * D + 32;      // bytes of a row in LDS: 16-byte reads of 32 rows, transposed reads of 8, on different banks
    constexpr int UNITS = KEYS * T;                          // of 16 channels, of K or of V
    constexpr int N = (2 * UNITS + NT - 1) / NT;             // a thread's
    typedef typename pool_codes<BITS>::type code_t;
    __shared__ __align__(16) unsigned char k_lds[2][KEYS * KROW], v_lds[2][KEYS * VROW];
    __shared__ unsigned int largest[4][2];                   // bits of the largest scale of a tile, K and V
    __shared__ unsigned int unknown[4];                      // a key of the tile lies in a page that does not exist
    __shared__ unsigned char known[2][KEYS];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
    const int total = a.chunk_before[a.s.n_seq];
    const int w = srft_block_by_die();
    const pool_shares shares(total, gridDim.x, 1);
    if (total == 0 || w >= shares.groups) return;            // (uniform)
    const int end = shares.begin(w + 1);
    int unit = shares.begin(w);
    int seq = __builtin_amdgcn_readfirstlane(pool_sequence_of(a.chunk_before, a.s.n_seq, unit));
    const int R = 1 << a.s.log_R, n_scales = D / a.g;

    // a thread's units: K's first, then V's; which key of the tile, which 16 channels
    int u_key[N], u_at[N], u_scale[N];
    bool u_v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int u = min(tid + i * NT, 2 * UNITS - 1);      // (past the end: the last unit again)
        u_v[i] = u >= UNITS;
        const int r = u_v[i] ? u - UNITS : u;
        u_key[i] = r / T;
        u_at[i] = r - u_key[i] * T;
        u_scale[i] = 16 * u_at[i] / a.g;
    }

    for (bool at_begin = true; unit < end; at_begin = false) {
        while (seq + 1 < a.s.n_seq && a.chunk_before[seq + 1] <= unit) ++seq;
        const pool_seq q = pool_seq_of(a.s, seq);
        const int blocks = (q.n_new * a.group + ROWS - 1) / ROWS;
        const int per_head = __builtin_amdgcn_readfirstlane(pool_chunk_units(q, a.group, ROWS, KEYS, blocks));
        const int rel = unit - a.chunk_before[seq], head = rel / per_head;
        int t0 = rel - head * per_head, rt = 0, tiles = pool_tiles(pool_seen(q, a.group, ROWS, 0), q.full, KEYS);
        while (t0 >= tiles && rt + 1 < blocks) {             // the block of rows (those without a tile are passed over)
            t0 -= tiles;
            tiles = pool_tiles(pool_seen(q, a.group, ROWS, ++rt), q.full, KEYS);
        }
        const int t1 = min(tiles, t0 + end - unit);
        if (t1 <= t0) return;                                // (only if the device arrays were written during the call)
        const int seen = pool_seen(q, a.group, ROWS, rt), page_keys = min(seen, q.full), page_tiles = (max(page_keys, 0) + KEYS - 1) / KEYS, tail = q.length - q.full;
        const pool_row row = pool_row_of(q, head, a.group, rt * ROWS + wave * kPoolBlock + l32);
        const long long q_row = (long long)row.token * (a.heads * a.group) + row.head;
        const int32_t* const table = a.s.table + seq * a.s.max_pages;
        const bool window_there = pool_there(a.s.windows[2 * seq + 1], a.s.n_windows);
        // (the last token that any row of this wavefront sees; rows do not see less than those before them)
        int wave_last = row.last;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) wave_last = max(wave_last, __shfl_xor(wave_last, d));
        wave_last = __builtin_amdgcn_readfirstlane(wave_last);

        half8 qf[T];
        {
            const uint4* const q_at = reinterpret_cast<const uint4*>(a.q_rows + q_row * D) + half;
#pragma unroll
            for (int s = 0; s < T; ++s) qf[s] = __builtin_bit_cast(half8, q_at[2 * s]);
        }
        const float factor = a.q_factor[q_row];
        pool_block<D> b;
        b.clear();

        code_t code[N];
        float scale[N];
        bool there[N];
        int page[N];
        const auto pages = [&](int t) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < N; ++i) page[i] = q.full > 0 ? table[min(t * KEYS + u_key[i], q.full - 1) >> a.s.log_R] : -1;
        };
        const auto fetch = [&](int t) __attribute__((always_inline)) {
            if (t >= t1) return;                             // uniform, as below
            if (t < page_tiles) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const srft_pool_buffers& of = u_v[i] ? a.vb : a.kb;
                    there[i] = pool_there(page[i], a.s.n_pages);
                    const long long at = ((long long)(there[i] ? page[i] : 0) * a.heads + head << a.s.log_R) + (min(t * KEYS + u_key[i], q.full - 1) & (R - 1));
                    code[i] = reinterpret_cast<const code_t*>(of.codes_dev + at * CB)[u_at[i]];
                    scale[i] = of.scales_dev[at * n_scales + u_scale[i]];
                }
            } else {                                         // the window's tokens: the row's factor (their rows are loaded where they are used)
                constexpr float kUp = BITS == 4 ? 4096.0f : 256.0f;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const long long at = ((long long)((u_v[i] ? a.s.n_seq : 0) + seq) * a.heads + head << a.s.log_R) + min((t - page_tiles) * KEYS + u_key[i], tail - 1);
                    there[i] = window_there;
                    scale[i] = there[i] ? a.tail_factor[at] * kUp : 0.0f;
                }
            }
        };
        // the largest scale of the tile that has been fetched
        const auto publish = [&](int t) __attribute__((always_inline)) {
            if (t >= t1) return;
            float mk = 0.0f, mv = 0.0f;
            bool all = true;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                scale[i] = there[i] ? scale[i] : 0.0f;
                mk = fmaxf(mk, u_v[i] ? 0.0f : scale[i]);
                mv = fmaxf(mv, u_v[i] ? scale[i] : 0.0f);
                all &= there[i];
            }
            mk = pool_wave_max(mk);
            mv = pool_wave_max(mv);
            const bool some = __ballot(!all) != 0;
            if (lane == 0) {
                atomicMax(&largest[t & 3][0], __float_as_uint(mk));
                atomicMax(&largest[t & 3][1], __float_as_uint(mv));
                if (some) unknown[t & 3] = 1;
            }
        };
        int ev = kPoolNoExponent;                            // of the tile decoded last
        const auto decode = [&](int t) __attribute__((always_inline)) {
            if (t >= t1) return;
            const int ek = pool_exponent<BITS>(__uint_as_float(largest[t & 3][0]));
            ev = max(ev, pool_exponent<BITS>(__uint_as_float(largest[t & 3][1])));
            const float uk = pool_power(-ek), uv = pool_power(-ev);
            if (t < page_tiles) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    half8 x, y;
                    pool_decode16(code[i], (_Float16)(scale[i] * (u_v[i] ? uv : uk)), x, y);
                    unsigned char* const dst = u_v[i] ? &v_lds[t & 1][u_key[i] * VROW] : &k_lds[t & 1][u_key[i] * KROW];
                    reinterpret_cast<uint4*>(dst)[2 * u_at[i]] = __builtin_bit_cast(uint4, x);
                    reinterpret_cast<uint4*>(dst)[2 * u_at[i] + 1] = __builtin_bit_cast(uint4, y);
                    if (!u_v[i] && u_at[i] == 0) known[t & 1][u_key[i]] = there[i];
                }
            } else {
                constexpr float kDown = BITS == 4 ? 1.0f / 4096.0f : 1.0f / 256.0f;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const long long at = ((long long)((u_v[i] ? a.s.n_seq : 0) + seq) * a.heads + head << a.s.log_R) + min((t - page_tiles) * KEYS + u_key[i], tail - 1);
                    const uint4* const src = reinterpret_cast<const uint4*>(a.tail_rows + at * D) + 2 * u_at[i];
                    const _Float16 f = (_Float16)(scale[i] * kDown * (u_v[i] ? uv : uk));
                    const uint4 zero = make_uint4(0, 0, 0, 0);
                    unsigned char* const dst = u_v[i] ? &v_lds[t & 1][u_key[i] * VROW] : &k_lds[t & 1][u_key[i] * KROW];
                    reinterpret_cast<uint4*>(dst)[2 * u_at[i]] = __builtin_bit_cast(uint4, pool_times(there[i] ? src[0] : zero, f));
                    reinterpret_cast<uint4*>(dst)[2 * u_at[i] + 1] = __builtin_bit_cast(uint4, pool_times(there[i] ? src[1] : zero, f));
                    if (!u_v[i] && u_at[i] == 0) known[t & 1][u_key[i]] = there[i];
                }
            }
        };

        // ---- the first tiles
        __syncthreads();                                     // (the segment before has read its last tile)
        if (tid < 8) largest[tid >> 1][tid & 1] = 0;
        if (tid < 4) unknown[tid] = 0;
        pages(t0);
        fetch(t0);
        pages(t0 + 1);
        __syncthreads();
        publish(t0);
        __syncthreads();
        decode(t0);
        int ev_now = ev;
        fetch(t0 + 1);
        pages(t0 + 2);
        publish(t0 + 1);

        for (int t = t0; t < t1; ++t) {
            __syncthreads();                                 // tile t is in LDS, tile t + 1's scales in the ring
            const int ek_now = pool_exponent<BITS>(__uint_as_float(largest[t & 3][0]));
            ev_now = ev;
            const bool some_unknown = unknown[t & 3] != 0;
            if (tid < 2) largest[(t + 3) & 3][tid] = 0;      // (last read before this barrier, next written behind the next one)
            if (tid == 2) unknown[(t + 3) & 3] = 0;
            decode(t + 1);
            fetch(t + 2);
            pages(t + 3);
            const bool window = t >= page_tiles;
            const int key0 = window ? q.full + (t - page_tiles) * KEYS : t * KEYS;
            if (key0 <= wave_last) {                         // (uniform over the wavefront)
                floatx16 s[KB];
                const unsigned char* const kr = &k_lds[t & 1][l32 * KROW + 16 * half];
#pragma unroll
                for (int n = 0; n < KB; ++n) {
                    s[n] = floatx16{0};
#pragma unroll
                    for (int i = 0; i < T; ++i)
                        s[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, *reinterpret_cast<const uint4*>(kr + 32 * n * KROW + 32 * i)), qf[i], s[n], 0, 0, 0);
                }
                const int last = min(row.last, window ? q.length - 1 : q.full - 1) - key0;
                if (__ballot(last < KEYS - 1) || some_unknown) {
#pragma unroll
                    for (int n = 0; n < KB; ++n)
#pragma unroll
                        for (int v = 0; v < 16; ++v) {
                            const int key = 32 * n + 8 * (v / 4) + 4 * half + v % 4;
                            s[n][v] = key <= last && known[t & 1][key] ? s[n][v] : -__builtin_inff();
                        }
                }
                pool_weights<D, KB>(b, s, fmaxf(factor * pool_power(ek_now), 1.17549435e-38f), ev_now, b.e == kPoolNoExponent);
                const unsigned char* const vr = &v_lds[t & 1][(4 * half + (lane & 15) / 4) * VROW + (16 * (lane >> 4 & 1) + 4 * (lane & 3)) * 2];
#pragma unroll
                for (int i = 0; i < 2 * KB; ++i) {
                    const half8 p = pool_half8(s[i / 2], i % 2);
#pragma unroll
                    for (int c = 0; c < D / 32; ++c)
                        b.sums[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(pool_transposed(vr + 16 * i * VROW + 64 * c, vr + (16 * i + 8) * VROW + 64 * c), p, b.sums[c], 0, 0, 0);
                }
            }
            publish(t + 2);
        }
        b.den = pool_halves_sum(b.den);
        if (t0 == 0 && t1 == tiles) {
            char* const dst = row.there ? a.out + row.token * a.out_token + row.head * a.out_head : nullptr;
            pool_finish<D>(b, a.out_table, a.out_unscale, dst, a.bf16, lane);
        } else {
            b.put(a.chunk_parts + ((2LL * w + (at_begin ? 0 : 1)) * W + wave) * kPoolPart<D>, lane);
        }
        unit += t1 - t0;
    }
}

template <int D> pool_attention_kernel_t pick(int bits) { return bits == 8 ? srft_pool_chunk_kernel<D, 8> : srft_pool_chunk_kernel<D, 4>; }
pool_attention_kernel_t dispatch(int d, int bits) { SRFT_DISPATCH_D(d, pick, bits) }

}  // namespace

pool_attention_kernel_t srft_pick_pool_chunk(int d, int bits) { return dispatch(d, bits); }
