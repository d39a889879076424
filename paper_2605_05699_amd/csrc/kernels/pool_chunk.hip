// Attention over a pool for many rows a key head (a chunk of a prompt): 256 rows (tokens x query heads of the group) a workgroup.
//
// 2048 new tokens behind 14,336, 32 query heads on 8 key heads, d = 128, 4 bits: 584 to 616 us the call in a row of calls (boxes differ), 39 of
// them the transform and the merge; in the profiler, which lets no launches overlap, the scan has 588 to 678.  The two products alone, the same loop
// without softmax, decoding and reads of LDS, took 370 (the rate of a large library product, 1.4 PFLOP/s, at the power limit).  What bounds it is that
// matrix and vector instructions hardly overlap: of a SIMD's 1.11 M clocks the matrix unit is busy for 0.49 M and the vector ALU for 0.60 M,
// 98 % together.  The energy of data that toggle comes on top: on zeros, the same instructions, the scan takes 500 to 513 us.
// Tried on that without a gain: priorities (s_setprio) for either half of the wavefronts, decoding before the products in one half and
// behind them in the other, a softmax spread between the matrix instructions of the values, and rows of LDS without bank conflicts at
// the writes.  Each of these left the order within a wavefront to the fences (sched_barrier) around the matrix instructions.
//
// A tile of keys is
// decoded once for all the workgroup's rows, by all its wavefronts, into LDS (two buffers: the next tile is decoded while this one is
// used, one barrier a tile); each of the eight wavefronts (four: 946 us against 838 then) takes 32 rows through it with the scheme of pool_decode.h: keys on the
// rows of the score product, so that scores, weights and the running softmax of a row stay in one lane and its neighbour across the
// wavefront, and weights go into the second product as they are.
//
// A tile is decoded under powers of two of K's and of V's scales that all wavefronts share.  They are running: they change only where a scale
// outgrows them (kRoom powers of two above what they were taken from), which a wavefront sees when its part of a tile arrives, one
// comparison; only then it tells the others, through a ring in LDS that all look into before they decode.
// Loads are straight-line, two tiles ahead of their use; a wavefront's part of a tile lies in one or two blocks of 16 keys, whose pages
// make scalar addresses, the same for K and V.  At d = 256 the registers are full: a reload of a spilled address behind loads in
// flight waited for these (119 us, now 78, for two prompts' chunks of 500 and 386 tokens among others, 8 query heads).
#include "../pool_attention.h"

namespace {

constexpr int kAhead = 2;                                    // reads of LDS ahead of the matrix instructions (739 us without); 4 and 6 measure the same up to d = 128 and spill above
constexpr int kRoom = 2;                                     // powers of two that scales may grow before the exponent changes

template <int D, int BITS>
__global__ void __launch_bounds__(64 * kPoolChunkWaves, 2) srft_pool_chunk_kernel(const pool_attention_args a) {
    constexpr int W = kPoolChunkWaves, NT = 64 * W, KEYS = kPoolChunkKeys<D>, ROWS = kPoolBlock * W, KB = KEYS / 32;
    constexpr int T = D / 16, CB = D * BITS / 8;
    constexpr int KROW = 2 * D + 16, VROW = 2 * D + 32;      // bytes of a row in LDS: 16-byte reads of 32 rows, transposed reads of 8, on different banks
    constexpr int UNITS = KEYS * T;                          // of 16 channels, of K and of V each
    constexpr int N = 2 * UNITS <= NT ? 1 : 2;               // a thread's: one of K or of V (then all of the wavefront's), or one place of both
    static_assert(UNITS % 64 == 0 && UNITS <= NT && (N == 2 || 64 * W % UNITS == 0), "whole wavefronts");
    typedef typename pool_codes<BITS>::type code_t;
    __shared__ __align__(16) unsigned char k_lds[2][KEYS * KROW], v_lds[2][KEYS * VROW];
    __shared__ uint4 ring[4];                                // of tile t % 4: largest scales (bits) of K, of V where they outgrew the exponents; blocks of 16
                                                             // keys whose pages do not exist

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
    const int total = a.chunk_before[a.s.n_seq];
    const int w = srft_block_by_die();
    const pool_shares shares(total, gridDim.x, 1);
    if (total == 0 || w >= shares.groups) return;            // (uniform)
    const int end = shares.begin(w + 1);
    int unit = shares.begin(w);
    int seq = __builtin_amdgcn_readfirstlane(pool_sequence_of(a.chunk_before, a.s.n_seq, unit));
    const int R = 1 << a.s.log_R, n_scales = D / a.g;

    // a thread's units: which key of the tile, which 16 channels (wavefronts beyond the last unit take units that others have too)
    const int r0 = N == 1 ? wave * 64 % UNITS : min(wave * 64, UNITS - 64), r = r0 + lane;
    const bool only_v = N == 1 && (wave * 64 / UNITS & 1) == 1;
    const auto is_v = [&](int i) __attribute__((always_inline)) { return N == 2 ? i == 1 : only_v; };
    const int u_key = r / T, u_at = r - u_key * T, u_block = r0 / T / 16;
    const bool second = u_key / 16 != u_block;               // the key is in the second block of 16 that the wavefront's units touch
    const uint32_t off_code = (u_key & 15) * CB + u_at * (int)sizeof(code_t), off_scale = 4 * ((u_key & 15) * n_scales + 16 * u_at / a.g);
    unsigned char *const k_dst = k_lds[0] + u_key * KROW + 32 * u_at, *const v_dst = v_lds[0] + u_key * VROW + 32 * u_at;    // in the first buffer

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
        const int seen = pool_seen(q, a.group, ROWS, rt), page_tiles = (max(min(seen, q.full), 0) + KEYS - 1) / KEYS, tail = q.length - q.full;
        pool_row row = pool_row_of(q, head, a.group, rt * ROWS + wave * kPoolBlock + l32);
        const long long q_row = (long long)row.token * (a.heads * a.group) + row.head;
        const int row_last = row.last;
        const int32_t* const table = a.s.table + seq * a.s.max_pages;
        // (the last token that any row of this wavefront sees; rows do not see less than those before them)
        int wave_last = row_last;
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
        int ek = kPoolNoExponent, ev = kPoolNoExponent;      // of the tile decoded last

        // ---- the rows of a decoded tile: buffer, its first token, the last that may count, missing blocks of 16 keys, exponents
        const auto compute = [&](int buffer, int key0, int last_key, uint32_t missing, int ek_now, int ev_now) __attribute__((always_inline)) {
            if (key0 > wave_last) return;                    // (uniform over the wavefront)
            floatx16 s[KB];
            const unsigned char* const kr = &k_lds[buffer][l32 * KROW + 16 * half];
            const unsigned char* const vr = &v_lds[buffer][(4 * half + (lane & 15) / 4) * VROW + (16 * (lane >> 4 & 1) + 4 * (lane & 3)) * 2];
            // Both products read their operands kAhead matrix instructions ahead; the fences keep the compiler from moving the reads to their uses.
            half8 f[kAhead];
            const auto read_k = [&](int j) __attribute__((always_inline)) {          // of the scores' j-th: block of keys j % KB, channels from 16 (j / KB) on
                return __builtin_bit_cast(half8, *reinterpret_cast<const uint4*>(kr + 32 * (j % KB) * KROW + 32 * (j / KB)));
            };
            const auto read_v = [&](int j) __attribute__((always_inline)) {          // of the sums': channels from 32 (j % (D / 32)) on, keys from 16 (j / (D / 32)) on
                const unsigned char* const at = vr + 16 * (j / (D / 32)) * VROW + 64 * (j % (D / 32));
                return pool_transposed(at, at + 8 * VROW);
            };
#pragma unroll
            for (int j = 0; j < kAhead; ++j) f[j] = read_k(j);
#pragma unroll
            for (int n = 0; n < KB; ++n) s[n] = floatx16{0};
#pragma unroll
            for (int j = 0; j < T * KB; ++j) {
                __builtin_amdgcn_sched_barrier(0);
                s[j % KB] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[j % kAhead], qf[j / KB], s[j % KB], 0, 0, 0);
                if (j + kAhead < T * KB) f[j % kAhead] = read_k(j + kAhead);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < kAhead; ++j) f[j] = read_v(j);
            const int last = min(row_last, last_key) - key0;
            if (__ballot(last < KEYS - 1) || missing) {
                const int limit = last - 4 * half;           // (compared with constants)
#pragma unroll
                for (int n = 0; n < KB; ++n)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const int key = 32 * n + 8 * (v / 4) + v % 4;
                        s[n][v] = key <= limit && !(missing >> (key >> 4) & 1) ? s[n][v] : -__builtin_inff();
                    }
            }
            pool_weights<D, KB>(b, s, fmaxf(factor * pool_power(ek_now), 1.17549435e-38f), ev_now, b.e == kPoolNoExponent);
            half8 p{};
#pragma unroll
            for (int j = 0; j < 2 * KB * (D / 32); ++j) {
                if (j % (D / 32) == 0) p = pool_half8(s[j / (D / 32) / 2], j / (D / 32) % 2);
                __builtin_amdgcn_sched_barrier(0);
                b.sums[j % (D / 32)] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[j % kAhead], p, b.sums[j % (D / 32)], 0, 0, 0);
                if (j + kAhead < 2 * KB * (D / 32)) f[j % kAhead] = read_v(j + kAhead);
            }
            __builtin_amdgcn_sched_barrier(0);
        };

        const int last_page_tile = min(t1, page_tiles) - 1;
        int t = t0;
        __syncthreads();                                     // (the segment before has read its last tile)
        if (tid < 4) ring[tid] = make_uint4(0, 0, 0, 0);
        if (t <= last_page_tile) {
            code_t code[N];
            typedef float pair __attribute__((ext_vector_type(2)));
            pair scale{0, 0};                                // (a native vector: an array ends up in LDS)
            uint32_t there = 0;                              // of the tile fetched last: the pages of its two blocks (bits)
            // the pages of the wavefront's blocks of 16 keys, in lanes 0 and 1; behind the last page, the last block again
            const auto pages_of = [&](int tile) __attribute__((always_inline)) {
                return table[min(tile * KEYS + 16 * (u_block + (lane & 1)), q.full - 16) >> a.s.log_R];
            };
            const auto fetch = [&](int tile, int pages) __attribute__((always_inline)) {
                there = 0;
                constexpr bool ONE = 64 % T == 0 && 64 / T <= 16;            // the wavefront's units lie in one block
                uint64_t at[2];
#pragma unroll
                for (int k = 0; k < (ONE ? 1 : 2); ++k) {
                    const int page = __builtin_amdgcn_readlane(pages, k), slot = min(tile * KEYS + 16 * (u_block + k), q.full - 16) & (R - 1);
                    const bool ok = pool_there(page, a.s.n_pages);
                    there |= (ok ? 1u : 0u) << k;
                    at[k] = ((uint64_t)((ok ? page : 0) * (uint64_t)a.heads + head) << a.s.log_R) + slot;
                }
                if (ONE) there |= there << 1;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    typedef __attribute__((address_space(1))) const char* global_t;
                    const auto load = [&](const void* base, uint64_t bytes, uint32_t off, auto* to) __attribute__((always_inline)) {
                        // a scalar address for each block (the asm keeps the compiler from adding a lane's offset to the base, a pair of registers for each array)
                        global_t p0 = (global_t)base + at[0] * bytes, p1 = p0;
                        if constexpr (!ONE) p1 = (global_t)base + at[1] * bytes;
                        asm("" : "+s"(p0));
                        if constexpr (!ONE) asm("" : "+s"(p1));
                        *to = *(__attribute__((address_space(1))) const std::remove_reference_t<decltype(*to)>*)((ONE || !second ? p0 : p1) + off);
                    };
                    float f;
                    load(is_v(i) ? (const void*)a.vb.codes_dev : a.kb.codes_dev, CB, off_code, &code[i]);
                    load(is_v(i) ? (const void*)a.vb.scales_dev : a.kb.scales_dev, 4 * n_scales, off_scale, &f);
                    scale[i] = f;
                }
            };
            // what of the fetched tile the others have to know: scales that outgrow the exponents, missing pages
            const auto check = [&](int tile) __attribute__((always_inline)) {
                const float most_k = pool_power(ek + 15 - kPoolAmp<BITS>), most_v = pool_power(ev + 15 - kPoolAmp<BITS>);
                bool news = there != 3;                      // uniform
#pragma unroll
                for (int i = 0; i < N; ++i) news |= __ballot(!(scale[i] < (is_v(i) ? most_v : most_k))) != 0;
                if (news) {
                    const bool ok = there >> (second ? 1 : 0) & 1;
                    uint32_t* const at = reinterpret_cast<uint32_t*>(&ring[tile & 3]);
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        scale[i] = ok ? scale[i] : 0.0f;
                        const float m = pool_wave_max(scale[i]);
                        if (lane == 0) atomicMax(&at[is_v(i) ? 1 : 0], __float_as_uint(m));
                    }
                    if (!ok) atomicOr(&at[2], 1u << (u_key >> 4));
                }
            };
            const auto decode = [&](int tile) __attribute__((always_inline)) {
                const float uk = pool_power(-ek), uv = pool_power(-ev);
                const int buffer = tile & 1;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    half8 x, y;
                    pool_decode16(code[i], (_Float16)(scale[i] * (is_v(i) ? uv : uk)), x, y);
                    uint4* const to = reinterpret_cast<uint4*>((is_v(i) ? v_dst : k_dst) + buffer * (is_v(i) ? KEYS * VROW : KEYS * KROW));
                    to[0] = __builtin_bit_cast(uint4, x);
                    to[1] = __builtin_bit_cast(uint4, y);
                }
            };
            // exponents for tile t, from the ring: kept unless a scale has outgrown them, else with room to grow
            uint32_t missing = 0;
            const auto look = [&](int tile) __attribute__((always_inline)) {
                const uint4 x = ring[tile & 3];
                const uint32_t k = __builtin_amdgcn_readfirstlane(x.x), v = __builtin_amdgcn_readfirstlane(x.y);
                missing = __builtin_amdgcn_readfirstlane(x.z);
                if (k) ek = max(ek, pool_exponent<BITS>(__uint_as_float(k)) + (__uint_as_float(k) < pool_power(ek + 15 - kPoolAmp<BITS>) ? -1000 : kRoom));
                if (v) ev = max(ev, pool_exponent<BITS>(__uint_as_float(v)) + (__uint_as_float(v) < pool_power(ev + 15 - kPoolAmp<BITS>) ? -1000 : kRoom));
            };
            fetch(t, pages_of(t));
            int pages = pages_of(min(t + 1, last_page_tile));
            __syncthreads();                                 // the ring is clear
            check(t);
            __syncthreads();
            look(t);
            ek = max(ek, -99 + kPoolAmp<BITS> - 14);         // (a tile of zeros)
            ev = max(ev, -99 + kPoolAmp<BITS> - 14);
            decode(t);
            fetch(min(t + 1, last_page_tile), pages);
            pages = pages_of(min(t + 2, last_page_tile));
            check(t + 1);
            for (; t <= last_page_tile; ++t) {
                __syncthreads();                             // tile t is in LDS, what tile t + 1 has to say in the ring
                const int ek_now = ek, ev_now = ev;
                const uint32_t missing_now = missing;
                if (tid == 0) ring[(t + 3) & 3] = make_uint4(0, 0, 0, 0);            // (last read before this barrier, next written behind the next one)
                look(t + 1);
                decode(t + 1);                               // (behind the last tile: that one again, which nobody reads)
                fetch(min(t + 2, last_page_tile), pages);
                pages = pages_of(min(t + 3, last_page_tile));
                compute(t & 1, t * KEYS, q.full - 1, missing_now, ek_now, ev_now);
                check(t + 2);
            }
        }
        // ---- the window's tokens: rows in fp16 under a power of two each
        if (t < t1 && pool_there(a.s.windows[2 * seq + 1], a.s.n_windows)) {             // (uniform)
            for (; t < t1; ++t) {
                const int key0 = (t - page_tiles) * KEYS;
                constexpr float kUp = BITS == 4 ? 4096.0f : 256.0f;          // 2^(15 - AMP): a row's values are below 2^15, not 2^AMP
                uint4 x[N][2];
                float f[N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const long long at = ((long long)((is_v(i) ? a.s.n_seq : 0) + seq) * a.heads + head << a.s.log_R) + min(key0 + u_key, tail - 1);
                    const uint4* const src = reinterpret_cast<const uint4*>(a.tail_rows + at * D) + 2 * u_at;
                    x[i][0] = src[0];
                    x[i][1] = src[1];
                    f[i] = a.tail_factor[at];
                }
                __syncthreads();                             // (the tile before has been read, its ring entries too)
                if (tid < 4) ring[tid] = make_uint4(0, 0, 0, 0);
                __syncthreads();
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float m = pool_wave_max(f[i] * kUp);
                    if (lane == 0) atomicMax(reinterpret_cast<uint32_t*>(&ring[0]) + (is_v(i) ? 1 : 0), __float_as_uint(m));
                }
                __syncthreads();
                ek = pool_exponent<BITS>(__uint_as_float(ring[0].x));
                ev = max(ev, pool_exponent<BITS>(__uint_as_float(ring[0].y)));
                const float uk = pool_power(-ek), uv = pool_power(-ev);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const _Float16 up = (_Float16)(f[i] * (is_v(i) ? uv : uk));
                    uint4* const to = reinterpret_cast<uint4*>(is_v(i) ? v_dst : k_dst);
                    to[0] = __builtin_bit_cast(uint4, pool_times(x[i][0], up));
                    to[1] = __builtin_bit_cast(uint4, pool_times(x[i][1], up));
                }
                __syncthreads();
                compute(0, q.full + key0, q.length - 1, 0, __builtin_amdgcn_readfirstlane(ek), __builtin_amdgcn_readfirstlane(ev));
            }
        }
        b.den = pool_halves_sum(b.den);
        if (t0 == 0 && t1 == tiles) {
            int again = lane;                                // (computed again: kept, the row took registers that the loop lacks at 256 dimensions)
            asm("" : "+v"(again));
            row = pool_row_of(q, head, a.group, rt * ROWS + wave * kPoolBlock + (again & 31));
            char* const to = row.there ? a.out + row.token * a.out_token + row.head * a.out_head : nullptr;
            pool_finish<D>(b, a.out_table, a.out_unscale, to, a.bf16, lane);
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
