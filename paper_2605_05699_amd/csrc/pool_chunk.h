// pool_chunk.h -- attention over a pool for many rows a key head (a chunk of a prompt): 256 rows (tokens x query heads of the group) a workgroup.
//
// 2048 new tokens behind 14,336, 32 query heads on 8 key heads, d = 128, 4 bits: 572 to 616 us the call in a row of calls (boxes differ), 39 of
// them the transform and the merge; in the profiler, which lets no launches overlap, the scan has 588 to 678.  The two products alone, the same loop
// without softmax, decoding and reads of LDS, took 370 (the rate of a large library product, 1.4 PFLOP/s, at the power limit).  What bounds it is
// that matrix and vector instructions hardly overlap: of a SIMD's 1.11 M clocks the matrix unit is busy for 0.49 M and the vector ALU for 0.60 M, 98
// % together.  The energy of data that toggle comes on top: on zeros, the same instructions, the scan takes 500 to 513 us.  Tried on that without a
// gain: priorities (s_setprio) for either half of the wavefronts, decoding before the products in one half and behind them in the other, a softmax
// spread between the matrix instructions of the values, and rows of LDS without bank conflicts at the writes.  Each of these left the order within a
// wavefront to the fences (sched_barrier) around the matrix instructions.
//
// A tile of keys is
// decoded once for all the workgroup's rows, by all its wavefronts, into LDS (two buffers: the next tile is decoded while this one is
// used, one barrier a tile); each of the eight wavefronts (four: 946 us against 838 then) takes 32 rows through it with the scheme of pool_decode.h:
// keys on the rows of the score product, so that scores, weights and the running softmax of a row stay in one lane and its neighbour across the
// wavefront, and weights go into the second product as they are.
//
// A tile is decoded under powers of two of K's and of V's scales that all wavefronts share.  They are running: they change only where a scale
// outgrows them (kPoolRoom powers of two above what they were taken from), which a wavefront sees when its part of a tile arrives, one
// comparison; only then it tells the others, through a ring in LDS that all look into before they decode.
// Loads are straight-line, two tiles ahead of their use; a wavefront's part of a tile lies in one or two blocks of 16 keys, whose pages
// make scalar addresses, the same for K and V.  At d = 256 the registers are full: a reload of a spilled address behind loads in
// flight waited for these (119 us, then 78, for two prompts' chunks of 500 and 386 tokens among others, 8 query heads).
// Registers spilled, causal / sliding / shared form: 192 dimensions 0 / 2 / 25, 224 9 / 26 / 56, 256 36 / 51 / 90; of the shared form's at 256 ten
// are read again for every tile (causal four), at 192 none.  8 questions of 40 to 300 tokens behind 12,000 in common, 32 query heads on 8 key heads,
// the shared call and the causal one over the same tokens: d = 192, 4 bits 452 and 486 us, d = 224, 8 bits 579 and 535, d = 256 615 and 581.
#ifndef SRFT_POOL_CHUNK_H
#define SRFT_POOL_CHUNK_H
#include "pool_attention.h"

constexpr int kPoolAhead = 2;                                    // reads of LDS ahead of the matrix instructions (739 us without); 4 and 6 measure the same up to d = 128 and spill above
constexpr int kPoolRoom = 2;                                     // powers of two that scales may grow before the exponent changes

// How a workgroup goes through its blocks of rows (see there), and what is the same in all lanes then in scalar registers.  Not so in the causal form
// above 192 dimensions: in the registers that are left there its loop takes 6 % longer for it (8192 new tokens behind 8192, 2 query heads to each of
// 4: 947 -> 1010 us).
template <int D, int FORM> constexpr bool kPoolWalk = FORM != kPoolCausal || D <= 192;
template <bool WALK> __device__ __forceinline__ int pool_same(int x) { return WALK ? __builtin_amdgcn_readfirstlane(x) : x; }
template <bool WALK> __device__ __forceinline__ pool_view pool_same(pool_view v) {
    v.q.start = pool_same<WALK>(v.q.start), v.q.n_new = pool_same<WALK>(v.q.n_new), v.q.length = pool_same<WALK>(v.q.length);
    v.q.before = pool_same<WALK>(v.q.before), v.q.full = pool_same<WALK>(v.q.full);
    v.seq = pool_same<WALK>(v.seq), v.first_page = pool_same<WALK>(v.first_page), v.group = pool_same<WALK>(v.group);
    return v;
}
template <bool WALK, int FORM> __device__ __forceinline__ pool_gap<FORM> pool_same(pool_gap<FORM> g) {
    g.begin = pool_same<WALK>(g.begin), g.skip = pool_same<WALK>(g.skip), g.low = pool_same<WALK>(g.low), g.sinks = pool_same<WALK>(g.sinks);
    return g;
}

// Rows end with the matrix by way of LDS (pool_finish_together) where segments are short, in the sliding form, and registers allow it: at 192
// dimensions and more the loop spills for it.  8192 tokens, 4 query heads to each of 8, that see 64: 164 us, now 153 (d = 128), that see 1024: 300,
// now 288; d = 160, 4 heads: 127 and 118.
template <int D, int FORM> constexpr bool kPoolTogether = FORM == kPoolSliding && D <= 160;

template <int D, int BITS, int FORM>
__global__ void __launch_bounds__(64 * kPoolChunkWaves, 2) srft_pool_chunk_kernel(const pool_attention_args a) {
    constexpr int W = kPoolChunkWaves, NT = 64 * W, KEYS = kPoolChunkKeys<D>, ROWS = kPoolBlock * W, KB = KEYS / 32;
    constexpr int T = D / 16, CB = D * BITS / 8;
    constexpr int KROW = 2 * D + 16, VROW = 2 * D + 32;      // bytes of a row in LDS: 16-byte reads of 32 rows, transposed reads of 8, on different banks
    constexpr int UNITS = KEYS * T;                          // of 16 channels, of K and of V each
    constexpr int N = 2 * UNITS <= NT ? 1 : 2;               // a thread's: one of K or of V (then all of the wavefront's), or one place of both
    static_assert(UNITS % 64 == 0 && UNITS <= NT && (N == 2 || 64 * W % UNITS == 0), "whole wavefronts");
    static_assert(!kPoolTogether<D, FORM> || kPoolSlab<D> * 16 <= 2 * KEYS * KROW, "room for the end");
    typedef typename pool_codes<BITS>::type code_t;
    __shared__ __align__(16) unsigned char k_lds[2][KEYS * KROW], v_lds[2][KEYS * VROW];
    __shared__ uint4 ring[4];                                // of tile t % 4: largest scales (bits) of K, of V where they outgrew the exponents; blocks of 16
                                                             // keys whose pages do not exist

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
    const int n_seq = pool_count<FORM>(a), total = a.chunk_before[n_seq];
    const int w = srft_block_by_die();
    const pool_shares shares(total, gridDim.x, kPoolChunkLeast<FORM>);
    if (total == 0 || w >= shares.groups) return;            // (uniform)
    constexpr bool WALK = kPoolWalk<D, FORM>;
    const int end = pool_same<WALK>(shares.begin(w + 1));
    int unit = pool_same<WALK>(shares.begin(w));
    const int R = 1 << a.s.log_R, n_scales = D / a.g;

    // a thread's units: which key of the tile, which 16 channels (wavefronts beyond the last unit take units that others have too)
    const int r0 = N == 1 ? wave * 64 % UNITS : min(wave * 64, UNITS - 64), r = r0 + lane;
    const bool only_v = N == 1 && (wave * 64 / UNITS & 1) == 1;
    const auto is_v = [&](int i) __attribute__((always_inline)) { return N == 2 ? i == 1 : only_v; };
    const int u_key = r / T, u_at = r - u_key * T, u_block = r0 / T / 16;
    const bool second = u_key / 16 != u_block;               // the key is in the second block of 16 that the wavefront's units touch
    const uint32_t off_code = (u_key & 15) * CB + u_at * (int)sizeof(code_t), off_scale = 4 * ((u_key & 15) * n_scales + 16 * u_at / a.g);
    unsigned char *const k_dst = k_lds[0] + u_key * KROW + 32 * u_at, *const v_dst = v_lds[0] + u_key * VROW + 32 * u_at;    // in the first buffer

    // The block of rows that a share begins in is found by a lane each, and the next ones in their order.  (Found by counting from a key head's first
    // one every time, 8192 new tokens that see 64, 8 query heads to each of 4 of 64 channels, took 388 us, now 118; that see 1024, 4 to each of 8 of
    // 128, 394, now 291.)
    int seq = pool_sequence_of(a.chunk_before, n_seq, unit), head = 0, rt = 0, t0 = 0, blocks = 0, tiles = 0;
    pool_view view;
    const auto take = [&]() __attribute__((always_inline)) {
        view = pool_same<WALK>(pool_view_of<FORM>(a, seq));
        blocks = pool_same<WALK>((view.q.n_new * a.group + ROWS - 1) / ROWS);
    };
    const auto tiles_of = [&](int rt) __attribute__((always_inline)) { return pool_same<WALK>(pool_chunk_tiles<FORM>(a, view.q, ROWS, KEYS, rt)); };
    const auto locate = [&]() __attribute__((always_inline)) {
        take();
        const int per_head = __builtin_amdgcn_readfirstlane(pool_chunk_units<FORM>(a, view.q, ROWS, KEYS, blocks));
        const int rel = pool_same<WALK>(unit - a.chunk_before[seq]);
        head = pool_same<WALK>(rel / per_head);
        t0 = rel - head * per_head;
        rt = 0;
        if constexpr (WALK) {
            const pool_block_at at = pool_chunk_block_of<FORM>(a, view.q, ROWS, KEYS, blocks, t0);
            rt = at.rt;
            t0 -= at.before;
            tiles = tiles_of(rt);
        } else {
            tiles = tiles_of(0);
            while (t0 >= pool_chunk_cost<FORM>(tiles) && rt + 1 < blocks) {
                t0 -= pool_chunk_cost<FORM>(tiles);
                tiles = tiles_of(++rt);
            }
        }
    };
    const auto next = [&]() __attribute__((always_inline)) {                 // whether there is another (those without a tile are passed over)
        t0 = 0;
        do {
            if (++rt < blocks) continue;
            rt = 0;
            if (++head == a.heads) {
                head = 0;
                do
                    if (++seq >= n_seq) return false;
                while (pool_same<WALK>(a.chunk_before[seq + 1]) <= unit);
                take();
            }
        } while ((tiles = tiles_of(rt)) == 0);
        return true;
    };
    if constexpr (WALK) locate();
    for (bool at_begin = true;; at_begin = false) {
        if (!at_begin && unit >= end) return;
        if constexpr (WALK) {
            if (!at_begin && !next()) return;
        } else {
            while (seq + 1 < n_seq && a.chunk_before[seq + 1] <= unit) ++seq;
            locate();
        }
        const pool_seq& q = view.q;
        int t1 = min(pool_chunk_cost<FORM>(tiles), t0 + end - unit);
        if (t1 <= t0) return;                                // (only if the device arrays were written during the call)
        unit += t1 - t0;
        if constexpr (kPoolChunkStart<FORM> > 0) {           // the units in front are the start's
            t0 = max(t0 - kPoolChunkStart<FORM>, 0);
            t1 -= kPoolChunkStart<FORM>;
            if (t1 <= t0) continue;
        }
        const int seen = pool_same<WALK>(pool_chunk_seen<FORM>(a, q, ROWS, rt)), all_page_tiles = (max(min(seen, q.full), 0) + KEYS - 1) / KEYS, tail = q.length - q.full;
        const pool_gap<FORM> gap = pool_same<WALK>(pool_chunk_gap<FORM>(a, q, ROWS, KEYS, rt));
        const int page_tiles = all_page_tiles - gap.in_pages(all_page_tiles);
        pool_row row = pool_row_of(q, head, a.group, rt * ROWS + wave * kPoolBlock + l32);
        const long long q_row = (long long)row.token * (a.heads * a.group) + row.head;
        const int row_last = row.last;
        const int32_t* const table = a.s.table + view.seq * a.s.max_pages + view.first_page;
        // (the last token that any row of this wavefront sees; rows do not see less than those before them)
        int wave_last = row_last;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) wave_last = max(wave_last, __shfl_xor(wave_last, d));
        wave_last = __builtin_amdgcn_readfirstlane(wave_last);
        const int row_first = row_last - a.recent + 1;       // (sliding: the first recent token of the row, and of the wavefront's first row)
        const int wave_first = FORM == kPoolSliding ? __builtin_amdgcn_readfirstlane(row_first) : 0;

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
            if (FORM == kPoolSliding && key0 + KEYS <= wave_first && key0 >= a.sinks) return;
            floatx16 s[KB];
            const unsigned char* const kr = &k_lds[buffer][l32 * KROW + 16 * half];
            const unsigned char* const vr = &v_lds[buffer][(4 * half + (lane & 15) / 4) * VROW + (16 * (lane >> 4 & 1) + 4 * (lane & 3)) * 2];
            // Both products read their operands kPoolAhead matrix instructions ahead; the fences keep the compiler from moving the reads to their
            // uses.
            half8 f[kPoolAhead];
            const auto read_k = [&](int j) __attribute__((always_inline)) {          // of the scores' j-th: block of keys j % KB, channels from 16 (j / KB) on
                return __builtin_bit_cast(half8, *reinterpret_cast<const uint4*>(kr + 32 * (j % KB) * KROW + 32 * (j / KB)));
            };
            const auto read_v = [&](int j) __attribute__((always_inline)) {          // of the sums': channels from 32 (j % (D / 32)) on, keys from 16 (j / (D / 32)) on
                const unsigned char* const at = vr + 16 * (j / (D / 32)) * VROW + 64 * (j % (D / 32));
                return pool_transposed(at, at + 8 * VROW);
            };
#pragma unroll
            for (int j = 0; j < kPoolAhead; ++j) f[j] = read_k(j);
#pragma unroll
            for (int n = 0; n < KB; ++n) s[n] = floatx16{0};
#pragma unroll
            for (int j = 0; j < T * KB; ++j) {
                __builtin_amdgcn_sched_barrier(0);
                s[j % KB] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[j % kPoolAhead], qf[j / KB], s[j % KB], 0, 0, 0);
                if (j + kPoolAhead < T * KB) f[j % kPoolAhead] = read_k(j + kPoolAhead);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < kPoolAhead; ++j) f[j] = read_v(j);
            const int last = min(row_last, last_key) - key0;
            if (FORM == kPoolSliding && key0 <= wave_last - a.recent) {        // (a row's recent tokens begin in the tile: `last` as below)
                const int limit = last - 4 * half, from = row_first - key0 - 4 * half, sinks = a.sinks - key0 - 4 * half;
#pragma unroll
                for (int n = 0; n < KB; ++n)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const int key = 32 * n + 8 * (v / 4) + v % 4;
                        s[n][v] = key <= limit && (key >= from || key < sinks) && !(missing >> (key >> 4) & 1) ? s[n][v] : -__builtin_inff();
                    }
            } else if (__ballot(last < KEYS - 1) || missing) {
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
                b.sums[j % (D / 32)] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[j % kPoolAhead], p, b.sums[j % (D / 32)], 0, 0, 0);
                if (j + kPoolAhead < 2 * KB * (D / 32)) f[j % kPoolAhead] = read_v(j + kPoolAhead);
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
                return table[min(gap.tile(tile) * KEYS + 16 * (u_block + (lane & 1)), q.full - 16) >> a.s.log_R];
            };
            const auto fetch = [&](int tile, int pages) __attribute__((always_inline)) {
                there = 0;
                constexpr bool ONE = 64 % T == 0 && 64 / T <= 16;            // the wavefront's units lie in one block
                uint64_t at[2];
#pragma unroll
                for (int k = 0; k < (ONE ? 1 : 2); ++k) {
                    const int page = __builtin_amdgcn_readlane(pages, k), key = min(gap.tile(tile) * KEYS + 16 * (u_block + k), q.full - 16), slot = key & (R - 1);
                    const bool ok = pool_there(page, a.s.n_pages) && !gap.hides(key);    // (of the block that is read)
                    there |= (ok ? 1u : 0u) << k;
                    at[k] = ((uint64_t)((ok ? page : 0) * (uint64_t)a.heads + head) << a.s.log_R) + slot;
                }
                if (ONE) there |= there << 1;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    typedef __attribute__((address_space(1))) const char* global_t;
                    const auto load = [&](const void* base, uint64_t bytes, uint32_t off, auto* to) __attribute__((always_inline)) {
                        // a scalar address for each block (the asm keeps the compiler from adding a lane's offset to the base, a pair of registers
                        // for each array)
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
                if (k) ek = max(ek, pool_exponent<BITS>(__uint_as_float(k)) + (__uint_as_float(k) < pool_power(ek + 15 - kPoolAmp<BITS>) ? -1000 : kPoolRoom));
                if (v) ev = max(ev, pool_exponent<BITS>(__uint_as_float(v)) + (__uint_as_float(v) < pool_power(ev + 15 - kPoolAmp<BITS>) ? -1000 : kPoolRoom));
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
                compute(t & 1, gap.tile(t) * KEYS, q.full - 1, missing_now, ek_now, ev_now);
                check(t + 2);
            }
        }
        // ---- the window's tokens: rows in fp16 under a power of two each
        if (t < t1 && pool_there(a.s.windows[2 * view.seq + 1], a.s.n_windows)) {             // (uniform)
            for (; t < t1; ++t) {
                const int key0 = (gap.tile(t) - all_page_tiles) * KEYS;
                constexpr float kUp = BITS == 4 ? 4096.0f : 256.0f;          // 2^(15 - AMP): a row's values are below 2^15, not 2^AMP
                uint4 x[N][2];
                float f[N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const long long at = ((long long)((is_v(i) ? a.s.n_seq : 0) + view.seq) * a.heads + head << a.s.log_R) + min(key0 + u_key, tail - 1);
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
        if (FORM == kPoolShared && t0 == 0 && t1 == tiles && (seq >= a.s.n_seq || view.group >= 0)) {           // whole, but to be joined: by rows
            row = pool_row_of(q, head, a.group, rt * ROWS + wave * kPoolBlock + l32);
            if (row.there) {
                const int which = seq >= a.s.n_seq;
                const long long at = (long long)row.token * (a.heads * a.group) + row.head;
#pragma unroll
                for (int k = 0; k < D / 32; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<floatx4*>(a.joint_rows[which] + at * D + 8 * (4 * k + i) + 4 * half) =
                            floatx4{b.sums[k][4 * i], b.sums[k][4 * i + 1], b.sums[k][4 * i + 2], b.sums[k][4 * i + 3]};
                if (half == 0) reinterpret_cast<floatx4*>(a.joint_heads[which])[at] = b.head();
            }
        } else if (t0 == 0 && t1 == tiles) {
            int again = lane;                                // (computed again: kept, the row took registers that the loop lacks at 256 dimensions)
            asm("" : "+v"(again));
            row = pool_row_of(q, head, a.group, rt * ROWS + wave * kPoolBlock + (again & 31));
            char* const to = row.there ? a.out + row.token * a.out_token + row.head * a.out_head : nullptr;
            if constexpr (kPoolTogether<D, FORM>)
                pool_finish_together<D, NT>(b, a.out_table, a.out_unscale, to, a.bf16, tid, reinterpret_cast<uint4*>(k_lds), reinterpret_cast<uint4*>(v_lds));
            else
                pool_finish<D>(b, a.out_table, a.out_unscale, to, a.bf16, lane);
        } else if (FORM == kPoolCausal || rt * ROWS + wave * kPoolBlock < q.n_new * a.group) {     // (sums of no row: nobody reads them)
            b.put(a.chunk_parts + ((2LL * w + (at_begin ? 0 : 1)) * W + wave) * kPoolPart<D>, lane, FORM == kPoolShared && seq >= a.s.n_seq);
        }
    }
}

template <int D, int FORM> pool_attention_kernel_t pool_pick_chunk(int bits) {
    return bits == 8 ? srft_pool_chunk_kernel<D, 8, FORM> : srft_pool_chunk_kernel<D, 4, FORM>;
}

#endif  // SRFT_POOL_CHUNK_H
