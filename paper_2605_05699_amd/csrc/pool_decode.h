// pool_decode.h -- attention over a pool for few rows a key head (a decode step: the query heads of a group; a few speculated
// tokens of them): the scan over the keys, and the merge of what its workgroups leave.
//
// Bound by the chain of a tile in a wavefront, its loads, decoding and products one after the other: 24 sequences up to 32,768 tokens, 8 key heads
// of 128 channels, 4 bits: 388 MB in 112 us, 3.5 TB/s, where a kernel that only reads gets 6.2 to 6.5 (62 us).  The vector ALU is busy for 54 % of a
// SIMD's clocks (66 % of a wavefront's life), the matrix unit for 14 %; neither they nor the bytes bind alone, and two wavefronts a SIMD, which
// is what the registers leave, do not cover each other's waits.  Codes are loaded past the L2, where nobody reads them again: 6 % slower without that.  A wavefront has
// a tile of KEYS keys to itself, keys on the rows of the score product and 16 query rows on its columns (16x16x32; CB blocks of
// them): a lane holds, for ITS row (lane % 16), the keys of its quarter of the wavefront (lane / 16), which is what the running maximum
// and sum want and what the product with the values takes as its B operand.  Scores and weights stay in registers.
//   scores: one group of 32 channels a step, the codes (exact in fp16) against q' as fp16 hi + lo, and the group's scale on the result in
//           fp32: no rounding but fp32's.  (The codes themselves, not the 1024 + code that half of the decoding gives: what the offsets add up to
//           is a thousand times the queries' sum, in whose last bits a group is lost whose large queries meet small codes.)
//   values: the codes go through the wavefront's LDS to be read transposed; a weight times the scale of the key and group, under a running power
//           of two, is rounded to fp16 once.
// Loads are straight-line, one tile ahead; a tile's pages are found by 16-key blocks (a page holds at least 16 tokens), their
// numbers a tile further ahead, and turned into scalar addresses.  Four wavefronts of a workgroup take the tiles of a segment in turn,
// with no barrier until its end, where their sums meet in LDS in a fixed order.
#ifndef SRFT_POOL_DECODE_H
#define SRFT_POOL_DECODE_H
#include "pool_attention.h"
#include "rotated_queries.h"

typedef int pool_v2i __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float pool_quarters_max(float m) {
    const uint2 a = swap16(__float_as_uint(m), __float_as_uint(m));
    return other_half_max(fmaxf(__uint_as_float(a.x), __uint_as_float(a.y)));
}
__device__ __forceinline__ float pool_quarters_sum(float s) {
    const uint2 a = swap16(__float_as_uint(s), __float_as_uint(s));
    return pool_halves_sum(__uint_as_float(a.x) + __uint_as_float(a.y));
}

// ---- the end of 16 rows, by a workgroup of four wavefronts: wavefront w holds the sums of the channels 16 c .. for c = w, w + 4, ...
// (o[i], lane l: channels 16 c + 4 (l / 16) + 0 .. 3 of row l % 16).
template <int D> constexpr int kPoolOwn = (D / 16 + kPoolTeam - 1) / kPoolTeam;
template <int D> constexpr int kPoolFinishBytes = D / 32 * 2 * 64 * 16 + kPoolTeam * 16 * 4;
// lds: kPoolFinishBytes<D>, free before and after a barrier of the caller's.  dst: the lane's row or null.  AHEAD: the matrix is asked for before
// it is needed (6.6 -> 5.8 us for the merge of 24 sequences; the scan's registers do not hold it).
template <int D, bool AHEAD>
__device__ __forceinline__ void pool_finish16(const floatx4 (&o)[kPoolOwn<D>], float den, int e2, unsigned char* lds, const uint4* __restrict__ table,
                                              float unscale, char* dst, int bf16, int wave, int lane) {
    uint2* const ops = reinterpret_cast<uint2*>(lds);        // [k-step][hi, lo][lane][half of 8]
    float* const tops = reinterpret_cast<float*>(lds + D / 32 * 2 * 64 * 16);
    const int l16 = lane & 15, a = lane >> 4;
    u32x4 ah[D / 32], al[D / 32];                            // of the matrix, where a block of 16 outputs is read ahead
    const auto fetch = [&](int n) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            ah[s] = reinterpret_cast<const u32x4*>(table)[((n * (D / 32) + s) * 2 + 0) * 64 + lane];
            al[s] = reinterpret_cast<const u32x4*>(table)[((n * (D / 32) + s) * 2 + 1) * 64 + lane];
        }
    };
    if constexpr (AHEAD) fetch(min(wave, D / 16 - 1));
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < kPoolOwn<D>; ++i)
        if (wave + kPoolTeam * i < D / 16)
#pragma unroll
            for (int k = 0; k < 4; ++k) m = fmaxf(m, fabsf(o[i][k]));
    m = pool_quarters_max(m);
    if (a == 0) tops[wave * 16 + l16] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kPoolTeam; ++w) m = fmaxf(m, tops[w * 16 + l16]);
    const int e = max((int)((__float_as_uint(m) >> 23) & 0xFF) - 127, -100);
    const float up = pool_power(14 - e), down = (den > 0.0f ? 1.0f / den : 0.0f) * unscale, p0 = pool_power(e - 14), p1 = pool_power(e2);
#pragma unroll
    for (int i = 0; i < kPoolOwn<D>; ++i) {
        const int c = wave + kPoolTeam * i;
        if (c < D / 16) {                                    // uniform
            uint32_t hi[2], lo[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float x = o[i][2 * k] * up, y = o[i][2 * k + 1] * up;
                const half2v h = {(_Float16)x, (_Float16)y}, l = {(_Float16)(x - (float)h[0]), (_Float16)(y - (float)h[1])};
                hi[k] = __builtin_bit_cast(uint32_t, h);
                lo[k] = __builtin_bit_cast(uint32_t, l);
            }
            ops[((c / 2 * 2 + 0) * 64 + lane) * 2 + c % 2] = make_uint2(hi[0], hi[1]);
            ops[((c / 2 * 2 + 1) * 64 + lane) * 2 + c % 2] = make_uint2(lo[0], lo[1]);
        }
    }
    __syncthreads();
    for (int n = wave; n < D / 16; n += kPoolTeam) {
        floatx4 acc{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            half8 h, l;
            if constexpr (AHEAD) {
                h = __builtin_bit_cast(half8, ah[s]);
                l = __builtin_bit_cast(half8, al[s]);
            } else {
                h = __builtin_bit_cast(half8, table[((n * (D / 32) + s) * 2 + 0) * 64 + lane]);
                l = __builtin_bit_cast(half8, table[((n * (D / 32) + s) * 2 + 1) * 64 + lane]);
            }
            const half8 bh = __builtin_bit_cast(half8, reinterpret_cast<const uint4*>(ops)[(s * 2 + 0) * 64 + lane]);
            const half8 bl = __builtin_bit_cast(half8, reinterpret_cast<const uint4*>(ops)[(s * 2 + 1) * 64 + lane]);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(h, bh, acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(l, bh, acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(h, bl, acc, 0, 0, 0);
        }
        if constexpr (AHEAD) fetch(min(n + kPoolTeam, D / 16 - 1));
        if (dst) {
            uint32_t r[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float x = acc[2 * k] * down * p0 * p1, y = acc[2 * k + 1] * down * p0 * p1;
                typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
                r[k] = bf16 ? __builtin_bit_cast(uint32_t, bf2{(__bf16)x, (__bf16)y}) : pack_half2(x, y);
            }
            *reinterpret_cast<uint2*>(dst + 2 * (16 * n + 4 * a)) = make_uint2(r[0], r[1]);
        }
    }
}

// Sums of 16 rows that a segment leaves: [D / 16][64 lanes] float4, then per lane maximum, sum of weights, V's exponent.
template <int D> constexpr int kPoolPart16 = 16 * D + 3 * 64;

// D, BITS: of the plans.  CB: blocks of 16 rows.  GM: groups of 16, of 32, or of more channels (kGroupWide).
template <int D, int BITS, int CB, int GM>
struct pool_decode {
    static constexpr bool FINE = GM == kGroup16;
    static constexpr int G = D / 32, NS = FINE ? 2 * G : G;  // runs of 32 channels; columns of scales
    static constexpr int KEYS = pool_decode_keys(D, CB), KQ = KEYS / 4, BK = KEYS / 16, W = kPoolTeam;
    static constexpr int CBY = D * BITS / 8, P = CBY / 16;   // bytes of a row of codes, 16-byte pieces of it
    static constexpr int NV = (P * KEYS + 63) / 64;          // a lane's pieces of a tile of codes
    static constexpr int NH = KEYS == 64 ? NS : (NS + 1) / 2;                        // a lane's columns of scales
    static constexpr int ROW = CBY + 16;                     // of codes in LDS, padded: 16 rows on different banks
    static constexpr int VTILE = KEYS * ROW + 4 * 8;         // (and the values' quarters apart)
    static constexpr int WAVE_BYTES = VTILE + 2 * NS * KEYS * 4;
    static constexpr int MEET = 8;                           // blocks of 16 channels that meet at a time
    static constexpr int MEET_BYTES = W * (MEET * 64 * 16 + 3 * 64 * 4);
    static constexpr int LDS = std::max(W * WAVE_BYTES, std::max(MEET_BYTES, kPoolFinishBytes<D>));
    typedef std::conditional_t<BITS == 4, uint32_t, uint2> unit_t;                   // eight codes
    static __device__ __forceinline__ half8 eight(uint32_t c) { return __builtin_bit_cast(half8, decode8(c)); }
    static __device__ __forceinline__ half8 eight(uint2 c) {
        const uint2 x = decode4_bytes(c.x), y = decode4_bytes(c.y);
        return __builtin_bit_cast(half8, make_uint4(x.x, x.y, y.x, y.y));
    }
    // which of a quarter's eight keys of a step is element e of an operand of decoded codes
    static constexpr int key_of(int e) { return BITS == 4 ? e / 2 + 4 * (e % 2) : (e & 4) + ((e & 1) << 1) + ((e & 2) >> 1); }
};

template <int N> using pool_floats = float __attribute__((ext_vector_type(N), aligned(4)));     // (native vectors: arrays of classes end up in memory)

// weight times scale, rounded once to fp16: two of them.  They go straight into a matrix instruction and are therefore written for the compiler: it
// has to wait two states between a vector instruction and a matrix instruction that reads its result, which it does not do behind inline
// asm.  (As asm, the scan for two blocks of rows at d = 32, 4 bits and groups of 16 had a weight written one state before its product, and gave
// wrong rows.)
__device__ __forceinline__ uint32_t pool_product2(float a, float f, float b, float g) {
    const half2v r = {(_Float16)__builtin_fmaf(a, f, 0.0f), (_Float16)__builtin_fmaf(b, g, 0.0f)};       // v_fma_mixlo_f16, v_fma_mixhi_f16
    return __builtin_bit_cast(uint32_t, r);
}

// Wavefronts per SIMD asked of the compiler.  Two fit (LDS, and 256 registers each).  Asked for one it fills the latencies with what registers there
// are, and mostly ends at 256 or below, so that two fit all the same; that is the faster form then (24 sequences up to 32,768 tokens, 8 rows a key
// head, 4 bits, the whole call, asked for one / two, us: d = 64 84 / 89, 128 123 / 132, 256 212 / 237; 192 at 8 bits 215 / 221).  Where it ends
// above, one wavefront is left, and asking for two is faster as long as that spills no more than some 40 registers.  Formats that do, groups of
// 16, 32 and d: 8 bits, d = 96 in groups of 16 199 / 156; d = 128 248 / 193, 183 / 161, 180 / 159; d = 192 with one group 260 / 225;
// d = 224 418 / 328, 335 / 278, 320 / 276; d = 256 472 / 380, 371 / 311, 359 / 309; 4 bits, d = 224 with one group 293 / 227.  With two blocks
// of rows (24 rows a key head): 8 bits, d = 96 in groups of 16 289 / 211, d = 128 in groups of 32 280 / 211, with one 279 / 212; 4 bits, the same three
// 282 / 196, 274 / 187, 275 / 187.  Beyond 40: d = 128 in groups of 16, two blocks, at 4 bits (87 spilled) 332 / 414, at 8 (120) 361 / 566.
// (All formats: profiles/pool_decode_registers.txt.)
constexpr int pool_decode_waves(int d, int bits, int cb, int gm) {
    if (cb == 2) return d == (gm == kGroup16 ? 96 : 128) ? 2 : 1;
    if (bits == 4) return d == 224 && gm == kGroupWide ? 2 : 1;
    return d == 128 || d >= 224 || (d == 96 && gm == kGroup16) || (d == 192 && gm == kGroupWide) ? 2 : 1;
}
// Whether a segment's first tile is asked for before its queries are in LDS (4 bits, groups of 32, with / without: d = 64 84 / 85, 96 104 / 107,
// 160 147 / 148).  Not where the registers are full: at d = 128 one wavefront is left with it (149 / 123), nor above 160 (256: 209 -> 291 when it was tried).
constexpr bool pool_decode_early(int d, int bits, int cb, int gm) { return pool_decode_waves(d, bits, cb, gm) == 1 && d <= 160 && d != 128; }
template <int D, int BITS, int CB, int GM>
__global__ void __launch_bounds__(64 * kPoolTeam, pool_decode_waves(D, BITS, CB, GM)) srft_pool_decode_kernel(const pool_attention_args a) {
    using P = pool_decode<D, BITS, CB, GM>;
    constexpr bool FINE = P::FINE;
    constexpr int G = P::G, NS = P::NS, KEYS = P::KEYS, KQ = P::KQ, BK = P::BK, W = P::W, CBY = P::CBY, NV = P::NV, NH = P::NH, NB = D / 16;
    typedef typename P::unit_t unit_t;
    __shared__ __align__(16) unsigned char lds[P::LDS];
    __shared__ uint4 qs[CB * G * 2 * 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, quarter = lane >> 4;
    // The first segment's sequence: where the sequences fit the lanes, all that it takes comes with one round of loads (a step of 4
    // sequences up to 1000 tokens: 12.6 us with this and with the first tile's loads before the queries are in LDS, 13.5 to 14 one after the other).
    const int n_seq = a.s.n_seq;
    const bool few = n_seq < 64;
    int of_before = 0, of_start = 0, of_length = 0;          // lane b: of sequence b
    if (few) {
        of_before = a.decode_before[min(lane, n_seq)];
        of_start = a.s.starts[min(lane, n_seq)];
        of_length = a.s.lengths[min(lane, n_seq - 1)];
    }
    const int total = few ? __builtin_amdgcn_readlane(of_before, n_seq) : a.decode_before[n_seq];
    const int w = srft_block_by_die();
    const pool_shares shares(total, gridDim.x, W);
    if (total == 0 || w >= shares.groups) return;            // (uniform)
    const int end = shares.begin(w + 1);
    int unit = shares.begin(w), seq, units_before;
    pool_seq q;
    if (few) {
        seq = min((int)__popcll(__ballot(lane <= n_seq && of_before <= unit)) - 1, n_seq - 1);
        units_before = __builtin_amdgcn_readlane(of_before, seq);
        q = pool_seq_from(a.s, __builtin_amdgcn_readlane(of_start, seq), __builtin_amdgcn_readlane(of_start, seq + 1), __builtin_amdgcn_readlane(of_length, seq));
    } else {
        seq = __builtin_amdgcn_readfirstlane(pool_sequence_of(a.decode_before, n_seq, unit));
        units_before = a.decode_before[seq];
        q = pool_seq_of(a.s, seq);
    }
    const int R = 1 << a.s.log_R, n_scales = D / a.g;
    unsigned char* const kt = lds + wave * P::WAVE_BYTES;    // this wavefront's keys, and then values, and scales
    unsigned char* const vt = kt;
    float* const ks = reinterpret_cast<float*>(vt + P::VTILE);               // [column][key]
    float* const vs = ks + NS * KEYS;
    const auto v_at = [&](int row) __attribute__((always_inline)) { return vt + row * P::ROW + (row / KQ) * 8; };
    // Which key of the tile is row l16 of block b of the score product: KQ (l16 / 4) + 4 b + l16 % 4, so that result register i of quarter q is
    // key KQ q + 4 b + i.  Neighbouring lanes load neighbouring pieces of rows (64 bytes of four lanes are one access; a lane's own row, read
    // as the operand wants it, was 1024 accesses of 4 bytes a tile, and they, not the bytes, took 130 of 160 us over 390 MB); keys and
    // values go through LDS, one after the other in the same place.
    const unsigned char* const k_src = kt + (KQ * (l16 >> 2) + (l16 & 3)) * P::ROW + quarter * BITS;
    int piece_off[NV], piece_block[NV];                      // of piece i: offset in the bytes of its block of 16 keys, which block
    unsigned char *k_dst[NV], *v_dst[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int u = P::P * KEYS % 64 == 0 ? lane + 64 * i : min(lane + 64 * i, P::P * KEYS - 1), row = u / P::P, piece = u - row * P::P;
        piece_block[i] = P::P == 4 ? i : row >> 4;
        piece_off[i] = (row & 15) * CBY + 16 * piece;
        k_dst[i] = kt + row * P::ROW + 16 * piece;
        v_dst[i] = v_at(row) + 16 * piece;
    }
    const int s_key = lane & (KEYS - 1), s_first = min(KEYS == 64 ? 0 : lane / 32 * NH, NS - NH);      // a lane's scales: of this key, these columns
    const int s_skip = GM == kGroupWide ? 0 : 4 * s_first;     // bytes behind the row's first scale
    for (bool at_begin = true; unit < end; at_begin = false) {
        if (!at_begin) {
            while (seq + 1 < n_seq && a.decode_before[seq + 1] <= unit) ++seq;
            units_before = a.decode_before[seq];
            q = pool_seq_of(a.s, seq);
        }
        const int tiles = pool_tiles(q.length, q.full, KEYS), page_tiles = (q.full + KEYS - 1) / KEYS, tail = q.length - q.full;
        const int rel = unit - units_before, item = rel / tiles, t0 = rel - item * tiles, t1 = min(tiles, t0 + end - unit);
        const int blocks_of_rows = (q.n_new * a.group + 16 * CB - 1) / (16 * CB), head = item / blocks_of_rows, r0 = 16 * CB * (item - head * blocks_of_rows);
        if (t1 <= t0) return;                                // (only if the device arrays were written during the call)
        const int32_t* const table = a.s.table + seq * a.s.max_pages;
        const int last_page_tile = min(t1, page_tiles) - 1;
        int t = t0 + wave;
        u32x4 kc[NV], vc[NV];
        pool_floats<NH> kf, vf;
        // pages of the tile's blocks of 16 keys (lane i: block i % (KEYS / 16)); behind the last page, the last block again
        const auto page_of = [&](int tile) __attribute__((always_inline)) {
            return table[min(tile * KEYS + 16 * (lane & (KEYS / 16 - 1)), q.full - 16) >> a.s.log_R];
        };
        uint32_t there = 0;
        uint64_t c0 = 0, c1 = 0, c2 = 0, c3 = 0;         // blocks' codes
        const auto code_of = [&](int block) __attribute__((always_inline)) {
            uint64_t r = block & 1 ? c1 : c0;
            if constexpr (KEYS == 64) r = block & 2 ? block & 1 ? c3 : c2 : r;
            return r;
        };
        const auto fetch_values = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < NV; ++i) vc[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.vb.codes_dev + (code_of(piece_block[i]) + piece_off[i])));
        };
        const auto fetch = [&](int tile, int pages) __attribute__((always_inline)) {
            // Blocks' addresses in scalar registers: in bytes of codes, and of scales.  (The empty asm keeps the choice between them a
            // choice of registers: the compiler makes branches of it otherwise.)
            uint32_t known = 0;
            uint64_t f0, f1, f2 = 0, f3 = 0;
            const auto address = [&](int i, uint64_t& code, uint64_t& scale) __attribute__((always_inline)) {
                const int page = __builtin_amdgcn_readlane(pages, i), slot = min(tile * KEYS + 16 * i, q.full - 16) & (R - 1);
                const bool ok = pool_there(page, a.s.n_pages);
                known |= (ok ? 1u : 0u) << i;
                const uint64_t row = ((uint64_t)((ok ? page : 0) * (uint64_t)a.heads + head) << a.s.log_R) + slot;
                code = row * CBY;
                scale = row * (4 * n_scales);
                asm("" : "+s"(code), "+s"(scale));
            };
            address(0, c0, f0);
            address(1, c1, f1);
            if constexpr (KEYS == 64) {
                address(2, c2, f2);
                address(3, c3, f3);
            }
            there = known;
            uint64_t f = s_key & 16 ? f1 : f0;
            if constexpr (KEYS == 64) f = s_key & 32 ? s_key & 16 ? f3 : f2 : f;
            const uint64_t s_at = f + (s_key & 15) * (4 * n_scales) + s_skip;
            const char *const sk = (const char*)a.kb.scales_dev + s_at, *const sv = (const char*)a.vb.scales_dev + s_at;
            if constexpr (GM == kGroupWide) {
#pragma unroll
                for (int i = 0; i < NH; ++i) {           // (the offset is uniform but for the half of the wavefront)
                    const int at = (s_first + i) * 32 / a.g;
                    kf[i] = reinterpret_cast<const float*>(sk)[at];
                    vf[i] = reinterpret_cast<const float*>(sv)[at];
                }
            } else {
                kf = *reinterpret_cast<const pool_floats<NH>*>(sk);
                vf = *reinterpret_cast<const pool_floats<NH>*>(sv);
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) kc[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.kb.codes_dev + (code_of(piece_block[i]) + piece_off[i])));
        };
        constexpr bool EARLY = pool_decode_early(D, BITS, CB, GM);
        // the first tile: its pages, then the queries, then its codes are on their way
        int pages = 0;
        if (EARLY && t <= last_page_tile) pages = page_of(t);
        pool_row row[CB];
        float factor[CB];
        constexpr int NQ = (2 * G + W - 1) / W;
        u32x4 x[CB][NQ];
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            row[c] = pool_row_of(q, head, a.group, r0 + 16 * c + l16);
            const long long q_row = (long long)row[c].token * (a.heads * a.group) + row[c].head;
            factor[c] = fmaxf(a.q_factor[q_row], 1.17549435e-38f);
#pragma unroll
            for (int i = 0; i < NQ; ++i) {                   // (hi and lo of run j / 2)
                const int j = min(wave + W * i, 2 * G - 1);
                x[c][i] = reinterpret_cast<const u32x4*>((j % 2 ? a.q_rows_low : a.q_rows) + q_row * D)[4 * (j / 2) + quarter];
            }
        }
        if (EARLY && t <= last_page_tile) {
            fetch(t, pages);
            pages = page_of(min(t + W, last_page_tile));
        }
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                qs[(c * G * 2 + min(wave + W * i, 2 * G - 1)) * 64 + lane] = __builtin_bit_cast(uint4, x[c][i]);     // (past the last, the last again)
            }
        __syncthreads();
        floatx4 acc[CB][NB];
        float top[CB], den[CB];
        int e_now = kPoolNoExponent;
#pragma unroll
        for (int c = 0; c < CB; ++c) {
#pragma unroll
            for (int n = 0; n < NB; ++n) acc[c][n] = floatx4{0, 0, 0, 0};
            top[c] = kPoolLowest;
            den[c] = 0.0f;
        }
        float p[CB][BK][4];                                  // scores, then weights: keys KQ quarter + 4 b + i of row l16
        // ---- scores -> weights under top (see pool_weights); key_of(b, i): which key of the tile p[.][b][i] is, counted from first_key
        const auto weights = [&](auto key_of, int first_key, int last_key, uint32_t blocks, int e, bool first) __attribute__((always_inline)) {
            const int e_new = max(e_now, e);                 // (uniform)
            bool changed = e_new != e_now;
            float m[CB], down[CB];
#pragma unroll
            for (int c = 0; c < CB; ++c) {
                const int last = min(row[c].last, last_key) - first_key;
                if (__ballot(last < KEYS - 1) || blocks != (1u << (KEYS / 16)) - 1) {
#pragma unroll
                    for (int b = 0; b < BK; ++b)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int key = key_of(b, i);
                            p[c][b][i] = key <= last && (blocks >> (key >> 4) & 1) ? p[c][b][i] : -__builtin_inff();
                        }
                }
                m[c] = p[c][0][0];
#pragma unroll
                for (int v = 1; v < 4 * BK; ++v) m[c] = fmaxf(m[c], p[c][v / 4][v % 4]);
                m[c] = fmaxf(pool_quarters_max(m[c]) * factor[c], kPoolLowest);
                changed |= __ballot(m[c] > top[c] + kLazy) != 0;
            }
            if (changed) {                                   // uniform
#pragma unroll
                for (int c = 0; c < CB; ++c) {
                    const float t = m[c] > top[c] + kLazy ? m[c] : top[c];
                    down[c] = __builtin_amdgcn_exp2f(top[c] - t);
                    top[c] = t;
                    den[c] *= down[c];
                    const float f = down[c] * pool_power(e_now - e_new);
                    if (!first)
#pragma unroll
                        for (int n = 0; n < NB; ++n) acc[c][n] *= f;
                }
                e_now = e_new;
            }
#pragma unroll
            for (int c = 0; c < CB; ++c)
#pragma unroll
                for (int v = 0; v < 4 * BK; ++v) {
                    float& x = p[c][v / 4][v % 4];
                    x = __builtin_amdgcn_exp2f(fmaf(x, factor[c], -top[c]));
                    den[c] += x;
                }
        };

        bool first = true;
        if (t <= last_page_tile) {
            if constexpr (!EARLY) {
                fetch(t, page_of(t));
                pages = page_of(min(t + W, last_page_tile));
            }
            fetch_values();
            for (; t <= last_page_tile; t += W) {
                // ---- scales and keys to LDS (of one wavefront: its accesses complete in program order)
                const uint32_t blocks = there;
                const bool mine = blocks >> (s_key >> 4) & 1;
                float most = 0.0f;
#pragma unroll
                for (int i = 0; i < NH; ++i) {
                    vf[i] = mine ? vf[i] : 0.0f;
                    most = fmaxf(most, vf[i]);
                }
                const int e = max(e_now, max((int)((__builtin_amdgcn_readfirstlane(__float_as_uint(pool_wave_max(most))) >> 23) & 0xFF) - 127, -99) - 6);
                const float up = pool_power(-e);             // the largest scale is 2^6 .. 2^7 then, a weight at most 2^kLazy
#pragma unroll
                for (int i = 0; i < NH; ++i) {
                    ks[(s_first + i) * KEYS + s_key] = kf[i];
                    vs[(s_first + i) * KEYS + s_key] = vf[i] * up;
                }
#pragma unroll
                for (int i = 0; i < NV; ++i) *reinterpret_cast<u32x4*>(k_dst[i]) = kc[i];
                // the next tile's loads (past the end the last one again): keys and scales here, values when these have gone to LDS
                fetch(min(t + W, last_page_tile), pages);
                pages = page_of(min(t + 2 * W, last_page_tile));
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                // ---- scores
#pragma unroll
                for (int j = 0; j < G; ++j) {
#pragma unroll
                    for (int half = 0; half < (FINE ? 2 : 1); ++half) {
                        const int column = FINE ? 2 * j + half : j;
#pragma unroll
                        for (int b = 0; b < BK; ++b) {
                            const unit_t codes = *reinterpret_cast<const unit_t*>(k_src + 4 * b * P::ROW + 4 * BITS * j);
                            half8 k = P::eight(codes);
                            if constexpr (FINE) {            // (the other group's half of the step: zeros)
                                const uint4 z = make_uint4(0, 0, 0, 0);
                                k = quarter >> 1 == half ? k : __builtin_bit_cast(half8, z);
                            }
                            const float4 f = *reinterpret_cast<const float4*>(&ks[column * KEYS + KQ * quarter + 4 * b]);
                            const float fv[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
                            for (int c = 0; c < CB; ++c) {
                                floatx4 s = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, __builtin_bit_cast(half8, qs[((c * G + j) * 2 + 0) * 64 + lane]), floatx4{0, 0, 0, 0}, 0, 0, 0);
                                s = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, __builtin_bit_cast(half8, qs[((c * G + j) * 2 + 1) * 64 + lane]), s, 0, 0, 0);
#pragma unroll
                                for (int i = 0; i < 4; ++i) p[c][b][i] = column == 0 ? s[i] * fv[i] : fmaf(s[i], fv[i], p[c][b][i]);
                            }
                        }
                    }
                    if (j % 2 || CB > 1) __builtin_amdgcn_sched_barrier(0);        // two groups' operands at a time (registers)
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    reinterpret_cast<uint2*>(v_dst[i])[0] = make_uint2(vc[i][0], vc[i][1]);          // (8-byte aligned)
                    reinterpret_cast<uint2*>(v_dst[i])[1] = make_uint2(vc[i][2], vc[i][3]);
                }
                fetch_values();
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_sched_barrier(0);           // (the values' operands are formed as they are used, not all ahead)
                weights([&](int b, int i) { return KQ * quarter + 4 * b + i; }, t * KEYS, q.full - 1, blocks, e, first);
                first = false;
                // ---- values: channels on the rows; step s takes keys 8 s .. 8 s + 7 of every quarter, in the order of decoded codes
#pragma unroll
                for (int column = 0; column < NS; ++column) {
                    half8 pw[CB][BK / 2];
#pragma unroll
                    for (int s = 0; s < BK / 2; ++s) {
                        const float4 f0 = *reinterpret_cast<const float4*>(&vs[column * KEYS + KQ * quarter + 8 * s]);
                        const float4 f1 = *reinterpret_cast<const float4*>(&vs[column * KEYS + KQ * quarter + 8 * s + 4]);
                        const float fv[8] = {f0.x, f0.y, f0.z, f0.w, f1.x, f1.y, f1.z, f1.w};
#pragma unroll
                        for (int c = 0; c < CB; ++c)
{
                            const auto two = [&](int x) __attribute__((always_inline)) {
                                const int y = P::key_of(x), z = P::key_of(x + 1);
                                return pool_product2(p[c][2 * s + y / 4][y % 4], fv[y], p[c][2 * s + z / 4][z % 4], fv[z]);
                            };
                            pw[c][s] = __builtin_bit_cast(half8, make_uint4(two(0), two(2), two(4), two(6)));
                        }
                    }
#pragma unroll
                    for (int h = 0; h < 32 / (FINE ? 32 : 16); ++h) {
                        const int n = FINE ? column : 2 * column + h;                    // block of 16 channels
                        half8 vd[BK / 2];
                        if constexpr (BITS == 4) {
                            const pool_v2i r = __builtin_amdgcn_ds_read_tr4_b64_v2i32(
                                (__attribute__((address_space(3))) pool_v2i*)(v_at(KQ * quarter + (l16 & (KQ - 1))) + 8 * n));
#pragma unroll
                            for (int s = 0; s < BK / 2; ++s) vd[s] = P::eight((uint32_t)r[s]);
                        } else {
#pragma unroll
                            for (int s = 0; s < BK / 2; ++s) {
                                const pool_v2i r = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                                    (__attribute__((address_space(3))) pool_v2i*)(v_at(KQ * quarter + 8 * s + l16 / 2) + 16 * n + 8 * (l16 & 1)));
                                if constexpr (BITS == 8) vd[s] = P::eight(make_uint2((uint32_t)r[0], (uint32_t)r[1]));
                            }
                        }
#pragma unroll
                        for (int c = 0; c < CB; ++c)
#pragma unroll
                            for (int s = 0; s < BK / 2; ++s) acc[c][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vd[s], pw[c][s], acc[c][n], 0, 0, 0);
                    }
                    if (column % 2 || CB > 1) __builtin_amdgcn_sched_barrier(0);
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            }
        }
        // ---- the window's tokens: rows in fp16 under a power of two each, the values' rows transposed.  Block b is the tokens 16 b .. 16 b + 15
        // of the tile here; those behind the last token are passed over.  Loads are unconditional (behind the last token, of it
        // again: its weights there are zero), so that a block's are on their way together.
        for (; t < t1; t += W) {
            if (!pool_there(a.s.windows[2 * seq + 1], a.s.n_windows)) break;             // (uniform)
            const int key0 = (t - page_tiles) * KEYS, held = tail - key0;                // slot of the tile's first token; tokens from there on
            const long long of_k = (long long)(seq * a.heads + head) << a.s.log_R, of_v = of_k + ((long long)a.s.n_seq * a.heads << a.s.log_R);
            float fv[BK][4], most = 0.0f;
#pragma unroll
            for (int b = 0; b < BK; ++b) {
                if (16 * b < held) {                         // uniform
                    u32x4 kr[G];
                    float fk[4];
                    const int slot = min(key0 + 16 * b + l16, tail - 1);
#pragma unroll
                    for (int j = 0; j < G; ++j) kr[j] = reinterpret_cast<const u32x4*>(a.tail_rows + (of_k + slot) * D)[4 * j + quarter];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = min(key0 + 16 * b + 4 * quarter + i, tail - 1);
                        fk[i] = a.tail_factor[of_k + key];
                        fv[b][i] = a.tail_factor[of_v + key];
                        most = fmaxf(most, fv[b][i]);
                    }
#pragma unroll
                    for (int c = 0; c < CB; ++c) {
                        floatx4 s{0, 0, 0, 0};
#pragma unroll
                        for (int j = 0; j < G; ++j) {
                            const half8 k = __builtin_bit_cast(half8, kr[j]);
                            s = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, __builtin_bit_cast(half8, qs[((c * G + j) * 2 + 0) * 64 + lane]), s, 0, 0, 0);
                            s = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, __builtin_bit_cast(half8, qs[((c * G + j) * 2 + 1) * 64 + lane]), s, 0, 0, 0);
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) p[c][b][i] = s[i] * fk[i];
                    }
                } else {                                     // (masked: keys behind the last)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        fv[b][i] = 0.0f;
#pragma unroll
                        for (int c = 0; c < CB; ++c) p[c][b][i] = 0.0f;
                    }
                }
            }
            // (a row's values are below 2^15: the sums of a few of them stay far inside fp32)
            const int e = max(e_now, max((int)((__builtin_amdgcn_readfirstlane(__float_as_uint(pool_wave_max(most))) >> 23) & 0xFF) - 127, -99) - 6);
            const float up = pool_power(-e);
            weights([&](int b, int i) { return 16 * b + 4 * quarter + i; }, q.full + key0, q.length - 1, (1u << (KEYS / 16)) - 1, e, first);
            first = false;
#pragma unroll
            for (int s = 0; s < BK / 2; ++s) {
                if (32 * s >= held) continue;                // uniform
                half8 pw[CB];
#pragma unroll
                for (int c = 0; c < CB; ++c)
#pragma unroll
                    for (int x = 0; x < 8; ++x) pw[c][x] = (_Float16)(p[c][2 * s + x / 4][x % 4] * (fv[2 * s + x / 4][x % 4] * up));
                // four tokens each of two blocks, next to each other in [channel][R]; past the last token, those that hold it
                const int slot0 = min(key0 + 32 * s + 4 * quarter, (tail - 1) & ~3), slot1 = min(key0 + 32 * s + 16 + 4 * quarter, (tail - 1) & ~3);
                const unsigned short* const at = a.tail_columns + (((long long)seq * a.heads + head) * D + l16 << a.s.log_R);
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    const uint2 x = *reinterpret_cast<const uint2*>(at + (16 * n << a.s.log_R) + slot0), y = *reinterpret_cast<const uint2*>(at + (16 * n << a.s.log_R) + slot1);
                    const half8 vd = __builtin_bit_cast(half8, make_uint4(x.x, x.y, y.x, y.y));
#pragma unroll
                    for (int c = 0; c < CB; ++c) acc[c][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vd, pw[c], acc[c][n], 0, 0, 0);
                }
            }
        }
        // ---- the wavefronts' sums meet: wavefront w adds up the channels 16 c .. of c = w, w + 4, ...
        const bool whole = t0 == 0 && t1 == tiles;
        float* const meet = reinterpret_cast<float*>(lds);   // [wavefront][maximum, sum, exponent][64], then [wavefront][MEET][64] float4
        floatx4* const sums = reinterpret_cast<floatx4*>(lds + W * 3 * 64 * 4);
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            __syncthreads();                                 // (the tiles, the sums before)
            const float d = pool_quarters_sum(den[c]);
            meet[(wave * 3 + 0) * 64 + lane] = top[c];
            meet[(wave * 3 + 1) * 64 + lane] = d;
            meet[(wave * 3 + 2) * 64 + lane] = __uint_as_float((uint32_t)e_now);
            floatx4 mine[kPoolOwn<D>];
            float f[W], t_all = kPoolLowest, d_all = 0.0f;
            int e_all = kPoolNoExponent;
#pragma unroll
            for (int part = 0; part < (NB + P::MEET - 1) / P::MEET; ++part) {
                if (part > 0) __syncthreads();
#pragma unroll
                for (int n = 0; n < P::MEET; ++n)
                    if (part * P::MEET + n < NB) sums[(wave * P::MEET + n) * 64 + lane] = acc[c][part * P::MEET + n < NB ? part * P::MEET + n : 0];
                __syncthreads();
                if (part == 0) {
#pragma unroll
                    for (int k = 0; k < W; ++k) {
                        t_all = fmaxf(t_all, meet[(k * 3 + 0) * 64 + lane]);
                        e_all = max(e_all, (int)__float_as_uint(meet[(k * 3 + 2) * 64 + lane]));
                    }
#pragma unroll
                    for (int k = 0; k < W; ++k) {
                        const float g = __builtin_amdgcn_exp2f(meet[(k * 3 + 0) * 64 + lane] - t_all);
                        d_all = fmaf(meet[(k * 3 + 1) * 64 + lane], g, d_all);
                        f[k] = g * pool_power((int)__float_as_uint(meet[(k * 3 + 2) * 64 + lane]) - e_all);
                    }
                }
#pragma unroll
                for (int i = 0; i < P::MEET / W; ++i)
                    if (part * (P::MEET / W) + i < kPoolOwn<D>) {            // (channels past the last: what is there is not looked at)
                        floatx4 x = sums[(wave + W * i) * 64 + lane] * f[0];
#pragma unroll
                        for (int k = 1; k < W; ++k) x += sums[(k * P::MEET + wave + W * i) * 64 + lane] * f[k];
                        mine[part * (P::MEET / W) + i < kPoolOwn<D> ? part * (P::MEET / W) + i : 0] = x;
                    }
            }
            __syncthreads();
            if (whole) {
                char* const dst = row[c].there ? a.out + row[c].token * a.out_token + row[c].head * a.out_head : nullptr;
                pool_finish16<D, false>(mine, d_all, e_all, lds, a.out_table16, a.out_unscale, dst, a.bf16, wave, lane);
            } else {
                float* const part = a.decode_parts + ((2LL * w + (at_begin ? 0 : 1)) * CB + c) * kPoolPart16<D>;
#pragma unroll
                for (int i = 0; i < kPoolOwn<D>; ++i)
                    if (wave + W * i < NB) reinterpret_cast<floatx4*>(part)[(wave + W * i) * 64 + lane] = mine[i];
                if (wave == 0) {
                    part[16 * D + lane] = t_all;
                    part[16 * D + 64 + lane] = d_all;
                    part[16 * D + 128 + lane] = __uint_as_float((uint32_t)e_all);
                }
            }
        }
        __syncthreads();                                     // (the next segment's tiles go where the sums were, its queries where these are)
        unit += t1 - t0;
    }
}

// The parts of a key head's rows that went to several workgroups, in the order of the keys; rows of sequences without a tile are zero.  One
// workgroup of four wavefronts per sequence and key head, each with a quarter of the channels, all parts of them on their way at once
// (up to AHEAD).
template <int D, int CB>
__device__ __forceinline__ void pool_decode_merge(const pool_attention_args& a, unsigned block, unsigned char* lds) {
    constexpr int NB = D / 16, W = kPoolTeam, AHEAD = 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int all = (a.decode_rows + 16 * CB - 1) / (16 * CB), at = (int)(block / (unsigned)all), rb = (int)block - at * all;
    const int seq = at / a.heads, head = at - seq * a.heads;
    const int units = a.decode_before[a.s.n_seq], units_before = a.decode_before[seq];       // (with the sequence's, in one round of loads)
    const pool_seq q = pool_seq_of(a.s, seq);
    const int rows = q.n_new * a.group, blocks_of_rows = (rows + 16 * CB - 1) / (16 * CB);
    if (rows == 0 || !pool_is_decode(q, a.group, a.decode_rows) || rb >= blocks_of_rows) return;
    const int tiles = pool_tiles(q.length, q.full, a.decode_keys);
    if (tiles == 0) {
        for (int i = threadIdx.x + rb * 16 * CB * (D / 8); i < min(rows, (rb + 1) * 16 * CB) * (D / 8); i += 64 * W) {
            const pool_row r = pool_row_of(q, head, a.group, i / (D / 8));
            reinterpret_cast<uint4*>(a.out + r.token * a.out_token + r.head * a.out_head)[i % (D / 8)] = make_uint4(0, 0, 0, 0);
        }
        return;
    }
    if (units == 0) return;                                  // (too many of them: see kPoolMostUnits)
    const pool_shares shares(units, a.decode_grid, W);
    const int first = units_before + (head * blocks_of_rows + rb) * tiles, w0 = shares.owner(first), w1 = shares.owner(first + tiles - 1);
    if (w0 == w1) return;
    const int behind = shares.begin(w0) != first ? 1 : 0;    // the first part's workgroup began with other rows
    const auto part = [&](int w, int c) __attribute__((always_inline)) {
        return a.decode_parts + ((2LL * w + (w == w0 ? behind : 0)) * CB + c) * kPoolPart16<D>;
    };
    for (int c = 0; c < CB; ++c) {
        float t_all = kPoolLowest, den = 0.0f;
        int e_all = kPoolNoExponent;
        floatx4 o[kPoolOwn<D>];
#pragma unroll
        for (int i = 0; i < kPoolOwn<D>; ++i) o[i] = floatx4{0, 0, 0, 0};
        for (int v = w0; v <= w1; v += AHEAD) {              // (one round of loads for AHEAD parts, the sums so far brought under their maximum)
            floatx4 x[AHEAD][kPoolOwn<D>];
            pool_part_head h[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const float* const at = part(min(v + k, w1), c);
                h[k].load(at + 16 * D, lane);
#pragma unroll
                for (int i = 0; i < kPoolOwn<D>; ++i) x[k][i] = reinterpret_cast<const floatx4*>(at)[min(wave + W * i, NB - 1) * 64 + lane];
            }
            const float before = pool_join(t_all, den, e_all, h, v, w1);
#pragma unroll
            for (int i = 0; i < kPoolOwn<D>; ++i) o[i] *= before;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
#pragma unroll
                for (int i = 0; i < kPoolOwn<D>; ++i) o[i] += x[k][i] * h[k].factor;
        }
        const pool_row r = pool_row_of(q, head, a.group, (rb * CB + c) * 16 + (lane & 15));
        char* const dst = r.there ? a.out + r.token * a.out_token + r.head * a.out_head : nullptr;
        if (c > 0) __syncthreads();
        pool_finish16<D, true>(o, den, e_all, lds, a.out_table16, a.out_unscale, dst, a.bf16, wave, lane);
    }
}

template <int D, int BITS, int CB>
pool_attention_kernel_t pool_pick_decode_groups(int gm) {
    return gm == kGroup16 ? srft_pool_decode_kernel<D, BITS, CB, kGroup16>
           : gm == kGroupWide ? srft_pool_decode_kernel<D, BITS, CB, kGroupWide> : srft_pool_decode_kernel<D, BITS, CB, kGroup32>;
}
template <int D, int BITS>
pool_attention_kernel_t pool_pick_decode(int cb, int gm) {
    if constexpr (D <= 128)
        if (cb == 2) return pool_pick_decode_groups<D, BITS, 2>(gm);
    return pool_pick_decode_groups<D, BITS, 1>(gm);
}

#endif  // SRFT_POOL_DECODE_H
