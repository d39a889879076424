// pool_attention.h -- attention of new tokens over a pool's pages: what its kernels share.
//
// The work is done in the rotated domain, as in kernels/decode_attention.hip: with x = R w the read path (w = code * scale, R = S Q^T
// diag(1 / max(lambda, 1e-6))), <q, k> = <R_k^T q, w_k> and sum_t p_t v_t = R_v (sum_t p_t w_t).  So
//   1. pool_rotate:  q' = R_k^T q for all rows, and w of the windows' tokens, both as fp16 with a power of two per row; and how many units of
//      work (a tile of keys of one sequence and key head) there are in front of each sequence;
//   2. pool_decode (few rows a key head) and pool_chunk (many): one pass over the keys with the running maximum and sum of the softmax.
//      Each workgroup takes an equal share of all units, in their order, whatever sequences they belong to; what it has of one
//      sequence, key head and block of rows is a segment.  A segment that is the whole of it is finished at once;
//   3. pool_merge: the others' sums are brought under one maximum, added in their order, and finished (one launch for both).
// Finishing is the division by the sum of weights and R_v, on the matrix cores.
//
// Roundings to 16 bits.  pool_decode, which memory bounds: codes go to the matrix cores as they are (exact in fp16) against q' as fp16
// hi + lo, scales on the results in fp32; a weight times the scale of its key and group is rounded to fp16 once.  pool_chunk, which the matrix
// cores bound, has one matrix instruction where that would take two: q', the dequantized w (code * scale, the scale rounded first) and
// the weights p are fp16, half a step (2^-11) each at most.  Against 64 bits that is 3e-4 and 1.2e-3 of an output's size (1.5e-3 where one scale
// serves a whole row), the output's own rounding to fp16 included.  Sums, maxima and exponents are fp32.  None of the operands can leave fp16's
// range: q' has a power of two per row, w a running one taken from the scales, the weights are at most 2^(kLazy + kHigh) in pool_chunk, and times a
// scale 2^(kLazy + 7) in pool_decode.
//
// Forms.  Causal: srft_pool_attention.  Sliding: rows see the last `recent` tokens and the first `sinks` ones; of a block's tiles those between its
// sinks and its first row's recent tokens are left out (pool_gap), what is left is numbered through.  Shared: sequences that have pages in
// common are taken apart into items: what a sequence has of its own, which is a sequence whose first page lies further along its table, and,
// for each group, the tokens in common with the rows of all of its sequences, which all see all of them.  Both leave unfinished sums, and the
// merge joins them (pool_item, joint_rows).
//
// Order of channels.  A dword of codes is decoded into eight fp16 values in the order 0 4 1 5 2 6 3 7 (4 bits; 0 2 1 3 at 8 bits), so
// all operands have their channels in that order within units of eight ("positions"), q' by the way it is stored, the output by the
// order of the columns of its matrix.
#ifndef SRFT_POOL_ATTENTION_H
#define SRFT_POOL_ATTENTION_H
#include "device_util.h"
#include "pool.h"

constexpr float kPoolLowest = -3.0e38f;                      // "no key yet": finite, so that differences of two are
constexpr int kPoolNoExponent = -200;                        // of V: "no value yet"
constexpr float kLazy = 8.0f;                                // how far (in powers of two) weights may grow past the maximum that they are taken from
// pool_chunk rounds weights to fp16, so it takes them as large as that allows: up to 2^(kLazy + kHigh).  What is lost then are weights below
// 2^-32 of a row's largest; under the maximum itself they were those below 2^-25, and behind one dominant key the others lost up to 2^-25 of it each
// (3 % of the output over 2^20 keys).  From kNear on, where an exponent's own rounding could take a weight past fp16's range, they have the older
// room.
constexpr float kHigh = 7.0f, kNear = 1048576.0f;
constexpr int kPoolDecodeRows = 32;                          // most rows of one key head that pool_decode takes, in blocks of 16
constexpr int kPoolTeam = 4;                                 // wavefronts of a workgroup of pool_decode and pool_merge
constexpr int pool_decode_keys(int d, int cb) { return d <= 128 && cb == 1 ? 64 : 32; }      // of a tile
constexpr int kPoolBlock = 32;                               // rows of a wavefront
template <int D> constexpr int kPoolChunkKeys = D <= 128 ? 64 : 32;
constexpr int kPoolChunkWaves = 8;

enum { kPoolCausal = 0, kPoolSliding = 1, kPoolShared = 2, kPoolForms = 3 };
// What the kernels of the shared form take for a sequence: first the sequences' own tokens, items 0 .. n_seq - 1, then the groups' in common.
struct pool_item {
    int start, n_new, length, before, full;                  // as pool_seq, without the tokens in front of first_page
    int seq, first_page;                                     // whose page table and windows; the first page of the item in it
    int group;                                               // the group that a sequence shares pages with, or -1
    int common_start, common_n_new, common;                  // of that group: rows of its new tokens, tokens in common
    int unused;
};
static_assert(sizeof(pool_item) == 48, "three loads");

struct pool_attention_args {
    pool_seqs s;
    srft_pool_buffers kb, vb;
    int heads, group, g;                                     // key heads, query heads to each, channels to a scale
    const char* q;                                           // strides in bytes
    char* out;
    long long q_token, q_head, out_token, out_head;
    int bf16;
    float exponent, sign;                                    // |softmax_scale| log2 e, and its sign
    const uint4 *q_table, *k_table, *v_table, *out_table, *out_table16;
    float q_unscale, k_unscale, v_unscale, out_unscale;
    int q_tiles, q_grid;                                     // passes of query rows in pool_rotate, workgroups that take them
    // workspace
    int *decode_before, *chunk_before;                       // [n_seq + 1]: units of work in front of a sequence
    int* blocks_before;                                      // [n_seq + 1]: blocks of 256 rows of pool_chunk's in front of a sequence (null where there are none)
    unsigned short *q_rows, *q_rows_low;                     // [n_new][n_q_heads][D] fp16: q', and what its rounding leaves
    float* q_factor;                                         // [n_new][n_q_heads]: exponent * what q_rows are to be multiplied with
    unsigned short* tail_rows;                               // [K, V][n_seq][heads][R][D] fp16
    float* tail_factor;                                      // [K, V][n_seq][heads][R]
    unsigned short* tail_columns;                            // V's [n_seq][heads][D channels][R]
    float *decode_parts, *chunk_parts;                       // sums of segments (pool_part)
    int decode_grid, chunk_grid;
    int decode_rows, decode_block, decode_keys;              // rows that go to pool_decode, those of a workgroup, keys of its tiles
    int decode_merges;                                       // workgroups of pool_merge that merge what pool_decode left
    unsigned merges;                                         // all of them (srft_grid)
    int recent, sinks;                                       // sliding
    const int *groups, *shared;                              // shared: the caller's
    int n_groups, bits;
    int common_rows;                                         // a group's rows up to which its tokens in common go to pool_decode
    int* bounds;                                             // [n_groups + 1]: groups, ascending and within n_seq (workspace)
    pool_item* items;                                        // [n_seq + n_groups] (workspace)
    float *joint_rows[2], *joint_heads[2];                   // [n_new][n_q_heads][D] and [4]: sums (by position from pool_chunk, by channel from pool_decode) and
                                                             // maximum, sum of weights, exponent, where one workgroup has had all of a row's own
                                                             // tokens [0], or of those in common [1] (workspace)
};
// Sums of a block of 32 rows that a segment leaves: [D / 8 float4][64 lanes], then per lane maximum, sum of weights and V's exponent.
template <int D> constexpr int kPoolPart = 32 * D + 3 * 64;
constexpr long long pool_part(int d) { return 32LL * d + 3 * 64; }

// ---- units of work.  A tile is of pages' keys or of the window's, never of both.
// Rows that belong to one sequence each come to less than kPoolMostUnits of them (the host's checks).  Starts that give the same rows to many
// sequences can come to more: then there are none, and nothing is answered.
constexpr unsigned kPoolMostUnits = 0x7FFFFF00;         // (sums of it and a small number are below 2^31)
__device__ __forceinline__ int pool_tiles(int seen, int full, int keys) {
    const int pages = max(min(seen, full), 0), window = max(seen - full, 0);
    return (pages + keys - 1) / keys + (window + keys - 1) / keys;
}
__device__ __forceinline__ bool pool_is_decode(const pool_seq& q, int group, int rows) { return q.n_new * group <= rows; }
template <int FORM> __device__ __forceinline__ bool pool_is_decode(const pool_attention_args& a, const pool_seq& q, int i) {
    return pool_is_decode(q, a.group, FORM == kPoolShared && i >= a.s.n_seq ? a.common_rows : a.decode_rows);
}
// tokens that the rows of block rt (of `rows` rows) see at most
__device__ __forceinline__ int pool_seen(const pool_seq& q, int group, int rows, int rt) {
    return q.before + (min((rt + 1) * rows, q.n_new * group) - 1) / group + 1;
}
// Tiles that a block of rows leaves out: `skip` of them from tile `begin` on.  (Sliding; none in the other forms.)
template <int FORM> struct pool_gap {
    int begin = 0, skip = 0;
    __device__ __forceinline__ int tile(int t) const {       // which tile of the sequence is the block's t-th
        if constexpr (FORM == kPoolSliding) return t < begin ? t : t + skip;
        return t;
    }
    __device__ __forceinline__ int in_pages(int page_tiles) const {          // how many of them are of pages
        if constexpr (FORM == kPoolSliding) return max(min(begin + skip, page_tiles) - min(begin, page_tiles), 0);
        return 0;
    }
    int low = 0, sinks = 0;
    // Whether no row of the block sees one of the 16 keys from `key` on: they are as if their page did not exist (what is in it need not be numbers).
    __device__ __forceinline__ bool hides(int key) const {
        if constexpr (FORM == kPoolSliding) return key + 16 <= low && key >= sinks;
        return false;
    }
};
// first: the block's first row's token (or an earlier one); seen: the tokens that its last row sees
template <int FORM>
__device__ __forceinline__ pool_gap<FORM> pool_gap_of(const pool_attention_args& a, const pool_seq& q, int first, int seen, int keys) {
    pool_gap<FORM> g;
    if constexpr (FORM == kPoolSliding) {
        g.low = max(first - a.recent + 1, 0);
        g.sinks = a.sinks;
        g.begin = pool_tiles(min(a.sinks, seen), q.full, keys);
        g.skip = max((g.low < q.full ? g.low / keys : (q.full + keys - 1) / keys + (g.low - q.full) / keys) - g.begin, 0);
    }
    return g;
}
// tokens that the rows of block rt of pool_chunk see at most, and the tiles that it leaves out
template <int FORM>
__device__ __forceinline__ int pool_chunk_seen(const pool_attention_args& a, const pool_seq& q, int rows, int rt) {
    const int seen = pool_seen(q, a.group, rows, rt);
    return FORM == kPoolShared ? min(seen, q.length) : seen;
}
template <int FORM>
__device__ __forceinline__ pool_gap<FORM> pool_chunk_gap(const pool_attention_args& a, const pool_seq& q, int rows, int keys, int rt) {
    return pool_gap_of<FORM>(a, q, q.before + rt * rows / a.group, pool_chunk_seen<FORM>(a, q, rows, rt), keys);
}
template <int FORM>
__device__ __forceinline__ int pool_chunk_tiles(const pool_attention_args& a, const pool_seq& q, int rows, int keys, int rt) {
    return pool_tiles(pool_chunk_seen<FORM>(a, q, rows, rt), q.full, keys) - pool_chunk_gap<FORM>(a, q, rows, keys, rt).skip;
}
// What a block of rows counts for when the work is shared out: its tiles, and the time that its start and its end take, in tiles, so that a
// workgroup with many short segments has fewer tiles (chunks of 8 sequences, 40 to 300 tokens, behind 12,000 in common: the workgroups with the
// own tokens' segments had 30 of them, 560 us; now 275, and with 4 or 8 for a start of pool_chunk 271 and 278; with 2 and 8 for one of pool_decode a
// batch of 8 groups takes 76 and 60 us where 4 takes 59).  Shares of pool_chunk are at least kPoolChunkLeast units: with 16, 500 tokens and less of 8
// sequences of up to 4096 at d = 256, 1000 of them seen, take 128 instead of 110 us, with 8, 512 tokens there that see 64 or 1024 94 and 74 instead
// of 55 and 64, and with 2, 64 tokens that see 4096 at d = 128 51 instead of 45 (4 query heads on each of 8).  The causal form counts tiles alone.
template <int FORM> constexpr int kPoolChunkStart = FORM == kPoolCausal ? 0 : 6;
template <int FORM> constexpr int kPoolDecodeStart = FORM == kPoolCausal ? 0 : 4;
template <int FORM> constexpr int kPoolChunkLeast = FORM == kPoolCausal ? 1 : 4;             // of units, a workgroup's of pool_chunk
template <int FORM> __device__ __forceinline__ int pool_chunk_cost(int tiles) { return tiles > 0 ? tiles + kPoolChunkStart<FORM> : 0; }
template <int FORM> __device__ __forceinline__ int pool_decode_cost(int tiles) { return tiles > 0 ? tiles + kPoolDecodeStart<FORM> : 0; }
// the same of pool_decode, whose blocks of a sequence have all the same tiles
template <int FORM>
__device__ __forceinline__ pool_gap<FORM> pool_decode_gap(const pool_attention_args& a, const pool_seq& q, int keys) {
    return pool_gap_of<FORM>(a, q, q.before, q.length, keys);
}
template <int FORM>
__device__ __forceinline__ int pool_decode_tiles(const pool_attention_args& a, const pool_seq& q, int keys) {
    return pool_tiles(q.length, q.full, keys) - pool_decode_gap<FORM>(a, q, keys).skip;
}
// A sequence, or item, of a call.
struct pool_view {
    pool_seq q;
    int seq, first_page;
    int group;                                               // whose tokens in common it has in front of its own, or -1
    pool_seq of_group;                                       // these, as a sequence (start, n_new, length and full are looked at)
};
template <int FORM> __device__ __forceinline__ int pool_count(const pool_attention_args& a) { return FORM == kPoolShared ? a.s.n_seq + a.n_groups : a.s.n_seq; }
template <int FORM>
__device__ __forceinline__ pool_view pool_view_of(const pool_attention_args& a, int i) {
    if constexpr (FORM == kPoolShared) {
        const pool_item t = a.items[i];
        return {{t.start, t.n_new, t.length, t.before, t.full}, t.seq, t.first_page, t.group, {t.common_start, t.common_n_new, t.common, t.common, t.common}};
    }
    return {pool_seq_of(a.s, i), i, 0, -1, {}};
}
// sum over the lanes of a wavefront, in all of them
__device__ __forceinline__ int pool_wave_sum(int x) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
    return x;
}
// tiles of the blocks of rows 0 .. n - 1 of one key head (by the whole wavefront)
template <int FORM>
__device__ __forceinline__ int pool_chunk_units(const pool_attention_args& a, const pool_seq& q, int rows, int keys, int n) {
    int sum = 0;
    for (int rt = threadIdx.x & 63; rt < n; rt += 64) sum += pool_chunk_cost<FORM>(pool_chunk_tiles<FORM>(a, q, rows, keys, rt));
    return pool_wave_sum(sum);
}
// The block of rows, of n, that unit u of one key head belongs to, and the units in front of it there (by the whole wavefront, a block a lane).
struct pool_block_at { int rt, before; };
template <int FORM>
__device__ __forceinline__ pool_block_at pool_chunk_block_of(const pool_attention_args& a, const pool_seq& q, int rows, int keys, int n, int u) {
    const int lane = (int)threadIdx.x & 63;
    int before = 0;
    for (int rt = 0;; rt += 64) {
        const int units = rt + lane < n ? pool_chunk_cost<FORM>(pool_chunk_tiles<FORM>(a, q, rows, keys, rt + lane)) : 0;
        int sum = units;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int other = __shfl_up(sum, d);
            if (lane >= d) sum += other;
        }
        const int below = (int)__popcll(__ballot(before + sum <= u));        // (ascending: the first ones)
        if (below < 64 || rt + 64 >= n) {
            const int i = max(min(below, min(n - rt, 64) - 1), 0);
            return {rt + i, before + __builtin_amdgcn_readlane(sum - units, i)};
        }
        before += __builtin_amdgcn_readlane(sum, 63);
    }
}
// The workgroups that take part, and where the share of workgroup w begins: the first `more` have a unit more than the others.
struct pool_shares {
    int units, groups, each, more;
    __device__ __forceinline__ pool_shares(int units_, int grid, int least) : units(units_), groups(max(min(grid, (units_ + least - 1) / least), 1)) {
        each = (int)((unsigned)units / (unsigned)groups);
        more = units - each * groups;
    }
    __device__ __forceinline__ int begin(int w) const { return w * each + min(w, more); }
    __device__ __forceinline__ int owner(int unit) const {
        const int longer = more * (each + 1);                // units of those with one more
        return unit < longer ? (int)((unsigned)unit / (unsigned)(each + 1)) : more + (int)((unsigned)(unit - longer) / (unsigned)max(each, 1));
    }
};
// the sequence that a unit belongs to (by the whole wavefront; units before before[0] = 0 are none): the last b with before[b] <= unit
__device__ __forceinline__ int pool_sequence_of(const int* before, int n_seq, int unit) {
    int at = 0, n = n_seq + 1;                               // the answer is among before[at .. at + n - 1]
    while (n > 1) {
        const int step = (n + 63) / 64, i = at + (int)(threadIdx.x & 63) * step;
        const int below = (int)__popcll(__ballot(i < at + n && before[min(i, n_seq)] <= unit));      // (ascending: the first ones)
        at += (below - 1) * step;
        n = min(step, n_seq + 1 - at);
    }
    return min(at, n_seq - 1);
}

// ---- exponents.  With E of the largest scale, code * scale * 2^-E is below 2^15 (codes below 2^AMP).
template <int BITS> constexpr int kPoolAmp = BITS == 4 ? 3 : 7;
template <int BITS>
__device__ __forceinline__ int pool_exponent(float scale) {
    return max((int)((__float_as_uint(scale) >> 23) & 0xFF) - 127, -99) + kPoolAmp<BITS> - 14;
}
__device__ __forceinline__ float pool_power(int e) { return __uint_as_float((uint32_t)(min(max(e, -126), 127) + 127) << 23); }

// ---- the merge: maximum, sum of weights and exponent of a part, and what its sums are to be multiplied with
struct pool_part_head {
    float top, den, e, factor;
    __device__ __forceinline__ void load(const float* p, int lane) { top = p[lane], den = p[64 + lane], e = p[128 + lane]; }
    __device__ __forceinline__ void load4(const float* p, bool in) {         // (a row that is not there counts for nothing)
        const floatx4 x = *reinterpret_cast<const floatx4*>(p);
        top = in ? x[0] : kPoolLowest;
        den = in ? x[1] : 0.0f;
        e = __uint_as_float(in ? __float_as_uint(x[2]) : (uint32_t)kPoolNoExponent);
    }
};
// Parts v .. v + N - 1 (those behind the last, w1, are it again and count for nothing) under one maximum with what has been added so far; what its
// sums are to be multiplied with.
template <int N>
__device__ __forceinline__ float pool_join(float& top, float& den, int& e, pool_part_head (&h)[N], int v, int w1) {
    float t = top;
    int m = e;
#pragma unroll
    for (int k = 0; k < N; ++k) t = fmaxf(t, h[k].top), m = max(m, (int)__float_as_uint(h[k].e));
    const float f = __builtin_amdgcn_exp2f(top - t), before = f * pool_power(e - m);
    den *= f;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const float g = v + k <= w1 ? __builtin_amdgcn_exp2f(h[k].top - t) : 0.0f;
        den = fmaf(h[k].den, g, den);
        h[k].factor = g * pool_power((int)__float_as_uint(h[k].e) - m);
    }
    top = t;
    e = m;
    return before;
}

// ---- 16 codes of a row (two dwords at 4 bits, four at 8) -> two units of eight fp16 values times a scale
template <int BITS> struct pool_codes;
template <> struct pool_codes<4> { typedef u32x2 type; };
template <> struct pool_codes<8> { typedef u32x4 type; };
__device__ __forceinline__ half8 pool_times(uint4 x, _Float16 f) {
    const half8 s = {f, f, f, f, f, f, f, f};
    return __builtin_bit_cast(half8, x) * s;
}
__device__ __forceinline__ void pool_decode16(u32x2 c, _Float16 f, half8& a, half8& b) {
    a = pool_times(decode8(c[0]), f);
    b = pool_times(decode8(c[1]), f);
}
__device__ __forceinline__ void pool_decode16(u32x4 c, _Float16 f, half8& a, half8& b) {
    const uint2 x = decode4_bytes(c[0]), y = decode4_bytes(c[1]), z = decode4_bytes(c[2]), w = decode4_bytes(c[3]);
    a = pool_times(make_uint4(x.x, x.y, y.x, y.y), f);
    b = pool_times(make_uint4(z.x, z.y, w.x, w.y), f);
}

// ---- lanes l and l ^ 32 hold the two halves of a row's keys
__device__ __forceinline__ float pool_halves_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// maximum over the 64 lanes of a non-negative number, in all of them
template <int CTRL> __device__ __forceinline__ float pool_row_rotated(float x) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float pool_wave_max(float x) {
    x = fmaxf(x, pool_row_rotated<0x128>(x));                // row_ror: 8, 4, 2, 1 within 16 lanes
    x = fmaxf(x, pool_row_rotated<0x124>(x));
    x = fmaxf(x, pool_row_rotated<0x122>(x));
    x = fmaxf(x, pool_row_rotated<0x121>(x));
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return other_half_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}

typedef short pool_v4i16 __attribute__((ext_vector_type(4)));
// Eight keys of one position: the transposed reads of two blocks of 4 keys x 16 positions by 16 lanes each.  Lane l of a 16 gives the
// address of key l / 4, positions 4 (l % 4) .., and receives its position (l) of the four keys.
__device__ __forceinline__ half8 pool_transposed(const unsigned char* keys0, const unsigned char* keys1) {
    const pool_v4i16 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) pool_v4i16*)keys0);
    const pool_v4i16 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) pool_v4i16*)keys1);
    const uint2 x = __builtin_bit_cast(uint2, a), y = __builtin_bit_cast(uint2, b);
    return __builtin_bit_cast(half8, make_uint4(x.x, x.y, y.x, y.y));
}

// What a wavefront holds of 32 rows: sums[b][v] is position 32 b + 8 (v / 4) + 4 (l / 32) + v % 4 of row l % 32.
template <int D> struct pool_block {
    floatx16 sums[D / 32];
    float top, den;                                          // what weights are taken under (an exponent, see kLazy and kHigh), sum of weights (of this lane's keys)
    int e;                                                   // sums are to be multiplied by 2^e
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int b = 0; b < D / 32; ++b) sums[b] = floatx16{0};
        top = kPoolLowest;
        den = 0.0f;
        e = kPoolNoExponent;
    }
    __device__ __forceinline__ void scale(float f) {
#pragma unroll
        for (int b = 0; b < D / 32; ++b) sums[b] *= f;
    }
    // of tokens in common: the three numbers of a row next to each other
    __device__ __forceinline__ floatx4 head() const { return floatx4{top, den, __uint_as_float((uint32_t)e), 0.0f}; }
    // p: kPoolPart<D> floats in memory or LDS
    __device__ __forceinline__ void put(float* p, int lane, bool common = false) const {
#pragma unroll
        for (int b = 0; b < D / 32; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                reinterpret_cast<floatx4*>(p)[(4 * b + i) * 64 + lane] = floatx4{sums[b][4 * i], sums[b][4 * i + 1], sums[b][4 * i + 2], sums[b][4 * i + 3]};
        if (common) {                                        // (uniform)
            if (lane < 32) reinterpret_cast<floatx4*>(p + 32 * D)[lane] = head();
            return;
        }
        p[32 * D + lane] = top;
        p[32 * D + 64 + lane] = den;
        p[32 * D + 128 + lane] = __uint_as_float((uint32_t)e);
    }
};

// A tile's weights.  s: scores of K keys, register v of 32 of them key 8 (v / 4) + 4 (l / 32) + v % 4; c > 0 turns them into
// exponents.  Masked scores are -infinity.  On return the weights, 2^(exponent - b.top); the block's sums are scaled where that grew.
template <int D, int N>
__device__ __forceinline__ void pool_weights(pool_block<D>& b, floatx16 (&s)[N], float c, int e, bool first) {
    float m = fmaxf(s[0][0], s[0][1]);
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int v = n == 0 ? 2 : 0; v < 16; ++v) m = fmaxf(m, s[n][v]);
    m = fmaxf(other_half_max(m) * c, kPoolLowest);
    // The sums are kept under an older maximum as long as no weight passes 2^kLazy: after the first tiles they are hardly ever scaled.
    const bool near = fabsf(b.top) < kNear;
    const bool grown = m > b.top + (near ? kLazy + kHigh : kLazy);
    const int e_new = max(b.e, e);                           // (uniform)
    if (__ballot(grown) || e_new != b.e) {
        const float t = grown ? m - (fabsf(m) < kNear ? kHigh : 0.0f) : b.top, f = __builtin_amdgcn_exp2f(b.top - t);
        if (!first) b.scale(f * pool_power(b.e - e_new));
        b.den *= f;
        b.top = t;
        b.e = e_new;
    }
    float sum = 0.0f;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            s[n][v] = __builtin_amdgcn_exp2f(fmaf(s[n][v], c, -b.top));
            sum += s[n][v];
        }
    b.den += sum;
}
// eight weights (registers 8 i .. 8 i + 7) as an operand
__device__ __forceinline__ half8 pool_half8(const floatx16& s, int i) {
    half8 h;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = (_Float16)s[8 * i + e];
    return h;
}

// 16 channels next to each other of the lane's row, times three factors (a power of two for each part: together they may leave fp32's range
// before the product does), to row dst from channel `first` on; nowhere if dst is null.
__device__ __forceinline__ void pool_store16(const floatx16& acc, float down, float p0, float p1, char* dst, int first, int bf16) {
    if (!dst) return;
    uint32_t o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = acc[2 * i] * down * p0 * p1, y = acc[2 * i + 1] * down * p0 * p1;
        typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
        o[i] = bf16 ? __builtin_bit_cast(uint32_t, bf2{(__bf16)x, (__bf16)y}) : pack_half2(x, y);
    }
    uint4* const p = reinterpret_cast<uint4*>(dst) + first / 8;
    p[0] = make_uint4(o[0], o[1], o[2], o[3]);
    p[1] = make_uint4(o[4], o[5], o[6], o[7]);
}

// The end of 32 rows: division by the sum of weights (over both halves' keys already) and R_v.  The sums are taken as fp16 hi + lo
// under a power of two per row, the matrix as hi + lo, so that nothing is lost here.  dst: the lane's row (l % 32), or null.
template <int D> struct pool_ending {
    half8 hi[D / 16], lo[D / 16];
    float down, p0, p1;
    __device__ __forceinline__ pool_ending(const pool_block<D>& b, float unscale) {
        float m = 0.0f;
#pragma unroll
        for (int k = 0; k < D / 32; ++k)
#pragma unroll
            for (int v = 0; v < 16; ++v) m = fmaxf(m, fabsf(b.sums[k][v]));
        m = other_half_max(m);
        const int e = max((int)((__float_as_uint(m) >> 23) & 0xFF) - 127, -100);
        const float up = pool_power(14 - e);
        down = (b.den > 0.0f ? 1.0f / b.den : 0.0f) * unscale, p0 = pool_power(e - 14), p1 = pool_power(b.e);
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = b.sums[k / 2][8 * (k % 2) + i] * up;
                hi[k][i] = (_Float16)x;
                lo[k][i] = (_Float16)(x - (float)hi[k][i]);
            }
    }
    // the outputs from 32 j on; at: the lane's units of the matrix's rows for them, [D / 16][hi, lo][64]
    __device__ __forceinline__ void rows(const uint4* at, int j, char* dst, int bf16, int half) const {
        floatx16 acc{0};
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            const half8 ah = __builtin_bit_cast(half8, at[(2 * k + 0) * 64]), al = __builtin_bit_cast(half8, at[(2 * k + 1) * 64]);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, hi[k], acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(al, hi[k], acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, lo[k], acc, 0, 0, 0);
        }
        pool_store16(acc, down, p0, p1, dst, 32 * j + 16 * half, bf16);
    }
};
template <int D> constexpr int kPoolSlab = D / 16 * 2 * 64;      // units of the matrix for 32 outputs
template <int D>
__device__ __forceinline__ void pool_finish(const pool_block<D>& b, const uint4* __restrict__ table, float unscale, char* dst, int bf16, int lane) {
    const pool_ending<D> end(b, unscale);
#pragma unroll 1
    for (int j = 0; j < D / 32; ++j) end.rows(table + j * kPoolSlab<D> + lane, j, dst, bf16, lane >> 5);
}
// The same by all NT / 64 wavefronts of a workgroup, the matrix by way of LDS, 32 outputs of it at a time in one of two buffers (read by every
// wavefront for itself, it is 512 KB a workgroup at d = 128).  lds0, lds1: kPoolSlab<D> units each, free behind a barrier that is here.
template <int D, int NT>
__device__ __forceinline__ void pool_finish_together(const pool_block<D>& b, const uint4* __restrict__ table, float unscale, char* dst, int bf16, int tid, uint4* lds0,
                                                     uint4* lds1) {
    constexpr int N = (kPoolSlab<D> + NT - 1) / NT;
    u32x4 x[N];
    const auto fetch = [&](int j) __attribute__((always_inline)) {           // (threads beyond the last unit load it again)
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = reinterpret_cast<const u32x4*>(table)[j * kPoolSlab<D> + min(tid + NT * i, kPoolSlab<D> - 1)];
    };
    const auto put = [&](uint4* to) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (kPoolSlab<D> % NT == 0 || tid + NT * i < kPoolSlab<D>) to[tid + NT * i] = __builtin_bit_cast(uint4, x[i]);
    };
    fetch(0);
    const pool_ending<D> end(b, unscale);
    __syncthreads();                                         // (the buffers have been read)
    put(lds0);
#pragma unroll 1
    for (int j = 0; j < D / 32; ++j) {
        __syncthreads();                                     // (these rows are there, those before have been read)
        const bool more = j + 1 < D / 32;                    // uniform
        if (more) fetch(j + 1);
        end.rows((j & 1 ? lds1 : lds0) + (tid & 63), j, dst, bf16, tid >> 5 & 1);
        if (more) put(j & 1 ? lds0 : lds1);
    }
}

// The lane's row of a block of rows that starts at row r0 of a key head's n_new * group: where it is in q and out, and the last
// token that it sees (-1: none, or no row).
struct pool_row {
    int token, head, last;
    bool there;
};
__device__ __forceinline__ pool_row pool_row_of(const pool_seq& q, int key_head, int group, int row) {
    const int n = q.n_new * group, r = min(row, n - 1), t = r / group;
    return {q.start + t, key_head * group + r - t * group, row < n ? min(q.before + t, q.length - 1) : -1, row < n};
}

typedef void (*pool_attention_kernel_t)(const pool_attention_args);
// (one translation unit for each form of the scans)
pool_attention_kernel_t srft_pick_pool_rotate(int d, int bits, int form);
pool_attention_kernel_t srft_pick_pool_decode_b4(int d, int cb, int gm);
pool_attention_kernel_t srft_pick_pool_decode_b8(int d, int cb, int gm);
pool_attention_kernel_t srft_pick_pool_decode_sliding_b4(int d, int cb, int gm);
pool_attention_kernel_t srft_pick_pool_decode_sliding_b8(int d, int cb, int gm);
pool_attention_kernel_t srft_pick_pool_decode_shared_b4(int d, int cb, int gm);
pool_attention_kernel_t srft_pick_pool_decode_shared_b8(int d, int cb, int gm);
pool_attention_kernel_t srft_pick_pool_chunk(int d, int bits);
pool_attention_kernel_t srft_pick_pool_chunk_sliding(int d, int bits);
pool_attention_kernel_t srft_pick_pool_chunk_shared(int d, int bits);
pool_attention_kernel_t srft_pick_pool_merge(int d, int cb, int form);

#endif  // SRFT_POOL_ATTENTION_H
