// Attention over a pool, the end: the sums of rows whose keys went to several workgroups are added in the order of the keys and
// finished; rows of sequences without a tile are zero.  The first a.decode_merges workgroups take the rows of the scan for few rows
// (pool_decode_merge), the others those of chunks, in one launch: apart, the first took 17 us beside the 29 of the others (d = 256).
// Chunks: one workgroup of four wavefronts per 32 rows of a key head, of the blocks of 256 rows that there are (by the longest sequence for each, 255
// decode steps beside a prompt of 4096 tokens, 64 query heads, were a million workgroups, nearly all of them empty: 1376 us, now 36), each with every
// fourth run of 32 positions of the sums and then of the outputs (one wavefront per 32 rows read every part, and the matrix, one after the other: 104
// us at d = 256, 28 at d = 128).  Bound by the chain of loads where parts are few (a first round for the maxima alone: 6.9 us, now 5.5, for a step of
// 4 sequences), by the parts' bytes where they are many (23 us for 67 MB at d = 128; more of them in flight is slower).  Shared forms: the parts of
// the tokens in common first, read by row; 64 conversations' 512 rows 16 us (28 with channels gathered one by one).  Rows that their scan has
// finished have nothing to do here.
#include "../pool_decode.h"

namespace {

// positions 4 half .. + 3 of a unit of eight channels
__device__ __forceinline__ floatx4 by_position(const float* unit, int half, int bits) {
    const floatx4 y = reinterpret_cast<const floatx4*>(unit)[0], z = reinterpret_cast<const floatx4*>(unit)[1];
    if (bits == 8) return half ? floatx4{z[0], z[2], z[1], z[3]} : floatx4{y[0], y[2], y[1], y[3]};
    return half ? floatx4{y[2], z[2], y[3], z[3]} : floatx4{y[0], z[0], y[1], z[1]};
}

template <int D, int FORM>
__device__ __forceinline__ void chunk_merge(const pool_attention_args& a, unsigned workgroup, uint4* ops, float (*tops)[32]) {
    constexpr int BLOCKS = kPoolChunkWaves, ROWS = kPoolBlock * BLOCKS, KEYS = kPoolChunkKeys<D>, G = D / 32, T = D / 16, OWN = (G + kPoolTeam - 1) / kPoolTeam, AHEAD = 2;
    // ops: [k-step][hi, lo][lane]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int of = (int)(workgroup / BLOCKS), block = (int)workgroup - of * BLOCKS, at = of / a.heads, head = of - at * a.heads;
    const int* const before = a.chunk_before;
    const int units = before[pool_count<FORM>(a)];           // (in one round of loads)
    if (at >= a.blocks_before[a.s.n_seq]) return;
    const int seq = a.s.n_seq == 1 ? 0 : __builtin_amdgcn_readfirstlane(pool_sequence_of(a.blocks_before, a.s.n_seq, at)), rt = at - a.blocks_before[seq];
    const pool_view view = pool_view_of<FORM>(a, seq);
    const pool_seq& q = view.q;
    const int units_before = before[seq];
    const int r0 = rt * ROWS + block * kPoolBlock;
    if (r0 >= q.n_new * a.group) return;
    const int tiles = pool_chunk_tiles<FORM>(a, q, ROWS, KEYS, rt);
    const auto row_here = [&]() __attribute__((always_inline)) { return pool_row_of(q, head, a.group, r0 + (lane & 31)); };
    const auto to = [&](const pool_row& r) __attribute__((always_inline)) { return r.there ? a.out + r.token * a.out_token + r.head * a.out_head : nullptr; };
    if (tiles == 0) {
        if (char* const dst = to(row_here()))
            for (int i = 2 * wave + half; i < D / 8; i += 2 * kPoolTeam) reinterpret_cast<uint4*>(dst)[i] = make_uint4(0, 0, 0, 0);
        return;
    }
    if (units == 0) return;                                  // (too many of them: see kPoolMostUnits)
    // Units of a key head's blocks of rows, and of those in front of this one: by one wavefront.  (By all four, each for itself, 8192 workgroups with
    // nothing to merge were 23 us, the vector ALU's time.)
    __shared__ int2 units_of;
    if (wave == 0) {
        int all = 0, in_front = 0;
        for (int i = lane; i * ROWS < q.n_new * a.group; i += 64) {
            const int cost = pool_chunk_cost<FORM>(pool_chunk_tiles<FORM>(a, q, ROWS, KEYS, i));
            all += cost;
            in_front += i < rt ? cost : 0;
        }
        all = pool_wave_sum(all);
        in_front = pool_wave_sum(in_front);
        if (lane == 0) units_of = make_int2(all, in_front);
    }
    __syncthreads();
    const int first = units_before + head * units_of.x + units_of.y;
    const pool_shares shares(units, a.chunk_grid, kPoolChunkLeast<FORM>);
    const int w0 = shares.owner(first + kPoolChunkStart<FORM>), w1 = shares.owner(first + pool_chunk_cost<FORM>(tiles) - 1);
    const bool joint = FORM == kPoolShared && view.group >= 0;
    if (w0 == w1 && !joint) return;
    const int behind = shares.begin(w0) < first ? 1 : 0;    // the first part's workgroup began with other rows
    const pool_row row = row_here();
    char* const dst = to(row);
    const auto part = [&](int w) __attribute__((always_inline)) {
        return a.chunk_parts + ((2LL * w + (w == w0 ? behind : 0)) * BLOCKS + block) * kPoolPart<D>;
    };
    float t_all = kPoolLowest, den = 0.0f;
    int e_all = kPoolNoExponent;
    floatx16 sums[OWN];
#pragma unroll
    for (int i = 0; i < OWN; ++i) sums[i] = floatx16{0};
    // parts v .. v + AHEAD - 1, up to w1, whose heads and sums (four of them: number n of the lane's) `heads` and `four` give
    const auto join = [&](int v, int w1, auto heads, auto four) __attribute__((always_inline)) {
        floatx4 x[AHEAD][OWN][4];
        pool_part_head h[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            heads(min(v + k, w1), h[k]);
#pragma unroll
            for (int i = 0; i < OWN; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) x[k][i][j] = four(min(v + k, w1), 4 * min(wave + kPoolTeam * i, G - 1) + j);
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
    };
    if (joint) {
        const long long r_at = (long long)row.token * (a.heads * a.group) + row.head;
        const pool_common p(a, view, head, KEYS);
        const bool common_chunk = p.chunk;
        // rows whose tokens (own: 0, in common: 1) one workgroup has had all of; the others as they are
        const auto whole = [&](int which, bool in) __attribute__((always_inline)) {
            pool_part_head h[1];
            h[0].load4(a.joint_heads[which] + 4 * r_at, in);
            const float before = pool_join(t_all, den, e_all, h, 0, 0);
#pragma unroll
            for (int i = 0; i < OWN; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int u = 4 * min(wave + kPoolTeam * i, G - 1) + j;
                    const floatx4 y = which == 1 && !common_chunk ? by_position(a.joint_rows[1] + r_at * D + 8 * u, half, a.bits)
                                                                  : *reinterpret_cast<const floatx4*>(a.joint_rows[which] + r_at * D + 8 * u + 4 * half);
#pragma unroll
                    for (int m = 0; m < 4; ++m) sums[i][4 * j + m] = fmaf(in ? y[m] : 0.0f, h[0].factor, sums[i][4 * j + m] * before);
                }
        };
        const int before_rows = (q.start - p.p.start) * a.group, n_rows = q.n_new * a.group, from = before_rows + r0, to = before_rows + min(r0 + 31, n_rows - 1);
        const int mine = min(from + (lane & 31), to);
        if (p.there && from >= 0 && to < p.p.n_new * a.group)       // (starts that are not ascending: anything)
            for (int b = from / p.rows; b <= to / p.rows; ++b) {
                const int v0 = p.first(b), v1 = p.last(b);
                const bool in = mine / p.rows == b;
                const int r = in ? mine - b * p.rows : 0;
                if (v0 == v1) {
                    whole(1, in);
                    continue;
                }
                for (int v = v0; v <= v1; v += AHEAD)
                    join(v, v1,
                         [&](int w, pool_part_head& h) __attribute__((always_inline)) {
                             h.load4(p.template heads<D>(p.template part<D>(a, b, w, w == v0, r), r), in);
                         },
                         [&](int w, int n) __attribute__((always_inline)) {
                             const floatx4 x = p.positions(p.template part<D>(a, b, w, w == v0, r), r, n, half, a.bits);
                             return in ? x : floatx4{0, 0, 0, 0};
                         });
            }
        if (w0 == w1) whole(0, true);
    }
    if (!joint || w0 != w1)
        for (int v = w0; v <= w1; v += AHEAD)
            join(v, w1, [&](int w, pool_part_head& h) __attribute__((always_inline)) { h.load(part(w) + 32 * D, lane); },
                 [&](int w, int n) __attribute__((always_inline)) { return reinterpret_cast<const floatx4*>(part(w))[n * 64 + lane]; });
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

// Four wavefronts a SIMD are asked for at 256 dimensions, where the registers would not allow them by themselves.  (Below they do; asked for all the
// same, a step of 4 sequences takes 0.1 us more.)
template <int D, int CB, int FORM>
__global__ void __launch_bounds__(64 * kPoolTeam, FORM == kPoolShared || D < 256 ? 1 : 4) srft_pool_merge_kernel(const pool_attention_args a) {
    constexpr int OPS = D / 16 * 2 * 64;
    __shared__ __align__(16) unsigned char lds[std::max(kPoolFinishBytes<D>, OPS * 16 + kPoolTeam * 32 * 4)];
    const unsigned workgroup = blockIdx.y * gridDim.x + blockIdx.x;          // (what follows is uniform)
    if (workgroup >= a.merges) return;
    if (workgroup < (unsigned)a.decode_merges)
        pool_decode_merge<D, CB, FORM>(a, workgroup, lds);
    else
        chunk_merge<D, FORM>(a, workgroup - a.decode_merges, reinterpret_cast<uint4*>(lds), reinterpret_cast<float (*)[32]>(lds + OPS * 16));
}

template <int D, int CB> pool_attention_kernel_t form_of(int form) {
    return form == kPoolShared ? srft_pool_merge_kernel<D, CB, kPoolShared>
           : form == kPoolSliding ? srft_pool_merge_kernel<D, CB, kPoolSliding> : srft_pool_merge_kernel<D, CB, kPoolCausal>;
}
template <int D> pool_attention_kernel_t pick(int cb, int form) {
    if constexpr (D <= 128)
        if (cb == 2) return form_of<D, 2>(form);
    return form_of<D, 1>(form);
}
pool_attention_kernel_t dispatch(int d, int cb, int form) { SRFT_DISPATCH_D(d, pick, cb, form) }

}  // namespace

pool_attention_kernel_t srft_pick_pool_merge(int d, int cb, int form) { return dispatch(d, cb, form); }
