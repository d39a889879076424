// Attention over a pool for few rows a key head (a decode step: the query heads of a group; a few speculated tokens of them).
//
// Bound by the records' bytes where there are enough of them, and by the vector instructions that decode them close behind.  A
// wavefront has a tile of 32 keys to itself: the keys are the rows of the score product and its 32 query rows the columns, so that a lane
// holds half of ONE key's record (D / 2 channels next to each other: one or two 16-byte loads) and decodes it straight into operands.  The
// scores come out with a lane's query row in its column, which is what the running maximum and sum and the second product (values on
// the rows, queries on the columns) want: weights stay in registers.  The values are decoded the same way and pass through the wavefront's
// own LDS once, to be read transposed.  Four wavefronts of a workgroup take the tiles of a segment in turn, with no barrier
// between them until the end of the segment, where their sums meet in LDS in a fixed order.
#include "../pool_attention.h"

namespace {

template <int D, int BITS>
__global__ void __launch_bounds__(64 * kPoolDecodeWaves, 2) srft_pool_decode_kernel(const pool_attention_args a) {
    constexpr int NU = D / 32;                               // units of 16 channels of a lane: half a row
    constexpr int T = D / 16;                                // k-steps of the score product
    constexpr int ROW = 2 * D + 32;                          // bytes of a row of values in LDS: 8 rows x 32 positions on different banks
    constexpr int KEYS = kPoolDecodeKeys, W = kPoolDecodeWaves, CB = D * BITS / 8;
    constexpr int VBYTES = KEYS * ROW, PART = kPoolPart<D> * 4;
    constexpr bool QLDS = D > 128;                           // (registers: the queries' operands are read again for every tile)
    typedef typename pool_codes<BITS>::type code_t;
    constexpr int LDS_BYTES = W * VBYTES > 2 * PART ? W * VBYTES : 2 * PART;
    __shared__ __align__(16) unsigned char lds[LDS_BYTES];
    __shared__ uint4 q_lds[QLDS ? T * 64 : 1];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
    const int total = a.decode_before[a.s.n_seq];
    const int w = srft_block_by_die();
    const pool_shares shares(total, gridDim.x, W);
    if (total == 0 || w >= shares.groups) return;            // (uniform)
    const int end = shares.begin(w + 1);
    int unit = shares.begin(w);
    int seq = __builtin_amdgcn_readfirstlane(pool_sequence_of(a.decode_before, a.s.n_seq, unit));
    unsigned char* const vt = lds + wave * VBYTES;
    const int R = 1 << a.s.log_R;
    int scale_at[NU];                                        // the scale of a lane's unit i
#pragma unroll
    for (int i = 0; i < NU; ++i) scale_at[i] = 16 * (half * NU + i) / a.g;
    const int n_scales = D / a.g;

    for (bool at_begin = true; unit < end; at_begin = false) {
        while (seq + 1 < a.s.n_seq && a.decode_before[seq + 1] <= unit) ++seq;
        const pool_seq q = pool_seq_of(a.s, seq);
        const int tiles = pool_tiles(q.length, q.full, KEYS), page_tiles = (q.full + KEYS - 1) / KEYS, tail = q.length - q.full;
        const int rel = unit - a.decode_before[seq], head = rel / tiles, t0 = rel - head * tiles, t1 = min(tiles, t0 + end - unit);
        if (t1 <= t0) return;                                // (only if the device arrays were written during the call)
        const pool_row row = pool_row_of(q, head, a.group, l32);
        const long long q_row = (long long)row.token * (a.heads * a.group) + row.head;
        const int32_t* const table = a.s.table + seq * a.s.max_pages;

        // ---- the queries' operands: k-step 2 i + j takes unit 2 (half NU + i) + j of the row
        half8 qf[QLDS ? 1 : T];
        const uint4* const q_at = reinterpret_cast<const uint4*>(a.q_rows + q_row * D) + 2 * half * NU;
        if constexpr (QLDS) {
            __syncthreads();                                 // (the segment before has read its own)
            for (int s = wave; s < T; s += W) q_lds[s * 64 + lane] = q_at[s];
            __syncthreads();
        } else {
#pragma unroll
            for (int s = 0; s < T; ++s) qf[s] = __builtin_bit_cast(half8, q_at[s]);
        }
        const float factor = a.q_factor[q_row];

        pool_block<D> b;
        b.clear();
        code_t kc[NU], vc[NU];
        float ks[NU], vs[NU];
        bool there = true;                                   // the page of the lane's key exists
        const auto page_of = [&](int t) __attribute__((always_inline)) { return q.full > 0 ? table[min(t * KEYS + l32, q.full - 1) >> a.s.log_R] : -1; };
        const auto fetch = [&](int t, int page) __attribute__((always_inline)) {
            if (t < page_tiles) {                            // uniform
                there = pool_there(page, a.s.n_pages);
                const long long at = ((long long)(there ? page : 0) * a.heads + head << a.s.log_R) + (min(t * KEYS + l32, q.full - 1) & (R - 1));
                const code_t* const k = reinterpret_cast<const code_t*>(a.kb.codes_dev + at * CB) + half * NU;
                const code_t* const v = reinterpret_cast<const code_t*>(a.vb.codes_dev + at * CB) + half * NU;
#pragma unroll
                for (int i = 0; i < NU; ++i) {
                    kc[i] = k[i];
                    vc[i] = v[i];
                }
                const float *const fk = a.kb.scales_dev + at * n_scales, *const fv = a.vb.scales_dev + at * n_scales;
#pragma unroll
                for (int i = 0; i < NU; ++i) {
                    ks[i] = fk[scale_at[i]];
                    vs[i] = fv[scale_at[i]];
                }
            }
        };
        int t = t0 + wave;
        int page_next = -1;
        if (t < t1) {
            fetch(t, page_of(t));
            page_next = page_of(min(t + W, t1 - 1));
        }
        for (bool first = true; t < t1; t += W, first = false) {
            const bool window = t >= page_tiles;             // uniform
            uint32_t known = 0xFFFFFFFFu;                    // keys whose page exists
            half8 kf[T];
            int ek, ev;
            if (!window) {
                float mk = 0.0f, mv = 0.0f;
#pragma unroll
                for (int i = 0; i < NU; ++i) {
                    ks[i] = there ? ks[i] : 0.0f;
                    vs[i] = there ? vs[i] : 0.0f;
                    mk = fmaxf(mk, ks[i]);
                    mv = fmaxf(mv, vs[i]);
                }
                ek = __builtin_amdgcn_readfirstlane(pool_exponent<BITS>(pool_wave_max(mk)));
                ev = max(b.e, __builtin_amdgcn_readfirstlane(pool_exponent<BITS>(pool_wave_max(mv))));
                known = (uint32_t)__ballot(there);
                const float uk = pool_power(-ek), uv = pool_power(-ev);
#pragma unroll
                for (int i = 0; i < NU; ++i) pool_decode16(kc[i], (_Float16)(ks[i] * uk), kf[2 * i], kf[2 * i + 1]);
#pragma unroll
                for (int i = 0; i < NU; ++i) {
                    half8 x, y;
                    pool_decode16(vc[i], (_Float16)(vs[i] * uv), x, y);
                    uint4* const dst = reinterpret_cast<uint4*>(vt + l32 * ROW + 32 * (half * NU + i));
                    dst[0] = __builtin_bit_cast(uint4, x);
                    dst[1] = __builtin_bit_cast(uint4, y);
                }
            } else {
                // the window's tokens: fp16 under a power of two per row already
                const int slot = min((t - page_tiles) * KEYS + l32, tail - 1);
                const long long at = ((long long)(seq * a.heads + head) << a.s.log_R) + slot, of_v = (long long)a.s.n_seq * a.heads << a.s.log_R;
                constexpr float kUp = BITS == 4 ? 4096.0f : 256.0f;          // 2^(15 - AMP): a row's values are below 2^15, not 2^AMP
                there = pool_there(a.s.windows[2 * seq + 1], a.s.n_windows);
                known = there ? 0xFFFFFFFFu : 0u;
                const float fk = there ? a.tail_factor[at] : 0.0f, fv = there ? a.tail_factor[of_v + at] : 0.0f;
                ek = __builtin_amdgcn_readfirstlane(pool_exponent<BITS>(pool_wave_max(fk * kUp)));
                ev = max(b.e, __builtin_amdgcn_readfirstlane(pool_exponent<BITS>(pool_wave_max(fv * kUp))));
                const _Float16 hk = (_Float16)(fk * pool_power(-ek)), hv = (_Float16)(fv * pool_power(-ev));
                const uint4 *const k = reinterpret_cast<const uint4*>(a.tail_rows + at * D) + 2 * half * NU,
                            *const v = reinterpret_cast<const uint4*>(a.tail_rows + (of_v + at) * D) + 2 * half * NU;
#pragma unroll
                for (int s = 0; s < T; ++s) {
                    const uint4 zero = make_uint4(0, 0, 0, 0);
                    kf[s] = pool_times(there ? k[s] : zero, hk);
                    reinterpret_cast<uint4*>(vt + l32 * ROW + 32 * half * NU)[s] = __builtin_bit_cast(uint4, pool_times(there ? v[s] : zero, hv));
                }
            }
            // the next tile goes into the registers that have just been read
            if (t + W < t1) fetch(t + W, page_next);
            page_next = page_of(min(t + 2 * W, t1 - 1));

            floatx16 s[1];
            s[0] = floatx16{0};
#pragma unroll
            for (int i = 0; i < T; ++i) {
                const half8 qi = QLDS ? __builtin_bit_cast(half8, q_lds[i * 64 + lane]) : qf[QLDS ? 0 : i];
                s[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[i], qi, s[0], 0, 0, 0);
            }
            // keys behind the last one of the tile's kind, behind what a row sees, or in pages that do not exist
            const int key0 = window ? q.full + (t - page_tiles) * KEYS : t * KEYS, last = min(row.last, window ? q.length - 1 : q.full - 1) - key0;
            if (__ballot(last < KEYS - 1) || known != 0xFFFFFFFFu) {
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int key = 8 * (v / 4) + 4 * half + v % 4;
                    s[0][v] = key <= last && (known >> key & 1) ? s[0][v] : -__builtin_inff();
                }
            }
            pool_weights<D, 1>(b, s, fmaxf(factor * pool_power(ek), 1.17549435e-38f), ev, first);
            const half8 p[2] = {pool_half8(s[0], 0), pool_half8(s[0], 1)};
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            // transposed reads: the 16 lanes of a quarter take positions 16 (quarter % 2) .. and keys 4 (quarter / 2) ..
            const unsigned char* const vr = vt + (4 * half + (lane & 15) / 4) * ROW + (16 * (lane >> 4 & 1) + 4 * (lane & 3)) * 2;
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    b.sums[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(pool_transposed(vr + 16 * i * ROW + 64 * c, vr + (16 * i + 8) * ROW + 64 * c), p[i],
                                                                       b.sums[c], 0, 0, 0);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        // ---- the wavefronts' sums meet, in the order (0 + 2) + (1 + 3)
        b.den = pool_halves_sum(b.den);
        float* const meet = reinterpret_cast<float*>(lds);
        __syncthreads();
        if (wave >= 2) b.put(meet + (wave - 2) * kPoolPart<D>, lane);
        __syncthreads();
        if (wave < 2) b.add(meet + wave * kPoolPart<D>, lane);
        __syncthreads();
        if (wave == 1) b.put(meet, lane);
        __syncthreads();
        if (wave == 0) b.add(meet, lane);
        __syncthreads();                                     // (the next segment's values go where the sums were)
        if (wave == 0) {
            if (t0 == 0 && t1 == tiles) {
                char* const dst = row.there ? a.out + row.token * a.out_token + row.head * a.out_head : nullptr;
                pool_finish<D>(b, a.out_table, a.out_unscale, dst, a.bf16, lane);
            } else {
                b.put(a.decode_parts + (2LL * w + (at_begin ? 0 : 1)) * kPoolPart<D>, lane);
            }
        }
        unit += t1 - t0;
    }
}

template <int D> pool_attention_kernel_t pick(int bits) { return bits == 8 ? srft_pool_decode_kernel<D, 8> : srft_pool_decode_kernel<D, 4>; }
pool_attention_kernel_t dispatch(int d, int bits) { SRFT_DISPATCH_D(d, pick, bits) }

}  // namespace

pool_attention_kernel_t srft_pick_pool_decode(int d, int bits) { return dispatch(d, bits); }
