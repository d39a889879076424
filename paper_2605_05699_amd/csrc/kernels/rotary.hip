// Rotary positions: (a, b) -> factor (a cos t - b sin t, a sin t + b cos t) for pairs of channels, t = position * frequency.
//
// Bound by memory: a row is read once and written once, and a pair costs four multiplications.  What has to be kept out of the way
// is the angles: t grows with the position, so it is formed and brought into one turn in 64 bits (at position 10^6 an fp32 product is off
// by 0.03 radians), and a sine and a cosine are some 40 instructions.  A workgroup therefore takes one token with all its heads, of
// all tensors of the call: the token's rot / 2 angles are computed once into LDS, while the first rows are on their way, and serve every
// head (of 40 heads at d = 128 that leaves 1.6 sine-cosine pairs a thread).  A thread moves V pairs, or V of the channels behind
// them twice: two 16-byte loads and stores of 16-bit values.
// 168 MB in 33.7 us, 5.0 TB/s (8192 tokens, 40 heads of 128 channels; a copy of this card gets 5.5).
#include "../rotary_rows.h"

namespace {

struct rotary_args {
    srft_rotary_rows t[SRFT_ROTARY_MAX];
    int row_units[2];                       // of a row: those with pairs, all
    int rot, pairs_layout;
    float factor, sign;
    const int32_t* positions;
    const double* freq;
};

// V: pairs of a thread; IN, OUT: types.  One workgroup per token (srft_grid); LDS: rot / 2 pairs (cos, sin) times factor.
template <class IN, class OUT, int V>
__device__ __forceinline__ void rows_of_token(const rotary_args& a, const srft_rotary_rows& t, long long token, const float2* cs) {
    const IN* const in = (const IN*)t.in_dev + token * t.in_token;
    OUT* const out = (OUT*)t.out_dev + token * t.out_token;
    const int half = a.rot >> 1;
    for (int u = threadIdx.x; u < t.n_heads * a.row_units[1]; u += blockDim.x) {
        const int head = (unsigned)u / (unsigned)a.row_units[1], p = u - head * a.row_units[1];
        const IN* const x = in + head * t.in_head;
        OUT* const y = out + head * t.out_head;
        float f[V], g[V];
        if (p >= a.row_units[0]) {                              // behind the turned part
            const int c = a.rot + (p - a.row_units[0]) * 2 * V;
            load<IN, V>(f, x + c);
            load<IN, V>(g, x + c + V);
            store<OUT, V>(f, y + c);
            store<OUT, V>(g, y + c + V);
        } else if (a.pairs_layout) {
            const int c = 2 * V * p;
            load<IN, V>(f, x + c);
            load<IN, V>(g, x + c + V);
            if constexpr (V > 1) {
#pragma unroll
                for (int i = 0; i < V; i += 2) {
                    const float2 l = cs[V * p + i / 2], h = cs[V * p + V / 2 + i / 2];
                    const float f0 = f[i], g0 = g[i];
                    f[i] = f0 * l.x - f[i + 1] * l.y;
                    f[i + 1] = f0 * l.y + f[i + 1] * l.x;
                    g[i] = g0 * h.x - g[i + 1] * h.y;
                    g[i + 1] = g0 * h.y + g[i + 1] * h.x;
                }
            } else {
                const float2 l = cs[p];
                const float f0 = f[0];
                f[0] = f0 * l.x - g[0] * l.y;
                g[0] = f0 * l.y + g[0] * l.x;
            }
            store<OUT, V>(f, y + c);
            store<OUT, V>(g, y + c + V);
        } else {
            const int c = V * p;
            load<IN, V>(f, x + c);
            load<IN, V>(g, x + c + half);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float2 l = cs[c + i];
                const float f0 = f[i];
                f[i] = f0 * l.x - g[i] * l.y;
                g[i] = f0 * l.y + g[i] * l.x;
            }
            store<OUT, V>(f, y + c);
            store<OUT, V>(g, y + c + half);
        }
    }
}

template <class IN, class OUT, int V>
__global__ void __launch_bounds__(256) srft_rotary_kernel(const rotary_args a, int count, unsigned n_tokens) {
    __shared__ float2 cs[512];
    const long long token = blockIdx.y * gridDim.x + blockIdx.x;
    if (token >= n_tokens) return;                           // (uniform)
    const double pos = (double)a.positions[token];
    for (int i = threadIdx.x; i < a.rot / 2; i += blockDim.x) {
        const float2 t = turn(pos * a.freq[i]);
        cs[i] = make_float2(t.x * a.factor, t.y * a.sign);
    }
    __syncthreads();
    for (int k = 0; k < count; ++k) rows_of_token<IN, OUT, V>(a, a.t[k], token, cs);
}

typedef void (*rotary_kernel_t)(const rotary_args, int, unsigned);
template <class IN, class OUT> rotary_kernel_t pick(int v) {
    if (v == 8) return srft_rotary_kernel<IN, OUT, 8>;
    return v == 4 ? srft_rotary_kernel<IN, OUT, 4> : srft_rotary_kernel<IN, OUT, 1>;
}
template <class IN> rotary_kernel_t pick(int out, int v) {
    return out == SRFT_F32 ? pick<IN, float>(v) : out == SRFT_F16 ? pick<IN, _Float16>(v) : pick<IN, bf16>(v);
}
bool fits(const srft_rotary_rows& r, int rot, int d, int v) {
    return fits_row(rot, d, v) && fits(r.in_dev, r.in_token, r.in_head, r.in_type, v) && fits(r.out_dev, r.out_token, r.out_head, r.out_type, v);
}

}  // namespace

extern "C" int srft_rotary(const srft_rotary_rows* rows, int count, int64_t n_tokens, int d, int rot, int layout,
                           const int32_t* positions_dev, const double* freq_dev, double factor, int inverse, void* hip_stream) {
    if (count < 0 || count > SRFT_ROTARY_MAX || n_tokens < 0 || n_tokens >= (1LL << 31) || d < 2 || d > 1024 || d % 2 != 0 || rot < 0 || rot > d || rot % 2 != 0 ||
        (layout != SRFT_ROTARY_HALF && layout != SRFT_ROTARY_PAIRS))
        return SRFT_ERR_BAD_N;
    if (count > 0 && !rows) return SRFT_ERR_NULL;
    for (int i = 0; i < count; ++i)
        if (rows[i].n_heads < 1 || n_tokens * rows[i].n_heads >= (1LL << 31) || (int64_t)rows[i].n_heads * d >= (1LL << 31) || !type_known(rows[i].in_type) || !type_known(rows[i].out_type) ||
            rows[i].reserved != 0)
            return SRFT_ERR_BAD_N;
    if (count == 0 || n_tokens == 0) return SRFT_OK;
    if (!positions_dev || (rot > 0 && !freq_dev)) return SRFT_ERR_NULL;
    if (!srft_aligned(positions_dev, 4) || !srft_aligned(freq_dev, 8)) return SRFT_ERR_ALIGN;
    for (int i = 0; i < count; ++i) {
        if (!rows[i].in_dev || !rows[i].out_dev) return SRFT_ERR_NULL;
        if (!srft_aligned(rows[i].in_dev, type_bytes(rows[i].in_type)) || !srft_aligned(rows[i].out_dev, type_bytes(rows[i].out_type)))
            return SRFT_ERR_ALIGN;
        // in place a thread writes where it has read, and nowhere else
        if (rows[i].in_dev == rows[i].out_dev && (rows[i].in_type != rows[i].out_type || (n_tokens > 1 && rows[i].in_token != rows[i].out_token) ||
                                                  (rows[i].n_heads > 1 && rows[i].in_head != rows[i].out_head)))
            return SRFT_ERR_BAD_N;
    }
    // tensors of one pair of types and one width share a launch
    bool done[SRFT_ROTARY_MAX] = {};
    const bool pairs = layout == SRFT_ROTARY_PAIRS;
    const auto width = [&](const srft_rotary_rows& r) {
        const int most = r.in_type == SRFT_F32 && r.out_type == SRFT_F32 ? 4 : 8;
        return fits(r, rot, d, most) ? most : fits(r, rot, d, 4) ? 4 : 1;
    };
    for (int i = 0; i < count; ++i) {
        if (done[i]) continue;
        rotary_args a = {};
        const int v = width(rows[i]);
        int n = 0;
        long long units = 0;
        for (int k = i; k < count; ++k) {
            if (done[k] || rows[k].in_type != rows[i].in_type || rows[k].out_type != rows[i].out_type || width(rows[k]) != v) continue;
            done[k] = true;
            a.t[n++] = rows[k];
            units += rows[k].n_heads;
        }
        a.row_units[0] = rot / 2 / v;
        a.row_units[1] = a.row_units[0] + (d - rot) / (2 * v);
        a.rot = rot;
        a.pairs_layout = pairs;
        a.factor = (float)factor;
        a.sign = (float)(inverse ? -factor : factor);
        a.positions = positions_dev;
        a.freq = freq_dev;
        const rotary_kernel_t kernel = rows[i].in_type == SRFT_F32 ? pick<float>(rows[i].out_type, v)
                                       : rows[i].in_type == SRFT_F16 ? pick<_Float16>(rows[i].out_type, v)
                                                                     : pick<bf16>(rows[i].out_type, v);
        const int threads = (int)std::min(256LL, (units * a.row_units[1] + 63) / 64 * 64);
        const int rc = srft_launch(kernel, srft_grid(n_tokens), threads, (hipStream_t)hip_stream, a, n, (unsigned)n_tokens);
        if (rc != SRFT_OK) return rc;
    }
    return SRFT_OK;
}
