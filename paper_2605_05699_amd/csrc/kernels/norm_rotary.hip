// RMS norms of heads with their rotary positions, and the gradients of that.
//   forward   r = 1 / sqrt(mean x^2 + eps), y = turn(x r w)                     (turn: see rotary.hip; the channels from rot on are not turned)
//   backward  g = turn^-1(dy), dx = r (g w - x r^2 mean(g w x)), dw = sum over tokens and heads of g x r
// Sums are fp32; an output is rounded once.
//
// Bound by memory: x is read once and y written once (dy and x, and dx).  8192 tokens, 40 heads of 128, bf16 -> fp16: 168 MB in 36 us, 4.7 TB/s
// (norm and positions one after the other would move 336 MB); fp32, 336 MB, 58 us; the gradients, 252 MB, 47 us, 5.4 TB/s, and 5 more in the second
// kernel.  Rows that are not aligned to four of their elements, or whose pairs do not come in fours, go a channel an access: the same bf16 rows one
// element further on 65 us, rows of 80 channels with 10 pairs 64 (105 MB), their gradients 137 (157 MB).
// A row belongs to 2^log_lanes neighbouring lanes of a wavefront, K units of 2 V channels to each (rotary_rows.h), so that a row's sums meet
// within the wavefront and its values stay in registers between the loads and the stores.  A workgroup has `tokens` tokens with all their heads;
// their angles are computed once, into LDS.
// The weights' gradient: a lane has the same channels of every row, adds its rows up in registers, a workgroup its lanes in LDS, and a second
// kernel the workgroups: always in the same order.
#include "../rotary_rows.h"

namespace {

constexpr int kAngles = 1024;                                // pairs (cos, sin) of a workgroup's tokens
constexpr int kLeastBlocks = 2048;                           // workgroups of a tensor that several tokens in one shall leave
// Workgroups of a tensor whose sums of the weights' gradient meet: two to a compute unit.  8192 tokens with 32 and 8 heads of 128, bf16: 59 us,
// with 256 of them 72, with 1024 62; 1777 with 10 and 5 of 96, fp32: 14.8, 18.4 and 18.3.
constexpr int kGradBlocks = 512;

struct norm_shape {
    int row_units[2];                                        // of a row: those with pairs, all
    int d, rot, pairs_layout, log_lanes;
    float factor, eps;
    unsigned n_tokens;
    const int32_t* positions;
    const double* freq;
};
struct norm_args {
    norm_shape s;
    srft_norm_rows t[SRFT_ROTARY_MAX];
    int tokens[SRFT_ROTARY_MAX], wide[SRFT_ROTARY_MAX];      // tokens of a workgroup at a time; whether weights are read V at a time
};
struct grad_args {
    norm_shape s;
    srft_norm_grad_rows t[SRFT_ROTARY_MAX];
    int tokens[SRFT_ROTARY_MAX], wide[SRFT_ROTARY_MAX], blocks[SRFT_ROTARY_MAX];         // (blocks: workgroups)
    float* parts[SRFT_ROTARY_MAX];                           // [blocks][d] of a tensor whose weights' gradient is asked for, else null
};

// sum over groups of 2^log_lanes neighbouring lanes, in all of them
template <int CTRL> __device__ __forceinline__ float lane_moved(float x) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float sum16(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float sum32(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float row_sum(float x, int log_lanes) {           // (log_lanes is uniform)
    if (log_lanes > 0) x += lane_moved<0xB1>(x);             // quad_perm [1, 0, 3, 2]
    if (log_lanes > 1) x += lane_moved<0x4E>(x);             // quad_perm [2, 3, 0, 1]
    if (log_lanes > 2) x += lane_moved<0x141>(x);            // row_half_mirror
    if (log_lanes > 3) x += lane_moved<0x140>(x);            // row_mirror
    if (log_lanes > 4) x = sum16(x);
    if (log_lanes > 5) x = sum32(x);
    return x;
}
// sum over the groups of lanes of a wavefront: in every lane, that of the lanes with its place in their groups
__device__ __forceinline__ float groups_sum(float x, int log_lanes) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1)
        if (d >> log_lanes) x += __shfl_xor(x, d);
    return x;
}

// the first channels of the two accesses of unit p of a row
struct unit_at { int first, second; };
template <int V>
__device__ __forceinline__ unit_at unit_of(const norm_shape& s, int p) {
    const bool turned = p < s.row_units[0];
    const int c = turned ? (s.pairs_layout ? 2 * V * p : V * p) : s.rot + (p - s.row_units[0]) * 2 * V;
    return {c, turned && !s.pairs_layout ? c + (s.rot >> 1) : c + V};
}
// (f, g) of unit p turned by the angles cs of its token, or back
template <int V, bool BACK>
__device__ __forceinline__ void turn_unit(const norm_shape& s, int p, const float2* cs, float (&f)[V], float (&g)[V]) {
    if (p >= s.row_units[0]) return;
    const auto two = [&](float& a, float& b, float2 t) __attribute__((always_inline)) {
        const float y = BACK ? -t.y : t.y, x = a;
        a = x * t.x - b * y;
        b = x * y + b * t.x;
    };
    if (s.pairs_layout) {
        if constexpr (V > 1) {
#pragma unroll
            for (int i = 0; i < V; i += 2) {
                two(f[i], f[i + 1], cs[V * p + i / 2]);
                two(g[i], g[i + 1], cs[V * p + V / 2 + i / 2]);
            }
        } else {
            two(f[0], g[0], cs[p]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) two(f[i], g[i], cs[V * p + i]);
    }
}
// a lane's weights: of its K units (1 where there are none)
template <class T, int V>
__device__ __forceinline__ void weights_at(const T* w, int wide, float (&x)[V]) {
    if (wide) {
        load<T, V>(x, w);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (float)w[i];
    }
}
template <int V, int K>
__device__ __forceinline__ void weights_of(const norm_shape& s, const void* w, int type, int wide, int lane, float (&a)[K][V], float (&b)[K][V]) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int i = 0; i < V; ++i) a[k][i] = b[k][i] = 1.0f;
        if (!w) continue;                                    // (uniform, as what follows)
        const unit_at at = unit_of<V>(s, min(lane + (k << s.log_lanes), s.row_units[1] - 1));
        const auto both = [&](auto* p) __attribute__((always_inline)) {
            weights_at(p + at.first, wide, a[k]);
            weights_at(p + at.second, wide, b[k]);
        };
        if (type == SRFT_F32) both((const float*)w);
        else if (type == SRFT_F16) both((const _Float16*)w);
        else both((const bf16*)w);
    }
}
// angles of tokens first .. first + n - 1 (a barrier of the caller's behind)
__device__ __forceinline__ void angles_of(const norm_shape& s, unsigned first, int n, float2* cs) {
    const int half = s.rot >> 1;
    for (int i = threadIdx.x; i < n * half; i += blockDim.x) {
        const int token = i / half, pair = i - token * half;
        const float2 t = turn((double)s.positions[first + token] * s.freq[pair]);
        cs[i] = make_float2(t.x * s.factor, t.y * s.factor);
    }
}

// blockIdx.z: the tensor; one workgroup of it for a.tokens tokens (srft_grid).  The first rows and the weights are on their way before the
// angles are computed.
template <class IN, class OUT, int V, int K>
__global__ void __launch_bounds__(256) srft_norm_rotary_kernel(const norm_args a) {
    __shared__ float2 cs[kAngles];
    const norm_shape& s = a.s;
    const srft_norm_rows& t = a.t[blockIdx.z];
    const unsigned tokens = a.tokens[blockIdx.z], first = (blockIdx.y * gridDim.x + blockIdx.x) * tokens;
    if (first >= s.n_tokens) return;                         // (uniform)
    const int n = min(tokens, s.n_tokens - first), lane = threadIdx.x & ((1 << s.log_lanes) - 1), half = s.rot >> 1;
    const int heads = t.x.n_heads, rows = n * heads, step = blockDim.x >> s.log_lanes;
    float f[K][V], g[K][V], wa[K][V], wb[K][V];
    int token = 0, head = 0;
    const auto fetch = [&](int r) __attribute__((always_inline)) {           // (rows past the last: that one again)
        const int row = min(r, rows - 1);
        token = (unsigned)row / (unsigned)heads, head = row - token * heads;
        const IN* const x = (const IN*)t.x.in_dev + (first + token) * t.x.in_token + head * t.x.in_head;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const unit_at at = unit_of<V>(s, min(lane + (k << s.log_lanes), s.row_units[1] - 1));
            load<IN, V>(f[k], x + at.first);
            load<IN, V>(g[k], x + at.second);
        }
    };
    int r = threadIdx.x >> s.log_lanes;
    fetch(r);
    weights_of<V, K>(s, t.weight_dev, t.weight_type, a.wide[blockIdx.z], lane, wa, wb);
    angles_of(s, first, n, cs);
    __syncthreads();
    for (int r0 = 0;;) {
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float here = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) here = fmaf(f[k][i], f[k][i], fmaf(g[k][i], g[k][i], here));
            sum += lane + (k << s.log_lanes) < s.row_units[1] ? here : 0.0f;
        }
        const float scale = 1.0f / sqrtf(row_sum(sum, s.log_lanes) / (float)s.d + s.eps);
        OUT* const y = (OUT*)t.x.out_dev + (first + token) * t.x.out_token + head * t.x.out_head;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int p = lane + (k << s.log_lanes);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                f[k][i] = f[k][i] * scale * wa[k][i];
                g[k][i] = g[k][i] * scale * wb[k][i];
            }
            turn_unit<V, false>(s, p, cs + token * half, f[k], g[k]);
            if (r < rows && p < s.row_units[1]) {
                const unit_at at = unit_of<V>(s, p);
                store<OUT, V>(f[k], y + at.first);
                store<OUT, V>(g[k], y + at.second);
            }
        }
        r0 += step;
        r += step;
        if (r0 >= rows) break;                               // (uniform)
        fetch(r);
    }
}

// blockIdx.y: the tensor; workgroup x of a.blocks takes the tokens a.tokens x .., then a.blocks a.tokens further on, and so on.
template <class IN, class DY, int V, int K>
__global__ void __launch_bounds__(256) srft_norm_rotary_backward_kernel(const grad_args a) {
    __shared__ union {
        float2 cs[kAngles];
        float sums[4][1024];                                 // [wavefront][channel]
    } lds;
    float2* const cs = lds.cs;
    const norm_shape& s = a.s;
    const srft_norm_grad_rows& t = a.t[blockIdx.y];
    const unsigned tokens = a.tokens[blockIdx.y], blocks = a.blocks[blockIdx.y];
    if (blockIdx.x >= blocks) return;                        // (uniform)
    const int lane = threadIdx.x & ((1 << s.log_lanes) - 1), half = s.rot >> 1, heads = t.n_heads, step = blockDim.x >> s.log_lanes;
    float* const part = a.parts[blockIdx.y];
    float f[K][V], g[K][V], u[K][V], v[K][V], wa[K][V], wb[K][V], da[K][V], db[K][V];
    int token = 0, head = 0;
    const auto fetch = [&](unsigned first, int rows, int r) __attribute__((always_inline)) {
        const int row = min(r, rows - 1);
        token = (unsigned)row / (unsigned)heads, head = row - token * heads;
        const IN* const x = (const IN*)t.x_dev + (first + token) * t.x_token + head * t.x_head;
        const DY* const dy = (const DY*)t.dy_dev + (first + token) * t.dy_token + head * t.dy_head;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const unit_at at = unit_of<V>(s, min(lane + (k << s.log_lanes), s.row_units[1] - 1));
            load<IN, V>(f[k], x + at.first);
            load<IN, V>(g[k], x + at.second);
            load<DY, V>(u[k], dy + at.first);
            load<DY, V>(v[k], dy + at.second);
        }
    };
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) da[k][i] = db[k][i] = 0.0f;
    for (unsigned first = blockIdx.x * tokens; first < s.n_tokens; first += blocks * tokens) {
        const int n = min(tokens, s.n_tokens - first), rows = n * heads;
        int r = threadIdx.x >> s.log_lanes;
        fetch(first, rows, r);
        if (first == blockIdx.x * tokens) weights_of<V, K>(s, t.weight_dev, t.weight_type, a.wide[blockIdx.y], lane, wa, wb);
        __syncthreads();                                     // (the angles before have been read)
        angles_of(s, first, n, cs);
        __syncthreads();
        for (int r0 = 0;;) {
            float sum = 0.0f, both = 0.0f;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int p = lane + (k << s.log_lanes);
                turn_unit<V, true>(s, p, cs + token * half, u[k], v[k]);
                float squares = 0.0f, products = 0.0f;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    squares = fmaf(f[k][i], f[k][i], fmaf(g[k][i], g[k][i], squares));
                    products = fmaf(u[k][i] * wa[k][i], f[k][i], fmaf(v[k][i] * wb[k][i], g[k][i], products));
                }
                sum += p < s.row_units[1] ? squares : 0.0f;
                both += p < s.row_units[1] ? products : 0.0f;
            }
            const float scale = 1.0f / sqrtf(row_sum(sum, s.log_lanes) / (float)s.d + s.eps);
            const float along = row_sum(both, s.log_lanes) / (float)s.d * scale * scale;
            IN* const dx = (IN*)t.dx_dev + (first + token) * t.dx_token + head * t.dx_head;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int p = lane + (k << s.log_lanes);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    // (rows past the last are it again: they count for nothing)
                    da[k][i] += r < rows ? u[k][i] * (f[k][i] * scale) : 0.0f;
                    db[k][i] += r < rows ? v[k][i] * (g[k][i] * scale) : 0.0f;
                    f[k][i] = scale * (u[k][i] * wa[k][i] - f[k][i] * along);
                    g[k][i] = scale * (v[k][i] * wb[k][i] - g[k][i] * along);
                }
                if (r < rows && p < s.row_units[1]) {
                    const unit_at at = unit_of<V>(s, p);
                    store<IN, V>(f[k], dx + at.first);
                    store<IN, V>(g[k], dx + at.second);
                }
            }
            r0 += step;
            r += step;
            if (r0 >= rows) break;                           // (uniform)
            fetch(first, rows, r);
        }
    }
    if (!part) return;                                       // (uniform)
    // ---- the workgroup's sums: a wavefront's lanes with the same channels, then its wavefronts
    __syncthreads();                                         // (the last angles have been read)
    float (*const sums)[1024] = lds.sums;
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int p = lane + (k << s.log_lanes);
        const unit_at at = unit_of<V>(s, min(p, s.row_units[1] - 1));
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float x = groups_sum(da[k][i], s.log_lanes), y = groups_sum(db[k][i], s.log_lanes);
            if ((int)(threadIdx.x & 63) < 1 << s.log_lanes && p < s.row_units[1]) {
                sums[wave][at.first + i] = x;
                sums[wave][at.second + i] = y;
            }
        }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < s.d; c += blockDim.x) {
        float x = sums[0][c];
        for (int w = 1; w < waves; ++w) x += sums[w][c];
        part[(long long)blockIdx.x * s.d + c] = x;
    }
}

// dweight of a tensor (blockIdx.y), 16 channels a workgroup: the sum of its parts, 16 threads a channel, in the order of the parts.
struct grad_sums {
    const float* parts[SRFT_ROTARY_MAX];
    float* dweight[SRFT_ROTARY_MAX];
    int blocks[SRFT_ROTARY_MAX];
};
__global__ void __launch_bounds__(1024) srft_norm_rotary_sums_kernel(const grad_sums a, int d) {
    constexpr int TEAMS = 64;
    __shared__ float sums[TEAMS][17];
    const float* const parts = a.parts[blockIdx.y];
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), from = threadIdx.x >> 4, blocks = a.blocks[blockIdx.y];
    float x[kGradBlocks / TEAMS];
#pragma unroll
    for (int i = 0; i < kGradBlocks / TEAMS; ++i) {          // (all on their way together)
        const int b = from + TEAMS * i;
        x[i] = b < blocks ? parts[(long long)b * d + min(c, d - 1)] : 0.0f;
    }
    float sum = x[0];
#pragma unroll
    for (int i = 1; i < kGradBlocks / TEAMS; ++i) sum += x[i];
    sums[from][threadIdx.x & 15] = sum;
    __syncthreads();
    if (from > 0 || c >= d) return;
    float all = 0.0f;
    for (int i = 0; i < TEAMS; ++i) all += sums[i][threadIdx.x & 15];
    a.dweight[blockIdx.y][c] = all;
}

typedef void (*norm_kernel_t)(const norm_args);
typedef void (*grad_kernel_t)(const grad_args);
// the instance for V pairs a thread and K units a lane
template <class A, class B> norm_kernel_t norm_of(int v, int k) {
    if (v == 8) return srft_norm_rotary_kernel<A, B, 8, 1>;
    if (v == 4) return k == 1 ? srft_norm_rotary_kernel<A, B, 4, 1> : srft_norm_rotary_kernel<A, B, 4, 2>;
    return k == 1 ? srft_norm_rotary_kernel<A, B, 1, 1> : srft_norm_rotary_kernel<A, B, 1, 8>;
}
template <class A, class B> grad_kernel_t grad_of(int v, int k) {
    if (v == 8) return srft_norm_rotary_backward_kernel<A, B, 8, 1>;
    if (v == 4) return k == 1 ? srft_norm_rotary_backward_kernel<A, B, 4, 1> : srft_norm_rotary_backward_kernel<A, B, 4, 2>;
    return k == 1 ? srft_norm_rotary_backward_kernel<A, B, 1, 1> : srft_norm_rotary_backward_kernel<A, B, 1, 8>;
}
template <class A> norm_kernel_t norm_of(int b, int v, int k) {
    return b == SRFT_F32 ? norm_of<A, float>(v, k) : b == SRFT_F16 ? norm_of<A, _Float16>(v, k) : norm_of<A, bf16>(v, k);
}
template <class A> grad_kernel_t grad_of(int b, int v, int k) {
    return b == SRFT_F32 ? grad_of<A, float>(v, k) : b == SRFT_F16 ? grad_of<A, _Float16>(v, k) : grad_of<A, bf16>(v, k);
}
norm_kernel_t norm_of(int a, int b, int v, int k) {
    return a == SRFT_F32 ? norm_of<float>(b, v, k) : a == SRFT_F16 ? norm_of<_Float16>(b, v, k) : norm_of<bf16>(b, v, k);
}
grad_kernel_t grad_of(int a, int b, int v, int k) {
    return a == SRFT_F32 ? grad_of<float>(b, v, k) : a == SRFT_F16 ? grad_of<_Float16>(b, v, k) : grad_of<bf16>(b, v, k);
}

// ---- checks that both calls make
int check(int count, const void* rows, int64_t n_tokens, int d, int rot, int layout, double eps) {
    if (count < 0 || count > SRFT_ROTARY_MAX || n_tokens < 0 || n_tokens >= (1LL << 31) || d < 2 || d > 1024 || d % 2 != 0 || rot < 0 || rot > d || rot % 2 != 0 ||
        (layout != SRFT_ROTARY_HALF && layout != SRFT_ROTARY_PAIRS) || !(eps >= 1.17549435e-38 && eps <= 3.4e38))
        return SRFT_ERR_BAD_N;
    return count > 0 && !rows ? SRFT_ERR_NULL : SRFT_OK;
}
bool rows_fit(int64_t n_tokens, int heads, int d) { return heads >= 1 && n_tokens * heads < (1LL << 31) && (int64_t)heads * d < (1LL << 31); }
int check_angles(const int32_t* positions_dev, const double* freq_dev, int rot) {
    if (!positions_dev || (rot > 0 && !freq_dev)) return SRFT_ERR_NULL;
    return srft_aligned(positions_dev, 4) && srft_aligned(freq_dev, 8) ? SRFT_OK : SRFT_ERR_ALIGN;
}
// Two tensors at one address: a lane writes what it alone has read, if their rows are the same ones.
bool apart(const void* a, int a_type, int64_t a_token, int64_t a_head, const void* b, int b_type, int64_t b_token, int64_t b_head, int64_t n_tokens, int heads) {
    return a != b || (a_type == b_type && (n_tokens == 1 || a_token == b_token) && (heads == 1 || a_head == b_head));
}

// The widest V that fits all of `ok`'s tensors.
template <class F>
int width_of(int rot, int d, bool all_f32, F ok) {
    const int most = all_f32 ? 4 : 8;
    return fits_row(rot, d, most) && ok(most) ? most : fits_row(rot, d, 4) && ok(4) ? 4 : 1;
}
// a row's units and lanes; returns K
int split_rows(norm_shape& s, int v) {
    s.row_units[0] = s.rot / 2 / v;
    s.row_units[1] = s.row_units[0] + (s.d - s.rot) / (2 * v);
    s.log_lanes = 0;
    while (s.log_lanes < 6 && (1 << s.log_lanes) < s.row_units[1]) ++s.log_lanes;
    return (s.row_units[1] + (1 << s.log_lanes) - 1) >> s.log_lanes;
}
// Tokens of a workgroup of a tensor: up to four rows a lane, up to `most`, and as many as the LDS has angles for.
int tokens_of(const norm_shape& s, int heads, int64_t most) {
    const int64_t rows = 4 * (256 >> s.log_lanes), fit = s.rot > 0 ? kAngles / (s.rot / 2) : kAngles;
    return (int)std::max<int64_t>(1, std::min({rows / heads, fit, most}));
}
int threads_of(const norm_shape& s, int tokens, int heads) { return (int)std::min<int64_t>(256, (((int64_t)tokens * heads << s.log_lanes) + 63) / 64 * 64); }
}  // namespace

extern "C" {

int srft_norm_rotary(const srft_norm_rows* rows, int count, int64_t n_tokens, int d, int rot, int layout, const int32_t* positions_dev,
                     const double* freq_dev, double factor, double eps, void* hip_stream) {
    int rc = check(count, rows, n_tokens, d, rot, layout, eps);
    if (rc != SRFT_OK) return rc;
    for (int i = 0; i < count; ++i) {
        const srft_rotary_rows& x = rows[i].x;
        if (!rows_fit(n_tokens, x.n_heads, d) || !type_known(x.in_type) || !type_known(x.out_type) || !type_known(rows[i].weight_type) || x.reserved != 0 ||
            rows[i].reserved != 0)
            return SRFT_ERR_BAD_N;
    }
    if (count == 0 || n_tokens == 0) return SRFT_OK;
    rc = check_angles(positions_dev, freq_dev, rot);
    if (rc != SRFT_OK) return rc;
    for (int i = 0; i < count; ++i) {
        const srft_rotary_rows& x = rows[i].x;
        if (!x.in_dev || !x.out_dev) return SRFT_ERR_NULL;
        if (!srft_aligned(x.in_dev, type_bytes(x.in_type)) || !srft_aligned(x.out_dev, type_bytes(x.out_type)) ||
            !srft_aligned(rows[i].weight_dev, type_bytes(rows[i].weight_type)))
            return SRFT_ERR_ALIGN;
        if (!apart(x.in_dev, x.in_type, x.in_token, x.in_head, x.out_dev, x.out_type, x.out_token, x.out_head, n_tokens, x.n_heads)) return SRFT_ERR_BAD_N;
    }
    const auto width = [&](const srft_rotary_rows& x) {
        return width_of(rot, d, x.in_type == SRFT_F32 && x.out_type == SRFT_F32, [&](int v) {
            return fits(x.in_dev, x.in_token, x.in_head, x.in_type, v) && fits(x.out_dev, x.out_token, x.out_head, x.out_type, v);
        });
    };
    // tensors of one pair of types and one width share a launch
    bool done[SRFT_ROTARY_MAX] = {};
    for (int i = 0; i < count; ++i) {
        if (done[i]) continue;
        const srft_rotary_rows& x = rows[i].x;
        const int v = width(x);
        norm_args a = {};
        a.s = {{0, 0}, d, rot, layout == SRFT_ROTARY_PAIRS, 0, (float)factor, (float)eps, (unsigned)n_tokens, positions_dev, freq_dev};
        const int k = split_rows(a.s, v);
        int n = 0, threads = 64;
        int64_t blocks = 0;
        for (int j = i; j < count; ++j) {
            const srft_rotary_rows& y = rows[j].x;
            if (done[j] || y.in_type != x.in_type || y.out_type != x.out_type || width(y) != v) continue;
            done[j] = true;
            a.t[n] = rows[j];
            a.wide[n] = srft_aligned(rows[j].weight_dev, std::min(16, v * type_bytes(rows[j].weight_type)));
            a.tokens[n] = tokens_of(a.s, y.n_heads, n_tokens / kLeastBlocks);
            threads = std::max(threads, threads_of(a.s, a.tokens[n], y.n_heads));
            blocks = std::max(blocks, (n_tokens + a.tokens[n] - 1) / a.tokens[n]);
            ++n;
        }
        dim3 grid = srft_grid(blocks);
        grid.z = (unsigned)n;
        rc = srft_launch(norm_of(x.in_type, x.out_type, v, k), grid, threads, (hipStream_t)hip_stream, a);
        if (rc != SRFT_OK) return rc;
    }
    return SRFT_OK;
}

int64_t srft_norm_rotary_backward_workspace_bytes(int count, int d) {
    if (count < 0 || count > SRFT_ROTARY_MAX || d < 2 || d > 1024 || d % 2 != 0) return SRFT_ERR_BAD_N;
    return 4LL * count * kGradBlocks * d;
}

int srft_norm_rotary_backward(const srft_norm_grad_rows* rows, int count, int64_t n_tokens, int d, int rot, int layout, const int32_t* positions_dev,
                              const double* freq_dev, double factor, double eps, void* workspace_dev, void* hip_stream) {
    int rc = check(count, rows, n_tokens, d, rot, layout, eps);
    if (rc != SRFT_OK) return rc;
    bool sums = false;
    for (int i = 0; i < count; ++i) {
        const srft_norm_grad_rows& x = rows[i];
        if (!rows_fit(n_tokens, x.n_heads, d) || !type_known(x.x_type) || !type_known(x.dy_type) || !type_known(x.weight_type)) return SRFT_ERR_BAD_N;
        for (int k = 0; k < i; ++k)
            if (x.dweight_dev && x.dweight_dev == rows[k].dweight_dev) return SRFT_ERR_BAD_N;
        sums |= x.dweight_dev != nullptr;
    }
    if (count == 0 || (n_tokens == 0 && !sums)) return SRFT_OK;
    if (n_tokens > 0) {
        rc = check_angles(positions_dev, freq_dev, rot);
        if (rc != SRFT_OK) return rc;
    }
    if (sums && !workspace_dev) return SRFT_ERR_NULL;
    if (!srft_aligned(workspace_dev, 16)) return SRFT_ERR_ALIGN;
    for (int i = 0; i < count; ++i) {
        const srft_norm_grad_rows& x = rows[i];
        if (!srft_aligned(x.dweight_dev, 4)) return SRFT_ERR_ALIGN;
        if (n_tokens == 0) continue;
        if (!x.x_dev || !x.dy_dev || !x.dx_dev) return SRFT_ERR_NULL;
        if (!srft_aligned(x.x_dev, type_bytes(x.x_type)) || !srft_aligned(x.dx_dev, type_bytes(x.x_type)) || !srft_aligned(x.dy_dev, type_bytes(x.dy_type)) ||
            !srft_aligned(x.weight_dev, type_bytes(x.weight_type)))
            return SRFT_ERR_ALIGN;
        if (!apart(x.dx_dev, x.x_type, x.dx_token, x.dx_head, x.x_dev, x.x_type, x.x_token, x.x_head, n_tokens, x.n_heads) ||
            !apart(x.dx_dev, x.x_type, x.dx_token, x.dx_head, x.dy_dev, x.dy_type, x.dy_token, x.dy_head, n_tokens, x.n_heads))
            return SRFT_ERR_BAD_N;
    }
    const hipStream_t st = (hipStream_t)hip_stream;
    const auto width = [&](const srft_norm_grad_rows& x) {
        return width_of(rot, d, x.x_type == SRFT_F32 && x.dy_type == SRFT_F32, [&](int v) {
            return fits(x.x_dev, x.x_token, x.x_head, x.x_type, v) && fits(x.dx_dev, x.dx_token, x.dx_head, x.x_type, v) &&
                   fits(x.dy_dev, x.dy_token, x.dy_head, x.dy_type, v);
        });
    };
    const auto part = [&](int i) { return (float*)workspace_dev + (int64_t)i * kGradBlocks * d; };
    int part_blocks[SRFT_ROTARY_MAX] = {};
    bool done[SRFT_ROTARY_MAX] = {};
    for (int i = 0; i < count && n_tokens > 0; ++i) {
        if (done[i]) continue;
        const srft_norm_grad_rows& x = rows[i];
        const int v = width(x);
        grad_args a = {};
        a.s = {{0, 0}, d, rot, layout == SRFT_ROTARY_PAIRS, 0, (float)factor, (float)eps, (unsigned)n_tokens, positions_dev, freq_dev};
        const int k = split_rows(a.s, v);
        int n = 0, threads = 64, blocks = 0;
        for (int j = i; j < count; ++j) {
            const srft_norm_grad_rows& y = rows[j];
            if (done[j] || y.x_type != x.x_type || y.dy_type != x.dy_type || width(y) != v) continue;
            done[j] = true;
            a.t[n] = y;
            a.wide[n] = srft_aligned(y.weight_dev, std::min(16, v * type_bytes(y.weight_type)));
            a.tokens[n] = tokens_of(a.s, y.n_heads, (n_tokens + kGradBlocks - 1) / kGradBlocks);
            a.blocks[n] = part_blocks[j] = (int)std::min<int64_t>((n_tokens + a.tokens[n] - 1) / a.tokens[n], kGradBlocks);
            a.parts[n] = y.dweight_dev ? part(j) : nullptr;
            threads = std::max(threads, threads_of(a.s, a.tokens[n], y.n_heads));
            blocks = std::max(blocks, a.blocks[n]);
            ++n;
        }
        rc = srft_launch(grad_of(x.x_type, x.dy_type, v, k), dim3((unsigned)blocks, (unsigned)n), threads, st, a);
        if (rc != SRFT_OK) return rc;
    }
    if (!sums) return SRFT_OK;
    grad_sums g = {};
    int n = 0;
    for (int i = 0; i < count; ++i)
        if (rows[i].dweight_dev) {
            g.parts[n] = part(i);
            g.blocks[n] = part_blocks[i];
            g.dweight[n++] = rows[i].dweight_dev;
        }
    return srft_launch(srft_norm_rotary_sums_kernel, dim3((unsigned)((d + 15) / 16), (unsigned)n), 1024, st, g, d);
}

}  // extern "C"
