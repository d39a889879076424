// rotary_rows.h -- rows of heads and their angles: what kernels/rotary.hip and kernels/norm_rotary.hip share.
//
// A thread moves V pairs of channels at a time, or 2 V of the channels behind the pairs ("a unit"): two accesses of V channels.
#ifndef SRFT_ROTARY_ROWS_H
#define SRFT_ROTARY_ROWS_H
#include <algorithm>

#include "common.h"

namespace {

typedef __bf16 bf16;
template <class T, int V> struct alignas(sizeof(T) * V <= 16 ? sizeof(T) * V : 16) wide { T v[V]; };

template <class T, int V>
__device__ __forceinline__ void load(float (&x)[V], const T* p) {
    const wide<T, V> w = *reinterpret_cast<const wide<T, V>*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = (float)w.v[i];
}
template <class T, int V>
__device__ __forceinline__ void store(const float (&x)[V], T* p) {
    wide<T, V> w;
#pragma unroll
    for (int i = 0; i < V; ++i) w.v[i] = (T)x[i];
    *reinterpret_cast<wide<T, V>*>(p) = w;
}
// cos and sin of t, a position times radians per token
__device__ __forceinline__ float2 turn(double t) {
    const double n = rint(t * 0.15915494309189533577);
    double r = fma(n, -6.283185307179586232, t);                 // 2 pi as a sum of two numbers
    r = fma(n, -2.4492935982947063545e-16, r);
    float s, c;
    sincosf((float)r, &s, &c);
    return make_float2(c, s);
}

inline int type_bytes(int t) { return t == SRFT_F32 ? 4 : 2; }
inline bool type_known(int t) { return t == SRFT_F32 || t == SRFT_F16 || t == SRFT_BF16; }

// Whether threads can move V channels at once: whole vectors of a row, and, of each tensor, from and to addresses of a vector's alignment.
inline bool fits_row(int rot, int d, int v) { return rot / 2 % v == 0 && (d - rot) % (2 * v) == 0; }
inline bool fits(const void* p, int64_t token, int64_t head, int type, int v) {
    const int64_t bytes = std::min(16, v * type_bytes(type));
    return srft_aligned(p, bytes) && token * type_bytes(type) % bytes == 0 && head * type_bytes(type) % bytes == 0;
}

}  // namespace

#endif  // SRFT_ROTARY_ROWS_H
