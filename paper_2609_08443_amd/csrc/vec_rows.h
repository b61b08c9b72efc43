// Pieces of rows of any width and alignment, as fp32: 16-byte loads and stores at whatever
// alignment the element type allows, one by one where the row ends.
#pragma once

#include "tile_ops.h"

namespace sa {
namespace vec {

template <typename T>
struct Piece {
    static constexpr int N = 16 / sizeof(T);
    T v[N];
} __attribute__((packed, aligned(2)));

__device__ inline float value(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ inline float value(float x) { return x; }
__device__ inline void store(uint16_t* p, float v) { *p = tile::to_bf16(v); }
__device__ inline void store(float* p, float v) { *p = v; }

// N values (whole pieces) of a row of D from column c on; zeros past D
template <int N, typename T>
__device__ inline void load(const T* p, int c, int D, float* o) {
    constexpr int P = Piece<T>::N;
    static_assert(N % P == 0, "whole pieces");
    if (c + N <= D) {
#pragma unroll
        for (int i = 0; i < N; i += P) {
            Piece<T> x;
            __builtin_memcpy(&x, p + c + i, 16);
#pragma unroll
            for (int e = 0; e < P; ++e) o[i + e] = value(x.v[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) o[e] = c + e < D ? value(p[c + e]) : 0.f;
    }
}
__device__ inline void pack(const float* v, Piece<uint16_t>* x) {
    const uint32_t w[4] = {tile::pack_bf16x2(v[0], v[1]), tile::pack_bf16x2(v[2], v[3]), tile::pack_bf16x2(v[4], v[5]),
                           tile::pack_bf16x2(v[6], v[7])};
    __builtin_memcpy(x, w, 16);
}
__device__ inline void pack(const float* v, Piece<float>* x) { __builtin_memcpy(x, v, 16); }
template <int N, typename T>
__device__ inline void store(T* p, int c, int D, const float* v) {
    constexpr int P = Piece<T>::N;
    if (c + N <= D) {
#pragma unroll
        for (int i = 0; i < N; i += P) {
            Piece<T> x;
            pack(v + i, &x);
            __builtin_memcpy(p + c + i, &x, 16);
        }
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (c + e < D) store(p + c + e, v[e]);
    }
}

}  // namespace vec
}  // namespace sa
