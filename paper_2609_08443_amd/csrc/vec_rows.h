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

// Column sums of parts [n][C] fp32, in a fixed order: workgroup b does columns 16 b .. 16 b + 15, four threads
// side by side and 64 groups of them down the parts, whose sums are added up through LDS.  put(column, sum).
constexpr int kSumColumns = 16;
template <typename F>
__device__ inline void sum_parts(const float* __restrict__ parts, int n, int64_t C, F put) {
    __shared__ float acc[64][kSumColumns + 1];
    const int64_t c = (int64_t)blockIdx.x * kSumColumns + 4 * (threadIdx.x & 3);
    const int group = threadIdx.x >> 2;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (c + 4 <= C && C % 4 == 0) {
#pragma unroll 8
        for (int i = group; i < n; i += 64) {
            const float4 x = *reinterpret_cast<const float4*>(parts + i * C + c);
            s[0] += x.x; s[1] += x.y; s[2] += x.z; s[3] += x.w;
        }
    } else {
#pragma unroll 4
        for (int i = group; i < n; i += 64)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < C) s[e] += parts[i * C + c + e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[group][4 * (threadIdx.x & 3) + e] = s[e];
    __syncthreads();
    // 16 threads a column, four groups each, then across them
    const int col = threadIdx.x >> 4, g = threadIdx.x & 15;
    float v = (acc[g][col] + acc[g + 16][col]) + (acc[g + 32][col] + acc[g + 48][col]);
#pragma unroll
    for (int o = 1; o < 16; o *= 2) v += __shfl_xor(v, o, 64);
    const int64_t to = (int64_t)blockIdx.x * kSumColumns + col;
    if (g == 0 && to < C) put(to, v);
}

}  // namespace vec
}  // namespace sa
