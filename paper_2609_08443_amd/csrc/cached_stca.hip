// STCA over the sketch cache (sa_stca_cached_fwd / sa_stca_cached_bwd): the small kernels around
// the weights' gradients, and the row kernels of the path in separate products, in which
// the cached sketches are read into the workspace and the products run on the batched GEMM.
//
// A row is the k fp32 logits of one (user, target, head), of which the user's first n
// count; one wave per row.  Weights past n are zero, and all of them where n = 0.
#include <type_traits>

#include "cache.h"

namespace sa {

namespace {

__device__ inline float wave_max(float v) {
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) v = fmaxf(v, __shfl_xor(v, k, 64));
    return v;
}
__device__ inline float wave_sum(float v) {
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) v += __shfl_xor(v, k, 64);
    return v;
}
template <bool BF>
__device__ inline void put(void* p, int64_t i, float v) {
    if constexpr (BF) reinterpret_cast<uint16_t*>(p)[i] = tile::to_bf16(v);
    else reinterpret_cast<float*>(p)[i] = v;
}

// lse = log sum_j exp(s_j), -inf for no rows; alpha_j = exp(s_j - max) / sum
template <bool BF>
__global__ __launch_bounds__(256) void cached_softmax_kernel(CacheView c, const float* __restrict__ S, int64_t rows,
                                                             int32_t Rh, void* __restrict__ alpha,
                                                             float* __restrict__ lse) {
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    int32_t n;
    cache_slot(c, row / Rh, &n);
    const int lane = threadIdx.x & 63;
    const float* s = S + row * c.k;
    float mx = -INFINITY;
    for (int j = lane; j < n; j += 64) mx = fmaxf(mx, s[j]);
    mx = wave_max(mx);
    if (mx == -INFINITY) mx = 0.f;
    float z = 0.f;
    for (int j = lane; j < n; j += 64) z += __expf(s[j] - mx);
    z = wave_sum(z);
    const float inv = n ? 1.f / z : 0.f;
    for (int j = lane; j < c.k; j += 64) put<BF>(alpha, row * c.k + j, j < n ? __expf(s[j] - mx) * inv : 0.f);
    if (lane == 0) lse[row] = mx + __logf(z);
}

// ds_j = scale alpha_j (da_j - sum_i alpha_i da_i), alpha_j = exp(s_j - lse); and the row's part of the
// targets for the weights' gradients, zeros where n = 0 (what stands there may be NaN or
// infinite, and times the zeros of C, dU and dQp it would be NaN in every sum)
template <bool BF>
__global__ __launch_bounds__(256) void cached_softmax_bwd_kernel(CacheView c, const float* __restrict__ S,
                                                                 const float* __restrict__ lse,
                                                                 const float* __restrict__ dA, int64_t rows,
                                                                 int32_t Rh, float scale, void* __restrict__ ds,
                                                                 CachedTargets t) {
    using T = std::conditional_t<BF, uint16_t, float>;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    int32_t n;
    cache_slot(c, row / Rh, &n);
    const int lane = threadIdx.x & 63;
    const float *s = S + row * c.k, *da = dA + row * c.k;
    const float l = lse[row];
    float dot = 0.f, z = 0.f;
    for (int j = lane; j < n; j += 64) {
        const float p = __expf(s[j] - l);
        dot = __builtin_fmaf(p, da[j], dot);
        z += p;
    }
    // sum of the weights as they come out here, 1 up to rounding: the gradients' sum over a
    // row then vanishes to the last bit for one row, and no worse than rounding otherwise
    dot = wave_sum(dot) / wave_sum(z);
    for (int j = lane; j < c.k; j += 64)
        put<BF>(ds, row * c.k + j, j < n ? scale * __expf(s[j] - l) * (da[j] - dot) : 0.f);
    for (int j = lane; j < t.dh; j += 64) {
        const int64_t at = row * t.dh + j;
        reinterpret_cast<T*>(t.q0)[at] = n ? reinterpret_cast<const T*>(t.q)[at] : T(0);
        reinterpret_cast<T*>(t.dout0)[at] = n ? reinterpret_cast<const T*>(t.dout)[at] : T(0);
        if (!n) reinterpret_cast<T*>(t.Qp)[at] = T(0);
    }
}

// one thread per 8 columns of a row, the matrices one after the other
__global__ __launch_bounds__(256) void tail_rows_kernel(TailRows t, int32_t rows, uint16_t* __restrict__ to) {
    int i = blockIdx.x * 256 + threadIdx.x, at = 0;
#pragma unroll
    for (int m = 0; m < 6; ++m) {
        const int per = t.width[m] / 8, n = 64 * per;
        if (i >= 0 && i < n) {
            const int64_t row = (int64_t)(rows & ~63) + i / per;
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (row < rows) v = reinterpret_cast<const uint4*>(t.from[m])[row * per + i % per];
            reinterpret_cast<uint4*>(to)[at + i] = v;
        }
        i -= n;
        at += n;
    }
}

__global__ __launch_bounds__(256) void sum_parts_kernel(SumParts s) {
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    const int m = blockIdx.y;
    if (i >= s.n) return;
    const float* from = s.parts + (int64_t)m * s.splits * s.n + i;
    float4 v = *reinterpret_cast<const float4*>(from);
    for (int p = 1; p < s.splits; ++p) {
        const float4 x = *reinterpret_cast<const float4*>(from + p * s.n);
        v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
    }
    void* const to = m == 0 ? s.to[0] : m == 1 ? s.to[1] : s.to[2];
    if (s.bf16) *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(to) + i) = make_uint2(tile::pack_bf16x2(v.x, v.y), tile::pack_bf16x2(v.z, v.w));
    else *reinterpret_cast<float4*>(reinterpret_cast<float*>(to) + i) = v;
}

}  // namespace

hipError_t launch_sum_parts(const SumParts& s, hipStream_t stream) {
    hipLaunchKernelGGL(sum_parts_kernel, dim3((unsigned)((s.n / 4 + 255) / 256), 3), dim3(256), 0, stream, s);
    return hipGetLastError();
}

hipError_t launch_tail_rows(const TailRows& t, int32_t rows, uint16_t* to, hipStream_t stream) {
    int64_t n = 0;
    for (int m = 0; m < 6; ++m) n += 64 * (int64_t)(t.width[m] / 8);
    hipLaunchKernelGGL(tail_rows_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, stream, t, rows, to);
    return hipGetLastError();
}

hipError_t launch_cached_softmax(const CacheView& c, const float* S, int64_t rows, int32_t Rh, bool bf16, void* alpha,
                                 float* lse, hipStream_t stream) {
    if (rows <= 0) return hipSuccess;
    const dim3 grid((unsigned)((rows + 3) / 4));
    if (bf16) hipLaunchKernelGGL(cached_softmax_kernel<true>, grid, dim3(256), 0, stream, c, S, rows, Rh, alpha, lse);
    else hipLaunchKernelGGL(cached_softmax_kernel<false>, grid, dim3(256), 0, stream, c, S, rows, Rh, alpha, lse);
    return hipGetLastError();
}

hipError_t launch_cached_softmax_bwd(const CacheView& c, const float* S, const float* lse, const float* dA,
                                     int64_t rows, int32_t Rh, float scale, bool bf16, void* ds, const CachedTargets& t,
                                     hipStream_t stream) {
    if (rows <= 0) return hipSuccess;
    const dim3 grid((unsigned)((rows + 3) / 4));
    if (bf16)
        hipLaunchKernelGGL(cached_softmax_bwd_kernel<true>, grid, dim3(256), 0, stream, c, S, lse, dA, rows, Rh, scale, ds, t);
    else
        hipLaunchKernelGGL(cached_softmax_bwd_kernel<false>, grid, dim3(256), 0, stream, c, S, lse, dA, rows, Rh, scale, ds, t);
    return hipGetLastError();
}

}  // namespace sa
