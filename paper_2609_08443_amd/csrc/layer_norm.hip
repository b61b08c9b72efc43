// Layer norm over rows of D values and its gradients:
//
//   y = xh gamma + beta,  xh = (x - mean) rstd,  rstd = 1 / sqrt(var + eps)   (var: mean of (x - mean)^2)
//   g = dy gamma,  dx = rstd (g - mean(g) - xh mean(g xh)),  dgamma = sum over rows of dy xh,  dbeta = sum of dy
//
// Both are bound by memory: each value read once and written once.  A row is LANES lanes of a
// wave, or the WAVES waves of a workgroup, and stays in registers between the sums (the mean
// first, then the squares around it: a row far from zero keeps its variance).  Loads and stores
// are of 16 bytes at whatever alignment rows of odd width have.  The weights' gradients add
// up in registers over the rows that a workgroup walks, each thread its own columns, then over
// the workgroups in a second launch, in order: no atomics.  100,000 rows of 1,024 bf16 take 78 us,
// 5.2 TB/s (a copy of 2 GiB 4.95), the gradients of 61,003 take 70 and the second launch 5.
#include <algorithm>
#include <type_traits>

#include "sa_internal.h"
#include "vec_rows.h"

namespace sa {

namespace {

constexpr int kThreads = 256;

using vec::value;
template <typename T>
using Vec = vec::Piece<T>;

// a piece of a row of D, and back
template <typename T>
__device__ inline void load_vec(const T* p, int c, int D, float* o) { vec::load<Vec<T>::N>(p, c, D, o); }
template <typename T>
__device__ inline void store_vec(T* p, int c, int D, const float* v) { vec::store<Vec<T>::N>(p, c, D, v); }

// Sum over a row's threads; every one gets it.  WAVES > 1: through `part` [2][WAVES], of which
// calls use one half in turn, so that one barrier a call is enough.
template <int LANES, int WAVES>
__device__ inline float row_sum(float v, float* part) {
#pragma unroll
    for (int s = 1; s < LANES; s *= 2) v += __shfl_xor(v, s, 64);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += part[w];
    }
    return v;
}

// A row by LANES lanes (WAVES = 1) or by a workgroup's WAVES waves, NV vectors a thread.
// WALK: any width, the row read again for each sum.
template <typename T, int LANES, int WAVES, int NV, bool WALK>
__global__ __launch_bounds__(kThreads) void norm_fwd_kernel(const T* __restrict__ x, int64_t x_ld, const T* __restrict__ gamma,
                                                            const T* __restrict__ beta, int64_t N, int D, float eps,
                                                            T* __restrict__ y, float2* __restrict__ stats) {
    constexpr int V = Vec<T>::N, PER = LANES * WAVES, ROWS = kThreads / PER;
    __shared__ float part[2][4];
    const int t = threadIdx.x % PER;
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < N; r0 += (int64_t)gridDim.x * ROWS) {
        const int64_t row = r0 + threadIdx.x / PER;
        if (row >= N) return;   // (only where rows take no barrier)
        const T* xp = x + row * x_ld;
        float v[NV][V];
        float s = 0.f;
        const int steps = WALK ? (D + PER * V - 1) / (PER * V) : NV;
        auto each = [&](auto f) __attribute__((always_inline)) {
            if constexpr (WALK) {
                for (int i = 0; i < steps; ++i) {
                    load_vec(xp, (i * PER + t) * V, D, v[0]);
                    f(v[0], (i * PER + t) * V);
                }
            } else {
#pragma unroll
                for (int i = 0; i < NV; ++i) f(v[i], (i * PER + t) * V);
            }
        };
        if constexpr (!WALK) {
#pragma unroll
            for (int i = 0; i < NV; ++i) load_vec(xp, (i * PER + t) * V, D, v[i]);
        }
        each([&](const float* u, int) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < V; ++e) s += u[e];
        });
        const float mean = row_sum<LANES, WAVES>(s, part[0]) / (float)D;   // (exact for equal values)
        s = 0.f;
        each([&](const float* u, int c) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float z = c + e < D ? u[e] - mean : 0.f;
                s = __builtin_fmaf(z, z, s);
            }
        });
        const float rstd = 1.f / sqrtf(row_sum<LANES, WAVES>(s, part[1]) / (float)D + eps);
        each([&](const float* u, int c) __attribute__((always_inline)) {
            float ga[V], be[V], o[V];
            load_vec(gamma, c, D, ga);
            load_vec(beta, c, D, be);
#pragma unroll
            for (int e = 0; e < V; ++e) o[e] = __builtin_fmaf((u[e] - mean) * rstd, ga[e], be[e]);
            store_vec(y + row * D, c, D, o);
        });
        if (stats && t == 0) stats[row] = make_float2(mean, rstd);
    }
}

// A workgroup walks over rows; its column sums go to part [grid][2][D].
template <typename T, int LANES, int WAVES, int NV>
__global__ __launch_bounds__(kThreads) void norm_bwd_kernel(const T* __restrict__ x, int64_t x_ld, const T* __restrict__ gamma,
                                                            const float2* __restrict__ stats, const T* __restrict__ dy,
                                                            int64_t N, int D, T* __restrict__ dx, float* __restrict__ sums) {
    constexpr int V = Vec<T>::N, PER = LANES * WAVES, ROWS = kThreads / PER;
    __shared__ float part[2][4];
    __shared__ float cols[ROWS > 1 ? kThreads * V : 1];
    const int t = threadIdx.x % PER;
    const float inv = 1.f / (float)D;
    float ga[NV][V], dg[NV][V], db[NV][V];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        load_vec(gamma, (i * PER + t) * V, D, ga[i]);
#pragma unroll
        for (int e = 0; e < V; ++e) dg[i][e] = db[i][e] = 0.f;
    }
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < N; r0 += (int64_t)gridDim.x * ROWS) {
        const int64_t row = r0 + threadIdx.x / PER;
        if (row < N) {   // (all of the workgroup where rows take a barrier)
            const float2 st = stats[row];
            float xh[NV][V], g[NV][V];
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                load_vec(x + row * x_ld, (i * PER + t) * V, D, xh[i]);
                load_vec(dy + row * D, (i * PER + t) * V, D, g[i]);
            }
            float s = 0.f, sx = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    xh[i][e] = (i * PER + t) * V + e < D ? (xh[i][e] - st.x) * st.y : 0.f;
                    db[i][e] += g[i][e];
                    dg[i][e] = __builtin_fmaf(g[i][e], xh[i][e], dg[i][e]);
                    g[i][e] *= ga[i][e];
                    s += g[i][e];
                    sx = __builtin_fmaf(g[i][e], xh[i][e], sx);
                }
            s = row_sum<LANES, WAVES>(s, part[0]) * inv;
            sx = row_sum<LANES, WAVES>(sx, part[1]) * inv;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float o[V];
#pragma unroll
                for (int e = 0; e < V; ++e) o[e] = st.y * (g[i][e] - s - xh[i][e] * sx);
                store_vec(dx + row * D, (i * PER + t) * V, D, o);
            }
        }
    }
    // the workgroup's rows' threads, in order
    float* const out = sums + (int64_t)blockIdx.x * 2 * D;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const float(&v)[V] = which ? db[i] : dg[i];
            const int c0 = (i * PER + t) * V;
            if constexpr (ROWS > 1) {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < V; ++e) cols[threadIdx.x * V + e] = v[e];
                __syncthreads();
                for (int c = threadIdx.x; c < PER * V; c += kThreads) {
                    float s = 0.f;
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) s += cols[r * PER * V + c];
                    if (i * PER * V + c < D) out[which * D + i * PER * V + c] = s;
                }
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (c0 + e < D) out[which * D + c0 + e] = v[e];
            }
        }
}

// Wider rows: dx alone, the row read twice; the column sums by norm_cols_kernel.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_bwd_walk_kernel(const T* __restrict__ x, int64_t x_ld,
                                                                 const T* __restrict__ gamma,
                                                                 const float2* __restrict__ stats,
                                                                 const T* __restrict__ dy, int64_t N, int D,
                                                                 T* __restrict__ dx) {
    constexpr int V = Vec<T>::N;
    __shared__ float part[2][4];
    for (int64_t row = blockIdx.x; row < N; row += gridDim.x) {
        const float2 st = stats[row];
        float xv[V], g[V], ga[V];
        float s = 0.f, sx = 0.f;
        auto load = [&](int c) __attribute__((always_inline)) {
            load_vec(x + row * x_ld, c, D, xv);
            load_vec(dy + row * D, c, D, g);
            load_vec(gamma, c, D, ga);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                xv[e] = c + e < D ? (xv[e] - st.x) * st.y : 0.f;
                g[e] *= ga[e];
            }
        };
        for (int c = threadIdx.x * V; c < D; c += kThreads * V) {
            load(c);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                s += g[e];
                sx = __builtin_fmaf(g[e], xv[e], sx);
            }
        }
        s = row_sum<64, 4>(s, part[0]) / (float)D;
        sx = row_sum<64, 4>(sx, part[1]) / (float)D;
        for (int c = threadIdx.x * V; c < D; c += kThreads * V) {
            load(c);
            float o[V];
#pragma unroll
            for (int e = 0; e < V; ++e) o[e] = st.y * (g[e] - s - xv[e] * sx);
            store_vec(dx + row * D, c, D, o);
        }
        __syncthreads();
    }
}
// Column sums of 256 columns over every gridDim.y-th row: sums [gridDim.y][2][D]
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_cols_kernel(const T* __restrict__ x, int64_t x_ld,
                                                             const float2* __restrict__ stats, const T* __restrict__ dy,
                                                             int64_t N, int D, float* __restrict__ sums) {
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= D) return;
    float dg = 0.f, db = 0.f;
    for (int64_t row = blockIdx.y; row < N; row += gridDim.y) {
        const float2 st = stats[row];
        const float d = value(dy[row * D + c]);
        dg = __builtin_fmaf(d, (value(x[row * x_ld + c]) - st.x) * st.y, dg);
        db += d;
    }
    sums[(int64_t)blockIdx.y * 2 * D + c] = dg;
    sums[((int64_t)blockIdx.y * 2 + 1) * D + c] = db;
}

// dgamma and dbeta: sums over the parts, in order
__global__ __launch_bounds__(kThreads) void norm_sum_kernel(const float* __restrict__ sums, int n, int D,
                                                            float* __restrict__ dgamma, float* __restrict__ dbeta) {
    vec::sum_parts(sums, n, 2 * (int64_t)D, [&](int64_t c, float s) { (c < D ? dgamma[c] : dbeta[c - D]) = s; });
}

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// rows that a workgroup takes at a time; 0: wider than the registers hold
template <typename T>
int rows_at_once(int D) {
    const int vecs = (int)cdiv(D, Vec<T>::N);
    if (vecs <= 8) return 32;
    if (vecs <= 16) return 16;
    if (vecs <= 32) return 8;
    if (vecs <= 256) return 4;
    return vecs <= 1024 ? 1 : 0;
}

template <typename T, typename F>
hipError_t by_width(int D, F f) {
    const int vecs = (int)cdiv(D, Vec<T>::N);
#define SA_NORM(LANES, WAVES, NV) \
    f(std::integral_constant<int, LANES>{}, std::integral_constant<int, WAVES>{}, std::integral_constant<int, NV>{})
    if (vecs <= 8) SA_NORM(8, 1, 1);
    else if (vecs <= 16) SA_NORM(16, 1, 1);
    else if (vecs <= 32) SA_NORM(32, 1, 1);
    else if (vecs <= 64) SA_NORM(64, 1, 1);
    else if (vecs <= 128) SA_NORM(64, 1, 2);
    else if (vecs <= 256) SA_NORM(64, 1, 4);
    else if (vecs <= 512) SA_NORM(64, 4, 2);
    else SA_NORM(64, 4, 4);
#undef SA_NORM
    return hipGetLastError();
}

template <typename T>
int64_t bwd_parts(int64_t N, int D) {
    const int rows = rows_at_once<T>(D);
    if (rows == 0) return std::min<int64_t>(std::max<int64_t>(N, 1), 64);
    return std::max<int64_t>(1, std::min<int64_t>(cdiv(N, rows), 4 * (int64_t)device_cus()));
}

template <typename T>
hipError_t norm_fwd(const NormArgs& a, hipStream_t stream) {
    const T* x = reinterpret_cast<const T*>(a.x);
    const T *ga = reinterpret_cast<const T*>(a.gamma), *be = reinterpret_cast<const T*>(a.beta);
    T* y = reinterpret_cast<T*>(a.y);
    const int rows = rows_at_once<T>(a.D);
    const int64_t most = 1 << 20;
    const dim3 grid((unsigned)std::min(cdiv(a.N, rows ? rows : 1), most));
    if (rows == 0) {
        hipLaunchKernelGGL((norm_fwd_kernel<T, 64, 4, 1, true>), grid, dim3(kThreads), 0, stream, x, a.x_ld, ga, be, a.N, a.D,
                           a.eps, y, a.stats);
        return hipGetLastError();
    }
    return by_width<T>(a.D, [&](auto lanes, auto waves, auto nv) {
        hipLaunchKernelGGL((norm_fwd_kernel<T, lanes.value, waves.value, nv.value, false>), grid, dim3(kThreads), 0, stream, x,
                           a.x_ld, ga, be, a.N, a.D, a.eps, y, a.stats);
    });
}

template <typename T>
hipError_t norm_bwd(const NormArgs& a, hipStream_t stream) {
    const T* x = reinterpret_cast<const T*>(a.x);
    const T *ga = reinterpret_cast<const T*>(a.gamma), *dy = reinterpret_cast<const T*>(a.dy);
    T* dx = reinterpret_cast<T*>(a.y);
    const int64_t parts = bwd_parts<T>(a.N, a.D);
    hipError_t e;
    if (rows_at_once<T>(a.D) == 0) {
        // (the sums first: dx may be dy)
        hipLaunchKernelGGL(norm_cols_kernel<T>, dim3((unsigned)cdiv(a.D, kThreads), (unsigned)parts), dim3(kThreads), 0, stream,
                           x, a.x_ld, a.stats, dy, a.N, a.D, a.sums);
        if (a.N > 0)
            hipLaunchKernelGGL(norm_bwd_walk_kernel<T>, dim3((unsigned)std::min<int64_t>(a.N, 1 << 20)), dim3(kThreads), 0,
                               stream, x, a.x_ld, ga, a.stats, dy, a.N, a.D, dx);
        e = hipGetLastError();
    } else {
        e = by_width<T>(a.D, [&](auto lanes, auto waves, auto nv) {
            hipLaunchKernelGGL((norm_bwd_kernel<T, lanes.value, waves.value, nv.value>), dim3((unsigned)parts), dim3(kThreads),
                               0, stream, x, a.x_ld, ga, a.stats, dy, a.N, a.D, dx, a.sums);
        });
    }
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(norm_sum_kernel, dim3((unsigned)cdiv(2 * (int64_t)a.D, vec::kSumColumns)), dim3(kThreads), 0, stream, a.sums,
                       (int)parts, a.D, a.dgamma, a.dbeta);
    return hipGetLastError();
}

}  // namespace

int64_t norm_parts(int64_t N, int32_t D, bool bf16) { return bf16 ? bwd_parts<uint16_t>(N, D) : bwd_parts<float>(N, D); }

hipError_t launch_norm_fwd(const NormArgs& a, bool bf16, hipStream_t stream) {
    return bf16 ? norm_fwd<uint16_t>(a, stream) : norm_fwd<float>(a, stream);
}
hipError_t launch_norm_bwd(const NormArgs& a, bool bf16, hipStream_t stream) {
    return bf16 ? norm_bwd<uint16_t>(a, stream) : norm_bwd<float>(a, stream);
}

}  // namespace sa
