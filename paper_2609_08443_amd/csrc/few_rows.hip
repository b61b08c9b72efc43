// C [R][N] = A [R][K] W [K][N], bf16, for one or two rows: a serving call's single target.
// The weights' bytes bound it (2 MB at K = N = 1024); the batched product's 64 x 64 tiles give
// 16 compute units 16 slabs one after the other there.  Here a workgroup takes 32 columns and
// all of K, each thread eight columns of eight rows of W of every 1024: all its loads are on
// their way at once, 64 bytes of a row by four neighbouring lanes.  Sums are fp32, in a fixed order: the
// thread's rows, the wave's threads, the waves.  A call of STCA over the cache with one target
// (k = 512, D = 1024): 30.8 us with the batched product, 27.4 with this; two 31.0 and 28.5; with
// four 31.1 and 31.3, where the exchanges between the threads weigh more.
#include "sa_internal.h"
#include "tile_ops.h"

namespace sa {

namespace {

constexpr int kThreads = 512, kCols = 32, kSlices = kThreads / 4;

template <int R>
__global__ __launch_bounds__(kThreads) void few_rows_kernel(const uint16_t* __restrict__ A, const uint16_t* __restrict__ W,
                                                            uint16_t* __restrict__ Cb, float* __restrict__ Cf, int rows,
                                                            int K, int N) {
    __shared__ float part[kThreads / 64][R][kCols];
    const int slice = threadIdx.x >> 2, n0 = blockIdx.x * kCols + 8 * (threadIdx.x & 3);
    float acc[R][8];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[r][c] = 0.f;
    if (n0 < N) {   // (N is a multiple of 8)
        for (int k = 8 * slice; k < K; k += 8 * kSlices) {   // (K is a multiple of 8)
            uint4 w[8], a[R];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = *reinterpret_cast<const uint4*>(W + (int64_t)(k + i) * N + n0);
#pragma unroll
            for (int r = 0; r < R; ++r) a[r] = *reinterpret_cast<const uint4*>(A + (int64_t)min(r, rows - 1) * K + k);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t v[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
                float x[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) x[c] = (c & 1) ? tile::bf16_hi(v[c / 2]) : tile::bf16_lo(v[c / 2]);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const uint32_t q[4] = {a[r].x, a[r].y, a[r].z, a[r].w};
                    const float y = (i & 1) ? tile::bf16_hi(q[i / 2]) : tile::bf16_lo(q[i / 2]);
#pragma unroll
                    for (int c = 0; c < 8; ++c) acc[r][c] = __builtin_fmaf(y, x[c], acc[r][c]);
                }
            }
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            float s = acc[r][c];
            s += __shfl_xor(s, 4, 64);
            s += __shfl_xor(s, 8, 64);
            s += __shfl_xor(s, 16, 64);
            s += __shfl_xor(s, 32, 64);
            if ((threadIdx.x & 63) < 4) part[threadIdx.x >> 6][r][8 * (threadIdx.x & 3) + c] = s;
        }
    __syncthreads();
    for (int i = threadIdx.x; i < R * kCols; i += kThreads) {
        const int r = i / kCols, c = i % kCols, n = blockIdx.x * kCols + c;
        if (r >= rows || n >= N) continue;
        float s = 0.f;
#pragma unroll
        for (int v = 0; v < kThreads / 64; ++v) s += part[v][r][c];
        if (Cb) Cb[(int64_t)r * N + n] = tile::to_bf16(s);
        else Cf[(int64_t)r * N + n] = s;
    }
}

}  // namespace

bool few_rows_supported(int32_t rows, int32_t K, int32_t N) { return rows <= 2 && N % 8 == 0 && K % 8 == 0; }

hipError_t launch_few_rows(const uint16_t* A, const uint16_t* W, void* C, bool c_bf16, int32_t rows, int32_t K, int32_t N,
                           hipStream_t stream) {
    uint16_t* cb = c_bf16 ? reinterpret_cast<uint16_t*>(C) : nullptr;
    float* cf = c_bf16 ? nullptr : reinterpret_cast<float*>(C);
    const dim3 grid((unsigned)((N + kCols - 1) / kCols));
    if (rows <= 1) hipLaunchKernelGGL(few_rows_kernel<1>, grid, dim3(kThreads), 0, stream, A, W, cb, cf, rows, K, N);
    else hipLaunchKernelGGL(few_rows_kernel<2>, grid, dim3(kThreads), 0, stream, A, W, cb, cf, rows, K, N);
    return hipGetLastError();
}

}  // namespace sa
