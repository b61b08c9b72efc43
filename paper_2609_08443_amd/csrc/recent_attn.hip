// Attention of targets over their users' recent histories: the plan of the kernels over tiles
// of rows (recent_attn_rows.h) and the join of tiles that several workgroups share.
//
// Where a user's targets and tokens lie is on the device alone, so the plan is made there: every
// tile's keys, and the units of keys before it.  The units of all tiles and key heads, one after
// the other, are cut into equal pieces, one a workgroup: users with few and many tokens, targets
// that see little or everything, cost what they have to read, and no workgroup more.  A tile cut
// by a piece's border leaves partial results, added up in the pieces' order.
#include "recent_attn.h"

namespace sa {
namespace attn {

namespace {

constexpr int kPlanThreads = 1024;

// Users' first rows are looked up in LDS where they fit
constexpr int kUsersInLds = 4096;

// Inclusive sums over the workgroup's threads
__device__ inline int64_t scan(int64_t v, int64_t* sums) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        const int64_t o = __shfl_up(v, s, 64);
        if (lane >= s) v += o;
    }
    if (lane == 63) sums[w] = v;
    __syncthreads();
    for (int i = 0; i < w; ++i) v += sums[i];
    __syncthreads();
    return v;
}

// tiles of keys of user b
__device__ int32_t plan_keys(const View& a, int64_t b) {
    const User us = user_at(a, b);
    if (b == a.B) return (int32_t)((a.T - us.tok0 + kKeyTile - 1) / kKeyTile) * (a.skip < 0);
    return (int64_t)us.n * a.g <= a.skip ? 0 : (us.L + kKeyTile - 1) / kKeyTile;
}

// Few tiles: records and sums by one workgroup, a thread a tile.  Else every tile's units by the
// grid first (into prefix[t + 1]), then their sums.  A second workgroup of the sums does the keys'.
enum PlanStep { kAll, kTiles, kSums };
template <PlanStep STEP>
__global__ __launch_bounds__(STEP == kTiles ? 256 : kPlanThreads) void plan_kernel(View a, int32_t bq, int32_t unit,
                                                                                    int64_t tiles, TileRec* recs,
                                                                                    int64_t* prefix, int64_t* keys) {
    if constexpr (STEP == kTiles) {
        const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
        if (t < tiles) prefix[t + 1] = plan_tile(a, a.targets, bq, unit, t, recs + t);
    } else {
        __shared__ int64_t sums[kPlanThreads / 64];
        __shared__ int64_t carry;
        __shared__ int64_t first[STEP == kAll ? kUsersInLds + 1 : 1];
        const bool for_keys = blockIdx.x == 1;
        int64_t* const to = for_keys ? keys : prefix;
        const int64_t n = for_keys ? a.B + 1 : tiles;
        const int64_t* targets = a.targets;
        if (STEP == kAll && !for_keys && a.B <= kUsersInLds) {
            for (int64_t b = threadIdx.x; b <= a.B; b += kPlanThreads) first[b] = a.targets[b];
            targets = first;
        }
        if (threadIdx.x == 0) {
            carry = 0;
            to[0] = 0;
        }
        __syncthreads();
        for (int64_t t0 = 0; t0 < n; t0 += kPlanThreads) {
            const int64_t t = t0 + threadIdx.x;
            int64_t v = 0;
            if (t < n) v = for_keys ? plan_keys(a, t) : STEP == kAll ? plan_tile(a, targets, bq, unit, t, recs + t) : prefix[t + 1];
            v = scan(v, sums) + carry;
            if (t < n) to[t + 1] = v;
            __syncthreads();
            if (threadIdx.x == kPlanThreads - 1) carry = v;
            __syncthreads();
        }
    }
}

// Workgroup w: the tile that piece w began and others went on with.  Threads take a row's values
// four at a time, and where there are few rows, every `groups`-th piece, joined through LDS.
template <typename T, int D, bool BWD>
__global__ __launch_bounds__(256) void join_kernel(RowsArgs f) {
    constexpr int PER = D / 4;   // threads a row
    __shared__ float acc[256][5];
    const View& a = f.a;
    const int32_t bq = f.p.bq;
    const int64_t w = blockIdx.x;
    const Begun tile = f.begun[w];
    const int32_t n = tile.n, rows = tile.rows;
    if (n < 2) return;
    const int64_t stride = (int64_t)bq * (D + 2);
    // what piece w began is at 2 w + 1; piece v's part of a tile that it goes on with at 2 v
    auto part_of = [&](int32_t i) { return f.parts + (i == 0 ? 2 * w + 1 : 2 * (w + i)) * stride; };
    // threads side by side on one row's piece: as many groups of pieces as rows leave room for
    int32_t groups = 256 / (rows * PER);
    groups = groups < 1 ? 1 : groups;
    const int32_t group = rows * PER >= 256 ? 0 : threadIdx.x / (rows * PER);
    for (int32_t x = rows * PER >= 256 ? threadIdx.x : threadIdx.x % (rows * PER); x < rows * PER; x += 256) {
        const int32_t r = x / PER, d = 4 * (x % PER);
        const int32_t row = tile.row0 + r;
        const int64_t target = tile.t0 + row / a.g;
        const int32_t head = tile.kv * a.g + row % a.g;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        float m = -__builtin_inff(), l = 0.f;
        const bool in = group < groups;
        if (groups == 1 && !in) return;
        if constexpr (!BWD) {
            if (in) {
#pragma unroll 4
                for (int32_t i = group; i < n; i += groups) m = fmaxf(m, part_of(i)[bq * D + r]);
            }
        }
        const float ms = m == -__builtin_inff() ? 0.f : m;
        if (in) {
#pragma unroll 4
            for (int32_t i = group; i < n; i += groups) {
                const float* part = part_of(i);
                const float4 o = *reinterpret_cast<const float4*>(part + r * D + d);
                float fac = 1.f;
                if constexpr (!BWD) {
                    fac = exp2_(part[bq * D + r] - ms);
                    l = __builtin_fmaf(part[bq * D + bq + r], fac, l);
                }
                v[0] = __builtin_fmaf(o.x, fac, v[0]);
                v[1] = __builtin_fmaf(o.y, fac, v[1]);
                v[2] = __builtin_fmaf(o.z, fac, v[2]);
                v[3] = __builtin_fmaf(o.w, fac, v[3]);
            }
        }
        if (groups > 1) {   // (all threads come here once)
            float* mine = acc[threadIdx.x];
            __shared__ float tops[256];
            tops[threadIdx.x] = m;
            __syncthreads();
            float top = m;
            if constexpr (!BWD) {
                for (int32_t g = 0; g < groups; ++g) top = fmaxf(top, tops[g * rows * PER + x]);
            }
            const float fac = BWD || m == -__builtin_inff() ? (BWD ? 1.f : 0.f) : exp2_(m - top);
#pragma unroll
            for (int e = 0; e < 4; ++e) mine[e] = v[e] * fac;
            mine[4] = l * fac;
            __syncthreads();
            if (group != 0) return;
            m = top;
            l = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = 0.f;
            for (int32_t g = 0; g < groups; ++g) {
                const float* o = acc[g * rows * PER + x];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += o[e];
                l += o[4];
            }
        }
        const float inv = BWD ? a.scale : l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] *= inv;
        T* o = BWD ? reinterpret_cast<T*>(f.out) + target * f.dq_t + head * f.dq_h
                   : reinterpret_cast<T*>(f.out) + (target * a.h + head) * D;
        Tile32<T, D>::store4(o + d, v);
        if (!BWD && f.lse && d == 0) f.lse[target * a.h + head] = (m + __builtin_amdgcn_logf(l)) / kLog2e;
    }
}

template <typename T, int D>
hipError_t launch_join_t(const RowsArgs& f, bool bwd, hipStream_t stream) {
    const dim3 grid((unsigned)(f.grid - 1));
    if (bwd) hipLaunchKernelGGL((join_kernel<T, D, true>), grid, dim3(256), 0, stream, f);
    else hipLaunchKernelGGL((join_kernel<T, D, false>), grid, dim3(256), 0, stream, f);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_plan(const View& a, const Plan& p, TileRec* recs, int64_t* prefix, int64_t* keys, hipStream_t stream) {
    const dim3 one(keys ? 2 : 1);
    const int64_t tiles = p.tiles;
    if (tiles <= 4 * kPlanThreads) {
        hipLaunchKernelGGL(plan_kernel<kAll>, one, dim3(kPlanThreads), 0, stream, a, p.bq, p.unit, tiles, recs, prefix, keys);
    } else {
        hipLaunchKernelGGL(plan_kernel<kTiles>, dim3((unsigned)((tiles + 255) / 256)), dim3(256), 0, stream, a, p.bq,
                           p.unit, tiles, recs, prefix, keys);
        hipLaunchKernelGGL(plan_kernel<kSums>, one, dim3(kPlanThreads), 0, stream, a, p.bq, p.unit, tiles, recs, prefix, keys);
    }
    return hipGetLastError();
}

hipError_t launch_join(const RowsArgs& f, bool bf16, int32_t d, bool bwd, hipStream_t stream) {
    if (f.grid < 2) return hipSuccess;
    if (bf16) return d == 64 ? launch_join_t<uint16_t, 64>(f, bwd, stream) : launch_join_t<uint16_t, 128>(f, bwd, stream);
    return d == 64 ? launch_join_t<float, 64>(f, bwd, stream) : launch_join_t<float, 128>(f, bwd, stream);
}

}  // namespace attn
}  // namespace sa
