// Writing a sketch into its slot of the cache and reading it back (format in cache.h).
//
// Both are one pass over the values: bytes bound them (a value of 2 or 4 bytes on one
// side, half a byte or one on the other, and 1/32 byte of scale).  A wave takes an
// octet of rows by 64 values at a time, lane l row l % 8 and values 8 (l / 8) ..+7:
// each lane's values are whole 16-byte pieces, each row of the wave a run of 128
// (bf16) or 256 bytes, the codes of the wave 256 or 512 contiguous bytes, and the four
// lanes of a group's values find its largest magnitude in two exchanges.  Measured: 128
// sketches of 512 x 1024 from bf16 to 8 bits 43 us (203 MB, 4.7 TB/s) and back 32 us (the
// codes from the cache behind the L2), 64 of 1024 x 1024 from 4 bits to bf16 35 us (170 MB,
// 4.8 TB/s; 27 into the same 134 MB again and again, which that cache then holds); a copy
// of 1 GB runs at 5.0 TB/s.
#include "cache.h"

namespace sa {

namespace {

using namespace cachefmt;

constexpr int kTiles = 4;             // 8 x 64 tiles a wave, loads of all before the first store
constexpr int kClaimUsers = 1024;     // most users whose later writers every workgroup looks through

struct IoArgs {
    const void* in;          // write: Xs [B][k][D];  read: unused
    void* out;               // read: [B][k][D]
    uint8_t* data;
    int32_t* rows;           // [n_slots]
    const int64_t* slots;    // [B]
    const int32_t* n;        // write: rows of each user, or null for k
    int64_t B, n_slots, slot_bytes, scales_at;
    int32_t k, D, G, G2;     // G2 = ceil(G / 2) tiles across
    int32_t tiles, per_user; // tiles and workgroups of a user
    bool claimed;            // rows[] holds the last writer of each slot (k + 1 + b)
};

// 8 values of a row from column c (columns from D on: zeros).  VEC: D is a multiple
// of 8 (bf16) or 4 (fp32), so that pieces are aligned.  Read once, and not kept in the
// caches that the codes go into (128 sketches of 512 x 1024 bf16: write 58 -> 46 us).
template <bool BF, bool VEC>
__device__ inline void load8(const void* p, int64_t at, int c, int D, float (&v)[8]) {
    if constexpr (BF && VEC) {
        tile::u32x4 w = {0u, 0u, 0u, 0u};
        if (c < D) w = __builtin_nontemporal_load(reinterpret_cast<const tile::u32x4*>(reinterpret_cast<const uint16_t*>(p) + at + c));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = tile::bf16_lo(w[i]);
            v[2 * i + 1] = tile::bf16_hi(w[i]);
        }
    } else if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            tile::u32x4 q = {0u, 0u, 0u, 0u};
            if (c + 4 * i < D)
                q = __builtin_nontemporal_load(reinterpret_cast<const tile::u32x4*>(reinterpret_cast<const float*>(p) + at + c + 4 * i));
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * i + j] = __uint_as_float(q[j]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = 0.f;
            if (c + i < D) {
                if constexpr (BF) v[i] = tile::bf16_lo(reinterpret_cast<const uint16_t*>(p)[at + c + i]);
                else v[i] = reinterpret_cast<const float*>(p)[at + c + i];
            }
        }
    }
}

// Is user b the last of the batch to write its slot?  Every workgroup looks through
// the users after its own: at most kClaimUsers, of 8 bytes each, from L2.
__device__ inline bool last_writer(const IoArgs& a, int64_t b, int64_t slot) {
    int later = 0;
    for (int64_t i = b + 1 + threadIdx.x; i < a.B; i += 256) later |= a.slots[i] == slot ? 1 : 0;
    return __syncthreads_or(later) == 0;
}

template <int BITS, bool BF, bool VEC>
__global__ __launch_bounds__(256) void cache_write_kernel(IoArgs a) {
    const int64_t b = blockIdx.x / a.per_user;
    const int part = (int)(blockIdx.x % a.per_user);
    const int64_t slot = a.slots[b];
    if (slot < 0 || slot >= a.n_slots) return;
    if (a.claimed) {
        if (a.rows[slot] != a.k + 1 + (int32_t)b) return;
    } else if (!last_writer(a, b, slot)) {
        return;
    }
    const int32_t n = a.n ? min(max(a.n[b], 0), a.k) : a.k;
    if (!a.claimed && part == 0 && threadIdx.x == 0) a.rows[slot] = n;
    uint8_t* const codes = a.data + slot * a.slot_bytes;
    uint8_t* const scales = codes + a.scales_at;
    const int lane = threadIdx.x & 63, r = lane & 7, oct = lane >> 3;
    const int t0 = (part * 4 + (threadIdx.x >> 6)) * kTiles;
    if ((int64_t)(t0 / a.G2) * 8 >= n) return;
    float v[kTiles][8];
    bool ok[kTiles];
    int o[kTiles], g[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        const int t = t0 + i;
        o[i] = t / a.G2;
        g[i] = (t % a.G2) * 2 + (oct >> 2);
        ok[i] = t < a.tiles && 8 * o[i] + r < n && g[i] < a.G;
        if (ok[i]) {
            load8<BF, VEC>(a.in, (b * a.k + 8 * o[i] + r) * (int64_t)a.D, g[i] * kGroup + 8 * (oct & 3), a.D, v[i]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        // the largest magnitude as bits: infinities and NaN above every number
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[i][j]) & 0x7fffffffu);
        top = max(top, (uint32_t)__shfl_xor((int)top, 8, 64));
        top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
        if (!ok[i]) continue;
        const bool fine = top < 0x7f800000u;
        const int e = scale_exp<BITS>(__uint_as_float(top));
        uint32_t w[BITS / 4];
        encode8<BITS>(v[i], exp_float(-e), w);
        uint8_t* const to = codes + (((int64_t)o[i] * a.G + g[i]) * 4 + (oct & 3)) * (8 * kRowBytes<BITS>) + r * kRowBytes<BITS>;
        if constexpr (BITS == 4) *reinterpret_cast<uint32_t*>(to) = fine ? w[0] : 0u;
        else *reinterpret_cast<uint2*>(to) = fine ? make_uint2(w[0], w[1]) : make_uint2(0u, 0u);
        if ((oct & 3) == 0) scales[((int64_t)o[i] * a.G + g[i]) * 8 + r] = (uint8_t)(fine ? e + 127 : kBadScale);
    }
}

// Batches of more than kClaimUsers users: rows[] of a slot, cleared of what it held (a
// count past k would outdo a writer's number), first takes the number of its last writer,
// above every count of rows, and its count once the rows are written.
template <bool CLEAR>
__global__ __launch_bounds__(256) void cache_claim_kernel(IoArgs a) {
    const int64_t b = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (b >= a.B) return;
    const int64_t slot = a.slots[b];
    if (slot < 0 || slot >= a.n_slots) return;
    if constexpr (CLEAR) a.rows[slot] = 0;
    else atomicMax(a.rows + slot, a.k + 1 + (int32_t)b);
}
__global__ __launch_bounds__(256) void cache_settle_kernel(IoArgs a) {
    const int64_t b = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (b >= a.B) return;
    const int64_t slot = a.slots[b];
    if (slot < 0 || slot >= a.n_slots || a.rows[slot] != a.k + 1 + (int32_t)b) return;
    a.rows[slot] = a.n ? min(max(a.n[b], 0), a.k) : a.k;
}

template <int BITS, bool BF, bool VEC>
__global__ __launch_bounds__(256) void cache_read_kernel(IoArgs a) {
    const int64_t b = blockIdx.x / a.per_user;
    const int part = (int)(blockIdx.x % a.per_user);
    const int64_t slot = a.slots[b];
    const bool hit = slot >= 0 && slot < a.n_slots;
    const int32_t n = hit ? min(max(a.rows[slot], 0), a.k) : 0;
    const uint8_t* const codes = a.data + (hit ? slot : 0) * a.slot_bytes;
    const uint8_t* const scales = codes + a.scales_at;
    const int lane = threadIdx.x & 63, r = lane & 7, oct = lane >> 3;
    const int t0 = (part * 4 + (threadIdx.x >> 6)) * kTiles;
    uint32_t w[kTiles][BITS / 4];
    uint32_t sc[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        const int t = t0 + i, o = t / a.G2, g = (t % a.G2) * 2 + (oct >> 2);
        w[i][0] = 0u;
        if constexpr (BITS == 8) w[i][1] = 0u;
        sc[i] = 127u;
        if (t < a.tiles && 8 * o + r < n && g < a.G) {
            const uint8_t* from = codes + (((int64_t)o * a.G + g) * 4 + (oct & 3)) * (8 * kRowBytes<BITS>) + r * kRowBytes<BITS>;
            if constexpr (BITS == 4) {
                w[i][0] = *reinterpret_cast<const uint32_t*>(from);
            } else {
                const uint2 q = *reinterpret_cast<const uint2*>(from);
                w[i][0] = q.x;
                w[i][1] = q.y;
            }
            sc[i] = scales[((int64_t)o * a.G + g) * 8 + r];
        }
    }
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        const int t = t0 + i, o = t / a.G2, c = ((t % a.G2) * 8 + oct) * 8, row = 8 * o + r;
        if (t >= a.tiles || row >= a.k || c >= a.D) continue;
        const uint4 q = decode8<BITS>(w[i], scale_float(sc[i]));
        const int64_t at = (b * a.k + row) * (int64_t)a.D + c;
        const uint32_t v[4] = {q.x, q.y, q.z, q.w};
        if constexpr (BF) {
            uint16_t* const to = reinterpret_cast<uint16_t*>(a.out) + at;
            if constexpr (VEC) {
                *reinterpret_cast<uint4*>(to) = q;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j < a.D) to[j] = (uint16_t)(v[j / 2] >> (16 * (j & 1)));
            }
        } else {
            float* const to = reinterpret_cast<float*>(a.out) + at;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float4 f = make_float4(tile::bf16_lo(v[2 * j]), tile::bf16_hi(v[2 * j]), tile::bf16_lo(v[2 * j + 1]),
                                             tile::bf16_hi(v[2 * j + 1]));
                if constexpr (VEC) {
                    if (c + 4 * j < a.D) *reinterpret_cast<float4*>(to + 4 * j) = f;
                } else {
                    const float e[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
                    for (int m = 0; m < 4; ++m)
                        if (c + 4 * j + m < a.D) to[4 * j + m] = e[m];
                }
            }
        }
    }
}

IoArgs io_args(const CacheView& c, int64_t B) {
    IoArgs a{};
    a.data = const_cast<uint8_t*>(c.data);
    a.rows = const_cast<int32_t*>(c.rows);
    a.slots = c.slots;
    a.B = B;
    a.n_slots = c.n_slots;
    a.slot_bytes = c.slot_bytes;
    a.scales_at = c.scales_at;
    a.k = c.k;
    a.D = c.D;
    a.G = c.G;
    a.G2 = (c.G + 1) / 2;
    a.tiles = (c.k + 7) / 8 * a.G2;
    a.per_user = (a.tiles + 4 * kTiles - 1) / (4 * kTiles);
    return a;
}

}  // namespace

int64_t cache_io_workgroups(int32_t k, int32_t D) {
    CacheView c{};
    c.k = k;
    c.D = D;
    c.G = (D + kGroup - 1) / kGroup;
    return io_args(c, 1).per_user;
}

hipError_t launch_cache_write(const CacheView& c, int bits, const void* Xs, bool bf16, const int32_t* n, int64_t B,
                              hipStream_t stream) {
    if (B <= 0) return hipSuccess;
    IoArgs a = io_args(c, B);
    a.in = Xs;
    a.n = n;
    a.claimed = B > kClaimUsers;
    const dim3 grid((unsigned)(B * a.per_user)), users((unsigned)((B + 255) / 256));
    if (a.claimed) {
        hipLaunchKernelGGL(cache_claim_kernel<true>, users, dim3(256), 0, stream, a);
        hipLaunchKernelGGL(cache_claim_kernel<false>, users, dim3(256), 0, stream, a);
    }
    const bool vec = c.D % (bf16 ? 8 : 4) == 0;
#define SA_LAUNCH(BITS, BF, VEC)                \
    if (bits == BITS && bf16 == BF && vec == VEC) \
        hipLaunchKernelGGL((cache_write_kernel<BITS, BF, VEC>), grid, dim3(256), 0, stream, a);
    SA_LAUNCH(4, true, true)
    SA_LAUNCH(4, true, false)
    SA_LAUNCH(4, false, true)
    SA_LAUNCH(4, false, false)
    SA_LAUNCH(8, true, true)
    SA_LAUNCH(8, true, false)
    SA_LAUNCH(8, false, true)
    SA_LAUNCH(8, false, false)
#undef SA_LAUNCH
    if (a.claimed) hipLaunchKernelGGL(cache_settle_kernel, users, dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_cache_read(const CacheView& c, int bits, void* out, bool bf16, int64_t B, hipStream_t stream) {
    if (B <= 0) return hipSuccess;
    IoArgs a = io_args(c, B);
    a.out = out;
    const dim3 grid((unsigned)(B * a.per_user));
    const bool vec = c.D % (bf16 ? 8 : 4) == 0;
#define SA_LAUNCH(BITS, BF, VEC)                \
    if (bits == BITS && bf16 == BF && vec == VEC) \
        hipLaunchKernelGGL((cache_read_kernel<BITS, BF, VEC>), grid, dim3(256), 0, stream, a);
    SA_LAUNCH(4, true, true)
    SA_LAUNCH(4, true, false)
    SA_LAUNCH(4, false, true)
    SA_LAUNCH(4, false, false)
    SA_LAUNCH(8, true, true)
    SA_LAUNCH(8, true, false)
    SA_LAUNCH(8, false, true)
    SA_LAUNCH(8, false, false)
#undef SA_LAUNCH
    return hipGetLastError();
}

}  // namespace sa
