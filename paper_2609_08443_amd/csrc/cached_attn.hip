// Attention over cached sketches in one kernel (bf16 mode, D up to 1024): per user the
// rows u [N = R h][D] against the n valid rows X [n][D] of its slot,
//
//   s = scale u X^T,  alpha = softmax over the n rows,  c = alpha X,
//
// with X read as its 4- or 8-bit codes and decoded in registers, once for the logits
// and once for the weighted sum.  4 N n D multiply-adds against (N D) 4 + n D / 2 or
// n D bytes: the matrix cores bound it from some 100 rows u on, the cache's bytes below.
//
// A workgroup has one wave per 128 columns and takes 16 RM rows u.  Its rows u lie in LDS
// for the logits, which the waves share by keys: a wave takes tiles of 16 keys, whose
// codes nobody else needs, straight from memory as operands of v_mfma_f32_16x16x32_bf16
// (a lane's 8 values of its key).  Keys are the result's rows and u's its columns, so
// that a lane holds four neighbouring keys of one u and the softmax's sums over keys are
// mostly within a lane; the weights go to LDS as bf16 (over the rows u, which are done
// with, where all keys fit one chunk).  For the weighted sum the waves share the
// columns: a lane loads a block of 8 keys x 8 columns (the cache's layout has them
// together), decodes it along the columns and pairs neighbouring keys with byte
// permutes, which makes the block eight operands of 8 keys each: no code passes LDS.
//
// The running maximum, the sum and both accumulators are fp32; the weights are rounded to
// bf16 as matrix-core operands, the result once.
#include <algorithm>
#include <cstdlib>
#include <type_traits>

#include "cache.h"

namespace sa {

namespace {

using namespace cachefmt;
using tile::bf16x8;
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct AttnArgs {
    CacheView c;
    const uint16_t* U;   // [B][N][D]
    uint16_t* C;         // [B][N][D]
    float* lse;          // [B][N]
    float* part_c;       // [splits][B][N][D], not yet divided by the sum
    float2* part_ml;     // [splits][B][N]: maximum (log2 units) and sum
    int64_t B;
    int32_t N, row_tiles, splits, split_keys;   // split_keys a multiple of 32
    float scale2;        // scale log2(e)
};

// keys of a chunk: KT tiles of 16 a wave
constexpr int chunk_keys(int KT, int waves) { return 16 * KT * waves; }

template <int RM, int KT, bool LOOP>
constexpr int lds_bytes(int waves) {
    const int u = 16 * RM * 128 * waves * 2, p = 16 * RM * chunk_keys(KT, waves) * 2;
    return (LOOP ? u + p : (u > p ? u : p)) + 16 * RM * 4 * 2 * waves;
}

// 16-byte chunk c of row r of an LDS tile of rows of `chunks` chunks (a multiple of 8):
// eight neighbouring rows' chunks lie in different banks
__device__ inline int at16(int r, int c, int chunks) { return (r * chunks + (c ^ (r & 7))) * 8; }

// 8 rows x 8 columns of codes with their rows' scales: the operand words of column 2 I
// and 2 I + 1, keys in pairs
template <int BITS, int I>
__device__ inline void turn(const uint32_t (&raw)[8][BITS / 4], const float (&sc)[8], uint4& lo, uint4& hi) {
    uint32_t e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = decode2<BITS, I>(raw[j], sc[j]);
    lo = make_uint4(__builtin_amdgcn_perm(e[1], e[0], 0x05040100u), __builtin_amdgcn_perm(e[3], e[2], 0x05040100u),
                    __builtin_amdgcn_perm(e[5], e[4], 0x05040100u), __builtin_amdgcn_perm(e[7], e[6], 0x05040100u));
    hi = make_uint4(__builtin_amdgcn_perm(e[1], e[0], 0x07060302u), __builtin_amdgcn_perm(e[3], e[2], 0x07060302u),
                    __builtin_amdgcn_perm(e[5], e[4], 0x07060302u), __builtin_amdgcn_perm(e[7], e[6], 0x07060302u));
}

template <int BITS>
struct Block {   // 8 keys x 8 columns of codes, and the keys' scale bytes
    uint4 w[BITS / 2];   // 32 or 64 bytes
    uint2 s;
};
template <int BITS>
__device__ inline void load_block(Block<BITS>& b, const uint8_t* codes, const uint8_t* scales, uint32_t at, uint32_t sat) {
#pragma unroll
    for (int i = 0; i < BITS / 2; ++i) b.w[i] = *reinterpret_cast<const uint4*>(codes + at + 16 * i);
    b.s = *reinterpret_cast<const uint2*>(scales + sat);
}

// Logits of NT tiles of 16 keys (tile t at keys kb + t kstep) against the 16 RM rows u in LDS.
// The next GB groups' codes are on their way while this batch's are multiplied.
template <int BITS, int RM, int NT, int KT>
__device__ inline void logits(const AttnArgs& a, const uint8_t* codes, const uint8_t* scales, const uint16_t* Ul, int chunks,
                              int kb, int kstep, int last, int lane, f32x4 (&S)[KT][RM]) {
    constexpr int kRegs = RM >= 2 && (RM == 2 || BITS == 8) ? 8 : 16;
    constexpr int GB = kRegs / NT > 0 ? kRegs / NT : 1;
    constexpr int W = BITS / 4;
    const int l16 = lane & 15, q = lane >> 4;
    const int G = a.c.G;
    uint32_t at[NT], sat[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int key = min(kb + t * kstep + l16, last);   // rows past the last read that one
        const uint32_t og = (uint32_t)(key >> 3) * (uint32_t)G;
        at[t] = (og * 4 + q) * (8 * BITS) + (key & 7) * BITS;
        sat[t] = og * 8 + (key & 7);
#pragma unroll
        for (int rm = 0; rm < RM; ++rm) S[t][rm] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    uint32_t w[2][GB][NT][W], sc[2][GB][NT];
    auto fetch = [&](int buf, int g0) {
#pragma unroll
        for (int i = 0; i < GB; ++i) {
            const uint32_t g = (uint32_t)min(g0 + i, G - 1);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const uint8_t* p = codes + at[t] + g * (32 * BITS);
                if constexpr (BITS == 4) {
                    w[buf][i][t][0] = *reinterpret_cast<const uint32_t*>(p);
                } else {
                    const uint2 v = *reinterpret_cast<const uint2*>(p);
                    w[buf][i][t][0] = v.x;
                    w[buf][i][t][1] = v.y;
                }
                sc[buf][i][t] = scales[sat[t] + g * 8];
            }
        }
    };
    auto multiply = [&](int buf, int g0) {
#pragma unroll
        for (int i = 0; i < GB; ++i) {
            if (g0 + i >= G) return;
            bf16x8 u[RM];
#pragma unroll
            for (int rm = 0; rm < RM; ++rm) u[rm] = tile::lds_b128(Ul, at16(rm * 16 + l16, (g0 + i) * 4 + q, chunks));
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const bf16x8 x = __builtin_bit_cast(bf16x8, decode8<BITS>(w[buf][i][t], scale_float(sc[buf][i][t])));
#pragma unroll
                for (int rm = 0; rm < RM; ++rm)
                    S[t][rm] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, u[rm], S[t][rm], 0, 0, 0);
            }
        }
    };
    fetch(0, 0);
    for (int g0 = 0; g0 < G; g0 += 2 * GB) {
        fetch(1, g0 + GB);
        multiply(0, g0);
        if (g0 + GB < G) {
            fetch(0, g0 + 2 * GB);
            multiply(1, g0 + GB);
        }
    }
}

template <int BITS, int RM, int KT, bool LOOP>
__global__ __launch_bounds__(512) void cached_attn_kernel(AttnArgs a) {
    extern __shared__ uint4 smem[];
    const int waves = blockDim.x >> 6, chunks = 16 * waves, KC = chunk_keys(KT, waves);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
    uint16_t* const Ul = reinterpret_cast<uint16_t*>(smem);
    uint16_t* const Pl = LOOP ? Ul + 16 * RM * 128 * waves : Ul;
    float* const wmax = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(smem) +
                                                 (lds_bytes<RM, KT, LOOP>(waves) - 16 * RM * 4 * 2 * waves));
    float* const wsum = wmax + 16 * RM * waves;      // [wave][row], as wmax

    const int64_t id = tile::xcd_range(blockIdx.x, gridDim.x);
    const int rt = (int)(id % a.row_tiles);
    const int sp = (int)(id / a.row_tiles % a.splits);
    const int64_t b = id / a.row_tiles / a.splits;
    int32_t n;
    const uint8_t* const codes = cache_slot(a.c, b, &n);
    const uint8_t* const scales = codes + a.c.scales_at;
    const int D = a.c.D, N = a.N, row0 = rt * 16 * RM;
    const int k0 = sp * a.split_keys, k1 = min(n, k0 + a.split_keys);
    const int rows = min(16 * RM, N - row0);
    const int64_t prow = ((int64_t)sp * a.B + b) * N + row0;   // partial results' rows
    const int64_t urow = b * N + row0;
    if (k1 <= k0) {
        if (a.splits > 1) {
            for (int r = threadIdx.x; r < rows; r += blockDim.x) a.part_ml[prow + r] = make_float2(-INFINITY, 0.f);
        } else {
            for (int r = threadIdx.x; r < rows; r += blockDim.x) a.lse[urow + r] = -INFINITY;
            for (int64_t i = threadIdx.x; i < (int64_t)rows * D; i += blockDim.x) a.C[urow * D + i] = 0;
        }
        return;
    }

    // rows u: chunks of 8 values, zeros past D (the codes there are zeros, but 0 NaN is none);
    // rows past the last repeat it
    if (D % 32 == 0) {
        const int per = D / 8;   // straight into LDS, each lane the chunk that belongs at its place
        for (int i = wave * 64; i < 16 * RM * chunks; i += waves * 64) {
            const int r = (i + lane) / chunks, c = ((i + lane) % chunks) ^ (r & 7);
            tile::load_lds16(a.U + (urow + min(r, rows - 1)) * D + 8 * min(c, per - 1), Ul + (int64_t)i * 8);
        }
        tile::wait_vmem();
    } else {
        for (int i = threadIdx.x; i < 16 * RM * chunks; i += blockDim.x) {
            const int r = i / chunks, c = i % chunks;
            const uint16_t* from = a.U + (urow + min(r, rows - 1)) * D + 8 * c;
            uint32_t v[4] = {0u, 0u, 0u, 0u};
            for (int j = 0; j < 8; ++j)
                if (8 * c + j < D) v[j / 2] |= (uint32_t)from[j] << (16 * (j & 1));
            *reinterpret_cast<uint4*>(Ul + at16(r, c, chunks)) = make_uint4(v[0], v[1], v[2], v[3]);
        }
    }
    __syncthreads();

    f32x4 acc[8][RM];
    float m[RM], l[RM];
    if constexpr (LOOP) {
#pragma unroll
        for (int rm = 0; rm < RM; ++rm) {
            m[rm] = -INFINITY;
            l[rm] = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j][rm] = (f32x4){0.f, 0.f, 0.f, 0.f};
        }
    }
    const int dj = min(wave * 16 + l16, a.c.G * 4 - 1);   // this lane's octet of columns
    for (int c0 = k0; c0 < k1; c0 += KC) {
        const int kend = min(k1, c0 + KC);
        const int nk = (kend - c0 + 31) / 32 * 32;
        // ---- logits of this wave's key tiles
        f32x4 S[KT][RM];
        const int kb = c0 + 16 * wave, kstep = 16 * waves;
        const int nt = nk > 16 * wave ? (nk - 16 * wave + kstep - 1) / kstep : 0;
        if (nt > KT / 2) logits<BITS, RM, KT, KT>(a, codes, scales, Ul, chunks, kb, kstep, n - 1, lane, S);
        else if (nt > KT / 4) logits<BITS, RM, KT / 2, KT>(a, codes, scales, Ul, chunks, kb, kstep, n - 1, lane, S);
        else if (nt > 0) logits<BITS, RM, KT / 4, KT>(a, codes, scales, Ul, chunks, kb, kstep, n - 1, lane, S);
        // ---- softmax: the maximum over the chunk's keys, of all waves
#pragma unroll
        for (int rm = 0; rm < RM; ++rm) {
            float mx = -INFINITY;
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool in = t < nt && kb + t * kstep + 4 * q + i < kend;
                    S[t][rm][i] = in ? S[t][rm][i] * a.scale2 : -INFINITY;
                    mx = fmaxf(mx, S[t][rm][i]);
                }
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            if (q == 0) wmax[wave * 16 * RM + rm * 16 + l16] = mx;
        }
        __syncthreads();   // the rows u have been read, too
        float cor[RM];
#pragma unroll
        for (int rm = 0; rm < RM; ++rm) {
            float mx = wmax[rm * 16 + l16];
            for (int v = 1; v < waves; ++v) mx = fmaxf(mx, wmax[v * 16 * RM + rm * 16 + l16]);
            if constexpr (LOOP) mx = fmaxf(mx, m[rm]);
            const float base = mx == -INFINITY ? 0.f : mx;   // (logits that are all -inf)
            if constexpr (LOOP) cor[rm] = exp2f(m[rm] - base);
            m[rm] = mx;
            float sum = 0.f;
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                if (t < nt) {
                    float p[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        p[i] = __builtin_amdgcn_exp2f(S[t][rm][i] - base);
                        sum += p[i];
                    }
                    const int key = 16 * wave + t * kstep + 4 * q;   // in the chunk
                    *reinterpret_cast<uint2*>(Pl + at16(rm * 16 + l16, key >> 3, KC >> 3) + (key & 7)) =
                        make_uint2(tile::pack_bf16x2(p[0], p[1]), tile::pack_bf16x2(p[2], p[3]));
                }
            }
            sum += __shfl_xor(sum, 16, 64);
            sum += __shfl_xor(sum, 32, 64);
            if (q == 0) wsum[wave * 16 * RM + rm * 16 + l16] = sum;
        }
        __syncthreads();
#pragma unroll
        for (int rm = 0; rm < RM; ++rm) {
            float sum = wsum[rm * 16 + l16];
            for (int v = 1; v < waves; ++v) sum += wsum[v * 16 * RM + rm * 16 + l16];
            if constexpr (LOOP) l[rm] = l[rm] * cor[rm] + sum;
            else l[rm] = sum;
            if constexpr (LOOP) {
                // lane l16 of each quarter holds row l16's factor; the accumulators' rows are 4 q + i
                if (c0 > k0) {
                    float f[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) f[i] = __shfl(cor[rm], 4 * q + i, 64);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[j][rm][i] *= f[i];
                }
            }
        }
        // ---- the weighted sum of this wave's 128 columns
        if constexpr (!LOOP) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int rm = 0; rm < RM; ++rm) acc[j][rm] = (f32x4){0.f, 0.f, 0.f, 0.f};
        }
        const int olast = (n - 1) >> 3;
        auto place = [&](int kk, uint32_t& at, uint32_t& sat) {
            const int o = min((c0 >> 3) + kk * 4 + q, olast);
            const uint32_t og = (uint32_t)o * (uint32_t)a.c.G;
            at = (og * 4 + dj) * (8 * BITS);
            sat = (og + (dj >> 2)) * 8;
            return o;
        };
        const int steps = nk / 32;
        Block<BITS> cur, nxt;
        uint32_t at, sat;
        int o = place(0, at, sat), onext = o;
        load_block<BITS>(cur, codes, scales, at, sat);
        for (int kk = 0; kk < steps; ++kk) {
            if (kk + 1 < steps) {
                onext = place(kk + 1, at, sat);
                load_block<BITS>(nxt, codes, scales, at, sat);
            }
            bf16x8 p[RM];
#pragma unroll
            for (int rm = 0; rm < RM; ++rm) p[rm] = tile::lds_b128(Pl, at16(rm * 16 + l16, kk * 4 + q, KC >> 3));
            uint32_t raw[8][BITS / 4];
            float sc[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t* words = reinterpret_cast<const uint32_t*>(cur.w);
#pragma unroll
                for (int x = 0; x < BITS / 4; ++x) raw[j][x] = words[j * (BITS / 4) + x];
                const uint32_t s = j < 4 ? cur.s.x : cur.s.y;
                sc[j] = scale_float((s >> (8 * (j & 3))) & 255u);
            }
            if (c0 + kk * 32 + 32 > (n & ~7)) {
                // bytes behind the slot's last row may be anything: their weights are zero, and so are they
                const int in = n - 8 * o;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j >= in) {
#pragma unroll
                        for (int x = 0; x < BITS / 4; ++x) raw[j][x] = 0u;
                        sc[j] = 1.f;
                    }
            }
            auto columns = [&](auto I) {
                constexpr int i = decltype(I)::value;
                uint4 lo, hi;
                turn<BITS, i>(raw, sc, lo, hi);
#pragma unroll
                for (int rm = 0; rm < RM; ++rm) {
                    acc[2 * i][rm] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p[rm], __builtin_bit_cast(bf16x8, lo), acc[2 * i][rm], 0, 0, 0);
                    acc[2 * i + 1][rm] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p[rm], __builtin_bit_cast(bf16x8, hi), acc[2 * i + 1][rm], 0, 0, 0);
                }
            };
            columns(std::integral_constant<int, 0>{});
            columns(std::integral_constant<int, 1>{});
            columns(std::integral_constant<int, 2>{});
            columns(std::integral_constant<int, 3>{});
            cur = nxt;
            o = onext;
        }
        if constexpr (!LOOP) break;   // all keys are in one chunk
    }
    // ---- results: rows rm 16 + 4 q + i, this lane's columns 8 (16 wave + l16) ..+7
    if (wave == 0 && q == 0) {
#pragma unroll
        for (int rm = 0; rm < RM; ++rm) {
            const int r = rm * 16 + l16;
            if (r < rows) {
                if (a.splits > 1) a.part_ml[prow + r] = make_float2(m[rm], l[rm]);
                else a.lse[urow + r] = (m[rm] + __builtin_amdgcn_logf(l[rm])) * 0.6931471805599453f;
            }
        }
    }
    const int col = 8 * (wave * 16 + l16);
#pragma unroll
    for (int rm = 0; rm < RM; ++rm) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float sum = __shfl(l[rm], 4 * q + i, 64);
            const int r = rm * 16 + 4 * q + i;
            if (r >= rows || col >= D) continue;
            if (a.splits > 1) {
                float* to = a.part_c + (prow + r) * D + col;
                if (D % 8 == 0) {
                    *reinterpret_cast<float4*>(to) = make_float4(acc[0][rm][i], acc[1][rm][i], acc[2][rm][i], acc[3][rm][i]);
                    *reinterpret_cast<float4*>(to + 4) = make_float4(acc[4][rm][i], acc[5][rm][i], acc[6][rm][i], acc[7][rm][i]);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (col + j < D) to[j] = acc[j][rm][i];
                }
            } else {
                const float inv = 1.f / sum;
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = acc[j][rm][i] * inv;
                uint16_t* to = a.C + (urow + r) * D + col;
                if (D % 8 == 0) {
                    *reinterpret_cast<uint4*>(to) = __builtin_bit_cast(uint4, tile::pack8(v));
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (col + j < D) to[j] = tile::to_bf16(v[j]);
                }
            }
        }
    }
}

// Joins the splits of each row: their sums and accumulators, each scaled to the common
// maximum.  One thread per 8 columns.
__global__ __launch_bounds__(256) void cached_join_kernel(AttnArgs a) {
    const int D = a.c.D, per = (D + 7) / 8;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t rows = a.B * a.N;
    if (i >= rows * per) return;
    const int64_t row = i / per;
    const int col = (int)(i % per) * 8;
    float m = -INFINITY;
    for (int s = 0; s < a.splits; ++s) m = fmaxf(m, a.part_ml[s * rows + row].x);
    const float base = m == -INFINITY ? 0.f : m;
    float sum = 0.f, v[8] = {};
    for (int s = 0; s < a.splits; ++s) {
        const float2 ml = a.part_ml[s * rows + row];
        if (ml.y == 0.f) continue;   // no keys: nothing was written
        const float f = exp2f(ml.x - base);
        sum += f * ml.y;
        const float* from = a.part_c + (s * rows + row) * D + col;
        if (D % 8 == 0) {
            const float4 x = *reinterpret_cast<const float4*>(from), y = *reinterpret_cast<const float4*>(from + 4);
            v[0] += f * x.x; v[1] += f * x.y; v[2] += f * x.z; v[3] += f * x.w;
            v[4] += f * y.x; v[5] += f * y.y; v[6] += f * y.z; v[7] += f * y.w;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (col + j < D) v[j] += f * from[j];
        }
    }
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    if (col == 0) a.lse[row] = (m + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
    uint16_t* to = a.C + row * D + col;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= inv;
    if (D % 8 == 0) {
        *reinterpret_cast<uint4*>(to) = __builtin_bit_cast(uint4, tile::pack8(v));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (col + j < D) to[j] = tile::to_bf16(v[j]);
    }
}

template <int BITS, int RM, int KT, bool LOOP>
hipError_t launch_instance(const AttnArgs& a, hipStream_t stream) {
    const int waves = (a.c.D + 127) / 128;
    const int lds = lds_bytes<RM, KT, LOOP>(waves);
    auto kern = cached_attn_kernel<BITS, RM, KT, LOOP>;
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    const int64_t blocks = a.B * a.row_tiles * a.splits;
    hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(64 * waves), lds, stream, a);
    return hipGetLastError();
}

struct AttnPlan {
    int variant;   // 0: 16 rows u a workgroup, 1: 32, 2: 64 with all keys in one chunk
    int row_tiles, splits, split_keys;
};

AttnPlan attn_plan(int64_t B, int32_t N, int32_t k, int32_t D) {
    AttnPlan p;
    const int waves = (D + 127) / 128;
    p.variant = N <= 16 ? 0 : N > 32 && k <= chunk_keys(8, waves) ? 2 : 1;
#ifdef SA_EXPERIMENT
    if (getenv("SA_V")) p.variant = atoi(getenv("SA_V"));
#endif
    const int rows = 16 << p.variant;
    p.row_tiles = (N + rows - 1) / rows;
    const int64_t wgs = B * p.row_tiles;
    int64_t most = std::max<int64_t>(1, device_cus() / std::max<int64_t>(wgs, 1));
    const int least = 16 * waves < 32 ? 32 : 16 * waves;   // keys that give every wave a tile
    int64_t keys = std::max<int64_t>(least, (k + most - 1) / most);
    p.split_keys = (int)((keys + 31) / 32 * 32);
    p.splits = (k + p.split_keys - 1) / p.split_keys;
    return p;
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

bool cached_attn_supported(int32_t D) { return D <= 1024; }

size_t cached_attn_workspace(int64_t B, int32_t N, int32_t k, int32_t D) {
    const AttnPlan p = attn_plan(B, N, k, D);
    if (p.splits <= 1) return 0;
    return up256((size_t)p.splits * B * N * sizeof(float2)) + (size_t)p.splits * B * N * D * 4;
}

hipError_t launch_cached_attn(const CacheView& c, int bits, const uint16_t* U, uint16_t* C, float* lse, void* part,
                              int64_t B, int32_t N, float scale, hipStream_t stream) {
    if (B <= 0 || N <= 0) return hipSuccess;
    const AttnPlan p = attn_plan(B, N, c.k, c.D);
    AttnArgs a;
    a.c = c;
    a.U = U;
    a.C = C;
    a.lse = lse;
    a.part_ml = reinterpret_cast<float2*>(part);
    a.part_c = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(part) + up256((size_t)p.splits * B * N * sizeof(float2)));
    a.B = B;
    a.N = N;
    a.row_tiles = p.row_tiles;
    a.splits = p.splits;
    a.split_keys = p.split_keys;
    a.scale2 = scale * tile::kLog2e;
    hipError_t e = hipErrorInvalidValue;
    if (bits == 4) {
        if (p.variant == 0) e = launch_instance<4, 1, 8, true>(a, stream);
        else if (p.variant == 1) e = launch_instance<4, 2, 8, true>(a, stream);
        else e = launch_instance<4, 4, 8, false>(a, stream);
    } else {
        if (p.variant == 0) e = launch_instance<8, 1, 8, true>(a, stream);
        else if (p.variant == 1) e = launch_instance<8, 2, 8, true>(a, stream);
        else e = launch_instance<8, 4, 8, false>(a, stream);
    }
    if (e != hipSuccess || p.splits == 1) return e;
    const int64_t threads = B * N * ((c.D + 7) / 8);
    hipLaunchKernelGGL(cached_join_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace sa
