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
// The running maximum, the sum and both accumulators are fp32.  Operands of the matrix cores
// are bf16, each rounded once: q W_Q, the rows u, the weights, the aggregates, and the result
// where it is asked for so.  Off by 0.36 to 0.39% by 2-norm with full sketches, a bf16 result
// alone by 0.17%.  In two bf16 parts u and the weights would double both contractions, and two
// parts of 48 rows u do not fit LDS; with q W_Q in two parts the result is off by 0.30 to 0.32%
// and a call takes 2% longer (one target, 16 users with 300, 32 with 40), with the aggregates
// besides 0.27% and 4 to 11%.
#include <algorithm>
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
    // whole heads: the projections around the attention, too
    const uint16_t *Qp, *Wk, *Wv;   // q W_Q [B][R][D]; [D][D]
    void* out;                      // [B][R][D], bf16 or fp32
    bool out_bf16;
    int32_t R, h, dh;               // dh a multiple of 32; N = R h, row_tiles tiles of targets a head
    // backward: out is dQp (bf16), C is written too
    const uint16_t *q, *dout;       // [B][R][D]
    const float* Qf;                // Qp (whole heads), left in Qb as bf16
    uint16_t *Qb, *q0, *dout0;      // [B][R][D]: Qp, q and dout, zeros for users without rows
    const uint16_t* dC;             // [B][N][D] (else)
    uint16_t* dU;                   // [B][N][D]
    float scale;
};

// keys of a chunk: KT tiles of 16 a wave
constexpr int chunk_keys(int KT, int waves) { return 16 * KT * waves; }

// [rows u | weights (LOOP; else over the rows u) | maxima and sums of the waves | scales of the
// waves' keys]; before that (HEADS) [64 values of W_K's rows | of the targets]
template <int RM, int KT, bool LOOP>
constexpr int lds_tiles(int waves) {
    const int u = 16 * RM * 128 * waves * 2, p = 16 * RM * chunk_keys(KT, waves) * 2;
    return LOOP ? u + p : (u > p ? u : p);
}
// An octet of rows' scales in a wave's copy in LDS, padded so that octets lie in different banks
constexpr int scale_stride(int waves) { return 4 * waves * 8 + 8; }
template <int RM, int KT, bool LOOP, bool HEADS>
constexpr int lds_bytes(int waves) {
    const int s = lds_tiles<RM, KT, LOOP>(waves) + 16 * RM * 4 * 2 * waves + waves * 8 * scale_stride(waves);
    const int t = HEADS ? waves * 128 * 64 * 2 + 16 * RM * 64 * 2 * 2 : 0;   // (targets in two parts)
    return s > t ? s : t;
}

// 16-byte chunk c of row r of an LDS tile of rows of `chunks` chunks (a multiple of 8):
// eight neighbouring rows' chunks lie in different banks
__device__ inline int at16(int r, int c, int chunks) { return (r * chunks + (c ^ (r & 7))) * 8; }

// A user's codes and scale bytes as buffers: a lane's offset in a vector register, the step's in a
// scalar one (as sums of pointers they took two thirds of the logits' vector instructions
// besides the decoding), and nothing outside the slot is read.
struct Slot {
    __amdgpu_buffer_rsrc_t codes, scales;
};
__device__ inline __amdgpu_buffer_rsrc_t buffer_of(const uint8_t* p, int64_t bytes) {
    const uint64_t u = reinterpret_cast<uint64_t>(p);
    const uint64_t v = (uint64_t)__builtin_amdgcn_readfirstlane((int)(u >> 32)) << 32 |
                       (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)u);
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(v), 0, (int)bytes, 0x00027000);
}
__device__ inline Slot slot_of(const CacheView& c, const uint8_t* codes) {
    return {buffer_of(codes, c.scales_at), buffer_of(codes + c.scales_at, c.slot_bytes - c.scales_at)};
}

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
__device__ inline void load_block(Block<BITS>& b, const Slot& x, uint32_t at, uint32_t step, uint32_t sat, uint32_t sstep) {
#pragma unroll
    for (int i = 0; i < BITS / 2; ++i)
        b.w[i] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(x.codes, at + 16 * i, step, 0));
    b.s = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(x.scales, sat, sstep, 0));
}

// Logits of NT tiles of 16 keys from kb on against the 16 RM rows u in LDS, into S[T0 ..].
// The load path takes four lanes at a time and 64 bytes that lie together in one go:
// NT = 4, 64 keys: lane l16's keys are 32 j + 2 l16 and the next, in tiles 2 j and 2 j + 1, so
// that four lanes read one block of 8 rows x 8 values (with one key a lane, four lanes' rows,
// it was the load path that bound this loop; with four keys a lane, whose octets lie apart,
// more so), and the scales come through LDS, 256 bytes a row octet copied by the wave
// beforehand.  A lane's results S[T0 + 2 j + s][.][i] are keys 32 j + 8 q + 2 i + s.
// NT = 1: 16 keys, lane l16's the l16-th, results 4 q + i.
// The codes of the next GB groups are on their way while a group is multiplied.  The
// groups run to the end of the rows u in LDS (a multiple of 128 columns), which hold zeros
// from 32 G on; the codes read there are the last group's.  Octets past the slot's last
// valid one, olast, read that one.
template <int BITS, int RM, int T0, int NT, int KT>
__device__ __forceinline__ void logits(const AttnArgs& a, const Slot& x, const uint16_t* Ul, uint8_t* Sl, int chunks, int kb,
                                       int olast, int first, int lane, f32x4 (&S)[KT][RM]) {
    static_assert(NT == 1 || NT == 4, "one key a lane, or four");
    constexpr int GB = NT == 1 ? 16 : 4;
    constexpr int NJ = NT == 1 ? 1 : 2;             // loads a group
    constexpr int W = (NT == 1 ? 1 : 2) * BITS / 4;  // words of a load
    const int l16 = lane & 15, q = lane >> 4;
    const int G = a.c.G, Gp = chunks / 4, stride = 8 * Gp + 8;
    uint32_t at[NJ];
    uint32_t sat = 0;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const int key = kb + (NT == 1 ? l16 : 32 * j + 2 * l16);
        const uint32_t og = (uint32_t)min(key >> 3, olast) * (uint32_t)G;
        at[j] = (og * 4 + q) * (8 * BITS) + (key & 7) * BITS;
        if (NT == 1) sat = og * 8 + (key & 7);
    }
    if constexpr (NT == 4) {
        const int o = lane >> 3;
        const uint32_t from = (uint32_t)min((kb >> 3) + o, olast) * (uint32_t)G * 8;
        for (int g = lane & 7; g < Gp; g += 8)
            *reinterpret_cast<uint2*>(Sl + o * stride + 8 * g) =
                __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(x.scales, from + 8 * min(g, G - 1), 0, 0));
        tile::wave_lds_order();
    }
    const uint8_t* const sl = Sl + (l16 >> 2) * stride + 2 * (l16 & 3);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int rm = 0; rm < RM; ++rm) S[T0 + t][rm] = (f32x4){0.f, 0.f, 0.f, 0.f};
    uint32_t w[GB][NJ][W], sc[GB];
    auto fetch = [&](int i, int g) {
        g = min(g, G - 1);
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const uint32_t step = (uint32_t)g * (32 * BITS);
            if constexpr (W == 4) {
                const uint4 v = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(x.codes, at[j], step, 0));
                w[i][j][0] = v.x; w[i][j][1] = v.y; w[i][j][2 % W] = v.z; w[i][j][3 % W] = v.w;
            } else if constexpr (W == 2) {
                const uint2 v = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(x.codes, at[j], step, 0));
                w[i][j][0] = v.x;
                w[i][j][1 % W] = v.y;
            } else {
                w[i][j][0] = __builtin_amdgcn_raw_buffer_load_b32(x.codes, at[j], step, 0);
            }
        }
        if constexpr (NT == 1) sc[i] = __builtin_amdgcn_raw_buffer_load_b8(x.scales, sat, (uint32_t)g * 8, 0);
    };
    // the lane's chunk of rows rm 16 + l16 in groups of even and odd number; two groups on, 128 bytes
    const uint16_t* u[2][RM];
#pragma unroll
    for (int rm = 0; rm < RM; ++rm) {
        u[0][rm] = Ul + at16(l16, q, chunks) + rm * 16 * chunks * 8;
        u[1][rm] = Ul + at16(l16, 4 + q, chunks) + rm * 16 * chunks * 8;
    }
    // group base + i, base a multiple of four
    auto multiply = [&](int i, int base) {
        bf16x8 y[RM];
#pragma unroll
        for (int rm = 0; rm < RM; ++rm) y[rm] = tile::lds_b128(u[i & 1][rm] + (base >> 1) * 64, (i >> 1) * 64);
        const uint8_t* const sg = sl + 8 * base;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            uint32_t s2;
            if constexpr (NT == 1) s2 = sc[i];
            else s2 = *reinterpret_cast<const uint16_t*>(sg + j * 4 * stride + 8 * i);
#pragma unroll
            for (int t = 0; t < NT / NJ; ++t) {
                uint32_t c[BITS / 4];
#pragma unroll
                for (int v = 0; v < BITS / 4; ++v) c[v] = w[i][j][t * (BITS / 4) + v];
                const bf16x8 z = __builtin_bit_cast(bf16x8, decode8<BITS>(c, scale_float((s2 >> (8 * t)) & 255u)));
#pragma unroll
                for (int rm = 0; rm < RM; ++rm)
                    S[T0 + 2 * j + t][rm] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(z, y[rm], S[T0 + 2 * j + t][rm], 0, 0, 0);
            }
        }
    };
    if constexpr (NT == 4) {
        // from group `first` (a multiple of four, as Gp) round to it again
#pragma unroll
        for (int i = 0; i < 4; ++i) fetch(i, first + i);
        int base = first;
        for (int g0 = 0; g0 < Gp; g0 += 4) {
            const int next = base + 4 < Gp ? base + 4 : 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                multiply(i, base);
                fetch(i, next + i);
            }
            base = next;
        }
    } else {
#pragma unroll
        for (int i = 0; i < GB; ++i) fetch(i, i);
        for (int g0 = 0; g0 < Gp; g0 += GB) {
#pragma unroll
            for (int i = 0; i < GB; ++i) {
                if (g0 + i < Gp) multiply(i, g0);
                fetch(i, g0 + GB + i);
            }
        }
    }
}

// Rows u of one head's targets into LDS: U = Qp_i W_K^(i)T, a wave its 128 columns, 64 of the
// head's width at a time.  W_K's rows come through LDS in whole lines, wave by wave in the
// place that the rows u take afterwards (loaded as operands, 16 rows a load, they took four
// times the load path's time: 15,000 of 147,000 cycles of a workgroup of 64 rows and 1,024
// keys), and the targets' values once for all waves.  Columns of u are the result's rows, so
// that a lane writes four neighbouring ones; those past D are zeros.  fp32 targets go in as two
// bf16 parts, v = hi + lo to 2^-17 of v, and hi is left in Qb for a later product.
template <int RM, typename T>
__device__ __forceinline__ void project_rows(const T* Qp, const uint16_t* Wk, int D, int dh, int rows, int wave, int lane,
                                             uint16_t* Ul, int chunks, uint16_t* Ql, uint16_t* Qb = nullptr) {
    constexpr bool SPLIT = sizeof(T) == 4;
    const int l16 = lane & 15, q = lane >> 4;
    uint16_t* const mine = Ul + wave * (128 * 64);
    f32x4 u[8][RM];
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int rm = 0; rm < RM; ++rm) u[e][rm] = (f32x4){0.f, 0.f, 0.f, 0.f};
    const int r8 = lane >> 3, c8 = lane & 7;
    for (int k = 0; k < dh; k += 64) {
        // (a width that ends at 32 repeats W_K's first 32 there and multiplies them by zeros;
        // columns past D read the last's; D D values are counted in 32 bits)
        if (k) __syncthreads();   // the last 64 have been read
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int e = 8 * i + r8, c = c8 ^ (e & 7);
            tile::load_lds16(Wk + (uint32_t)(min(128 * wave + e, D - 1) * D + k + (k + 8 * c < dh ? 8 * c : 8 * c - 32)),
                             mine + i * 512);
        }
        for (int i = threadIdx.x; i < 16 * RM * 8; i += blockDim.x) {
            const int r = i >> 3, c = i & 7;
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            const int64_t at = (int64_t)min(r, rows - 1) * D + k + 8 * c;
            if constexpr (SPLIT) {
                uint4 lo = v;
                if (k + 8 * c < dh) {
                    const float4 x = *reinterpret_cast<const float4*>(Qp + at), y = *reinterpret_cast<const float4*>(Qp + at + 4);
                    v = make_uint4(tile::pack_bf16x2(x.x, x.y), tile::pack_bf16x2(x.z, x.w), tile::pack_bf16x2(y.x, y.y),
                                   tile::pack_bf16x2(y.z, y.w));
                    auto rest = [](uint32_t h, float a, float b) { return tile::pack_bf16x2(a - tile::bf16_lo(h), b - tile::bf16_hi(h)); };
                    lo = make_uint4(rest(v.x, x.x, x.y), rest(v.y, x.z, x.w), rest(v.z, y.x, y.y), rest(v.w, y.z, y.w));
                    if (r < rows) *reinterpret_cast<uint4*>(Qb + at) = v;
                }
                *reinterpret_cast<uint4*>(Ql + 16 * RM * 64 + at16(r, c, 8)) = lo;
            } else if (k + 8 * c < dh) {
                v = *reinterpret_cast<const uint4*>(Qp + at);
            }
            *reinterpret_cast<uint4*>(Ql + at16(r, c, 8)) = v;
        }
        tile::wait_vmem();
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            bf16x8 x[RM], lo[RM];
#pragma unroll
            for (int rm = 0; rm < RM; ++rm) {
                x[rm] = tile::lds_b128(Ql, at16(rm * 16 + l16, 4 * i + q, 8));
                if constexpr (SPLIT) lo[rm] = tile::lds_b128(Ql + 16 * RM * 64, at16(rm * 16 + l16, 4 * i + q, 8));
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bf16x8 w = tile::lds_b128(mine, at16(16 * e + l16, 4 * i + q, 8));
#pragma unroll
                for (int rm = 0; rm < RM; ++rm) {
                    if constexpr (SPLIT) u[e][rm] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, lo[rm], u[e][rm], 0, 0, 0);
                    u[e][rm] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x[rm], u[e][rm], 0, 0, 0);
                }
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int rm = 0; rm < RM; ++rm)
            *reinterpret_cast<uint2*>(Ul + at16(rm * 16 + l16, 16 * wave + 2 * e + (q >> 1), chunks) + 4 * (q & 1)) =
                128 * wave + 16 * e + 4 * q < D
                    ? make_uint2(tile::pack_bf16x2(u[e][rm][0], u[e][rm][1]), tile::pack_bf16x2(u[e][rm][2], u[e][rm][3]))
                    : make_uint2(0u, 0u);
}

// 16 RM rows of D values into LDS, zeros past D; rows past the last repeat it
template <int RM>
__device__ __forceinline__ void load_rows(const uint16_t* U, int D, int rows, int waves, int wave, int lane, uint16_t* Ul,
                                          int chunks) {
    if (D % 128 == 0) {   // straight into LDS, each lane the chunk that belongs at its place
        for (int i = wave * 64; i < 16 * RM * chunks; i += waves * 64) {
            const int r = (i + lane) / chunks, c = ((i + lane) % chunks) ^ (r & 7);
            tile::load_lds16(U + (int64_t)min(r, rows - 1) * D + 8 * c, Ul + (int64_t)i * 8);
        }
        tile::wait_vmem();
        return;
    }
    for (int i = threadIdx.x; i < 16 * RM * chunks; i += blockDim.x) {
        const int r = i / chunks, c = i % chunks;
        const uint16_t* from = U + (int64_t)min(r, rows - 1) * D + 8 * c;
        uint32_t v[4] = {0u, 0u, 0u, 0u};
        if (D % 8 == 0) {
            if (8 * c < D) {
                const uint4 x = *reinterpret_cast<const uint4*>(from);
                v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
            }
        } else {
            for (int j = 0; j < 8; ++j)
                if (8 * c + j < D) v[j / 2] |= (uint32_t)from[j] << (16 * (j & 1));
        }
        *reinterpret_cast<uint4*>(Ul + at16(r, c, chunks)) = make_uint4(v[0], v[1], v[2], v[3]);
    }
}

// out = c W of one head, c [16 RM][128 waves] in accumulators (rows rm 16 + 4 q + i, columns
// 8 (16 wave + l16) + j): each wave multiplies its own 128 columns of c, through its own part
// of LDS into operand order, with their rows of W [D][dh of D], 64 columns of out at a time;
// the waves' sums meet in LDS.  W's operands are blocks of 8 rows x 4 columns, paired by byte
// permutes as the codes are.  All waves have left LDS before.  SPLIT: c goes in as two bf16
// parts, its leading 8 bits and the next.
template <int RM, bool SPLIT>
__device__ __forceinline__ void project_out(const AttnArgs& a, const f32x4 (&acc)[8][RM], const float (&inv)[RM][4],
                                   const uint16_t* W, int rows, int64_t row0, int head, int waves, int wave, int lane,
                                   uint16_t* lds) {
    const int l16 = lane & 15, q = lane >> 4, D = a.c.D;
    uint16_t* const mine = lds + wave * (16 * RM * 128);
    const bool in = 8 * (16 * wave + l16) < D;
    // two 32-row steps of W ahead, the first two before c is turned (W's bytes from its head's
    // first column on are counted in 32 bits: D is at most 1024)
    uint2 w[2][8];
    auto fetch = [&](int k, int j0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {   // (rows past D meet c's zero columns; the last one's values are as good as any)
            const uint32_t at = (uint32_t)(min(128 * wave + 32 * k + 8 * q + e, D - 1) * D + min(j0 + 4 * l16, a.dh - 4));
            w[k & 1][e] = *reinterpret_cast<const uint2*>(W + at);
        }
    };
    fetch(0, 0);
    fetch(1, 0);
    bf16x8 c[SPLIT ? 2 : 1][4][RM];
#pragma unroll
    for (int part = 0; part < (SPLIT ? 2 : 1); ++part) {
#pragma unroll
        for (int rm = 0; rm < RM; ++rm)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[j] = in ? acc[j][rm][i] * inv[rm][i] : 0.f;
                    if (part == 1) v[j] -= tile::bf16_lo(tile::to_bf16(v[j]));
                }
                *reinterpret_cast<uint4*>(mine + at16(rm * 16 + 4 * q + i, l16, 16)) = __builtin_bit_cast(uint4, tile::pack8(v));
            }
        tile::wave_lds_order();
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int rm = 0; rm < RM; ++rm) c[part][k][rm] = tile::lds_b128(mine, at16(rm * 16 + l16, 4 * k + q, 16));
        tile::wave_lds_order();
    }
    for (int j0 = 0; j0 < a.dh; j0 += 64) {
        f32x4 o[4][RM];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int rm = 0; rm < RM; ++rm) o[j][rm] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint2(&x)[8] = w[k & 1];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    p[e] = __builtin_amdgcn_perm(j < 2 ? x[2 * e + 1].x : x[2 * e + 1].y, j < 2 ? x[2 * e].x : x[2 * e].y,
                                                 (j & 1) ? 0x07060302u : 0x05040100u);
                const bf16x8 b = __builtin_bit_cast(bf16x8, make_uint4(p[0], p[1], p[2], p[3]));
#pragma unroll
                for (int rm = 0; rm < RM; ++rm) {
                    if constexpr (SPLIT) o[j][rm] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(c[1][k][rm], b, o[j][rm], 0, 0, 0);
                    o[j][rm] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(c[0][k][rm], b, o[j][rm], 0, 0, 0);
                }
            }
            if (k < 2) fetch(k + 2, j0);
            else if (j0 + 64 < a.dh) fetch(k - 2, j0 + 64);
        }
        if (j0) __syncthreads();   // the last 64 columns' sums have been read
        float* const part = reinterpret_cast<float*>(mine);   // [row][64]
#pragma unroll
        for (int rm = 0; rm < RM; ++rm)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<float4*>(part + (rm * 16 + 4 * q + i) * 64 + 4 * l16) =
                    make_float4(o[0][rm][i], o[1][rm][i], o[2][rm][i], o[3][rm][i]);
        __syncthreads();
        for (int i = threadIdx.x; i < rows * 16; i += blockDim.x) {
            const int r = i >> 4, cc = 4 * (i & 15);
            if (j0 + cc >= a.dh) continue;
            const float* from = reinterpret_cast<const float*>(lds) + r * 64 + cc;
            float4 s = *reinterpret_cast<const float4*>(from);
            for (int v = 1; v < waves; ++v) {
                const float4 x = *reinterpret_cast<const float4*>(from + v * (16 * RM * 64));
                s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
            }
            const int64_t to = (row0 + r) * D + head * a.dh + j0 + cc;
            if (a.out_bf16)
                *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.out) + to) =
                    make_uint2(tile::pack_bf16x2(s.x, s.y), tile::pack_bf16x2(s.z, s.w));
            else
                *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + to) = s;
        }
    }
}

// The keys of a chunk that a wave's logits are of: up to KT / 4 runs of 64 (wide), or, where that
// would leave waves without keys, of 16; the first at kb of the chunk, the next kstep on.
struct Keys {
    int c0, kend, nk;   // the chunk's first and last key; their number in whole 32s
    bool wide;
    int run, kb, kstep, nt;
};
template <int KT>
__device__ inline Keys wave_keys(int c0, int kend, int waves, int wave) {
    Keys k;
    k.c0 = c0;
    k.kend = kend;
    k.nk = (kend - c0 + 31) / 32 * 32;
    k.wide = k.nk > 4 * KT * waves;
    k.run = k.wide ? 64 : 16;
    k.kb = k.run * wave;
    k.kstep = k.run * waves;
    k.nt = k.nk > k.kb ? min((k.nk - k.kb + k.kstep - 1) / k.kstep, KT / 4) : 0;
    return k;
}

// A wave's logits of its keys; `fill` where there is none
template <int BITS, int RM, int KT>
__device__ __forceinline__ void wave_logits(const AttnArgs& a, const Slot& x, const uint16_t* Ul, uint8_t* Sl, int chunks, const Keys& k, int n, int first,
                                            int lane, float fill, f32x4 (&S)[KT][RM]) {
    static_assert(KT == 4 || KT == 8, "one or two runs of four tiles");
    const int q = lane >> 4, olast = (n - 1) >> 3, at = k.c0 + k.kb;
    if (k.nt > 0) {
        if (k.wide) logits<BITS, RM, 0, 4, KT>(a, x, Ul, Sl, chunks, at, olast, first, lane, S);
        else logits<BITS, RM, 0, 1, KT>(a, x, Ul, Sl, chunks, at, olast, first, lane, S);
    }
    if constexpr (KT == 8) {
        if (k.nt > 1) {
            if (k.wide) logits<BITS, RM, 4, 4, KT>(a, x, Ul, Sl, chunks, at + k.kstep, olast, first, lane, S);
            else logits<BITS, RM, 4, 1, KT>(a, x, Ul, Sl, chunks, at + k.kstep, olast, first, lane, S);
        }
    }
    if (k.wide && k.nt == KT / 4 && at + (k.nt - 1) * k.kstep + 64 <= k.kend) return;   // a full share
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int key = at + (t >> 2) * k.kstep + (k.wide ? 16 * (t & 2) + 8 * q + 2 * i + (t & 1) : 4 * q + i);
            const bool in = (t >> 2) < k.nt && (k.wide || (t & 3) == 0) && key < k.kend;
#pragma unroll
            for (int rm = 0; rm < RM; ++rm) S[t][rm][i] = in ? S[t][rm][i] : fill;
        }
}

// A run's values p[i][tile] of row r into LDS as bf16, keys in order
__device__ __forceinline__ void put_run(uint16_t* Pl, int r, int run, const Keys& k, int KC, int q, const float (&p)[4][4]) {
    const int c = (k.kb + run * k.kstep) >> 3;   // in chunks of 8 keys
    if (k.wide) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
            *reinterpret_cast<uint4*>(Pl + at16(r, c + 4 * x + q, KC >> 3)) =
                make_uint4(tile::pack_bf16x2(p[0][2 * x], p[0][2 * x + 1]), tile::pack_bf16x2(p[1][2 * x], p[1][2 * x + 1]),
                           tile::pack_bf16x2(p[2][2 * x], p[2][2 * x + 1]), tile::pack_bf16x2(p[3][2 * x], p[3][2 * x + 1]));
    } else {
        *reinterpret_cast<uint2*>(Pl + at16(r, c + (q >> 1), KC >> 3) + 4 * (q & 1)) =
            make_uint2(tile::pack_bf16x2(p[0][0], p[1][0]), tile::pack_bf16x2(p[2][0], p[3][0]));
    }
}

// acc += P X over the chunk's keys: a wave its 128 columns (dj: the lane's octet of them)
template <int BITS, int RM>
__device__ __forceinline__ void weighted_sum(const AttnArgs& a, const Slot& x, const uint16_t* Pl, int KC, int c0, int nk, int n, int dj, int lane,
                                             f32x4 (&acc)[8][RM]) {
    const int l16 = lane & 15, q = lane >> 4;
    const int steps = nk / 32, tail = steps - 1;
    // A lane's block of a step lies a fixed number of bytes behind the last step's (the steps
    // move in scalar registers), but in the last step, where octets past the slot's last one
    // read that one
    const uint32_t G = (uint32_t)a.c.G;
    const int otail = min((c0 >> 3) + 4 * tail + q, (n - 1) >> 3);
    const uint32_t oq = (uint32_t)((c0 >> 3) + q) * G, ot = (uint32_t)otail * G - (uint32_t)(4 * tail) * G;
    const uint32_t at0 = (oq * 4 + dj) * (8 * BITS), at1 = (ot * 4 + dj) * (8 * BITS);
    const uint32_t sat0 = (oq + (dj >> 2)) * 8, sat1 = (ot + (dj >> 2)) * 8;
    Block<BITS> b0, b1;
    auto fetch = [&](Block<BITS>& to, int kk) {   // (past the last step: that one, not used)
        kk = min(kk, tail);
        const uint32_t at = kk == tail ? at1 : at0, sat = kk == tail ? sat1 : sat0;
        const uint32_t step = (uint32_t)(4 * kk) * G;
        load_block<BITS>(to, x, at, step * (32 * BITS), sat, step * 8);
    };
    auto multiply = [&](const Block<BITS>& from, int kk) {
        bf16x8 p[RM];
#pragma unroll
        for (int rm = 0; rm < RM; ++rm) p[rm] = tile::lds_b128(Pl, at16(rm * 16 + l16, kk * 4 + q, KC >> 3));
        uint32_t raw[8][BITS / 4];
        float sc[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t* words = reinterpret_cast<const uint32_t*>(from.w);
#pragma unroll
            for (int x = 0; x < BITS / 4; ++x) raw[j][x] = words[j * (BITS / 4) + x];
            const uint32_t s = j < 4 ? from.s.x : from.s.y;
            sc[j] = scale_float((s >> (8 * (j & 3))) & 255u);
        }
        if (c0 + kk * 32 + 32 > (n & ~7)) {
            // bytes behind the slot's last row may be anything: their weights are zero, and so are they
            const int in = n - 8 * otail;
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
    };
    fetch(b0, 0);
    int kk = 0;
    for (; kk + 1 < steps; kk += 2) {
        fetch(b1, kk + 1);
        multiply(b0, kk);
        fetch(b0, kk + 2);
        multiply(b1, kk + 1);
    }
    if (kk < steps) multiply(b0, kk);
}

template <int BITS, int RM, int KT, bool LOOP, bool HEADS>
__global__ __launch_bounds__(512) void cached_attn_kernel(AttnArgs a) {
    extern __shared__ uint4 smem[];
    const int waves = blockDim.x >> 6, chunks = 16 * waves, KC = chunk_keys(KT, waves);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
    uint16_t* const Ul = reinterpret_cast<uint16_t*>(smem);
    uint16_t* const Pl = LOOP ? Ul + 16 * RM * 128 * waves : Ul;
    float* const wmax = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(smem) + lds_tiles<RM, KT, LOOP>(waves));
    float* const wsum = wmax + 16 * RM * waves;      // [wave][row], as wmax

    uint8_t* const Sl = reinterpret_cast<uint8_t*>(wsum + 16 * RM * waves) + wave * 8 * scale_stride(waves);
    const uint32_t id = (uint32_t)tile::xcd_range(blockIdx.x, gridDim.x);
    const int D = a.c.D, N = a.N;
    int64_t b;
    int sp = 0, head = 0, row0, rows;   // rows u of this workgroup: from row0 on, of the user or of the head's targets
    if constexpr (HEADS) {
        const uint32_t bh = id / (uint32_t)a.row_tiles;
        row0 = (int)(id - bh * (uint32_t)a.row_tiles) * 16 * RM;
        b = bh / (uint32_t)a.h;
        head = (int)(bh - (uint32_t)b * (uint32_t)a.h);
        rows = min(16 * RM, a.R - row0);
    } else {
        const uint32_t bs = id / (uint32_t)a.row_tiles;
        row0 = (int)(id - bs * (uint32_t)a.row_tiles) * 16 * RM;
        b = bs / (uint32_t)a.splits;
        sp = (int)(bs - (uint32_t)b * (uint32_t)a.splits);
        rows = min(16 * RM, N - row0);
    }
    int32_t n;
    const uint8_t* const codes = cache_slot(a.c, b, &n);
    const Slot x = slot_of(a.c, codes);
    const int k0 = sp * a.split_keys, k1 = min(n, k0 + a.split_keys);
    const int64_t prow = ((int64_t)sp * a.B + b) * N + row0;   // partial results' rows
    const int64_t urow = HEADS ? b * a.R + row0 : b * N + row0;
    if (k1 <= k0) {
        if constexpr (HEADS) {
            for (int r = threadIdx.x; r < rows; r += blockDim.x) a.lse[(urow + r) * a.h + head] = -INFINITY;
            for (int i = threadIdx.x; i < rows * a.dh; i += blockDim.x) {
                const int64_t to = (urow + i / a.dh) * D + head * a.dh + i % a.dh;
                if (a.out_bf16) reinterpret_cast<uint16_t*>(a.out)[to] = 0;
                else reinterpret_cast<float*>(a.out)[to] = 0.f;
            }
        } else if (a.splits > 1) {
            for (int r = threadIdx.x; r < rows; r += blockDim.x) a.part_ml[prow + r] = make_float2(-INFINITY, 0.f);
        } else {
            for (int r = threadIdx.x; r < rows; r += blockDim.x) a.lse[urow + r] = -INFINITY;
            for (int64_t i = threadIdx.x; i < (int64_t)rows * D; i += blockDim.x) a.C[urow * D + i] = 0;
        }
        return;
    }

    if constexpr (HEADS) {
        project_rows<RM>(a.Qp + urow * D + head * a.dh, a.Wk + head * a.dh, D, a.dh, rows, wave, lane, Ul, chunks,
                         Ul + waves * 128 * 64);
    } else {
        load_rows<RM>(a.U + urow * D, D, rows, waves, wave, lane, Ul, chunks);
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
    // each wave starts its logits at a group of its own: octets of rows lie a power of two of bytes
    // apart (D = 1024), so that one group of all of them is in one channel of the L2
    const int first = 4 * (int)((uint32_t)(3 * wave + 5 * id) % (uint32_t)(chunks / 16));
    for (int c0 = k0; c0 < k1; c0 += KC) {
        const Keys keys = wave_keys<KT>(c0, min(k1, c0 + KC), waves, wave);
        f32x4 S[KT][RM];
        wave_logits<BITS, RM, KT>(a, x, Ul, Sl, chunks, keys, n, first, lane, -INFINITY, S);
        // ---- softmax: the maximum over the chunk's keys, of all waves (scale2 > 0: the largest
        // logit has the largest product)
#pragma unroll
        for (int rm = 0; rm < RM; ++rm) {
            float mx = -INFINITY;
#pragma unroll
            for (int t = 0; t < KT; ++t) mx = fmaxf(fmaxf(fmaxf(mx, S[t][rm][0]), fmaxf(S[t][rm][1], S[t][rm][2])), S[t][rm][3]);
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
            mx *= a.scale2;
            if constexpr (LOOP) mx = fmaxf(mx, m[rm]);
            const float base = mx == -INFINITY ? 0.f : mx;   // (logits that are all -inf)
            if constexpr (LOOP) cor[rm] = exp2f(m[rm] - base);
            m[rm] = mx;
            float sum = 0.f;
#pragma unroll
            for (int t = 0; t < KT; t += 4) {
                if ((t >> 2) >= keys.nt) break;
                float p[4][4];   // [i][tile]
#pragma unroll
                for (int i = 0; i < 4; ++i) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        p[i][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[t + j][rm][i], a.scale2, -base));
                    sum += (p[i][0] + p[i][1]) + (p[i][2] + p[i][3]);
                }
                put_run(Pl, rm * 16 + l16, t >> 2, keys, KC, q, p);
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
        weighted_sum<BITS, RM>(a, x, Pl, KC, c0, keys.nk, n, dj, lane, acc);
        if constexpr (!LOOP) break;   // all keys are in one chunk
    }
    // ---- results: rows rm 16 + 4 q + i, this lane's columns 8 (16 wave + l16) ..+7
    if (wave == 0 && q == 0) {
#pragma unroll
        for (int rm = 0; rm < RM; ++rm) {
            const int r = rm * 16 + l16;
            if (r < rows) {
                if (HEADS) a.lse[(urow + r) * a.h + head] = (m[rm] + __builtin_amdgcn_logf(l[rm])) * 0.6931471805599453f;
                else if (a.splits > 1) a.part_ml[prow + r] = make_float2(m[rm], l[rm]);
                else a.lse[urow + r] = (m[rm] + __builtin_amdgcn_logf(l[rm])) * 0.6931471805599453f;
            }
        }
    }
    if constexpr (HEADS) {
        float inv[RM][4];
#pragma unroll
        for (int rm = 0; rm < RM; ++rm)
#pragma unroll
            for (int i = 0; i < 4; ++i) inv[rm][i] = 1.f / __shfl(l[rm], 4 * q + i, 64);
        __syncthreads();   // the weights in LDS have been read
        project_out<RM, false>(a, acc, inv, a.Wv + head * a.dh, rows, urow, head, waves, wave, lane, reinterpret_cast<uint16_t*>(smem));
        return;
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

// The rows' part of q and dout, copied for the weights' gradients, which sum over the targets of
// all users: those of users without rows (a padded batch's) may be NaN or infinite, and their zeros
// in C, dU and dQp times those are NaN.  They go in as zeros, and so does their Qp.
template <bool HEADS>
__device__ inline void keep_targets(const AttnArgs& a, int64_t urow, int head, int rows, bool any) {
    const int D = a.c.D, dh = a.dh;
    // (a row u's dh values, wherever its row of [B][R][h] is)
    const int64_t first = HEADS ? urow * D + head * dh : urow * dh, next = HEADS ? D : dh;
    if (HEADS || dh % 8 == 0) {
        const int per = dh / 8;
        for (int i = threadIdx.x; i < rows * per; i += blockDim.x) {
            const int64_t at = first + i / per * next + 8 * (i % per);
            uint4 q = make_uint4(0u, 0u, 0u, 0u), d = q;
            if (any) {
                q = *reinterpret_cast<const uint4*>(a.q + at);
                d = *reinterpret_cast<const uint4*>(a.dout + at);
            } else {
                *reinterpret_cast<uint4*>(a.Qb + at) = q;
            }
            *reinterpret_cast<uint4*>(a.q0 + at) = q;
            *reinterpret_cast<uint4*>(a.dout0 + at) = d;
        }
        return;
    }
    for (int i = threadIdx.x; i < rows * dh; i += blockDim.x) {
        const int64_t at = first + i;
        a.q0[at] = any ? a.q[at] : (uint16_t)0;
        a.dout0[at] = any ? a.dout[at] : (uint16_t)0;
        if (!any) a.Qb[at] = 0;
    }
}

// a user without rows: no C, dU and dQp
template <bool HEADS>
__device__ inline void no_rows(const AttnArgs& a, int64_t urow, int head, int rows) {
    const int D = a.c.D;
    for (int i = threadIdx.x; i < rows * D; i += blockDim.x) {
        const int64_t to = (HEADS ? (urow + i / D) * a.h + head : urow + i / D) * D + i % D;
        a.C[to] = 0;
        a.dU[to] = 0;
    }
    if constexpr (HEADS)
        for (int i = threadIdx.x; i < rows * a.dh; i += blockDim.x) {
            const int64_t at = (urow + i / a.dh) * D + head * a.dh + i % a.dh;
            reinterpret_cast<uint16_t*>(a.out)[at] = 0;
        }
    keep_targets<HEADS>(a, urow, head, rows, false);
}

// accumulators times their rows' factors to [B][R][h][D], bf16
template <int RM, bool HEADS>
__device__ __forceinline__ void store_rows(const AttnArgs& a, uint16_t* to, const f32x4 (&acc)[8][RM], const float (&f)[RM][4],
                                           int64_t urow, int head, int rows, int wave, int lane) {
    const int l16 = lane & 15, q = lane >> 4, D = a.c.D, col = 8 * (wave * 16 + l16);
#pragma unroll
    for (int rm = 0; rm < RM; ++rm)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = rm * 16 + 4 * q + i;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = acc[j][rm][i] * f[rm][i];
            if (r >= rows || col >= D) continue;
            const int64_t at = (HEADS ? (urow + r) * a.h + head : urow + r) * D + col;
            if (HEADS || D % 8 == 0) {
                *reinterpret_cast<uint4*>(to + at) = __builtin_bit_cast(uint4, tile::pack8(v));
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (col + j < D) to[at + j] = tile::to_bf16(v[j]);
            }
        }
}

// The attention's backward: of rows u and their aggregates' gradients dC (in LDS one after the
// other)
//   alpha = softmax(scale U X^T),  C = alpha X,
//   dA = dC X^T,  ds = scale alpha (dA - sum alpha dA),  dU = ds X,
// C and dU for the weights' gradients.  All keys in one chunk: the weights wait in registers,
// fp32, while C is summed and dA computed.  Four products of the forward's kind, each decoding
// the codes once.  HEADS: the rows are one head's targets, and the workgroup makes
// U = Qp_i W_K^(i)T and dC = dout_i W_V^(i)T itself, and dQp_i = dU W_K^(i).  Roundings to bf16 in
// the way to dq: U, dC, ds, dQp and the result, as operands of products too large to run twice;
// Qp and dU, of small ones, go in as two parts (with them rounded, single targets' gradients were
// up to 0.5% off by 2-norm, now 0.4%).
template <int BITS, int RM, int KT, bool HEADS>
__global__ __launch_bounds__(512) void cached_attn_bwd_kernel(AttnArgs a) {
    extern __shared__ uint4 smem[];
    const int waves = blockDim.x >> 6, chunks = 16 * waves, KC = chunk_keys(KT, waves);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
    uint16_t* const Ul = reinterpret_cast<uint16_t*>(smem);
    uint16_t* const Pl = Ul;
    float* const wmax = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(smem) + lds_tiles<RM, KT, false>(waves));
    float* const wsum = wmax + 16 * RM * waves;      // [wave][row], as wmax
    uint8_t* const Sl = reinterpret_cast<uint8_t*>(wsum + 16 * RM * waves) + wave * 8 * scale_stride(waves);
    const uint32_t id = (uint32_t)tile::xcd_range(blockIdx.x, gridDim.x);
    const int D = a.c.D;
    const uint32_t bh = id / (uint32_t)a.row_tiles;
    const int row0 = (int)(id - bh * (uint32_t)a.row_tiles) * 16 * RM;
    const int64_t b = HEADS ? bh / (uint32_t)a.h : bh;
    const int head = HEADS ? (int)(bh - (uint32_t)b * (uint32_t)a.h) : 0;
    const int rows = min(16 * RM, (HEADS ? a.R : a.N) - row0);
    int32_t n;
    const uint8_t* const codes = cache_slot(a.c, b, &n);
    const Slot x = slot_of(a.c, codes);
    const int64_t urow = b * (HEADS ? a.R : a.N) + row0;
    if (n <= 0) {
        no_rows<HEADS>(a, urow, head, rows);
        return;
    }
    const int first = 4 * (int)((uint32_t)(3 * wave + 5 * id) % (uint32_t)(chunks / 16));
    const int dj = min(wave * 16 + l16, a.c.G * 4 - 1);
    const Keys keys = wave_keys<KT>(0, n, waves, wave);
    uint16_t* const Ql = Ul + waves * 128 * 64;

    if constexpr (HEADS)
        project_rows<RM>(a.Qf + urow * D + head * a.dh, a.Wk + head * a.dh, D, a.dh, rows, wave, lane, Ul, chunks, Ql,
                         a.Qb + urow * D + head * a.dh);
    else
        load_rows<RM>(a.U + urow * D, D, rows, waves, wave, lane, Ul, chunks);
    __syncthreads();
    f32x4 S[KT][RM];   // logits, then weights before their division by the sum
    wave_logits<BITS, RM, KT>(a, x, Ul, Sl, chunks, keys, n, first, lane, -INFINITY, S);
#pragma unroll
    for (int rm = 0; rm < RM; ++rm) {
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < KT; ++t) mx = fmaxf(fmaxf(fmaxf(mx, S[t][rm][0]), fmaxf(S[t][rm][1], S[t][rm][2])), S[t][rm][3]);
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        if (q == 0) wmax[wave * 16 * RM + rm * 16 + l16] = mx;
    }
    __syncthreads();
#pragma unroll
    for (int rm = 0; rm < RM; ++rm) {
        float mx = wmax[rm * 16 + l16];
        for (int v = 1; v < waves; ++v) mx = fmaxf(mx, wmax[v * 16 * RM + rm * 16 + l16]);
        if (mx == -INFINITY) mx = 0.f;
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < KT; t += 4) {
            float p[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    {
                    // (the difference first: the largest weight is 1 exactly, and a row alone has no gradient)
                    p[i][j] = __builtin_amdgcn_exp2f((S[t + j][rm][i] - mx) * a.scale2);
                    S[t + j][rm][i] = p[i][j];
                }
                sum += (p[i][0] + p[i][1]) + (p[i][2] + p[i][3]);
            }
            if ((t >> 2) < keys.nt) put_run(Pl, rm * 16 + l16, t >> 2, keys, KC, q, p);
        }
        sum += __shfl_xor(sum, 16, 64);
        sum += __shfl_xor(sum, 32, 64);
        if (q == 0) wsum[wave * 16 * RM + rm * 16 + l16] = sum;
    }
    __syncthreads();
    float inv[RM];   // 1 / sum of row l16
#pragma unroll
    for (int rm = 0; rm < RM; ++rm) {
        float sum = wsum[rm * 16 + l16];
        for (int v = 1; v < waves; ++v) sum += wsum[v * 16 * RM + rm * 16 + l16];
        inv[rm] = 1.f / sum;
    }
    f32x4 acc[8][RM];
    auto clear = [&] {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int rm = 0; rm < RM; ++rm) acc[j][rm] = (f32x4){0.f, 0.f, 0.f, 0.f};
    };
    clear();
    weighted_sum<BITS, RM>(a, x, Pl, KC, 0, keys.nk, n, dj, lane, acc);
    {
        float f[RM][4];
#pragma unroll
        for (int rm = 0; rm < RM; ++rm)
#pragma unroll
            for (int i = 0; i < 4; ++i) f[rm][i] = __shfl(inv[rm], 4 * q + i, 64);
        store_rows<RM, HEADS>(a, a.C, acc, f, urow, head, rows, wave, lane);
    }
    keep_targets<HEADS>(a, urow, head, rows, true);
    __syncthreads();   // the weights in LDS have been read
    if constexpr (HEADS)
        project_rows<RM>(a.dout + urow * D + head * a.dh, a.Wv + head * a.dh, D, a.dh, rows, wave, lane, Ul, chunks, Ql);
    else
        load_rows<RM>(a.dC + urow * D, D, rows, waves, wave, lane, Ul, chunks);
    __syncthreads();
    f32x4 T[KT][RM];   // gradients of the weights
    wave_logits<BITS, RM, KT>(a, x, Ul, Sl, chunks, keys, n, first, lane, 0.f, T);
#pragma unroll
    for (int rm = 0; rm < RM; ++rm) {
        float dot = 0.f;
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) dot = __builtin_fmaf(S[t][rm][i], T[t][rm][i], dot);
        dot += __shfl_xor(dot, 16, 64);
        dot += __shfl_xor(dot, 32, 64);
        if (q == 0) wmax[wave * 16 * RM + rm * 16 + l16] = dot;
    }
    __syncthreads();
#pragma unroll
    for (int rm = 0; rm < RM; ++rm) {
        float dot = wmax[rm * 16 + l16];
        for (int v = 1; v < waves; ++v) dot += wmax[v * 16 * RM + rm * 16 + l16];
        dot *= inv[rm];
        const float f = a.scale * inv[rm];
#pragma unroll
        for (int t = 0; t < KT; t += 4) {
            if ((t >> 2) >= keys.nt) break;
            float p[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) p[i][j] = f * S[t + j][rm][i] * (T[t + j][rm][i] - dot);
            put_run(Pl, rm * 16 + l16, t >> 2, keys, KC, q, p);
        }
    }
    __syncthreads();
    clear();
    weighted_sum<BITS, RM>(a, x, Pl, KC, 0, keys.nk, n, dj, lane, acc);
    float one[RM][4];
#pragma unroll
    for (int rm = 0; rm < RM; ++rm)
#pragma unroll
        for (int i = 0; i < 4; ++i) one[rm][i] = 1.f;
    store_rows<RM, HEADS>(a, a.dU, acc, one, urow, head, rows, wave, lane);
    if constexpr (!HEADS) return;
    __syncthreads();
    project_out<RM, true>(a, acc, one, a.Wk + head * a.dh, rows, urow, head, waves, wave, lane, Ul);
}

// The same where the keys fill several chunks, in two passes over them: the first carries the
// maximum, the sum, sum alpha dA and C from chunk to chunk, the second has the final ones and sums
// dU.  Logits and dA are computed in both, six products instead of four, and U and dC stay in LDS
// side by side: 16 or 32 rows a workgroup.
template <int BITS, int RM, int KT, bool HEADS>
__global__ __launch_bounds__(512) void cached_attn_bwd_loop_kernel(AttnArgs a) {
    extern __shared__ uint4 smem[];
    const int waves = blockDim.x >> 6, chunks = 16 * waves, KC = chunk_keys(KT, waves);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
    uint16_t* const Ul = reinterpret_cast<uint16_t*>(smem);
    uint16_t* const Dl = Ul + 16 * RM * 128 * waves;
    uint16_t* const Pl = Dl + 16 * RM * 128 * waves;
    float* const wmax = reinterpret_cast<float*>(Pl + 16 * RM * KC);
    float* const wsum = wmax + 16 * RM * waves;      // [wave][row], all three
    float* const wdot = wsum + 16 * RM * waves;
    uint8_t* const Sl = reinterpret_cast<uint8_t*>(wdot + 16 * RM * waves) + wave * 8 * scale_stride(waves);
    const uint32_t id = (uint32_t)tile::xcd_range(blockIdx.x, gridDim.x);
    const int D = a.c.D;
    const uint32_t bh = id / (uint32_t)a.row_tiles;
    const int row0 = (int)(id - bh * (uint32_t)a.row_tiles) * 16 * RM;
    const int64_t b = HEADS ? bh / (uint32_t)a.h : bh;
    const int head = HEADS ? (int)(bh - (uint32_t)b * (uint32_t)a.h) : 0;
    const int rows = min(16 * RM, (HEADS ? a.R : a.N) - row0);
    int32_t n;
    const uint8_t* const codes = cache_slot(a.c, b, &n);
    const Slot x = slot_of(a.c, codes);
    const int64_t urow = b * (HEADS ? a.R : a.N) + row0;
    if (n <= 0) {
        no_rows<HEADS>(a, urow, head, rows);
        return;
    }
    const int first = 4 * (int)((uint32_t)(3 * wave + 5 * id) % (uint32_t)(chunks / 16));
    const int dj = min(wave * 16 + l16, a.c.G * 4 - 1);
    if constexpr (HEADS) {   // (W_K's and W_V's rows pass through LDS behind what is there already)
        project_rows<RM>(a.Qf + urow * D + head * a.dh, a.Wk + head * a.dh, D, a.dh, rows, wave, lane, Ul, chunks,
                         Ul + waves * 128 * 64, a.Qb + urow * D + head * a.dh);
        __syncthreads();
        project_rows<RM>(a.dout + urow * D + head * a.dh, a.Wv + head * a.dh, D, a.dh, rows, wave, lane, Dl, chunks,
                         Dl + waves * 128 * 64);
    } else {
        load_rows<RM>(a.U + urow * D, D, rows, waves, wave, lane, Ul, chunks);
        load_rows<RM>(a.dC + urow * D, D, rows, waves, wave, lane, Dl, chunks);
    }
    __syncthreads();

    f32x4 acc[8][RM];
    float m[RM], l[RM], dot[RM];   // of row l16: maximum, sum of weights, of weights times dA
    auto clear = [&] {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int rm = 0; rm < RM; ++rm) acc[j][rm] = (f32x4){0.f, 0.f, 0.f, 0.f};
    };
    clear();
#pragma unroll
    for (int rm = 0; rm < RM; ++rm) m[rm] = -INFINITY, l[rm] = 0.f, dot[rm] = 0.f;
    for (int c0 = 0; c0 < n; c0 += KC) {
        const Keys keys = wave_keys<KT>(c0, min(n, c0 + KC), waves, wave);
        f32x4 S[KT][RM], T[KT][RM];
        wave_logits<BITS, RM, KT>(a, x, Ul, Sl, chunks, keys, n, first, lane, -INFINITY, S);
        wave_logits<BITS, RM, KT>(a, x, Dl, Sl, chunks, keys, n, first, lane, 0.f, T);
#pragma unroll
        for (int rm = 0; rm < RM; ++rm) {
            float mx = -INFINITY;
#pragma unroll
            for (int t = 0; t < KT; ++t) mx = fmaxf(fmaxf(fmaxf(mx, S[t][rm][0]), fmaxf(S[t][rm][1], S[t][rm][2])), S[t][rm][3]);
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            if (q == 0) wmax[wave * 16 * RM + rm * 16 + l16] = mx;
        }
        __syncthreads();   // the last chunk's weights have been read, too
        float cor[RM];
#pragma unroll
        for (int rm = 0; rm < RM; ++rm) {
            float mx = m[rm];
            for (int v = 0; v < waves; ++v) mx = fmaxf(mx, wmax[v * 16 * RM + rm * 16 + l16]);
            const float base = mx == -INFINITY ? 0.f : mx;
            cor[rm] = __builtin_amdgcn_exp2f((m[rm] - base) * a.scale2);
            m[rm] = mx;
            float sum = 0.f, d = 0.f;
#pragma unroll
            for (int t = 0; t < KT; t += 4) {
                if ((t >> 2) >= keys.nt) break;
                float p[4][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        p[i][j] = __builtin_amdgcn_exp2f((S[t + j][rm][i] - base) * a.scale2);
                        d = __builtin_fmaf(p[i][j], T[t + j][rm][i], d);
                    }
                    sum += (p[i][0] + p[i][1]) + (p[i][2] + p[i][3]);
                }
                put_run(Pl, rm * 16 + l16, t >> 2, keys, KC, q, p);
            }
            sum += __shfl_xor(sum, 16, 64);
            sum += __shfl_xor(sum, 32, 64);
            d += __shfl_xor(d, 16, 64);
            d += __shfl_xor(d, 32, 64);
            if (q == 0) {
                wsum[wave * 16 * RM + rm * 16 + l16] = sum;
                wdot[wave * 16 * RM + rm * 16 + l16] = d;
            }
        }
        __syncthreads();
#pragma unroll
        for (int rm = 0; rm < RM; ++rm) {
            float sum = 0.f, d = 0.f;
            for (int v = 0; v < waves; ++v) {
                sum += wsum[v * 16 * RM + rm * 16 + l16];
                d += wdot[v * 16 * RM + rm * 16 + l16];
            }
            l[rm] = l[rm] * cor[rm] + sum;
            dot[rm] = dot[rm] * cor[rm] + d;
            if (c0 > 0) {
                float f[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) f[i] = __shfl(cor[rm], 4 * q + i, 64);
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[j][rm][i] *= f[i];
            }
        }
        weighted_sum<BITS, RM>(a, x, Pl, KC, c0, keys.nk, n, dj, lane, acc);
    }
    float f[RM][4], inv[RM];
#pragma unroll
    for (int rm = 0; rm < RM; ++rm) {
        inv[rm] = 1.f / l[rm];
        dot[rm] *= inv[rm];
        if (m[rm] == -INFINITY) m[rm] = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) f[rm][i] = __shfl(inv[rm], 4 * q + i, 64);
    }
    store_rows<RM, HEADS>(a, a.C, acc, f, urow, head, rows, wave, lane);
    keep_targets<HEADS>(a, urow, head, rows, true);
    clear();
    for (int c0 = 0; c0 < n; c0 += KC) {
        const Keys keys = wave_keys<KT>(c0, min(n, c0 + KC), waves, wave);
        f32x4 S[KT][RM], T[KT][RM];
        wave_logits<BITS, RM, KT>(a, x, Ul, Sl, chunks, keys, n, first, lane, -INFINITY, S);
        wave_logits<BITS, RM, KT>(a, x, Dl, Sl, chunks, keys, n, first, lane, 0.f, T);
        __syncthreads();   // the last weights have been read
#pragma unroll
        for (int rm = 0; rm < RM; ++rm) {
            const float g = a.scale * inv[rm];
#pragma unroll
            for (int t = 0; t < KT; t += 4) {
                if ((t >> 2) >= keys.nt) break;
                float p[4][4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        p[i][j] = g * __builtin_amdgcn_exp2f((S[t + j][rm][i] - m[rm]) * a.scale2) * (T[t + j][rm][i] - dot[rm]);
                put_run(Pl, rm * 16 + l16, t >> 2, keys, KC, q, p);
            }
        }
        __syncthreads();
        weighted_sum<BITS, RM>(a, x, Pl, KC, c0, keys.nk, n, dj, lane, acc);
    }
#pragma unroll
    for (int rm = 0; rm < RM; ++rm)
#pragma unroll
        for (int i = 0; i < 4; ++i) f[rm][i] = 1.f;
    store_rows<RM, HEADS>(a, a.dU, acc, f, urow, head, rows, wave, lane);
    if constexpr (!HEADS) return;
    __syncthreads();
    project_out<RM, true>(a, acc, f, a.Wk + head * a.dh, rows, urow, head, waves, wave, lane, Ul);
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

template <int BITS, int RM, int KT, bool LOOP, bool HEADS>
hipError_t launch_instance(const AttnArgs& a, hipStream_t stream) {
    const int waves = (a.c.D + 127) / 128;
    const int lds = lds_bytes<RM, KT, LOOP, HEADS>(waves);
    auto kern = cached_attn_kernel<BITS, RM, KT, LOOP, HEADS>;
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    const int64_t blocks = a.B * a.row_tiles * (HEADS ? a.h : a.splits);
    hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(64 * waves), lds, stream, a);
    return hipGetLastError();
}

// (a launch has fewer than 2^32 threads)
bool fits_a_grid(int64_t workgroups, int waves) { return workgroups * 64 * waves < (int64_t(1) << 32); }

// The forward's workgroups: 16 rm rows u, of one head's targets (heads; rm 1 to 4) or of all of a
// user's (rm 1, 2 or 4, and splits of its keys where workgroups would be too few).  rm above 2
// takes all keys in one chunk.
struct AttnPlan {
    bool heads = false;
    int rm = 0, row_tiles = 0, splits = 1, split_keys = 0;
};

// By estimated time (us).  Measured at k = 512, D = 1024, h = 16, fp4, whole calls: heads in 16,
// 32, 48, 64 rows / all rows in 16, 32, 64:
//   R = 1,   B = 1      31   36   40   47 /  34   36   42
//   R = 1,   B = 64    105  125  140  165 /  41   43   48
//   R = 4,   B = 64    105  125  141  165 /  44   55   65
//   R = 8,   B = 64    105  126  141  165 /  68   53   78
//   R = 16,  B = 16     35   40   44   50 /  47   55   64
//   R = 16,  B = 64    105  126  141  166 / 107   83   68
//   R = 40,  B = 32    146  126   78   91 / 129  108  103
//   R = 300, B = 1      55   38   43   49 /  66   52   73
//   R = 300, B = 4     122   94   76   88 / 127  107  103
// that is, heads: 9 and a round of workgroups 5 + 2.5 rm and 13.5 + 2.7 rm for 512 keys (at
// k = 1024 40, 46, 54, 63 a round); all rows: 27, 3 and the partial sums' bytes to join splits, and a round 5 and 15, 22 or
// 33 for 512 keys.  Widths below 1024 scale both, not below a half: latency.  (fp8 counts as fp4, and
// every slot as k rows: the host does not know how many it holds.)
AttnPlan attn_plan(int64_t B, int32_t R, int32_t h, int32_t k, int32_t D) {
    const int waves = (D + 127) / 128;
    const int64_t slots = (int64_t)device_cus() * std::max(1, 8 / waves);   // eight waves a compute unit
    const double width = std::max(0.5, D / 1024.0);
    B = std::max<int64_t>(B, 1);
    const bool one = k <= chunk_keys(8, waves);
    AttnPlan p;
    double best = 0;
    auto consider = [&](AttnPlan c, int64_t wgs, double cost) {
        if (fits_a_grid(wgs, waves) && (p.rm == 0 || cost < best)) p = c, best = cost;
    };
    if (D % h == 0 && (D / h) % 32 == 0) {
        for (int rm = 1; rm <= (one ? 4 : 2); ++rm) {
            AttnPlan c;
            c.heads = true;
            c.rm = rm;
            c.row_tiles = (R + 16 * rm - 1) / (16 * rm);
            c.split_keys = (k + 31) / 32 * 32;
            const int64_t wgs = B * h * c.row_tiles, rounds = (wgs + slots - 1) / slots;
            consider(c, wgs, 9 + rounds * width * (5 + 2.5 * rm + (13.5 + 2.7 * rm) * k / 512));
        }
    }
    const int64_t N = (int64_t)R * h;
    for (int rm = 1; rm <= (one ? 4 : 2); rm *= 2) {
        AttnPlan c;
        c.rm = rm;
        c.row_tiles = (int)((N + 16 * rm - 1) / (16 * rm));
        const int64_t wgs = B * c.row_tiles, most = std::max<int64_t>(1, slots / wgs);
        const int least = std::max(32, 16 * waves);   // keys that give every wave a tile
        const int64_t keys = std::max<int64_t>(least, (k + most - 1) / most);
        c.split_keys = (int)((keys + 31) / 32 * 32);
        c.splits = (k + c.split_keys - 1) / c.split_keys;
        const int64_t rounds = (wgs * c.splits + slots - 1) / slots;
        const double key = rm == 1 ? 15 : rm == 2 ? 22 : 33;
        const double join = c.splits > 1 ? 3 + 8.0 * c.splits * B * N * D / 5e6 : 0;   // written and read at 5 TB/s
        consider(c, wgs * c.splits, 27 + join + rounds * width * (5 + key * std::min(k, c.split_keys) / 512));
    }
    return p;
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

template <int BITS>
hipError_t launch_plan(const AttnPlan& p, const AttnArgs& a, hipStream_t stream) {
    if (p.heads) {
        if (p.rm == 1) return launch_instance<BITS, 1, 8, true, true>(a, stream);
        if (p.rm == 2) return launch_instance<BITS, 2, 8, true, true>(a, stream);
        if (p.rm == 3) return launch_instance<BITS, 3, 8, false, true>(a, stream);
        return launch_instance<BITS, 4, 8, false, true>(a, stream);
    }
    if (p.rm == 1) return launch_instance<BITS, 1, 8, true, false>(a, stream);
    if (p.rm == 2) return launch_instance<BITS, 2, 8, true, false>(a, stream);
    return launch_instance<BITS, 4, 8, false, false>(a, stream);
}

}  // namespace

int cached_attn_kind(int64_t B, int32_t R, int32_t h, int32_t k, int32_t D) {
    if (D > 1024) return 0;
    const AttnPlan p = attn_plan(B, R, h, k, D);
    return p.rm == 0 ? 0 : p.heads ? 2 : 1;
}

size_t cached_attn_workspace(int64_t B, int32_t R, int32_t h, int32_t k, int32_t D) {
    const AttnPlan p = attn_plan(B, R, h, k, D);
    if (p.splits <= 1) return 0;
    const size_t rows = (size_t)p.splits * B * R * h;
    return up256(rows * sizeof(float2)) + rows * D * 4;
}

hipError_t launch_cached_attn(const CacheView& c, int bits, const CachedAttnArgs& f, hipStream_t stream) {
    const AttnPlan p = attn_plan(f.B, f.R, f.h, c.k, c.D);
    AttnArgs a{};
    a.c = c;
    a.U = f.U;
    a.C = f.C;
    a.lse = f.lse;
    a.B = f.B;
    a.R = f.R;
    a.h = f.h;
    a.N = f.R * f.h;
    a.row_tiles = p.row_tiles;
    a.splits = p.splits;
    a.split_keys = p.split_keys;
    a.scale2 = f.scale * tile::kLog2e;
    a.part_ml = reinterpret_cast<float2*>(f.part);
    a.part_c = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(f.part) + up256((size_t)p.splits * f.B * a.N * sizeof(float2)));
    a.Qp = f.Qp;
    a.Wk = f.Wk;
    a.Wv = f.Wv;
    a.out = f.out;
    a.out_bf16 = f.out_bf16;
    a.dh = c.D / f.h;
    const hipError_t e = bits == 4 ? launch_plan<4>(p, a, stream) : launch_plan<8>(p, a, stream);
    if (e != hipSuccess || p.splits == 1) return e;
    const int64_t threads = f.B * a.N * ((c.D + 7) / 8);
    hipLaunchKernelGGL(cached_join_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

namespace {

// The backward's workgroups: rm 16s of rows, of one head's targets (heads) or of all of a
// user's; rm = 0 where it does not take the shape.  Keys that do not fit a chunk go in chunks
// (loop), in as many rows as LDS holds twice.
struct BwdPlan {
    int rm = 0;
    bool heads = false, loop = false;
};
template <int RM, int KT, bool HEADS>
constexpr int bwd_loop_lds(int waves) {
    const int s = 2 * 16 * RM * 128 * waves * 2 + 16 * RM * chunk_keys(KT, waves) * 2 + 3 * 16 * RM * 4 * waves +
                  waves * 8 * scale_stride(waves);
    const int t = HEADS ? 16 * RM * 128 * waves * 2 + waves * 128 * 64 * 2 + 16 * RM * 64 * 2 * 2 : 0;
    return s > t ? s : t;
}
// (up to half the width all of them fit)
static_assert(bwd_loop_lds<2, 4, true>(4) <= 160 * 1024 && bwd_loop_lds<1, 8, true>(4) <= 160 * 1024, "LDS");
BwdPlan bwd_plan(int64_t B, int32_t R, int32_t h, int32_t k, int32_t D) {
    BwdPlan p;
    const int waves = (D + 127) / 128;
    if (D > 1024) return p;
    // Chunks of keys one after the other, up to 16 and at half the width; elsewhere the separate
    // products are faster.  In chunks / in products (us a call):
    //   D = 256:  16 users, R = 20, k = 512    61 /  70;  10 users, R = 60, k = 3000  316 / 464
    //   D = 512:  20 users, R = 30, k = 1024  135 / 150;  64 users, R = 8, k = 2048   163 / 240
    //   D = 1024: 14 users, R = 1, k = 2048   201 / 142;  4 users, R = 100, k = 2048  392 / 334
    //   D = 64, 24 chunks: 2 users, R = 2, k = 3000  244 / 193
    p.loop = k > chunk_keys(8, waves);
    if (p.loop && (D > 512 || k > 16 * chunk_keys(8, waves))) return p;
    // Microseconds: rounds of workgroups, each 12.5 for every 16 rows at k = 512, D = 1024, and 22
    // (heads: 26) for the rest at D = 1024; 15 for the three products around the rows' form.
    // Measured there, heads in 16, 32, 48 rows / rows in 16, 32, 48 (us a call):
    //   R = 1,  B = 16     71   82   89 /  74   82   88
    //   R = 1,  B = 128   342  430  477 /  79   87   94
    //   R = 8,  B = 64    199  242  267 / 129  111  115
    //   R = 16, B = 32    122  143  156 / 129  110  114
    //   R = 40, B = 32    287  260  179 / 245  221  194
    //   R = 100, B = 8    261  211  224 / 264  225  240
    // (loop: six products for four)
    const double rest = D / 1024.0, row16 = (p.loop ? 18.75 : 12.5) * rest * (k / 512.0);
    double best = 0;
    for (int heads = 0; heads < 2; ++heads) {
        if (heads && (D % h != 0 || (D / h) % 32 != 0)) continue;
        for (int rm = 1; rm <= (k <= chunk_keys(4, waves) ? 3 : 2); ++rm) {
            const int64_t wgs = heads ? B * h * ((R + 16 * rm - 1) / (16 * rm)) : B * (((int64_t)R * h + 16 * rm - 1) / (16 * rm));
            const double rounds = (double)((wgs + device_cus() - 1) / device_cus());
            const double cost = rounds * (rm * row16 + (heads ? 26 : 22) * rest) + (heads ? 0 : 15);
            if (fits_a_grid(wgs, waves) && (p.rm == 0 || cost <= best)) p.rm = rm, p.heads = heads != 0, best = cost;
        }
    }
    return p;
}

template <int BITS, int RM, int KT, bool HEADS>
hipError_t launch_bwd_instance(const AttnArgs& a, hipStream_t stream) {
    const int waves = (a.c.D + 127) / 128;
    const int lds = lds_bytes<RM, KT, false, HEADS>(waves);
    auto kern = cached_attn_bwd_kernel<BITS, RM, KT, HEADS>;
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)(a.B * a.row_tiles * (HEADS ? a.h : 1))), dim3(64 * waves), lds, stream, a);
    return hipGetLastError();
}
template <int BITS, int RM, int KT, bool HEADS>
hipError_t launch_bwd_loop(const AttnArgs& a, hipStream_t stream) {
    const int waves = (a.c.D + 127) / 128, lds = bwd_loop_lds<RM, KT, HEADS>(waves);
    auto kern = cached_attn_bwd_loop_kernel<BITS, RM, KT, HEADS>;
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)(a.B * a.row_tiles * (HEADS ? a.h : 1))), dim3(64 * waves), lds, stream, a);
    return hipGetLastError();
}
template <int BITS, bool HEADS>
hipError_t launch_bwd_rows(const AttnArgs& a, int rm, bool loop, hipStream_t stream) {
    if (loop) return rm == 1 ? launch_bwd_loop<BITS, 1, 8, HEADS>(a, stream) : launch_bwd_loop<BITS, 2, 4, HEADS>(a, stream);
    if (rm == 1) return launch_bwd_instance<BITS, 1, 8, HEADS>(a, stream);
    if (rm == 2) return launch_bwd_instance<BITS, 2, 8, HEADS>(a, stream);
    if (rm == 3) return launch_bwd_instance<BITS, 3, 4, HEADS>(a, stream);
    return hipErrorInvalidValue;
}

}  // namespace

int cached_bwd_kind(int64_t B, int32_t R, int32_t h, int32_t k, int32_t D) {
    const BwdPlan p = bwd_plan(B, R, h, k, D);
    return p.rm == 0 ? 0 : p.heads ? 2 : 1;
}

hipError_t launch_cached_bwd(const CacheView& c, int bits, const CachedBwdArgs& f, hipStream_t stream) {
    const BwdPlan p = bwd_plan(f.B, f.R, f.h, c.k, c.D);
    AttnArgs a{};
    a.c = c;
    a.U = f.U;
    a.C = f.C;
    a.B = f.B;
    a.N = f.R * f.h;
    a.row_tiles = ((p.heads ? f.R : a.N) + 16 * p.rm - 1) / (16 * p.rm);
    a.scale2 = f.scale * tile::kLog2e;
    a.q = f.q;
    a.q0 = f.q0;
    a.dout0 = f.dout0;
    a.Qf = f.Qf;
    a.Qb = f.Qb;
    a.Wk = f.Wk;
    a.Wv = f.Wv;
    a.out = f.dQp;
    a.out_bf16 = true;
    a.R = f.R;
    a.h = f.h;
    a.dh = c.D / f.h;
    a.dout = f.dout;
    a.dC = f.dC;
    a.dU = f.dU;
    a.scale = f.scale;
    if (bits == 4) return p.heads ? launch_bwd_rows<4, true>(a, p.rm, p.loop, stream) : launch_bwd_rows<4, false>(a, p.rm, p.loop, stream);
    return p.heads ? launch_bwd_rows<8, true>(a, p.rm, p.loop, stream) : launch_bwd_rows<8, false>(a, p.rm, p.loop, stream);
}

}  // namespace sa
