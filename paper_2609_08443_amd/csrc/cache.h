// The sketch cache's format and its device-side conversions (sa_cache_write in
// sa_sketch.h states the format), shared by the kernels that write, read and
// attend over it.
//
// A slot of k rows of D values: with O = ceil(k / 8) octets of rows and
// G = ceil(D / 32) groups of values, the codes as blocks of 8 rows x 8 values,
// [O][G][4][8 rows][8 values], then the scale bytes [O][G][8 rows].  The block is
// what both contractions of the attention read whole: along a row's values (logits:
// a lane takes its row's 8 values, 16 rows 2 x 32 or 2 x 64 contiguous bytes) and
// along the rows (weighted sums: a lane takes a whole block and turns it in
// registers), so that neither needs the codes transposed through LDS.
#pragma once

#include "sa_internal.h"
#include "tile_ops.h"

namespace sa {
namespace cachefmt {

constexpr int kGroup = 32;       // values sharing a scale
constexpr int kMinExp = -100;    // least scale exponent: products with bf16 values stay normal numbers
constexpr int kBadScale = 255;   // scale byte of a group with an infinity or a NaN: reads as NaN

// bytes of 8 values
template <int BITS>
constexpr int kRowBytes = BITS;

// Scale exponent of a group: the least e with amax <= L 2^e, L = 7 (4 bits) or 464
// (8 bits), the largest magnitudes that round to the largest code's value (6, 448):
// no value of the group is off by more than half a step of its own size.
template <int BITS>
__device__ inline int scale_exp(float amax) {
    const uint32_t w = __float_as_uint(amax);
    const int p = (int)(w >> 23) - 127;   // amax = 1.f 2^p (numbers below 2^-126 end at kMinExp)
    const uint32_t f = w & 0x7fffffu;
    int e;
    if constexpr (BITS == 4) e = p - (f <= 0x600000u ? 2 : 1);   // 7 = 1.75 2^2
    else e = p - (f <= 0x680000u ? 8 : 7);                        // 464 = 1.8125 2^8
    return max(kMinExp, min(e, BITS == 4 ? 125 : 119));
}
__device__ inline float exp_float(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// the scale of a byte; of kBadScale an infinity, with which the conversions below give NaN
__device__ inline float scale_float(uint32_t byte) { return __uint_as_float(byte << 23); }

// 8 values to codes: v inv, inv = 2^-e, rounded to nearest even; magnitudes past the
// largest code (only where e is held at its upper end) saturate.
template <int BITS>
__device__ inline void encode8(const float (&v)[8], float inv, uint32_t (&w)[BITS / 4]) {
    constexpr float top = BITS == 4 ? 6.f : 448.f;
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = fminf(fmaxf(v[i] * inv, -top), top);
    if constexpr (BITS == 4) {
        uint32_t r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, y[0], y[1], 1.f, 0);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, y[2], y[3], 1.f, 1);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, y[4], y[5], 1.f, 2);
        w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, y[6], y[7], 1.f, 3);
    } else {
        typedef short s16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s16x2 r = {0, 0};
            r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, y[4 * i], y[4 * i + 1], 1.f, false);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, y[4 * i + 2], y[4 * i + 3], 1.f, true);
            w[i] = __builtin_bit_cast(uint32_t, r);
        }
    }
}

// Values 2 i and 2 i + 1 of a row's 8 codes, as bf16 (exact: at most four significant bits)
template <int BITS, int I>
__device__ inline uint32_t decode2(const uint32_t (&w)[BITS / 4], float scale) {
    if constexpr (BITS == 4)
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, I));
    else
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[I / 2], scale, (I & 1) != 0));
}
template <int BITS>
__device__ inline uint4 decode8(const uint32_t (&w)[BITS / 4], float scale) {
    return make_uint4(decode2<BITS, 0>(w, scale), decode2<BITS, 1>(w, scale), decode2<BITS, 2>(w, scale),
                      decode2<BITS, 3>(w, scale));
}

}  // namespace cachefmt

// A cache's place in device memory: slots of slot_bytes bytes, valid rows of each.
struct CacheView {
    const uint8_t* data;
    const int32_t* rows;
    const int64_t* slots;   // [B]
    int64_t n_slots, slot_bytes;
    int32_t k, D, G;        // G = ceil(D / 32)
    int64_t scales_at;      // byte offset of the scales in a slot
};

// user b's slot and its valid rows; none (0) for a slot outside the cache
__device__ inline const uint8_t* cache_slot(const CacheView& c, int64_t b, int32_t* n) {
    const int64_t s = c.slots[b];
    const bool hit = s >= 0 && s < c.n_slots;
    const int64_t at = hit ? s : 0;
    *n = hit ? min(max(c.rows[at], 0), c.k) : 0;
    return c.data + at * c.slot_bytes;
}

}  // namespace sa
