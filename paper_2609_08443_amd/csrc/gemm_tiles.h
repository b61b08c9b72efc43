// Operand slabs of the bf16 products in LDS: GBK = 64 deep, k-contiguous ones as [rows][64 k]
// swizzled by swz<64>, m- (n-) contiguous ones as they lie in memory, [64 k][R].
#pragma once

#include "tile_ops.h"

namespace sa {
namespace tile {

constexpr int GBK = 64;

// 16-byte chunk swizzle of an m- (n-) contiguous slab ([64 k][R] bf16, LPR = R / 8
// chunks per row): the eight k rows one transposing read touches (64 bytes of rows
// k0 + 0..3 and k0 + 8..11) fall in four different 64-byte windows of the 256
// bytes of banks instead of one.  Rows of 256 bytes or more start on the same
// bank, so row k moves by (k mod 4) windows; 128-byte rows alternate between the
// two halves, so row k moves by one window when bit 1 of k is set.  Measured: 8%
// less time on a product with both operands transposed, 2% on one.
__device__ __forceinline__ int tr_swizzle(int k, int lpr) {
    return lpr >= 16 ? (k & 3) << 2 : ((k >> 1) & 1) << 2;
}

// fragment (32 rows or columns from `first`, k step ks) of an operand slab in LDS:
// k-contiguous: ds_read_b128 of the swizzled rows; otherwise two transposing
// reads: inside each 16-lane group, lane i receives element i % 4 of the 8-byte
// pieces addressed by lanes 4 e + i / 4 (e < 4), so lane 4 e + j addresses k row
// e (then e + 4) and columns 4 j .. 4 j + 3 of its group's 16 columns.
template <int R, bool KC>
__device__ __forceinline__ bf16x8 lt_frag(const uint8_t* lds, int first, int ks, int lane) {
    const int l32 = lane & 31, hl = lane >> 5;
    if constexpr (KC) {
        return lds_b128(reinterpret_cast<const uint16_t*>(lds), swz<64>(first + l32, 2 * ks + hl));
    } else {
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const int s = lane & 15, g = (lane >> 4) & 1;
        const int k = 16 * ks + 8 * hl + (s >> 2), col = first + 16 * g + 4 * (s & 3);
        typedef __attribute__((address_space(3))) short lds_short;
        constexpr int LPR = R / 8;
        lds_short* base = (lds_short*)(const_cast<uint8_t*>(lds));
        lds_short* p = base + k * R + 8 * ((col >> 3) ^ tr_swizzle(k, LPR)) + (col & 7);
        lds_short* q = base + (k + 4) * R + 8 * ((col >> 3) ^ tr_swizzle(k + 4, LPR)) + (col & 7);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)q);
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
}

}  // namespace tile
}  // namespace sa
