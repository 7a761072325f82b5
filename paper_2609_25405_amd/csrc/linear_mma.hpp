// One step of K of a 16x16 tile on the matrix cores, in the lane order of the packed weights.
#pragma once

#include <type_traits>
#include <utility>

#include "linear.hpp"

namespace orthrus {

#if defined(__HIP_DEVICE_COMPILE__)
// f(integral_constant 0), ..., f(integral_constant N - 1)
template <typename F, int... I> __device__ __forceinline__ void unrolled_of(F &&f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F> __device__ __forceinline__ void unrolled(F &&f) {
    unrolled_of(f, std::make_integer_sequence<int, N>{});
}

// the first n bytes of sixteen, the others zero (n >= 16: all)
__device__ __forceinline__ i32x4 first_bytes(i32x4 v, int n) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int left = n - 4 * i;
        v[i] = left >= 4 ? v[i] : left <= 0 ? 0 : v[i] & ((1 << 8 * left) - 1);
    }
    return v;
}

// both halves of a lane's 32 bytes of a step
__device__ __forceinline__ i32x8 both(i32x4 a, i32x4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }
template <int H> __device__ __forceinline__ bf16x8 half_of(i32x8 v) {
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v, v, 4 * H, 4 * H + 1, 4 * H + 2, 4 * H + 3));
}

// acc += W x^T over 128 bytes of K: lane l holds row l % 16 of the weight tile and of x, bytes 16 (l / 16) and
// 64 + 16 (l / 16) on; the sums are those of x row l % 16 and weight rows 4 (l / 16) + 0..3.  MX8: byte WB of sw and XB of sx are the scales of
// block l / 16 of those rows.  bfloat16 products are exact and added in fp32 (16x16x32); the scaled 16x16x128
// reads 8-bit products of eight neighbours against the largest of them, without what is below 2^-13 of its
// power of two (a product of normal data is 1.5e-5 off, whatever K), at 3.5 PFLOP/s in a stream of them.
template <int DT, int WB, int XB>
__device__ __forceinline__ void mma_step(f32x4 &acc, i32x8 w, i32x8 x, int sw, int sx) {
    if constexpr (DT == ORTHRUS_MX8) {
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, acc, 0, 0, WB, sw, XB, sx);
    } else {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(half_of<0>(w), half_of<0>(x), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(half_of<1>(w), half_of<1>(x), acc, 0, 0, 0);
    }
}

// The same on 32x32 tiles, over half SS of 128 bytes: lane l holds row l % 32 of each, bytes 64 SS + 16 (l / 32) and
// 64 SS + 32 + 16 (l / 32) on; the sums are those of x row l % 32 and weight rows 8 (i / 4) + 4 (l / 32) + i % 4.  MX8: the scale bytes are
// those of block 2 SS + l / 32 of the 128 bytes.
template <int DT, int WB, int XB>
__device__ __forceinline__ void mma_half_step(f32x16 &acc, i32x8 w, i32x8 x, int sw, int sx) {
    if constexpr (DT == ORTHRUS_MX8) {
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, x, acc, 0, 0, WB, sw, XB, sx);
    } else {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(half_of<0>(w), half_of<0>(x), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(half_of<1>(w), half_of<1>(x), acc, 0, 0, 0);
    }
}
#endif

// the weight tiles that a workgroup of linear_few.hip owns, and how many workgroups there can be
int few_tiles(const PackedShape &s, int rows, int groups, int gated, int y_dtype);
int64_t few_units(const PackedShape &s, int rows, int groups, int nt);
// row tiles of bm rows that `rows` rows in `groups` groups can have
int64_t most_row_tiles(int64_t rows, int64_t groups, int bm);

}  // namespace orthrus
