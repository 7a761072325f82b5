// Norms and products as operators: kernel arguments, the layout of packed weights, and the device
// code they share (8-bit blocks, what follows a product).
#pragma once

#include <cstdint>
#include <type_traits>

#include "orthrus/linear.h"

namespace orthrus {

constexpr int kBlock8 = ORTHRUS_MX8_BLOCK;
constexpr int kLeastExpMx = -100;   // least exponent of a block's scale

// Packed weights of one group.  A row's K bytes are cut into steps of 128 bytes (128 codes or 64
// bfloat16), zero behind the last element, and the rows into tiles of 16 (gated: tiles of the
// activated matrix and of the other one in turn), zero behind the last row.  A step of a tile is 2048 contiguous
// bytes in the order in which the lanes of a 16x16 MFMA take them: [half][lane][16], half h of lane l being row
// l % 16, bytes 64 h + 16 (l / 16) of the step.  Behind all tiles (MX8): scale bytes [tile / 4][step][lane][tile % 4],
// lane l being row l % 16, block l / 16 of the step: one word of a lane serves four tiles.
constexpr int kStepBytes = 128, kTileBytes = 16 * kStepBytes;
struct PackedShape {
    int tiles, steps, quads;              // tiles of 16 rows, steps of K, quads of tiles
    size_t tile_bytes, scale_at, bytes;   // of a tile's steps; of the scales in a group; of a group
};
inline PackedShape packed_shape(int dtype, int n, int k, int gated) {
    PackedShape p;
    p.tiles = (n + 15) / 16 * (gated ? 2 : 1);
    p.steps = (int)(((int64_t)k * (dtype == ORTHRUS_MX8 ? 1 : 2) + kStepBytes - 1) / kStepBytes);
    p.quads = (p.tiles + 3) / 4;
    p.tile_bytes = (size_t)p.steps * kTileBytes;
    p.scale_at = p.tiles * p.tile_bytes;
    p.bytes = p.scale_at + (dtype == ORTHRUS_MX8 ? (size_t)p.quads * p.steps * 256 : 0);
    return p;
}

// Runs of bytes, `stride` apart: what a call reads or writes of a matrix.
struct Runs {
    __int128 at, stride, bytes, rows;
};
// Do two share a byte?  Rows of one matrix often lie between those of another (columns of one buffer).
constexpr bool runs_meet(Runs a, Runs b) {
    if (a.rows < 1 || b.rows < 1 || a.bytes < 1 || b.bytes < 1) return false;
    if (a.at + (a.rows - 1) * a.stride + a.bytes <= b.at || b.at + (b.rows - 1) * b.stride + b.bytes <= a.at) return false;
    if (a.stride == b.stride && a.rows > 1 && b.rows > 1) {
        // row j of b and row i of a share one where -b.bytes < b.at - a.at + (j - i) stride < a.bytes: the least such j - i, and
        // is it one of two rows?
        const __int128 least = a.at - b.at - b.bytes + 1, s = a.stride;
        __int128 k = least >= 0 ? (least + s - 1) / s : -(-least / s);
        if (k < 1 - a.rows) k = 1 - a.rows;
        return k < b.rows && b.at - a.at + k * s < a.bytes;
    }
    if (a.rows > b.rows) {
        const Runs c = a;
        a = b;
        b = c;
    }
    for (__int128 i = 0; i < a.rows; ++i) {
        // the first row of b that ends behind where this one of a begins
        const __int128 p = a.at + i * a.stride, past = p - b.at - b.bytes;
        const __int128 j = past < 0 ? 0 : b.rows == 1 ? 1 : past / b.stride + 1;
        if (j < b.rows && b.at + j * b.stride < p + a.bytes) return true;
    }
    return false;
}

// rows of a matrix, strides in elements (scales: bytes)
struct Mat {
    char *data;
    uint8_t *scale;
    int64_t stride, scale_stride;
    int dtype;
};

// what follows a product
struct Epilogue {
    const float *bias;
    Mat res, y;
    int act, n;
};

struct Product {
    const char *w;
    size_t group_bytes;
    PackedShape shape;
    const char *x;
    const uint8_t *x_scale;
    int64_t x_stride, x_scale_stride;   // bytes
    int k_bytes, k_blocks;              // of a row
    int rows, dtype, gated, groups;
    const int32_t *offsets;             // null: one group of all rows
    int splits;                         // > 1: part s of K goes to slab + s * rows * tiles * 16
    float *slab;
    Epilogue e;
};

// Where the copies of linear_tile.hip read, in bytes from the tile's first row of x (first tile of the weights): the part of the address
// that a lane holds, which is compared with the buffer's length, and the part that all lanes share, on whose part in that comparison
// nothing here relies.  A tile's rows may be fewer than its copies', and a step's bytes more than what is left of a row: of x all of the
// address is the lane's (buffers that begin at the shared part cost as much: 8192^3 442 to 450 us, 438 to 440 so).  The weights' tiles are
// whole, and a tile that is not there is told by the lane's part.
struct CopyAt {
    unsigned lane, shared;
};
// 16 bytes of a row of x, of a step of K; the buffer ends with the last row's last 16 bytes
constexpr CopyAt x_copy(int row, int chunk, int step, unsigned stride) {
    return CopyAt{row * stride + step * kStepBytes + chunk * 16, 0};
}
constexpr int64_t x_room(int rows, int64_t stride, int k_bytes) { return (rows - 1) * stride + (k_bytes + 15) / 16 * 16; }
// a word of scales of a row of x; `row` is 16 rows' first, `lane_row` the one of them, `words` that of four steps' first
constexpr CopyAt x_scale_copy(int row, int lane_row, int words, int lane_word, unsigned stride) {
    return CopyAt{(row + lane_row) * stride + (words + lane_word) * 4, 0};
}
constexpr int64_t x_scale_room(int rows, int64_t stride, int k_blocks) { return (rows - 1) * stride + (k_blocks + 3) / 4 * 4; }
// 16 bytes of a half of a weight tile's step, and a lane's word of scales of a quad of tiles
constexpr CopyAt w_copy(int half, int lane, int step, unsigned tile_bytes) {
    return CopyAt{half / 2 * tile_bytes + half % 2 * 1024 + lane * 16, (unsigned)step * kTileBytes};
}
constexpr CopyAt w_scale_copy(int quad, int lane, int step, unsigned steps) {
    return CopyAt{quad * steps * 256 + lane * 4, (unsigned)step * 256};
}

// the cover of a product by workgroups
struct ProductPlan {
    int shape;          // of linear_tile.hip, or -1: few rows (linear_few.hip)
    int splits;
    int m_tiles_most;   // row tiles of all groups together, the most there can be
};
// joint: one group of all rows, whose K may be cut
ProductPlan plan_product(const PackedShape &s, int rows, int groups, bool joint);
size_t slab_bytes(const PackedShape &s, int rows, int splits);

}  // namespace orthrus

#ifdef __HIPCC__
#include <hip/hip_runtime.h>

#include "common.hpp"

namespace orthrus {

struct NormOp {
    Mat x, add, total, y;
    const float *gain;
    float eps;
    int rows, width;
};
hipError_t launch_norm_op(const NormOp &a, hipStream_t s);
hipError_t launch_convert(const Mat &x, const Mat &y, int rows, int width, hipStream_t s);
hipError_t launch_pack(const orthrus_linear_weights &w, const PackedShape &p, const Mat &m, const Mat &up, hipStream_t s);
hipError_t launch_few(const Product &p, hipStream_t s);
hipError_t launch_tile(const Product &p, const ProductPlan &plan, hipStream_t s);
hipError_t launch_join(const Product &p, hipStream_t s);

#if defined(__HIP_DEVICE_COMPILE__)
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// ------------------------------------------------------------------------------ 8-bit blocks
// Magnitudes from here on would round to 2^128: not a number, as infinities are.
constexpr float kPastRangeMx = 0x1.fp127f;
// the byte of the least power of two s with amax <= 448 s = 1.75 * 2^8 s, from amax's exponent and mantissa
__device__ __forceinline__ int scale_byte(float amax) {
    const uint32_t b = __float_as_uint(amax);
    int e = (int)(b >> 23) - 8;
    if ((b & 0x7fffffu) > 0x600000u) ++e;
    return max(e, kLeastExpMx + 127);
}
// 2^-e of the byte e + 127: what a value is multiplied by before its rounding (e is at most 120)
__device__ __forceinline__ float inverse_scale(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }
// 2^e of any byte; 0 is the subnormal 2^-127
__device__ __forceinline__ float scale_value(int byte) {
    return byte == 0 ? 0x1p-127f : byte == 255 ? NAN : __uint_as_float((uint32_t)byte << 23);
}
// e4m3 codes of four values times `inv`, rounded to nearest even; |v inv| <= 448, or not a number
__device__ __forceinline__ uint32_t encode4_mx(float a, float b, float c, float d, float inv) {
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, w, true);
}
template <int CTRL> __device__ __forceinline__ float quad_lane(float v) {
    return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// the largest of four neighbouring lanes'
__device__ __forceinline__ float quad_max(float v) {
    v = fmaxf(v, quad_lane<0xB1>(v));
    return fmaxf(v, quad_lane<0x4E>(v));
}
// A block held by four neighbouring lanes, eight neighbours each: its scale's byte and this lane's codes.  A maximum passes by what is
// not a number, whose code comes by itself; only where it is infinite or past the range is anything looked at one by one.
__device__ __forceinline__ uint2 encode_block(const float (&v)[8], int &byte) {
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(v[i]));
    amax = quad_max(amax);
    if (amax < kPastRangeMx) {
        byte = scale_byte(amax);
        const float inv = inverse_scale(byte);
        return uint2{encode4_mx(v[0], v[1], v[2], v[3], inv), encode4_mx(v[4], v[5], v[6], v[7], inv)};
    }
    float fine[8];
    amax = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bool ok = fabsf(v[i]) < kPastRangeMx;
        amax = fmaxf(amax, ok ? fabsf(v[i]) : 0.f);
        fine[i] = ok ? v[i] : NAN;
    }
    byte = scale_byte(quad_max(amax));
    const float inv = inverse_scale(byte);
    return uint2{encode4_mx(fine[0], fine[1], fine[2], fine[3], inv), encode4_mx(fine[4], fine[5], fine[6], fine[7], inv)};
}

// ------------------------------------------------------------------------------ what follows a product
// (exponentials and reciprocals of the hardware, a step of fp32 or two off: a division by the book costs the epilogue of
// a large tile more than all else in it)
constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float over_one_plus_exp(float v, float u) {      // v / (1 + exp(-u))
    return v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * u));
}
template <int ACT> __device__ __forceinline__ float activate(float v) {
    if constexpr (ACT == ORTHRUS_ACT_RELU) return v < 0.f ? 0.f : v;      // (not a number stays)
    if constexpr (ACT == ORTHRUS_ACT_SILU) return over_one_plus_exp(v, v);
    if constexpr (ACT == ORTHRUS_ACT_GELU) {
        // v (1 - q) or v q, q = erfc(|v| / sqrt(2)) / 2 = exp(-v^2 / 2) P(t), t = 1 / (1 + 0.3 |v|): P is the polynomial of degree
        // eight without a constant whose largest error relative to q exp(v^2 / 2) over |v| <= 13.2 is least, 1.2e-7 (one of degree
        // seven: 7e-7).  What far negative v leave is right relative to itself; the exponent's roundings are the most of its error,
        // v^2 2^-24.  (Formula 7.1.26 of Abramowitz and Stegun, with three products less: 5e-5 at -3, a hundredth at -8.)
        const float x = fabsf(v), t = __builtin_amdgcn_rcpf(fmaf(0.3f, x, 1.f));
        float poly = 0.0360888392f;
        poly = fmaf(poly, t, -0.158933744f);
        poly = fmaf(poly, t, 0.209346414f);
        poly = fmaf(poly, t, -0.0564501211f);
        poly = fmaf(poly, t, 0.130032629f);
        poly = fmaf(poly, t, 0.0994650573f);
        poly = fmaf(poly, t, 0.120826319f);
        poly = fmaf(poly, t, 0.11962454f);
        const float q = poly * t * __builtin_amdgcn_exp2f(-0.5f * kLog2e * (x * x));
        return v * (v < 0.f ? q : 1.f - q);
    }
    // 1 + tanh(u) = 2 / (1 + exp(-2 u))
    if constexpr (ACT == ORTHRUS_ACT_GELU_TANH) return over_one_plus_exp(v, 1.59576912160573071f * (v + 0.044715f * v * v * v));
    return v;
}

// Runs of eight elements at any address: the hardware takes wide accesses at any byte, and a row of odd width costs
// less so than element by element (777 x 4001 x 1003 in bf16 with bias and gelu: 16.0 us, 21.5 in pieces).
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
// eight neighbouring columns from `col` (a multiple of eight) of a row; those behind n zero.  WHOLE: n is a multiple of eight
template <bool WHOLE = false> __device__ __forceinline__ void load_cols(const Mat &m, int64_t row, int col, int n, float (&v)[8]) {
    if (m.dtype == ORTHRUS_F32) {
        const float *p = (const float *)m.data + row * m.stride + col;
        if (WHOLE || col + 7 < n) {
            const f32x4_any a = *(const f32x4_any *)p, b = *(const f32x4_any *)(p + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = col + i < n ? p[i] : 0.f;
    } else {
        const uint16_t *p = (const uint16_t *)m.data + row * m.stride + col;
        if (WHOLE || col + 7 < n) {
            const u32x4_any w = *(const u32x4_any *)p;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[2 * i] = bf16_lo(w[i]), v[2 * i + 1] = bf16_hi(w[i]);
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = col + i < n ? __uint_as_float((uint32_t)p[i] << 16) : 0.f;
    }
}
template <bool WHOLE = false> __device__ __forceinline__ void store_cols(const Mat &m, int64_t row, int col, int n, const float (&v)[8]) {
    if (m.dtype == ORTHRUS_F32) {
        float *p = (float *)m.data + row * m.stride + col;
        if (WHOLE || col + 7 < n) {
            *(f32x4_any *)p = f32x4{v[0], v[1], v[2], v[3]};
            *(f32x4_any *)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < n) p[i] = v[i];
    } else {
        uint16_t *p = (uint16_t *)m.data + row * m.stride + col;
        if (WHOLE || col + 7 < n) {
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
            *(u32x4_any *)p = w;
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < n) p[i] = (uint16_t)f2bf_bits(v[i]);
    }
}
// eight neighbours of a block that four neighbouring lanes hold, which all take part; zero behind n.  The lanes of rows that are
// not stored say so
template <bool WHOLE = false>
__device__ __forceinline__ void store_cols_mx(const Mat &m, int64_t row, int col, int n, const float (&v)[8], bool ok) {
    int byte;
    const uint2 w = encode_block(v, byte);
    if (!ok || col >= n) return;
    uint8_t *p = (uint8_t *)m.data + row * m.stride + col;
    if (WHOLE || col + 7 < n) {
        *(u32x2_any *)p = u32x2_any{w.x, w.y};
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < n) p[i] = (uint8_t)((i < 4 ? w.x : w.y) >> 8 * (i % 4));
    }
    if (col % kBlock8 == 0) m.scale[row * m.scale_stride + col / kBlock8] = (uint8_t)byte;
}

// sums of eight neighbouring columns -> y; up: the other matrix's sums of gated weights.  Four neighbouring lanes hold the
// 32 columns of a block of one row; all lanes take part, those with nothing to store say so.
template <bool GATED, int ACT>
__device__ __forceinline__ void finish_cols(const Epilogue &e, int group, int row, int col, bool ok, float (&v)[8], float (&up)[8]) {
    const int n = e.n;
    ok = ok && col < n;
    if (ok) {
        float r[8] = {};
        if (e.res.data) load_cols(e.res, row, col, n, r);
        if (e.bias) {
            const Mat b{(char *)(e.bias + (size_t)group * n * (GATED ? 2 : 1)), nullptr, n, 0, ORTHRUS_F32};
            float c[8];
            load_cols(b, 0, col, n, c);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += c[i];
            if constexpr (GATED) {
                load_cols(b, 1, col, n, c);
#pragma unroll
                for (int i = 0; i < 8; ++i) up[i] += c[i];
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = activate<ACT>(v[i]);
            if constexpr (GATED) v[i] *= up[i];
            v[i] += r[i];
        }
    }
    if (e.y.dtype == ORTHRUS_MX8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = ok && col + i < n ? v[i] : 0.f;
        store_cols_mx(e.y, row, col, n, v, ok);
    } else if (ok) {
        store_cols(e.y, row, col, n, v);
    }
}
// f(integral_constant of the activation): the choice outside of the loops over rows
template <typename F> __device__ __forceinline__ void with_act(int act, F &&f) {
    switch (act) {
        case ORTHRUS_ACT_RELU: f(std::integral_constant<int, ORTHRUS_ACT_RELU>{}); break;
        case ORTHRUS_ACT_SILU: f(std::integral_constant<int, ORTHRUS_ACT_SILU>{}); break;
        case ORTHRUS_ACT_GELU: f(std::integral_constant<int, ORTHRUS_ACT_GELU>{}); break;
        case ORTHRUS_ACT_GELU_TANH: f(std::integral_constant<int, ORTHRUS_ACT_GELU_TANH>{}); break;
        default: f(std::integral_constant<int, ORTHRUS_ACT_NONE>{});
    }
}

// A wave's sums in LDS -> y: `rows` rows of NT weight tiles' columns, `ld` floats between rows, the first of them
// row0 and tile0 of the product.  An even number of tiles, gated of pairs.  U runs of rows at a time, each kind of access and the
// arithmetic for all of them together: a tile's waves are alone on their SIMDs, and nothing else would hide their latencies.
template <bool GATED, int NT, int U>
__device__ __forceinline__ void finish_rows(const Epilogue &e, int group, const float *sums, int ld, int rows, int row0, int row_end, int tile0,
                                            int lane) {
    constexpr int STEP = GATED ? 2 : 1, LANES = NT / STEP * 2, RUN = 64 / LANES;        // lanes of a row, rows of a run
    static_assert(64 % LANES == 0, "whole rows in a wave");
    const int part = lane % LANES, tile = part / 2 * STEP, in_tile = part % 2 * 8, col = (tile0 / STEP + part / 2) * 16 + in_tile, n = e.n;
    rows = min(rows, row_end - row0);
    if (rows <= 0) return;
    const bool in = col < n;
    float bias[8] = {}, bias_up[8] = {};
    if (e.bias && in) {
        const Mat b{(char *)(e.bias + (size_t)group * n * STEP), nullptr, n, 0, ORTHRUS_F32};
        load_cols(b, 0, col, n, bias);
        if constexpr (GATED) load_cols(b, 1, col, n, bias_up);
    }
    with_act(e.act, [&](auto act_c) {
        constexpr int ACT = decltype(act_c)::value;
        for (int r0 = 0; r0 < rows; r0 += U * RUN) {
            float v[U][8], up[U][8];
            bool ok[U];
            int64_t row[U];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int r = r0 + k * RUN + lane / LANES;
                ok[k] = in && r < rows;
                row[k] = row0 + r;
                const float *p = sums + min(r, rows - 1) * ld + tile * 16 + in_tile;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const f32x4 a = *(const f32x4 *)(p + 4 * h), b = *(const f32x4 *)(p + 16 * (STEP - 1) + 4 * h);
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[k][4 * h + i] = a[i] + bias[4 * h + i], up[k][4 * h + i] = b[i] + bias_up[4 * h + i];
                }
            }
            if (e.res.data) {
                float res[U][8];
#pragma unroll
                for (int k = 0; k < U; ++k) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) res[k][i] = 0.f;
                    if (ok[k]) load_cols(e.res, row[k], col, n, res[k]);
                }
#pragma unroll
                for (int k = 0; k < U; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[k][i] = (GATED ? activate<ACT>(v[k][i]) * up[k][i] : activate<ACT>(v[k][i])) + res[k][i];
            } else {
#pragma unroll
                for (int k = 0; k < U; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[k][i] = GATED ? activate<ACT>(v[k][i]) * up[k][i] : activate<ACT>(v[k][i]);
            }
            if (e.y.dtype == ORTHRUS_MX8) {
#pragma unroll
                for (int k = 0; k < U; ++k) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[k][i] = col + i < n ? v[k][i] : 0.f;
                    store_cols_mx(e.y, row[k], col, n, v[k], ok[k]);
                }
            } else if (e.y.dtype == ORTHRUS_F32) {      // (the same call: store_cols then knows the type, once for all runs)
#pragma unroll
                for (int k = 0; k < U; ++k)
                    if (ok[k]) store_cols(e.y, row[k], col, n, v[k]);
            } else {
#pragma unroll
                for (int k = 0; k < U; ++k)
                    if (ok[k]) store_cols(e.y, row[k], col, n, v[k]);
            }
        }
    });
}

// ------------------------------------------------------------------------------ groups
// The work unit of a workgroup: its group's weights and rows, the row tile and the column tile
// in it.  Units are numbered group by group; within a group by bands of BAND row tiles, in a band by column tiles, row tiles
// fastest, so that the 32 units that an XCD works on at a time are BAND x 32 / BAND tiles, which share the most
// rows and weights in its L2.  False: there is no such unit.
constexpr int kBand = 8;
struct Unit {
    int group, row0, row_end, n_tile;
};
// unit `in` of a group of m_tiles x n_tiles
__device__ __forceinline__ void place_unit(int in, int m_tiles, int n_tiles, int &m, int &n) {
    const int band = in / (kBand * n_tiles), first = band * kBand, high = min(kBand, m_tiles - first);
    in -= band * kBand * n_tiles;
    n = in / high;
    m = first + in - n * high;
}
__device__ __forceinline__ int clamp_offset(int v, int rows) { return min(max(v, 0), rows); }
// inclusive scans over a wave of values >= 0: within rows of 16 lanes, then each row's last lane into the rows behind it
template <int CTRL, int ROWS> __device__ __forceinline__ int lanes_before(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int wave_scan_max(int v) {
    v = max(v, lanes_before<0x111, 0xf>(v));
    v = max(v, lanes_before<0x112, 0xf>(v));
    v = max(v, lanes_before<0x114, 0xf>(v));
    v = max(v, lanes_before<0x118, 0xf>(v));
    v = max(v, lanes_before<0x142, 0xa>(v));
    return max(v, lanes_before<0x143, 0xc>(v));
}
__device__ __forceinline__ int wave_scan_sum(int v) {
    v += lanes_before<0x111, 0xf>(v);
    v += lanes_before<0x112, 0xf>(v);
    v += lanes_before<0x114, 0xf>(v);
    v += lanes_before<0x118, 0xf>(v);
    v += lanes_before<0x142, 0xa>(v);
    return v + lanes_before<0x143, 0xc>(v);
}
// XCD-contiguous order: blocks are dealt round-robin to the 8 XCDs, and each XCD walks a run of
// consecutive units, so re-reads stay inside one L2
__device__ __forceinline__ int xcd_run_of(int b, int n) {
    const int x = b % 8, q = n / 8, r = n % 8;
    return x * q + min(x, r) + b / 8;
}
__device__ __forceinline__ bool find_unit(const Product &p, int block, int bm, int n_tiles, Unit &u) {
    if (!p.offsets) {
        const int m_tiles = (p.rows + bm - 1) / bm, total = m_tiles * n_tiles;
        if (block >= total) return false;
        int m;
        place_unit(xcd_run_of(block, total), m_tiles, n_tiles, m, u.n_tile);
        u.group = 0;
        u.row0 = m * bm;
        u.row_end = p.rows;
        return true;
    }
    const int lane = threadIdx.x & 63;
    // 64 groups' rows and row tiles at a time, behind `carry` rows and `before` tiles of the groups ahead
    struct Walk {
        int begin, end, m_tiles, sum, carry, before;
    } w;
    auto walk = [&](int g0) {
        const int g = g0 + lane;
        w.end = g < p.groups ? clamp_offset(p.offsets[g + 1], p.rows) : 0;
        w.end = max(w.carry, wave_scan_max(w.end));
        w.begin = __shfl_up(w.end, 1, 64);
        if (lane == 0) w.begin = w.carry;
        w.m_tiles = (w.end - w.begin + bm - 1) / bm;
        w.sum = wave_scan_sum(w.m_tiles);
    };
    auto step = [&]() {
        w.before += __builtin_amdgcn_readlane(w.sum, 63);
        w.carry = __builtin_amdgcn_readlane(w.end, 63);
    };
    const int start = clamp_offset(p.offsets[0], p.rows);
    int total = 0;
    w.carry = start;
    w.before = 0;
    walk(0);
    if (p.groups <= 64) {
        total = __builtin_amdgcn_readlane(w.sum, 63);
    } else {
        step();
        for (int g0 = 64; g0 < p.groups; g0 += 64) {
            walk(g0);
            step();
        }
        total = w.before;
        w.carry = start;
        w.before = 0;
        walk(0);
    }
    total *= n_tiles;
    if (block >= total) return false;
    const int id = xcd_run_of(block, total);
    for (int g0 = 0;;) {
        const int first = (w.before + w.sum - w.m_tiles) * n_tiles;
        const uint64_t hit = __ballot(id >= first && id < first + w.m_tiles * n_tiles);
        if (hit) {
            const int at = __builtin_ctzll(hit);
            int m;
            place_unit(id - __builtin_amdgcn_readlane(first, at), __builtin_amdgcn_readlane(w.m_tiles, at), n_tiles, m, u.n_tile);
            u.group = g0 + at;
            u.row0 = __builtin_amdgcn_readlane(w.begin, at) + m * bm;
            u.row_end = __builtin_amdgcn_readlane(w.end, at);
            return true;
        }
        step();
        g0 += 64;
        if (g0 >= p.groups) return false;
        walk(g0);
    }
}
#endif  // __HIP_DEVICE_COMPILE__

}  // namespace orthrus
#endif
