// RMS norm with the residual's addition, and conversion between element types and 8-bit blocks, as
// operators.  Both read and write every element once; memory is what bounds them.
#include "linear.hpp"

namespace orthrus {

namespace {

#if defined(__HIP_DEVICE_COMPILE__)
// A value in two parts, high + low: a row's factor, so that it adds nothing to its elements' own roundings, and an element that is
// formed again (in 64 bits the operands would take half as many registers more, kept for a branch that is hardly taken: 42 us for 30)
struct Two {
    float high, low;
};
__device__ __forceinline__ Two add(float a, float b) {
    const float s = a + b, t = s - a;
    return Two{s, (a - (s - t)) + (b - t)};
}
template <int CTRL> __device__ __forceinline__ double other_lane(double v) {
    const uint64_t b = (uint64_t)__double_as_longlong(v);
    const uint32_t lo = __builtin_amdgcn_mov_dpp((uint32_t)b, CTRL, 0xf, 0xf, true), hi = __builtin_amdgcn_mov_dpp((uint32_t)(b >> 32), CTRL, 0xf, 0xf, true);
    return __longlong_as_double((int64_t)((uint64_t)hi << 32 | lo));
}
// the sum of all threads' v; two calls in a row are given different places
template <int NT> __device__ __forceinline__ double block_sum(double v, double *shared) {
    v += __shfl_xor(v, 32, 64);
    v += __shfl_xor(v, 16, 64);
    v += other_lane<0x140>(v);      // 15 - lane of 16, 7 - lane of 8, the neighbouring pair, the neighbour
    v += other_lane<0x141>(v);
    v += other_lane<0x4E>(v);
    v += other_lane<0xB1>(v);
    if constexpr (NT == 64) return v;
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
    __syncthreads();
    v = shared[0];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) v += shared[i];
    return v;
}
// 1 / sqrt(sum / width + eps), share = 1 / width.  A sum past fp32's range is infinite.
__device__ __forceinline__ Two row_factor(double sum, double share, float eps) {
    if (!(sum <= 0x1.fffffep127)) sum = (float)sum;
    const double m = fma(sum, share, (double)eps);
    const float f = 1.f / sqrtf((float)m);
    const double e = fma(-(double)f * f, m, 1.0);
    return Two{f, fabs(e) < 1.0 ? 0.5f * (float)e * f : 0.f};
}
__device__ __forceinline__ float element(const Mat &m, int64_t row, int col) {
    if (m.dtype == ORTHRUS_F32) return ((const float *)m.data)[row * m.stride + col];
    return __uint_as_float((uint32_t)((const uint16_t *)m.data)[row * m.stride + col] << 16);
}
// s g f where fp32 is too near the middle between two codes to tell: in two parts, the second as the first one's last bit, which no
// middle has
__device__ __forceinline__ float beside_middle(Two s, float g, Two f) {
    const float sg = s.high * g, rest = fmaf(sg, f.low, (fmaf(s.high, g, -sg) + s.low * g) * f.high), high = fmaf(sg, f.high, rest);
    const float low = fmaf(sg, f.high, -high) + rest;
    if (!(fabsf(low) > 0.f) || !isfinite(high)) return high;
    const uint32_t bits = __float_as_uint(high) - ((low < 0.f) != (high < 0.f) ? 1 : 0);
    return __uint_as_float(bits | 1);
}
#endif

// A row a workgroup at a time, kept in registers: thread t holds eight neighbours from 8 t on, and V - 1 more
// such runs 8 NT apart; the gain stays, and the next row is on its way while a row is worked on (30 -> 24.6 us at 8192 x 4096 with all in
// fp32).  V = 0: any width, the row is read twice.  8192 rows of 4096 in bf16 to 8 bits: 30.2 us, 3.4 TB/s, to bf16 27.7, 4.8 TB/s; vector
// work bounds the former.
// Squares are added in 64 bits, whose products and sums cost as much as fp32's (in fp32, and at the end in two parts, 29.5 us here, 38.9 for
// 36.2 of 2048 x 16384): an element beside the middle between two codes of three mantissa bits gets the code of the definition; smaller
// codes, and the scale where a block's maximum lies on its border, are those of y in fp32.  With the factor and the products rounded in
// fp32 14 to 30 of 33 million codes are not the definition's, in 24.6 us.
template <int NT, int V, bool WHOLE>
__global__ __launch_bounds__(NT, NT == 256 && V == 1 ? 6 : 1) void norm_op_kernel(NormOp a) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ double shared[2][NT / 64];
    const double share = 1.0 / a.width;
    const int t = threadIdx.x;
    auto sum_at = [&](int64_t row, int col, float (&s)[8]) {
        load_cols<WHOLE>(a.x, row, col, a.width, s);
        if (a.add.data) {
            float b[8];
            load_cols<WHOLE>(a.add, row, col, a.width, b);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] += b[i];
        }
    };
    auto put = [&](int64_t row, int col, const float (&s)[8], const float (&g)[8], Two f, bool in) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float sg = s[i] * g[i];
            y[i] = fmaf(sg, f.high, sg * f.low);
        }
        if (a.y.dtype == ORTHRUS_MX8) {
            // within four steps of fp32 of the middle between two codes (a code keeps three bits of the mantissa)?
            uint32_t nearest = ~0u;
#pragma unroll
            for (int i = 0; i < 8; ++i) nearest = min(nearest, (__float_as_uint(y[i]) - 0x7fffcu) & 0xfffffu);
            if (nearest <= 8) {
                // (with what the addition rounded off, from the rows again: total, which may be one of them, is stored last)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (((__float_as_uint(y[i]) - 0x7fffcu) & 0xfffffu) <= 8 && col + i < a.width) {
                        Two whole{s[i], 0.f};
                        if (a.add.data) whole = add(element(a.x, row, col + i), element(a.add, row, col + i));
                        y[i] = beside_middle(whole, g[i], f);
                    }
            }
            store_cols_mx<WHOLE>(a.y, row, col, a.width, y, true);
        } else if (in) {
            store_cols<WHOLE>(a.y, row, col, a.width, y);
        }
        if (in && a.total.data) store_cols<WHOLE>(a.total, row, col, a.width, s);
    };
    auto gain_at = [&](int col, bool in, float (&g)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = a.gain ? 0.f : 1.f;
        if (in && a.gain) load_cols<WHOLE>(Mat{(char *)a.gain, nullptr, 0, 0, ORTHRUS_F32}, 0, col, a.width, g);
    };
    auto factor = [&](double sq, int turn) { return row_factor(block_sum<NT>(sq, shared[turn & 1]), share, a.eps); };
    int turn = 0;
    if constexpr (V > 0) {
        float s[V][8], g[V][8];
        auto load = [&](int64_t row) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int col = 8 * (v * NT + t);
#pragma unroll
                for (int i = 0; i < 8; ++i) s[v][i] = 0.f;
                if (col < a.width) sum_at(row, col, s[v]);
            }
        };
        load(blockIdx.x);
#pragma unroll
        for (int v = 0; v < V; ++v) gain_at(8 * (v * NT + t), 8 * (v * NT + t) < a.width, g[v]);
        for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
            float c[V][8];
            double sq = 0.0;
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    c[v][i] = s[v][i];
                    sq = fma((double)c[v][i], (double)c[v][i], sq);
                }
            if (row + gridDim.x < a.rows) load(row + gridDim.x);
            const Two f = factor(sq, turn++);
#pragma unroll
            for (int v = 0; v < V; ++v) put(row, 8 * (v * NT + t), c[v], g[v], f, 8 * (v * NT + t) < a.width);
        }
    } else {
        for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
            float s[8], g[8];
            double sq = 0.0;
            for (int col = 8 * t; col < a.width; col += 8 * NT) {
                sum_at(row, col, s);
#pragma unroll
                for (int i = 0; i < 8; ++i) sq = fma((double)s[i], (double)s[i], sq);
            }
            const Two f = factor(sq, turn++);
            for (int c0 = 0; c0 < a.width; c0 += 8 * NT) {
                const int col = c0 + 8 * t;
                const bool in = col < a.width;
#pragma unroll
                for (int i = 0; i < 8; ++i) s[i] = 0.f;
                if (in) sum_at(row, col, s);
                gain_at(col, in, g);
                put(row, col, s, g, f, in);
            }
        }
    }
#endif
}

// Blocks of rows: four lanes a block of 32.  Bound by memory, as the way back is: 8192 x 4096 from bf16 23.2 us, 4.4 TB/s, from fp32 31.5, 5.4
// TB/s; back to bf16 17.4 us, 5.9 TB/s.
__global__ __launch_bounds__(256) void to_blocks_kernel(Mat x, Mat y, int rows, int width) {
#if defined(__HIP_DEVICE_COMPILE__)
    const int per_row = (width + kBlock8 - 1) / kBlock8 * 4;
    const int64_t n = (int64_t)rows * per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / per_row;
        const int col = (int)(i - row * per_row) * 8;
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = 0.f;
        if (col < width) load_cols(x, row, col, width, v);
        store_cols_mx(y, row, col, width, v, true);
    }
#endif
}

__global__ __launch_bounds__(256) void from_blocks_kernel(Mat x, Mat y, int rows, int width) {
#if defined(__HIP_DEVICE_COMPILE__)
    const int per_row = (width + 7) / 8;
    const int64_t n = (int64_t)rows * per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / per_row;
        const int col = (int)(i - row * per_row) * 8;
        const uint8_t *p = (const uint8_t *)x.data + row * x.stride + col;
        uint32_t w[2] = {0, 0};
        if (col + 7 < width) {
            const u32x2_any q = *(const u32x2_any *)p;
            w[0] = q[0], w[1] = q[1];
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (col + k < width) w[k / 4] |= (uint32_t)p[k] << 8 * (k % 4);
        }
        const float s = scale_value(x.scale[row * x.scale_stride + col / kBlock8]);
        float v[8];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
            v[4 * k] = lo[0] * s, v[4 * k + 1] = lo[1] * s, v[4 * k + 2] = hi[0] * s, v[4 * k + 3] = hi[1] * s;
        }
        store_cols(y, row, col, width, v);
    }
#endif
}

}  // namespace

hipError_t launch_norm_op(const NormOp &a, hipStream_t s) {
    auto go = [&](auto nt_c, auto v_c) {
        constexpr int NT = decltype(nt_c)::value, V = decltype(v_c)::value;
        // What the CUs hold at once by their registers (95 of 512 a lane for two runs a thread, 80 for one): 8192 rows of 4096 with five
        // workgroups a CU 30 us, with six 35, since the sixth then runs alone
        constexpr int PER_CU = NT > 256 ? 1024 / NT : NT == 256 && V == 2 ? 5 : 1536 / NT;
        const int most = 256 * PER_CU, blocks = a.rows < most ? a.rows : most;
        if (a.width % 8 == 0) hipLaunchKernelGGL((norm_op_kernel<NT, V, true>), dim3(blocks), dim3(NT), 0, s, a);
        else hipLaunchKernelGGL((norm_op_kernel<NT, V, false>), dim3(blocks), dim3(NT), 0, s, a);
        return hipGetLastError();
    };
    constexpr std::integral_constant<int, 0> twice;
    constexpr std::integral_constant<int, 1> one;
    constexpr std::integral_constant<int, 2> two;
    // The fewest waves that hold a row in two runs a thread, or in one where that is a wave or four.  65536 x 512 in bf16 to 8 bits: 29.7 us on
    // 64 threads, 85.7 on 256; 16384 x 2048 30.2 on 256, 35.2 on 128 with two runs; 8192 x 4096 30.2, 40.0 on 512 with one; 4096 x 4104 and x 8192
    // 22.4 and 32.4, on 1024 with one 27.5 and 41.5; 2048 x 16384 36.2, read twice 41.2
    if (a.width <= 512) return go(std::integral_constant<int, 64>{}, one);
    if (a.width <= 2048) return go(std::integral_constant<int, 256>{}, one);
    if (a.width <= 4096) return go(std::integral_constant<int, 256>{}, two);
    if (a.width <= 8192) return go(std::integral_constant<int, 512>{}, two);
    if (a.width <= 16384) return go(std::integral_constant<int, 1024>{}, two);
    return go(std::integral_constant<int, 1024>{}, twice);
}

hipError_t launch_convert(const Mat &x, const Mat &y, int rows, int width, hipStream_t s) {
    const bool to = y.dtype == ORTHRUS_MX8;
    const int64_t lanes = (int64_t)rows * (to ? (width + kBlock8 - 1) / kBlock8 * 4 : (width + 7) / 8);
    const int64_t blocks = (lanes + 255) / 256;
    const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : 1 << 20));
    if (to) hipLaunchKernelGGL(to_blocks_kernel, grid, dim3(256), 0, s, x, y, rows, width);
    else hipLaunchKernelGGL(from_blocks_kernel, grid, dim3(256), 0, s, x, y, rows, width);
    return hipGetLastError();
}

}  // namespace orthrus
