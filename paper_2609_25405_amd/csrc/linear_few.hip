// Products of few rows: tiles of at most 16 rows of x, bound by reading the weights once: 1 x 6144 x 4096 in 8 bits 6.6 us, 3.9 TB/s
// with the launch (64 x 128 tiles in four parts of K: 10.3); 8 x 4096 x 14336 12.3, 4.8 TB/s (15.5).
//
// A workgroup owns NT tiles of 16 weight rows and one tile of x; its waves deal the steps
// of K out among themselves, so that together they read one contiguous stream, keep DEPTH steps
// of loads on their way in registers (nothing is staged in LDS: the packed order is the lanes' own, and
// the few rows of x sit in the caches), and add their sums through LDS at the end.
#include "linear.hpp"
#include "linear_mma.hpp"

namespace orthrus {

namespace {

constexpr int kRows = 16, kWaves = 8;

template <int DT, int NT, int DEPTH, bool GATED> __global__ __launch_bounds__(64 * kWaves) void few_kernel(Product p) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr bool MX = DT == ORTHRUS_MX8;
    constexpr int LD = NT * 16 + 4;
    __shared__ f32x4 part[kWaves][NT][64];
    __shared__ __attribute__((aligned(16))) float sums[kRows * LD];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int n_tiles = (p.shape.tiles + NT - 1) / NT, steps = p.shape.steps;
    Unit u;
    if (!find_unit(p, blockIdx.x, kRows, n_tiles, u)) return;
    const int tile0 = u.n_tile * NT;
    const char *const w = p.w + u.group * p.group_bytes;
    const char *wt[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) wt[t] = w + min(tile0 + t, p.shape.tiles - 1) * p.shape.tile_bytes + lane * 16;
    const char *const ws = w + p.shape.scale_at + (size_t)(tile0 / 4) * steps * 256 + lane * 4;
    const int64_t row = min(u.row0 + r, u.row_end - 1);      // (rows past the end repeat the last: not stored)
    const char *const xr = p.x + row * p.x_stride + 16 * g;
    const uint8_t *const xs = MX ? p.x_scale + row * p.x_scale_stride + g : nullptr;
    const bool tail = p.k_bytes % kStepBytes != 0;

    struct Frags {
        i32x4 w[NT][2], x[2];
        int sw, sx;
    };
    auto load = [&](Frags &f, int s) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) f.w[t][h] = *(const i32x4 *)(wt[t] + (size_t)s * kTileBytes + h * 1024);
        if constexpr (MX) f.sw = *(const int *)(ws + (size_t)s * 256);
        if (tail && s == steps - 1) {
            // what lies behind a row's end may be anything: read as zero, under a scale of one
            const int left = p.k_bytes - s * kStepBytes;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int n = left - 64 * h - 16 * g;
                f.x[h] = n > 0 ? first_bytes(*(const i32x4 *)(xr + (int64_t)s * kStepBytes + h * 64), n) : i32x4{0, 0, 0, 0};
            }
            if constexpr (MX) f.sx = 4 * s + g < p.k_blocks ? xs[4 * s] : 127;
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) f.x[h] = *(const i32x4 *)(xr + (int64_t)s * kStepBytes + h * 64);
            if constexpr (MX) f.sx = xs[4 * s];
        }
    };
    f32x4 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int shift = 8 * (tile0 & 3);
    auto mul = [&](const Frags &f) {
        const int sw = MX ? f.sw >> shift : 0;
        unrolled<NT>([&](auto t_c) {
            constexpr int t = decltype(t_c)::value;
            mma_step<DT, t, 0>(acc[t], both(f.w[t][0], f.w[t][1]), both(f.x[0], f.x[1]), sw, MX ? f.sx : 0);
        });
    };
    Frags f[DEPTH];
    const int n = (steps - wave + kWaves - 1) / kWaves;      // steps of this wave: `wave`, and every eighth after it
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (d < n) load(f[d], wave + d * kWaves);
    for (int i = 0; i < n; i += DEPTH)
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            if (i + d < n) {
                mul(f[d]);
                if (i + d + DEPTH < n) load(f[d], wave + (i + d + DEPTH) * kWaves);
            }

#pragma unroll
    for (int t = 0; t < NT; ++t) part[wave][t][lane] = acc[t];
    __syncthreads();
    // the rows' sums side by side, then whole runs of columns
    for (int t = wave; t < NT; t += kWaves) {
        f32x4 v = part[0][t][lane];
#pragma unroll
        for (int k = 1; k < kWaves; ++k) v += part[k][t][lane];
        *(f32x4 *)(&sums[r * LD + t * 16 + 4 * g]) = v;
    }
    __syncthreads();
    if (wave == 0) finish_rows<GATED, NT, 1>(p.e, u.group, sums, LD, kRows, u.row0, u.row_end, tile0, lane);
#endif
}

template <int DT, int NT, bool GATED> hipError_t go(const Product &p, hipStream_t s) {
    // Two steps on their way in each of eight waves: three and four are as fast at most sizes (1 x 6144 x 4096 in 8 bits 7.3, 7.6, 7.4 us;
    // 16 x 12300 x 2048 8.6, 8.5, 8.8) and slower where a wave has many steps (8 x 4096 x 14336 12.3, 12.8, 13.4)
    constexpr int DEPTH = 2;
    hipLaunchKernelGGL((few_kernel<DT, NT, DEPTH, GATED>), dim3((unsigned)few_units(p.shape, p.rows, p.groups, NT)), dim3(64 * kWaves), 0, s, p);
    return hipGetLastError();
}
template <int DT> hipError_t go_tiles(const Product &p, hipStream_t s) {
    const int nt = few_tiles(p.shape, p.rows, p.groups, p.gated, p.e.y.dtype);
    if (p.gated) return nt == 4 ? go<DT, 4, true>(p, s) : go<DT, 2, true>(p, s);
    return nt == 4 ? go<DT, 4, false>(p, s) : nt == 2 ? go<DT, 2, false>(p, s) : go<DT, 1, false>(p, s);
}

}  // namespace

hipError_t launch_few(const Product &p, hipStream_t s) {
    return p.dtype == ORTHRUS_MX8 ? go_tiles<ORTHRUS_MX8>(p, s) : go_tiles<ORTHRUS_BF16>(p, s);
}

}  // namespace orthrus
