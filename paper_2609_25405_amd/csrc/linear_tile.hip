// Products of more than a few rows, y = act(x W^T + bias) (* (x U^T + bias_u)) + residual: tiles of BM rows of x by BN weight
// rows.  Large ones are bound by the chip's power and by what feeds the matrix cores: 4096 x 28672 x 4096 in 8 bits 400 us, 2.4
// PFLOP/s, the matrix pipe 0.57 busy at 1.93 GHz (8192^3: 440 us, 2.5 PFLOP/s; of an earlier 425 us 357 were left without the copies into LDS,
// 416 without the epilogue); with few rows by the weights' bytes (64 x 28672 x 4096: 25 us, 4.7 TB/s).
//  - A wave holds 128 x 128 sums of a 256 x 256 tile in its accumulation registers: per product the fewest bytes from LDS, whose reads
//    and fills take three quarters of the products' time (of 128 x 256 all of it).
//  - 32x32x64 fragments: a half step's operands are live at a time, not a step's, so that nothing spills (16x16x128: 599 us).
//  - Copies go from memory to LDS without a register, and are issued between products: all at once they hold the products up (459
//    us at 8192^3).
//  - Neighbouring workgroups of an XCD share operands (place_unit): without, 8192^3 takes a quarter longer.
#include "linear.hpp"
#include "linear_mma.hpp"
#include "gemm_common.hpp"

namespace orthrus {

namespace {

typedef __attribute__((address_space(3))) void lds_void;
constexpr int kLdsMost = 160 * 1024;

// a stage: x, weights, the weights' scales; the scales of x lie beside the stages, four steps at a time
template <int DT, int BM, int BN> constexpr int stage_bytes() { return (BM + BN) * kStepBytes + (DT == ORTHRUS_MX8 ? BN * 4 : 0); }
constexpr int scale_sets(int r) { return r == 2 ? 2 : 4; }
template <int DT, int BM, int R> constexpr int x_scale_bytes() { return DT == ORTHRUS_MX8 ? scale_sets(R) * BM * 16 : 0; }

#if defined(__HIP_DEVICE_COMPILE__)
// bytes from p on as a buffer: what lies behind reads as zero
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void *p, size_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, (unsigned)bytes, 0x00020000);
}
#define SCHED_FENCE() __builtin_amdgcn_sched_barrier(0)
// what a wave wrote to LDS can be read by its other lanes
__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
// the most rows of TM, halved, that `row_bytes` each fit into `room`
template <int TM, int ROW_BYTES, int ROOM> constexpr int rows_at_once() {
    int n = TM;
    while (n * ROW_BYTES > ROOM) n /= 2;
    return n;
}
#endif

// WM x WN waves, R stages of one step of K in LDS.  A step is two half steps of FM x FN products of 32x32 fragments: those
// of x stay in registers for a half step, each half with a set of its own, those of the weights pass through a
// ring of RB register sets, PB columns ahead of their use.  A step's one barrier sits PB columns before
// its end, where its last fragments have been read: from there on the next step is read under the products
// of the last columns, and its place in LDS is filled with the step R further on.
template <int DT, int BM, int BN, int WM, int WN, int R, bool GATED>
__global__ __launch_bounds__(64 * WM * WN, 1) void tile_kernel(Product p) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr bool MX = DT == ORTHRUS_MX8;
    constexpr int W = WM * WN, TM = BM / WM, TN = BN / WN, FM = TM / 32, FN = TN / 32, C = 2 * FN, RB = 4, PB = RB - 1, QB = FN / 2;
    static_assert(C % RB == 0 && FN % 2 == 0 && TM % 32 == 0, "weight fragments go round their ring in a step");
    constexpr int A_I = BM / (8 * W), B_I = BN / (8 * W), SA_I = BM / (64 * W) > 0 ? BM / (64 * W) : 1, SB_N = BN / 64, COPIES = A_I + B_I + MX, INST = COPIES + (MX ? SA_I : 0);
    static_assert(A_I * 8 * W == BM && B_I * 8 * W == BN && (BM / 16) % (4 * SA_I) == 0 && W % SB_N == 0, "copies divide over the waves");
    constexpr int B_AT = BM * kStepBytes, SB_AT = B_AT + BN * kStepBytes, STAGE = stage_bytes<DT, BM, BN>(), SA_AT = R * STAGE;
    constexpr int LDS = SA_AT + x_scale_bytes<DT, BM, R>();
    static_assert(LDS <= kLdsMost, "LDS");
    __shared__ __attribute__((aligned(1024))) char smem[LDS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, g = lane >> 5;
    const int wm = wave / WN, wn = wave % WN;
    const int n_tiles = (p.shape.tiles + BN / 16 - 1) / (BN / 16);
    Unit u;
    if (!find_unit(p, blockIdx.x, BM, n_tiles, u)) return;
    const int split = blockIdx.y, steps = p.shape.steps;
    const int kt0 = (int)((int64_t)split * steps / p.splits), nk = (int)((int64_t)(split + 1) * steps / p.splits) - kt0;
    const int tile0 = u.n_tile * (BN / 16);

    // the tile's rows of x and of the weights as buffers: what lies behind the last row reads as zero
    const int valid = min(BM, u.row_end - u.row0), b_valid = min(BN / 16, p.shape.tiles - tile0);
    const char *const wg = p.w + u.group * p.group_bytes;
    const __amdgpu_buffer_rsrc_t ra = buffer_of(p.x + (int64_t)u.row0 * p.x_stride, x_room(valid, p.x_stride, p.k_bytes));
    const __amdgpu_buffer_rsrc_t rb = buffer_of(wg + tile0 * p.shape.tile_bytes, b_valid * p.shape.tile_bytes);
    const __amdgpu_buffer_rsrc_t rsa = buffer_of(MX ? (const char *)p.x_scale + (int64_t)u.row0 * p.x_scale_stride : nullptr,
                                                 MX ? x_scale_room(valid, p.x_scale_stride, p.k_blocks) : 0);
    const __amdgpu_buffer_rsrc_t rsb = buffer_of(MX ? wg + p.shape.scale_at + (size_t)(tile0 / 4) * steps * 256 : nullptr,
                                                 MX ? (size_t)((b_valid + 3) / 4) * steps * 256 : 0);
    // LDS row r of x holds 16-byte chunk c at chunk c ^ key(r), so that the 16 lanes of a pass of a fragment read (16
    // rows, the same chunk) hit distinct banks; a copy's lane l writes row r0 + l / 8 at chunk l % 8 and fetches
    // what is stored there.  Weights lie as they are packed: 1024 bytes a half of a tile of 16.
    auto key_of = [](int row) { return (row / 2) % 8; };
    auto x_at = [&](int i, int step) {
        const int row = 8 * (W * i + wave) + lane / 8;
        return x_copy(row, (lane % 8) ^ key_of(row), step, (unsigned)p.x_stride);
    };
    auto w_at = [&](int i, int step) { return w_copy(W * i + wave, lane, step, (unsigned)p.shape.tile_bytes); };
    const int sb_i = wave % SB_N;
    // The scales of x: a copy fetches the words of four steps of 16 rows, since a word a row would cost as many requests as the
    // codes do (at 2048 x 4096 x 14336 147 us against 125 without any).  Step t issues quarter (t + AHEAD) % 4 of the rows' words of
    // the four steps from 4 ((t + AHEAD) / 4) on: the last quarter R steps before the first of them.
    constexpr int QUARTER = BM / 16 / 4, AHEAD = R + 3, SETS = scale_sets(R);       // sixteens of rows in a quarter
    static_assert(R <= 6, "a set is read before it is filled again");
    auto copy_sa = [&](int i, int m, int q) {
        const int at = m * QUARTER + (W * i + wave) % QUARTER;          // (waves without rows of their own repeat another's)
        const CopyAt c = x_scale_copy(at * 16, lane / 4, kt0 + 4 * q, lane % 4, (unsigned)p.x_scale_stride);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsa, (lds_void *)(smem + SA_AT + ((q & (SETS - 1)) * (BM / 16) + at) * 256), 4, c.lane,
                                                 c.shared, 0, 0);
    };
    // copy i of a step: x, then weights, then the scales (which waves fetch more than once where there are few)
    auto copy = [&](auto i_c, int kt, char *st) {
        constexpr int i = decltype(i_c)::value;
        if constexpr (i < A_I) {
            const CopyAt c = x_at(i, kt0 + kt);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_void *)(st + (W * i + wave) * 1024), 16, c.lane, c.shared, 0, 0);
        } else if constexpr (i < A_I + B_I) {
            const CopyAt c = w_at(i - A_I, kt0 + kt);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_void *)(st + B_AT + (W * (i - A_I) + wave) * 1024), 16, c.lane, c.shared, 0, 0);
        } else {
            const CopyAt c = w_scale_copy(sb_i, lane, kt0 + kt, (unsigned)steps);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsb, (lds_void *)(st + SB_AT + sb_i * 256), 4, c.lane, c.shared, 0, 0);
        }
    };

    f32x16 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int k = 0; k < 16; ++k) acc[i][j][k] = 0.f;
    i32x8 fa[2][FM], fb[RB];
    int sa[FM] = {}, sb[QB] = {}, sa_raw[FM], sb_raw[QB];
    const int arow = wm * TM + r;
    int aoff[2][2];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int h = 0; h < 2; ++h) aoff[s][h] = arow * kStepBytes + (((4 * s + 2 * h + g) ^ key_of(arow)) << 4);
    // a lane's row of a pair of tiles of 16, chunk g of their half steps
    const int boff = B_AT + wn * (TN / 16) * kTileBytes + r / 16 * kTileBytes + (16 * g + r % 16) * 16;
    auto read_a = [&](auto s_c, int i, const char *st) {
        constexpr int s = decltype(s_c)::value;
        fa[s][i] = both(*(const i32x4 *)(st + aoff[s][0] + i * 32 * kStepBytes), *(const i32x4 *)(st + aoff[s][1] + i * 32 * kStepBytes));
    };
    // column q of a step: fragment q % FN of half q / FN
    auto read_b = [&](int q, const char *st) {
        const char *at = st + boff + q % FN * 2 * kTileBytes + q / FN * 1024;
        fb[q % RB] = both(*(const i32x4 *)at, *(const i32x4 *)(at + 512));
    };
    // a row's scales of the step's four blocks; the weights' of four tiles of 16, a lane's block of the first half step and (32 lanes
    // on) of the second
    auto read_sa = [&](int i, int kt) { sa_raw[i] = *(const int *)(smem + SA_AT + (((kt >> 2) & (SETS - 1)) * BM + arow + 32 * i) * 16 + (kt & 3) * 4); };
    int sb_next[QB] = {}, sb_raw2[QB];
    auto read_sb = [&](int q, const char *st) {
        const char *at = st + SB_AT + (wn * QB + q) * 256 + (16 * g + r % 16) * 4;
        sb_raw[q] = *(const int *)at;
        sb_raw2[q] = *(const int *)(at + 128);
    };
    // byte 0 and byte 2: this lane's block of each half step; this lane's tile of each pair
    const int a_shift = 8 * g, b_shift = 8 * (r / 16);
    auto take_scales = [&]() {
#pragma unroll
        for (int i = 0; i < FM; ++i) sa[i] = sa_raw[i] >> a_shift;
#pragma unroll
        for (int q = 0; q < QB; ++q) sb[q] = sb_raw[q] >> b_shift, sb_next[q] = sb_raw2[q] >> b_shift;
    };
    constexpr std::integral_constant<int, 0> first;
    constexpr std::integral_constant<int, 1> second;

    unrolled<R>([&](auto st_c) {
        constexpr int st = decltype(st_c)::value;
        unrolled<COPIES>([&](auto i) { copy(i, min(st, nk - 1), smem + st * STAGE); });
        // scales: those that steps from -AHEAD on would have issued, the oldest with the first stage
        if constexpr (MX) {
            constexpr int from = st == 0 ? 0 : 3 + st, to = 4 + st;
#pragma unroll
            for (int k = from; k < to; ++k)
#pragma unroll
                for (int i = 0; i < SA_I; ++i) copy_sa(i, k & 3, k >> 2);
        }
    });
    __builtin_amdgcn_s_waitcnt(vmcnt_imm<(R - 1) * INST>());
    ring_barrier();
#pragma unroll
    for (int i = 0; i < FM; ++i) read_a(first, i, smem);
#pragma unroll
    for (int q = 0; q < PB; ++q) read_b(q, smem);
    if constexpr (MX) {
#pragma unroll
        for (int i = 0; i < FM; ++i) read_sa(i, 0);
#pragma unroll
        for (int q = 0; q < QB; ++q) read_sb(q, smem);
        take_scales();
    }
    SCHED_FENCE();

    int buf = 0;
    auto step = [&](auto more_c, int kt) {
        constexpr bool more = decltype(more_c)::value;       // a step follows
        constexpr int A_FROM = FN > C - PB ? FN : C - PB;    // the first column under which the next step's first half is read
        constexpr int A_TO = C - FN < C - PB ? C - FN : C - PB;  // the columns under which this step's second half is read: before the barrier
        const int nbuf = buf == R - 1 ? 0 : buf + 1, ktc = min(kt + R, nk - 1);
        char *const st = smem + buf * STAGE;
        const char *const sn = smem + nbuf * STAGE;
        unrolled<C>([&](auto q_c) {
            constexpr int q = decltype(q_c)::value, s = q / FN, j = q % FN;
            if constexpr (more && q == C - PB) {
                SCHED_FENCE();
                __builtin_amdgcn_s_waitcnt(vmcnt_imm<(R - 2) * INST>());
                ring_barrier();
                SCHED_FENCE();
            }
            unrolled<FM>([&](auto i_c) {
                constexpr int i = decltype(i_c)::value;
                mma_half_step<DT, j % 2 * 2, s * 2>(acc[i][j], fb[q % RB], fa[s][i], MX ? (s ? sb_next : sb)[j / 2] : 0, MX ? sa[i] : 0);
                if constexpr (i == 0) {
                    if constexpr (q + PB < C) read_b(q + PB, st);
                    else if constexpr (more) read_b(q + PB - C, sn);
                }
                // (the last step has read its second half, and ended it, before)
                if constexpr (more && q < A_TO)
                    unrolled<FM>([&](auto k_c) {
                        constexpr int k = decltype(k_c)::value;
                        if constexpr (k * A_TO == q * FM + i) read_a(second, k, st);
                    });
                if constexpr (more && q >= A_FROM) {
                    constexpr int n = (q - A_FROM) * FM + i, slots = (C - A_FROM) * FM;
                    unrolled<FM>([&](auto k_c) {
                        constexpr int k = decltype(k_c)::value;
                        if constexpr (k * slots / FM == n) read_a(first, k, sn);
                    });
                    if constexpr (MX) {
                        if constexpr (n < FM) read_sa(n, kt + 1);
                        if constexpr (n < QB) read_sb(n, sn);
                    }
                }
                if constexpr (more && q >= C - PB) {
                    constexpr int n = (q - (C - PB)) * FM + i, slots = PB * FM;
                    unrolled<INST>([&](auto k_c) {
                        constexpr int k = decltype(k_c)::value;
                        if constexpr (k * slots / INST == n) {
                            if constexpr (k < COPIES) copy(k_c, ktc, st);
                            else copy_sa(k - COPIES, (kt + AHEAD) & 3, (kt + AHEAD) >> 2);
                        }
                    });
                }
                SCHED_FENCE();
            });
        });
        if constexpr (more && MX) take_scales();
        buf = nbuf;
    };
    for (int kt = 0; kt < nk - 1; ++kt) step(std::true_type{}, kt);
#pragma unroll
    for (int i = 0; i < FM; ++i) read_a(second, i, smem + buf * STAGE);
    const int last_bytes = p.k_bytes - (steps - 1) * kStepBytes;
    if (last_bytes < kStepBytes && kt0 + nk == steps) {
        // the rows end inside the last step: what follows is anything, and reads as zero under a scale of one
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int s = 0; s < 2; ++s)
                fa[s][i] = both(first_bytes(__builtin_shufflevector(fa[s][i], fa[s][i], 0, 1, 2, 3), last_bytes - 64 * s - 16 * g),
                                first_bytes(__builtin_shufflevector(fa[s][i], fa[s][i], 4, 5, 6, 7), last_bytes - 64 * s - 32 - 16 * g));
        if constexpr (MX) {
            const int left = p.k_blocks - 4 * (steps - 1) - g;      // blocks from this lane's first on
#pragma unroll
            for (int i = 0; i < FM; ++i) sa[i] = left <= 0 ? 0x7f7f7f7f : left <= 2 ? (sa[i] & 0xff) | 0x7f7f7f00 : sa[i];
        }
    }
    step(std::false_type{}, nk - 1);
    // the repeated copies of the last steps still write LDS: they end before its next use
    __builtin_amdgcn_s_waitcnt(vmcnt_imm<0>());

    // sums through LDS, a part of the wave's rows at a time, so that rows leave in whole runs
    constexpr int LD = TN + 4, CH = rows_at_once<TM, LD * 4 * W, LDS>();
    static_assert(CH >= 32, "sums in LDS");
    float *const sums = (float *)smem + wave * CH * LD;
    __syncthreads();
    unrolled<TM / CH>([&](auto c_c) {
        constexpr int c = decltype(c_c)::value;
#pragma unroll
        for (int i = 0; i < CH / 32; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const f32x16 &a = acc[c * (CH / 32) + i][j];
                    *(f32x4 *)(sums + (32 * i + r) * LD + 32 * j + 8 * k + 4 * g) = f32x4{a[4 * k], a[4 * k + 1], a[4 * k + 2], a[4 * k + 3]};
                }
        wave_fence();
        const int row0 = u.row0 + wm * TM + c * CH, tile = tile0 + wn * (TN / 16);
        if (p.splits > 1) {
            const int ld = p.shape.tiles * 16, cols = min(TN, ld - tile * 16), rows = min(CH, u.row_end - row0);
            float *o = p.slab + ((size_t)split * p.rows + row0) * ld + tile * 16;
            constexpr int LANES = TN / 4;
            for (int k = lane / LANES; k < rows; k += 64 / LANES)
                if (lane % LANES * 4 < cols) *(f32x4 *)(o + (size_t)k * ld + lane % LANES * 4) = *(const f32x4 *)(sums + k * LD + lane % LANES * 4);
        } else {
            finish_rows<GATED, TN / 16, 4>(p.e, u.group, sums, LD, CH, row0, u.row_end, tile, lane);
        }
        wave_fence();
    });
#endif
}

// The parts of K added up, in order, and what follows the product; four lanes a block of 32 columns.  Bound by the parts' bytes: three
// of 1280 x 4096 in 16 us, 5.3 TB/s.
template <bool GATED> __global__ __launch_bounds__(256) void join_kernel(Product p) {
#if defined(__HIP_DEVICE_COMPILE__)
    with_act(p.e.act, [&](auto act_c) {
    constexpr int ACT = decltype(act_c)::value;
    constexpr int STEP = GATED ? 2 : 1;
    const int per_row = (p.e.n + kBlock8 - 1) / kBlock8 * 4, ld = p.shape.tiles * 16;
    const int64_t n = (int64_t)p.rows * per_row;
    const size_t slab = (size_t)p.rows * ld;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int row = (int)(i / per_row), col = (int)(i - (int64_t)row * per_row) * 8;
        const bool in = col / 16 * STEP < p.shape.tiles;
        f32x4 v[2] = {}, up[2] = {};
        if (in) {
            const float *at = p.slab + (size_t)row * ld + col / 16 * 16 * STEP + col % 16;
            for (int s = 0; s < p.splits; ++s)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    v[h] += *(const f32x4 *)(at + s * slab + 4 * h);
                    if constexpr (GATED) up[h] += *(const f32x4 *)(at + s * slab + 16 + 4 * h);
                }
        }
        float a[8], b[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) a[k] = v[k / 4][k % 4], b[k] = up[k / 4][k % 4];
        finish_cols<GATED, ACT>(p.e, 0, row, col, true, a, b);
    }
    });
#endif
}

template <int DT, int BM, int BN, int WM, int WN, int R> hipError_t go(const Product &p, const ProductPlan &plan, hipStream_t s) {
    const int n_tiles = (p.shape.tiles + BN / 16 - 1) / (BN / 16);
    const dim3 grid(plan.m_tiles_most * n_tiles, p.splits), block(64 * WM * WN);
    if (p.gated) hipLaunchKernelGGL((tile_kernel<DT, BM, BN, WM, WN, R, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((tile_kernel<DT, BM, BN, WM, WN, R, false>), grid, block, 0, s, p);
    return hipGetLastError();
}
template <int DT> hipError_t go_shape(const Product &p, const ProductPlan &plan, hipStream_t s) {
    switch (plan.shape) {
        case 0: return go<DT, 256, 256, 2, 2, 2>(p, plan, s);
        case 1: return go<DT, 128, 256, 2, 2, 3>(p, plan, s);
        case 2: return go<DT, 128, 128, 2, 2, 3>(p, plan, s);
        case 3: return go<DT, 64, 128, 2, 2, 3>(p, plan, s);
        case 4: return go<DT, 64, 256, 1, 4, 3>(p, plan, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace

hipError_t launch_tile(const Product &p, const ProductPlan &plan, hipStream_t s) {
    return p.dtype == ORTHRUS_MX8 ? go_shape<ORTHRUS_MX8>(p, plan, s) : go_shape<ORTHRUS_BF16>(p, plan, s);
}

hipError_t launch_join(const Product &p, hipStream_t s) {
    const int64_t lanes = (int64_t)p.rows * ((p.e.n + kBlock8 - 1) / kBlock8 * 4), blocks = (lanes + 255) / 256;
    const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : 1 << 20));
    if (p.gated) hipLaunchKernelGGL(join_kernel<true>, grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL(join_kernel<false>, grid, dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace orthrus
