// C entries of the norms and products: argument checks, the cover of a product, packing.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "linear.hpp"
#include "linear_mma.hpp"

namespace orthrus {

namespace {

// The packed order from matrices of any stride, once for a matrix: a thread writes sixteen bytes of a lane, or a word of scales of four
// tiles (2 x 14336 x 4096 in 8 bits: 51 us).
template <int DT> __global__ __launch_bounds__(256) void pack_kernel(Mat m, Mat up, PackedShape p, char *dst, int n, int k, int gated,
                                                                    int64_t pieces, int64_t words, int groups) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int ES = DT == ORTHRUS_MX8 ? 1 : 2;
    const int64_t all = (pieces + words) * groups;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t group = i / (pieces + words), at = i - group * (pieces + words);
        char *const out = dst + group * p.bytes;
        // row of the matrices that a row of a tile is, or -1
        auto source = [&](int tile, int r, const Mat *&src) {
            src = gated && tile % 2 ? &up : &m;
            const int row = (gated ? tile / 2 : tile) * 16 + r;
            return tile < p.tiles && row < n ? group * n + row : (int64_t)-1;
        };
        const Mat *src;
        if (at < pieces) {
            const int64_t step_of = at / 128;
            const int lane = (int)(at % 64), half = (int)(at / 64 % 2), step = (int)(step_of % p.steps), tile = (int)(step_of / p.steps);
            const int64_t row = source(tile, lane % 16, src);
            const int e0 = (step * kStepBytes + half * 64 + lane / 16 * 16) / ES;
            uint32_t v[4] = {0, 0, 0, 0};
            if (row >= 0) {
                const char *from = src->data + (row * src->stride + e0) * ES;
                if (e0 + 16 / ES <= k) {
                    const u32x4_any w = *(const u32x4_any *)from;
                    v[0] = w[0], v[1] = w[1], v[2] = w[2], v[3] = w[3];
                } else if constexpr (ES == 1) {
#pragma unroll
                    for (int b = 0; b < 16; ++b)
                        if (e0 + b < k) v[b / 4] |= (uint32_t)(uint8_t)from[b] << 8 * (b % 4);
                } else {
#pragma unroll
                    for (int b = 0; b < 8; ++b)
                        if (e0 + b < k) v[b / 2] |= (uint32_t)((const uint16_t *)from)[b] << 16 * (b % 2);
                }
            }
            *(u32x4 *)(out + at * 16) = u32x4{v[0], v[1], v[2], v[3]};
        } else {
            const int64_t w = at - pieces, step_of = w / 64;
            const int lane = (int)(w % 64), step = (int)(step_of % p.steps), quad = (int)(step_of / p.steps);
            const int block = step * (kStepBytes / kBlock8) + lane / 16;
            uint32_t v = 0;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int64_t row = source(quad * 4 + t, lane % 16, src);
                const uint32_t byte = row >= 0 && block < (k + kBlock8 - 1) / kBlock8 ? src->scale[row * src->scale_stride + block] : 127;
                v |= byte << 8 * t;
            }
            *(uint32_t *)(out + p.scale_at + w * 4) = v;
        }
    }
#endif
}

}  // namespace

hipError_t launch_pack(const orthrus_linear_weights &w, const PackedShape &p, const Mat &m, const Mat &up, hipStream_t s) {
    const int64_t pieces = (int64_t)p.tiles * p.steps * 128, words = w.dtype == ORTHRUS_MX8 ? (int64_t)p.quads * p.steps * 64 : 0;
    const int64_t blocks = ((pieces + words) * w.groups + 255) / 256;
    const dim3 grid((unsigned)std::min<int64_t>(blocks, 1 << 20));
    auto *kernel = w.dtype == ORTHRUS_MX8 ? pack_kernel<ORTHRUS_MX8> : pack_kernel<ORTHRUS_BF16>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, m, up, p, (char *)const_cast<void *>(w.packed), w.n, w.k, w.gated, pieces, words,
                       w.groups);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------ covers
namespace {
constexpr int kMostSplits = 8, kLeastSteps = 4;     // parts of K, and steps of a part
constexpr size_t kMostSlab = (size_t)64 << 20;
constexpr int32_t kMostRows = 1 << 30;    // a row tile's end stays an int
constexpr int kCus = 256;
int div_up(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// Shapes of linear_tile.hip, in its order: microseconds of a step of K (128 bytes) of one tile alone on its CU, of two where two
// fit (their LDS: 79 KB each), and of the rest of a tile.  Measured in 8 bits at 256 x 6144 x 4096 (64 x 128: 14.3 us),
// 512 x 4096 x 4096 (128 x 128 18.4, 64 x 256 20.9), 2048 x 4096 x 4096 and x 14336 (128 x 256 38.3, 135), 4096 x 28672 x 4096 (256 x 256 411) and
// 1024 x 28672 x 4096 (64 x 128, 7 rounds of two a CU: 164); bfloat16 takes as long for a step of half as many elements.
struct TileShape {
    int bm, bn;
    double step, pair_step, rest;
};
constexpr TileShape kTiles[] = {{256, 256, 1.5, 0, 10}, {128, 256, 1.12, 0, 6}, {128, 128, 0.43, 0, 5}, {64, 128, 0.29, 0.65, 4}, {64, 256, 0.53, 0, 5}};
constexpr double kBytesPerUs = 4.7e6;     // a large copy's rate
constexpr double kJoinUs = 3.5;           // a second launch
constexpr double kUnhidden = 0.25;        // of the shorter of tiles and reading

// microseconds of `n` tiles of `steps` steps
double tiles_us(const TileShape &t, double n, double steps) {
    const double alone = steps * t.step + t.rest;
    if (t.pair_step == 0) return std::ceil(n / kCus) * alone;
    const double pair = steps * t.pair_step + t.rest, rounds = std::floor(n / (2 * kCus)), left = n - rounds * 2 * kCus;
    return rounds * pair + (left == 0 ? 0 : left <= kCus ? alone : pair);
}
}  // namespace

size_t slab_bytes(const PackedShape &s, int rows, int splits) { return splits > 1 ? (size_t)splits * rows * s.tiles * 64 : 0; }

// the most sums that plan_product leaves in a workspace, over all numbers of rows up to `rows`: what keeps it from cutting K, without
// its estimates
size_t most_slab(const PackedShape &s, int rows) {
    size_t most = 0;
    for (int split = 2; split <= kMostSplits && s.steps / split >= kLeastSteps; ++split)
        for (const TileShape &t : kTiles) {
            const int64_t cut = (int64_t)(2 * kCus - 1) / (split - 1) / div_up(s.tiles, t.bn / 16) * t.bm;     // the most rows in so many parts
            most = std::max(most, std::min(slab_bytes(s, (int)std::min<int64_t>(rows, cut), split), kMostSlab));
        }
    return most;
}

// a group of rows takes at most one tile more than its share
int64_t most_row_tiles(int64_t rows, int64_t groups, int bm) {
    return groups == 1 ? (rows + bm - 1) / bm : std::min(rows, rows / bm + std::min(rows, groups));
}

int64_t few_units(const PackedShape &s, int rows, int groups, int nt) { return div_up(s.tiles, nt) * most_row_tiles(rows, groups, 16); }
int few_tiles(const PackedShape &s, int rows, int groups, int gated, int y_dtype) {
    // Whole units of output, and more (so that x is read less often) while three quarters of the CUs have work: 16 x 6144 x 4096 in 8
    // bits 7.4 us with two tiles a workgroup, 9.6 with one; one row 6.8 with either
    int nt = (gated ? 2 : 1) * (y_dtype == ORTHRUS_MX8 ? 2 : 1);
    while (nt < 4 && few_units(s, rows, groups, 2 * nt) >= 192) nt *= 2;
    return nt;
}

// The cover whose estimated time is least: the rounds of its tiles over the CUs or the reading of the weights, whichever is
// longer, a part of the other (4096 rows over 64 groups of 2048 x 2048, gated: 64 x 256 64 us, 128 x 256 75, both shorter than
// the reading), and the joining of the parts where K is cut.
ProductPlan plan_product(const PackedShape &s, int rows, int groups, bool joint) {
    ProductPlan best{-1, 1, 0};
    const double used = std::min(rows, groups), weight_us = (double)s.bytes * used / kBytesPerUs;
    double best_us = 1e30;
    int bm = 0;
    const int n_shapes = (int)(sizeof(kTiles) / sizeof(kTiles[0]));
    for (int i = 0; i < n_shapes; ++i) {
        const TileShape &t = kTiles[i];
        // ragged groups: half a tile of each is empty, and most have one
        const double m_tiles = groups == 1 ? div_up(rows, t.bm) : std::max((double)rows / t.bm + 0.5 * used, 0.8 * used);
        const double tiles = m_tiles * div_up(s.tiles, t.bn / 16);
        for (int split = 1; split <= (joint ? kMostSplits : 1); ++split) {
            // (more parts than two rounds of tiles only cost)
            if (split > 1 && (s.steps / split < kLeastSteps || slab_bytes(s, rows, split) > kMostSlab || tiles * (split - 1) >= 2 * kCus)) break;
            const double tile_us = tiles_us(t, tiles * split, div_up(s.steps, split));
            double us = std::max(tile_us, weight_us) + kUnhidden * std::min(tile_us, weight_us);
            if (split > 1) us += kJoinUs + 2.0 * slab_bytes(s, rows, split) / kBytesPerUs;
            if (us < best_us) {
                best_us = us;
                best.shape = i;
                best.splits = split;
                bm = t.bm;
            }
        }
    }
    if (div_up(rows, groups) <= 16) {
        // One tile of 16 rows: the weights go straight to registers.  1 x 6144 x 4096 in 8 bits 7.3 us against 10.3, 8 x 4096 x 14336
        // 12.3 against 15.5; with many columns the tiles are as fast
        const double us = 2.0 + 1.25 * weight_us;
        if (us < best_us) {
            best.shape = -1;
            best.splits = 1;
            bm = 16;
        }
    }
    best.m_tiles_most = (int)most_row_tiles(rows, groups, bm);
    return best;
}

}  // namespace orthrus

using namespace orthrus;

namespace {

bool weights_ok(const orthrus_linear_weights *w) {
    return w && (w->dtype == ORTHRUS_BF16 || w->dtype == ORTHRUS_MX8) && w->n > 0 && w->k > 0 && w->groups > 0 &&
           (w->gated == 0 || w->gated == 1);
}
// sizes that the kernels' 32-bit offsets hold: a workgroup's tiles of the weights, all tiles' columns
bool weights_fit(const orthrus_linear_weights *w) { return w->k <= (1 << 22) && w->n <= (1 << 26); }

size_t element_bytes(int dtype) { return dtype == ORTHRUS_F32 ? 4 : dtype == ORTHRUS_BF16 ? 2 : 1; }
// rows of `width` elements at any alignment to an element
bool matrix_ok(const orthrus_matrix *m, int32_t width) {
    if (!m || !m->data || m->stride < width || (m->dtype != ORTHRUS_F32 && m->dtype != ORTHRUS_BF16 && m->dtype != ORTHRUS_MX8)) return false;
    if ((uintptr_t)m->data % element_bytes(m->dtype)) return false;
    return m->dtype != ORTHRUS_MX8 || (m->scale && m->scale_stride >= (width + (int64_t)kBlock8 - 1) / kBlock8);
}
Mat mat(const orthrus_matrix *m) {
    if (!m || !m->data) return Mat{nullptr, nullptr, 0, 0, ORTHRUS_F32};
    return Mat{(char *)m->data, (uint8_t *)m->scale, m->stride, m->scale_stride, m->dtype};
}

// what a call touches of a matrix: its elements, and the scales of 8-bit blocks
Runs elements_of(const orthrus_matrix *m, int64_t rows, int32_t width) {
    if (!m || !m->data) return Runs{0, 0, 0, 0};
    const int64_t es = element_bytes(m->dtype);
    return Runs{(__int128)(uintptr_t)m->data, (__int128)m->stride * es, (__int128)width * es, rows};
}
Runs scales_of(const orthrus_matrix *m, int64_t rows, int32_t width) {
    if (!m || !m->data || m->dtype != ORTHRUS_MX8) return Runs{0, 0, 0, 0};
    return Runs{(__int128)(uintptr_t)m->scale, m->scale_stride, (width + (int64_t)kBlock8 - 1) / kBlock8, rows};
}
Runs bytes_of(const void *p, size_t bytes) { return Runs{(__int128)(uintptr_t)p, 0, p ? (__int128)bytes : 0, 1}; }
// one matrix: every element is read by the lane that writes it, before
bool same_rows(const orthrus_matrix *a, const orthrus_matrix *b, int32_t rows) {
    return a && b && a->data == b->data && a->dtype == b->dtype && a->dtype != ORTHRUS_MX8 && (rows == 1 || a->stride == b->stride);
}
// does what is written of y share memory with itself or with x?
bool writes_meet(const orthrus_matrix *y, const Runs &x, int32_t rows, int32_t width) {
    return runs_meet(elements_of(y, rows, width), x) || runs_meet(scales_of(y, rows, width), x);
}
bool writes_meet(const orthrus_matrix *y, const orthrus_matrix *x, int32_t rows, int32_t width, int32_t x_width) {
    return writes_meet(y, elements_of(x, rows, x_width), rows, width) || writes_meet(y, scales_of(x, rows, x_width), rows, width);
}
bool meets_itself(const orthrus_matrix *y, int32_t rows, int32_t width) {
    return runs_meet(elements_of(y, rows, width), scales_of(y, rows, width));
}

int product(const orthrus_linear_weights *w, const orthrus_matrix *x, const int32_t *offsets, bool grouped, int32_t rows,
            const orthrus_epilogue *e, const orthrus_matrix *y, void *workspace, size_t ws_bytes, void *stream) {
    if (!weights_ok(w) || rows < 0 || (!grouped && w->groups != 1)) return ORTHRUS_EINVAL;
    if (rows == 0) return ORTHRUS_OK;
    if (!w->packed || (uintptr_t)w->packed % 256 || !x || !y || (grouped && (!offsets || (uintptr_t)offsets % 4))) return ORTHRUS_EINVAL;
    if (!matrix_ok(x, w->k) || !matrix_ok(y, w->n)) return ORTHRUS_EINVAL;
    if (x->dtype != w->dtype) return ORTHRUS_EUNSUPPORTED;
    const int64_t xs = x->stride * (int64_t)element_bytes(x->dtype);
    if ((uintptr_t)x->data % 16 || xs % 16) return ORTHRUS_EINVAL;
    if (x->dtype == ORTHRUS_MX8 && ((uintptr_t)x->scale % 4 || x->scale_stride % 4)) return ORTHRUS_EINVAL;
    if (e) {
        if (e->act < ORTHRUS_ACT_NONE || e->act > ORTHRUS_ACT_GELU_TANH || (uintptr_t)e->bias % 4) return ORTHRUS_EINVAL;
        if (e->residual.data) {
            if (!matrix_ok(&e->residual, w->n)) return ORTHRUS_EINVAL;
            if (e->residual.dtype == ORTHRUS_MX8) return ORTHRUS_EUNSUPPORTED;
        }
    }
    if (!weights_fit(w) || rows >= kMostRows || xs > 0x7fffffff / 256 || x->scale_stride > 0x7fffffff / 256) return ORTHRUS_ECAPACITY;
    Product p{};
    p.shape = packed_shape(w->dtype, w->n, w->k, w->gated);
    const ProductPlan plan = plan_product(p.shape, rows, w->groups, !grouped);
    // (a launch holds fewer than 2^32 threads in a direction)
    if (plan.shape < 0 ? few_units(p.shape, rows, w->groups, few_tiles(p.shape, rows, w->groups, w->gated, y->dtype)) >= (1 << 23)
                       : plan.m_tiles_most * (int64_t)div_up(p.shape.tiles, kTiles[plan.shape].bn / 16) >= (1 << 24))
        return ORTHRUS_ECAPACITY;
    const size_t need = slab_bytes(p.shape, rows, plan.splits);
    if (need > 0 && (!workspace || (uintptr_t)workspace % 16)) return ORTHRUS_EINVAL;
    if (ws_bytes < need) return ORTHRUS_ECAPACITY;
    const Runs kept[] = {bytes_of(w->packed, orthrus_linear_packed_bytes(w)), bytes_of(grouped ? offsets : nullptr, ((size_t)w->groups + 1) * 4),
                         bytes_of(e ? e->bias : nullptr, (size_t)w->groups * (w->gated ? 2 : 1) * w->n * 4)};
    const Runs room = bytes_of(workspace, need);
    const orthrus_matrix *res = e ? &e->residual : nullptr;
    if (meets_itself(y, rows, w->n) || writes_meet(y, x, rows, w->n, w->k) || writes_meet(y, room, rows, w->n)) return ORTHRUS_EINVAL;
    if (!same_rows(y, res, rows) && writes_meet(y, res, rows, w->n, w->n)) return ORTHRUS_EINVAL;
    for (const Runs &r : kept)
        if (writes_meet(y, r, rows, w->n) || runs_meet(room, r)) return ORTHRUS_EINVAL;
    if (runs_meet(room, elements_of(x, rows, w->k)) || runs_meet(room, scales_of(x, rows, w->k)) || runs_meet(room, elements_of(res, rows, w->n)))
        return ORTHRUS_EINVAL;
    p.w = (const char *)w->packed;
    p.group_bytes = (p.shape.bytes + 255) / 256 * 256;
    p.x = (const char *)x->data;
    p.x_scale = (const uint8_t *)x->scale;
    p.x_stride = xs;
    p.x_scale_stride = x->scale_stride;
    p.k_bytes = (int)(w->k * element_bytes(w->dtype));
    p.k_blocks = (w->k + kBlock8 - 1) / kBlock8;
    p.rows = rows;
    p.dtype = w->dtype;
    p.gated = w->gated;
    p.groups = w->groups;
    p.offsets = grouped ? offsets : nullptr;
    p.splits = plan.splits;
    p.slab = (float *)workspace;
    p.e.y = mat(y);
    p.e.n = w->n;
    p.e.res = Mat{nullptr, nullptr, 0, 0, ORTHRUS_F32};
    if (e) {
        p.e.bias = e->bias;
        p.e.act = e->act;
        p.e.res = mat(&e->residual);
    }
    hipStream_t s = (hipStream_t)stream;
    hipError_t rc = plan.shape < 0 ? launch_few(p, s) : launch_tile(p, plan, s);
    if (rc == hipSuccess && plan.splits > 1) rc = launch_join(p, s);
    return rc == hipSuccess ? ORTHRUS_OK : ORTHRUS_EHIP;
}

}  // namespace

extern "C" {

int orthrus_convert(const orthrus_matrix *x, const orthrus_matrix *y, int32_t rows, int32_t width, void *stream) {
    if (rows < 0 || width < 1) return ORTHRUS_EINVAL;
    if (rows == 0) return ORTHRUS_OK;
    if (!matrix_ok(x, width) || !matrix_ok(y, width)) return ORTHRUS_EINVAL;
    if ((x->dtype == ORTHRUS_MX8) == (y->dtype == ORTHRUS_MX8)) return ORTHRUS_EUNSUPPORTED;
    if (width > (1 << 30)) return ORTHRUS_ECAPACITY;
    if (meets_itself(y, rows, width) || writes_meet(y, x, rows, width, width)) return ORTHRUS_EINVAL;
    return launch_convert(mat(x), mat(y), rows, width, (hipStream_t)stream) == hipSuccess ? ORTHRUS_OK : ORTHRUS_EHIP;
}

int orthrus_norm(const orthrus_matrix *x, const orthrus_matrix *add, const orthrus_matrix *total, const float *gain, float eps,
                 const orthrus_matrix *y, int32_t rows, int32_t width, void *stream) {
    if (rows < 0 || width < 1 || !(eps >= 0.f)) return ORTHRUS_EINVAL;
    if (rows == 0) return ORTHRUS_OK;
    if (!matrix_ok(x, width) || !matrix_ok(y, width) || (add && !matrix_ok(add, width)) || (total && !matrix_ok(total, width)) ||
        (uintptr_t)gain % 4)
        return ORTHRUS_EINVAL;
    if (x->dtype == ORTHRUS_MX8 || (add && add->dtype == ORTHRUS_MX8) || (total && total->dtype == ORTHRUS_MX8)) return ORTHRUS_EUNSUPPORTED;
    if (width > (1 << 30)) return ORTHRUS_ECAPACITY;
    const Runs factors = bytes_of(gain, (size_t)width * 4);
    if (meets_itself(y, rows, width) || writes_meet(y, total, rows, width, width) || writes_meet(y, factors, rows, width) ||
        writes_meet(total, factors, rows, width))
        return ORTHRUS_EINVAL;
    for (const orthrus_matrix *read : {x, add})
        for (const orthrus_matrix *written : {y, total})
            if (!same_rows(written, read, rows) && writes_meet(written, read, rows, width, width)) return ORTHRUS_EINVAL;
    const NormOp a{mat(x), mat(add), mat(total), mat(y), gain, eps, rows, width};
    return launch_norm_op(a, (hipStream_t)stream) == hipSuccess ? ORTHRUS_OK : ORTHRUS_EHIP;
}

size_t orthrus_linear_packed_bytes(const orthrus_linear_weights *w) {
    if (!weights_ok(w) || !weights_fit(w)) return 0;
    return (packed_shape(w->dtype, w->n, w->k, w->gated).bytes + 255) / 256 * 256 * w->groups;
}

int orthrus_linear_pack(const orthrus_linear_weights *w, const orthrus_matrix *matrix, const orthrus_matrix *up, void *stream) {
    if (!weights_ok(w) || !w->packed || (uintptr_t)w->packed % 256 || !matrix_ok(matrix, w->k) || (w->gated != 0) != (up != nullptr) ||
        (up && !matrix_ok(up, w->k)))
        return ORTHRUS_EINVAL;
    if (matrix->dtype != w->dtype || (up && up->dtype != w->dtype)) return ORTHRUS_EUNSUPPORTED;
    if (!weights_fit(w)) return ORTHRUS_ECAPACITY;
    PackedShape p = packed_shape(w->dtype, w->n, w->k, w->gated);
    p.bytes = (p.bytes + 255) / 256 * 256;
    const Runs packed = bytes_of(w->packed, p.bytes * w->groups);
    const int64_t rows = (int64_t)w->groups * w->n;
    for (const orthrus_matrix *read : {matrix, up})
        if (runs_meet(packed, elements_of(read, rows, w->k)) || runs_meet(packed, scales_of(read, rows, w->k))) return ORTHRUS_EINVAL;
    return launch_pack(*w, p, mat(matrix), mat(up), (hipStream_t)stream) == hipSuccess ? ORTHRUS_OK : ORTHRUS_EHIP;
}

size_t orthrus_linear_bytes(const orthrus_linear_weights *w, int32_t rows) {
    if (!weights_ok(w) || !weights_fit(w) || rows < 1 || w->groups != 1) return 0;
    return most_slab(packed_shape(w->dtype, w->n, w->k, w->gated), rows);
}

int orthrus_linear(const orthrus_linear_weights *w, const orthrus_matrix *x, int32_t rows, const orthrus_epilogue *epilogue,
                   const orthrus_matrix *y, void *workspace, size_t ws_bytes, void *stream) {
    return product(w, x, nullptr, false, rows, epilogue, y, workspace, ws_bytes, stream);
}

int orthrus_linear_grouped(const orthrus_linear_weights *w, const orthrus_matrix *x, const int32_t *offsets, int32_t rows,
                           const orthrus_epilogue *epilogue, const orthrus_matrix *y, void *workspace, size_t ws_bytes, void *stream) {
    return product(w, x, offsets, true, rows, epilogue, y, workspace, ws_bytes, stream);
}

}  // extern "C"
