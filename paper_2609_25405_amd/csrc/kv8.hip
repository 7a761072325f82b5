// C entries of the 8-bit cache's operators: the rows handle, its plan's upload, argument checks.
#include <hip/hip_runtime.h>

#include <atomic>
#include <cmath>
#include <cstring>
#include <new>

#include "kv8.hpp"

namespace {
using namespace orthrus;

constexpr size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// one plan's copy from pinned host memory, which the kernel reads through its device address (a
// copy engine's hand-off leaves the GPU idle for longer than these few kilobytes take)
__global__ __launch_bounds__(256) void plan_upload_kernel(const int4 *src, int4 *dst, int n16) {
    for (int i = blockIdx.x * 256 + threadIdx.x; i < n16; i += gridDim.x * 256) dst[i] = src[i];
}

std::atomic<int32_t> next_stamp{1};

}  // namespace

struct orthrus_rows {
    orthrus_head_shape shape{};
    std::vector<double> turns;     // turns per position of each pair
    RowsPlan plan;
    bool planned = false;
    int device = -1, stamp = 0;
    char *ws = nullptr;
    int *err = nullptr;            // device error word
    // pinned staging, double-buffered; an event marks when a buffer's upload is done
    void *stage[2] = {nullptr, nullptr}, *stage_dev[2] = {nullptr, nullptr};
    size_t stage_bytes[2] = {0, 0};
    hipEvent_t ev[2] = {nullptr, nullptr};
    int next = 0;
};

namespace {

#define HIP_TRY(expr)                                   \
    do {                                                \
        if ((expr) != hipSuccess) {                     \
            (void)hipGetLastError();                    \
            return ORTHRUS_EHIP;                        \
        }                                               \
    } while (0)

bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

bool kv8_ok(const orthrus_kv8 *kv) {
    return kv && kv->k_cache && kv->v_cache && kv->k_scale && kv->v_scale && kv->block_table && kv->n_layers > 0 &&
           kv->n_pages > 0 && kv->n_seq > 0 && kv->max_blocks > 0 && aligned16(kv->k_cache) && aligned16(kv->v_cache);
}

float *partials_of(const orthrus_rows *r) { return (float *)(r->ws + kPlanOffset + up256(r->plan.meta.size() * 4)); }

// the checks every call on a plan makes, and its kernels' common arguments
int plan_args(const orthrus_rows *r, const orthrus_kv8 *kv, int32_t layer, Plan8 &p) {
    if (!r || !kv8_ok(kv) || layer < 0 || layer >= kv->n_layers || !r->planned) return ORTHRUS_EINVAL;
    if (kv->n_seq < r->plan.need_seq || kv->max_blocks < r->plan.need_blocks) return ORTHRUS_ECAPACITY;
    int dev = -1;
    HIP_TRY(hipGetDevice(&dev));
    if (dev != r->device) return ORTHRUS_EINVAL;
    const orthrus_head_shape &s = r->shape;
    const size_t heads = (size_t)kv->n_pages * s.n_kv_heads, bytes = heads * kPage8 * s.head_dim;
    p.meta = (const int32_t *)(r->ws + kPlanOffset);
    p.stamp = r->stamp;
    p.err = r->err;
    p.k = (uint8_t *)kv->k_cache + layer * bytes;
    p.v = (uint8_t *)kv->v_cache + layer * bytes;
    p.ks = kv->k_scale + layer * heads;
    p.vs = kv->v_scale + layer * heads;
    p.table = kv->block_table;
    p.n_pages = kv->n_pages;
    p.max_blocks = kv->max_blocks;
    p.nq = s.n_q_heads;
    p.nkv = s.n_kv_heads;
    p.hd = s.head_dim;
    p.group = s.n_q_heads / s.n_kv_heads;
    return ORTHRUS_OK;
}

bool rows_ok(const void *base, int64_t stride, int64_t least) {
    return base && aligned16(base) && stride >= least && stride % 8 == 0;
}

}  // namespace

namespace orthrus {

int rows_prepare(const orthrus_rows *r, const orthrus_kv8 *kv, const orthrus_segment *segments, int n, RowsPlan &p, size_t &bytes) {
    if (!r || !kv8_ok(kv)) return ORTHRUS_EINVAL;
    try {
        const int rc = plan_rows8(r->shape, r->turns, *kv, segments, n, p);
        if (rc) return rc;
        const size_t meta = up256(p.meta.size() * 4);
        p.meta.resize(meta / 4, 0);
        bytes = kPlanOffset + meta + (size_t)p.n_slots * kSmallCols * (r->shape.head_dim + kPartialPad) * 4;
    } catch (...) {
        return ORTHRUS_ECAPACITY;   // out of host memory
    }
    return ORTHRUS_OK;
}

int rows_upload(orthrus_rows *r, RowsPlan &&p, void *workspace, int *err, void *stream) {
    hipStream_t s = (hipStream_t)stream;
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    HIP_TRY(hipStreamIsCapturing(s, &cap));
    if (cap != hipStreamCaptureStatusNone) return ORTHRUS_EUNSUPPORTED;
    int dev = -1;
    HIP_TRY(hipGetDevice(&dev));
    if (r->device >= 0 && dev != r->device) return ORTHRUS_EINVAL;
    r->device = dev;
    const size_t meta = p.meta.size() * 4;
    const int stamp = next_stamp.fetch_add(1);
    p.meta[0] = stamp;
    const int i = r->next;
    if (r->ev[i]) HIP_TRY(hipEventSynchronize(r->ev[i]));
    else HIP_TRY(hipEventCreateWithFlags(&r->ev[i], hipEventDisableTiming));
    if (r->stage_bytes[i] < meta) {
        if (r->stage[i]) (void)hipHostFree(r->stage[i]);   // its last upload is done
        r->stage[i] = r->stage_dev[i] = nullptr;
        r->stage_bytes[i] = 0;
        HIP_TRY(hipHostMalloc(&r->stage[i], 2 * meta, hipHostMallocCoherent));
        HIP_TRY(hipHostGetDevicePointer(&r->stage_dev[i], r->stage[i], 0));
        r->stage_bytes[i] = 2 * meta;
    }
    std::memcpy(r->stage[i], p.meta.data(), meta);
    const int n16 = (int)(meta / 16), blocks = std::min((n16 + 255) / 256, 128);
    hipLaunchKernelGGL(plan_upload_kernel, dim3(blocks), dim3(256), 0, s, (const int4 *)r->stage_dev[i],
                       (int4 *)((char *)workspace + kPlanOffset), n16);
    HIP_TRY(hipGetLastError());
    HIP_TRY(hipEventRecord(r->ev[i], s));
    r->next ^= 1;
    r->plan = std::move(p);
    r->stamp = stamp;
    r->ws = (char *)workspace;
    r->err = err;
    r->planned = true;
    return ORTHRUS_OK;
}

int append_rows8(const orthrus_rows *r, const orthrus_kv8 *kv, int32_t layer, const void *qkv, int32_t qkv_dtype, int64_t row_stride,
                 int64_t slab, const float *q_gain, const float *k_gain, void *q_out, int64_t q_stride, void *stream) {
    Append8 a{};
    const int rc = plan_args(r, kv, layer, a.p);
    if (rc) return rc;
    const orthrus_head_shape &s = r->shape;
    if (qkv_dtype != ORTHRUS_F32 && qkv_dtype != ORTHRUS_BF16) return ORTHRUS_EINVAL;
    if (qkv_dtype == ORTHRUS_BF16 && s.dtype != ORTHRUS_BF16) return ORTHRUS_EUNSUPPORTED;
    if (r->plan.T == 0) return ORTHRUS_OK;
    const int64_t q_dim = (int64_t)s.n_q_heads * s.head_dim;
    if (!rows_ok(qkv, row_stride, q_dim + 2 * (int64_t)s.n_kv_heads * s.head_dim) || !rows_ok(q_out, q_stride, q_dim)) return ORTHRUS_EINVAL;
    if (!aligned16(q_gain) || !aligned16(k_gain)) return ORTHRUS_EINVAL;
    a.qkv = qkv;
    a.stride = row_stride;
    a.slab = slab;
    a.q_gain = q_gain;
    a.k_gain = k_gain;
    a.q_out = q_out;
    a.q_stride = q_stride;
    a.n_units = r->plan.n_units;
    a.most = r->plan.most_unit;
    a.rot = s.rot_dims;
    a.interleaved = s.interleaved;
    a.in_dtype = qkv_dtype;
    a.out_dtype = s.dtype;
    a.magnitude = s.rope_magnitude;
    a.eps = s.norm_eps;
    return launch_append8(a, (hipStream_t)stream) == hipSuccess ? ORTHRUS_OK : ORTHRUS_EHIP;
}

}  // namespace orthrus

extern "C" {

int orthrus_rows_create(const orthrus_head_shape *shape, orthrus_rows **out) {
    if (!shape || !out) return ORTHRUS_EINVAL;
    *out = nullptr;
    const int rc = validate_shape8(*shape);
    if (rc) return rc;
    orthrus_rows *r = new (std::nothrow) orthrus_rows;
    if (!r) return ORTHRUS_EINVAL;
    try {
        r->shape = *shape;
        for (int i = 0; i < shape->rot_dims / 2; ++i) {
            const double f = shape->rope_freq ? shape->rope_freq[i] : std::pow((double)shape->rope_base, -2.0 * i / shape->rot_dims);
            r->turns.push_back(f / (2.0 * M_PI));
        }
    } catch (...) {
        delete r;
        return ORTHRUS_EINVAL;
    }
    r->shape.rope_freq = nullptr;
    *out = r;
    return ORTHRUS_OK;
}

void orthrus_rows_destroy(orthrus_rows *r) {
    if (!r) return;
    for (int i = 0; i < 2; ++i) {
        if (r->ev[i]) {
            (void)hipEventSynchronize(r->ev[i]);
            (void)hipEventDestroy(r->ev[i]);
        }
        if (r->stage[i]) (void)hipHostFree(r->stage[i]);
    }
    delete r;
}

size_t orthrus_rows_workspace_bytes(const orthrus_rows *r, int32_t max_rows, int32_t max_segments, int32_t max_keys) {
    if (!r || max_rows < 0 || max_segments < 0 || max_keys < 0) return 0;
    size_t ints = 0, slots = 0;
    bound_rows8(r->shape, max_rows, max_segments, max_keys, ints, slots);
    return kPlanOffset + up256(ints * 4) + slots * kSmallCols * (size_t)(r->shape.head_dim + kPartialPad) * 4;
}

int orthrus_rows_items(const orthrus_rows *r, const orthrus_kv8 *kv, const orthrus_segment *segments, int32_t n,
                       int32_t counts[4], int32_t *items, int32_t cap) {
    if (!r || !kv8_ok(kv) || (items && cap < 0)) return ORTHRUS_EINVAL;
    try {
        RowsPlan p;
        const int rc = plan_rows8(r->shape, r->turns, *kv, segments, n, p);
        if (rc) return rc;
        if (counts) {
            counts[0] = p.n_small;
            counts[1] = p.n_tiles;
            counts[2] = p.n_merge;
            counts[3] = p.n_slots;
        }
        if (items) {
            const int m = std::min<int>(cap, p.n_small + p.n_tiles);   // small items, then tiles: one run of the meta
            std::memcpy(items, p.meta.data() + p.off_small, (size_t)m * kItem8Ints * 4);
        }
    } catch (...) {
        return ORTHRUS_ECAPACITY;   // out of host memory
    }
    return ORTHRUS_OK;
}

int orthrus_rows_plan(orthrus_rows *r, const orthrus_kv8 *kv, const orthrus_segment *segments, int32_t n, void *workspace,
                      size_t ws_bytes, void *stream) {
    if (!workspace || ((uintptr_t)workspace & 255)) return ORTHRUS_EINVAL;
    RowsPlan p;
    size_t bytes = 0;
    const int rc = rows_prepare(r, kv, segments, n, p, bytes);
    if (rc) return rc;
    if (ws_bytes < bytes) return ORTHRUS_ECAPACITY;
    return rows_upload(r, std::move(p), workspace, (int *)workspace, stream);
}

int orthrus_kv8_append(const orthrus_rows *r, const orthrus_kv8 *kv, int32_t layer, const void *qkv, int32_t qkv_dtype,
                       int64_t row_stride, const float *q_gain, const float *k_gain, void *q_out, int64_t q_stride,
                       void *stream) {
    return append_rows8(r, kv, layer, qkv, qkv_dtype, row_stride, 0, q_gain, k_gain, q_out, q_stride, stream);
}

int orthrus_kv8_read(const orthrus_rows *r, const orthrus_kv8 *kv, int32_t layer, void *k_out, void *v_out, void *stream) {
    Read8 a{};
    const int rc = plan_args(r, kv, layer, a.p);
    if (rc) return rc;
    if (r->plan.T == 0) return ORTHRUS_OK;
    if (!k_out || !v_out || !aligned16(k_out) || !aligned16(v_out)) return ORTHRUS_EINVAL;
    a.n_units = r->plan.n_units;
    a.most = r->plan.most_unit;
    a.k_out = (bf16 *)k_out;
    a.v_out = (bf16 *)v_out;
    return launch_read8(a, (hipStream_t)stream) == hipSuccess ? ORTHRUS_OK : ORTHRUS_EHIP;
}

int orthrus_kv8_attend(const orthrus_rows *r, const orthrus_kv8 *kv, int32_t layer, const void *q, int64_t q_stride,
                       float scale, void *out, int64_t out_stride, void *stream) {
    Attend8 a{};
    const int rc = plan_args(r, kv, layer, a.p);
    if (rc) return rc;
    const orthrus_head_shape &s = r->shape;
    if (scale == 0.f) scale = 1.0f / std::sqrt((float)s.head_dim);
    const float scale2 = 1.4426950408889634f * scale;
    if (!(scale > 0.f) || !std::isfinite(scale2)) return ORTHRUS_EINVAL;
    if (r->plan.T == 0) return ORTHRUS_OK;
    const int64_t q_dim = (int64_t)s.n_q_heads * s.head_dim;
    if (!rows_ok(q, q_stride, q_dim) || !rows_ok(out, out_stride, q_dim)) return ORTHRUS_EINVAL;
    a.q = q;
    a.out = out;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.dtype = s.dtype;
    a.n_small = r->plan.n_small;
    a.n_tiles = r->plan.n_tiles;
    a.n_merge = r->plan.n_merge;
    a.merge_slots = r->plan.merge_slots;
    a.small_cols = r->plan.small_cols;
    a.wide = r->plan.wide;
    a.joint = r->plan.joint;
    a.off_small = r->plan.off_small;
    a.off_tiles = r->plan.off_tiles;
    a.off_merge = r->plan.off_merge;
    a.scale = scale2;
    a.partials = partials_of(r);
    return launch_attend8(a, (hipStream_t)stream) == hipSuccess ? ORTHRUS_OK : ORTHRUS_EHIP;
}

}  // extern "C"
