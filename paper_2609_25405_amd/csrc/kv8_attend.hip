// Causal attention of ragged rows over the 8-bit paged cache.
//
// Both kernels turn codes into bf16 by v_cvt_scalef32_pk_bf16_fp8 (two codes an instruction, exact) and
// multiply on bf16 MFMA, with an online softmax in fp32 (exp2 domain).  fp32 rows go through the
// same products in parts: q and the weights as three bf16 parts each (24 bits, all of an fp32 value), each part a
// product of its own into the same sums.
//
// Small items ((rows, query heads of one KV head) pairs of a segment, at most 16): the pairs are the 16 columns
// of a 16x16x32 MFMA, so all query heads and rows that share a key read it once, and the arithmetic
// hides behind the cache's bytes.  A wave walks steps of 64 keys (4 pages): a page's keys are one
// 2-KB run (head_dim 128) of which lane (quarter, key) reads the quarter's dims; the scores then lie
// with lane (quarter, column) holding keys 4 quarter .. + 3 of each page, which is also how the
// cache lays out its values (slot / 4 outermost), so weights feed the second product without
// moving between lanes.  Bound by the cache's bytes: 256 rows of 4096 to 8192 keys over 8 KV heads of 128 dims 540 us, 6.0 TB/s.
//
// Tiles (128 pairs of a longer segment): four waves of 32 pairs; 64-key blocks are turned into bf16 once
// per workgroup on their way into LDS (two buffers, the next block's codes in flight in registers).  Bound by the matrix pipe with
// the softmax's vector work beside it: 2 x 512 rows after 7680 keys, 32 query heads over 8, 134 GFLOP in 142 us and the
// merge of their pieces in 11.  fp32 rows have three times the products: 64 rows of 1024 to 4096 keys 81 us, those chunks 388.
//
// Long key ranges come as pieces that leave (max, sum, unnormalised output) to a merge launch.  (Joining
// them in the workgroup that arrives last was five times slower: its device-scope release and acquire write back and
// drop the L2 that all other workgroups read through.)
#include <type_traits>

#include "kv8.hpp"

namespace orthrus {
namespace {

__device__ __forceinline__ float2 partner16(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return float2{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ float2 partner32(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return float2{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
// over the four quarters (16 lanes each) of a wave
__device__ __forceinline__ float quarters_max(float v) {
    float2 p = partner16(v);
    v = fmaxf(p.x, p.y);
    p = partner32(v);
    return fmaxf(p.x, p.y);
}
__device__ __forceinline__ float quarters_sum(float v) {
    float2 p = partner16(v);
    v = p.x + p.y;
    p = partner32(v);
    return p.x + p.y;
}

__device__ __forceinline__ float first_lane(float v) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v))); }

// a barrier that orders LDS only: loads from global memory stay in flight across it
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

__device__ __forceinline__ bf16x8 as_bf16x8(uint2 a, uint2 b) { return __builtin_bit_cast(bf16x8, u32x4{a.x, a.y, b.x, b.y}); }

// eight values as N bf16 parts whose sum they are (to 8 N bits)
template <int N> __device__ __forceinline__ void parts_of(const float (&x)[8], bf16x8 (&out)[N]) {
    float r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = x[j];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = pack_bf16x2(r[2 * j], r[2 * j + 1]);
        out[k] = __builtin_bit_cast(bf16x8, w);
        if (k + 1 < N) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                r[2 * j] -= bf16_lo(w[j]);
                r[2 * j + 1] -= bf16_hi(w[j]);
            }
        }
    }
}
// eight consecutive q values as NQ parts
template <typename T, int NQ> __device__ __forceinline__ void load_q(const T *p, bf16x8 (&out)[NQ]) {
    if constexpr (NQ == 1) {
        out[0] = *(const bf16x8 *)p;
    } else {
        const f32x4 a = *(const f32x4 *)p, b = *(const f32x4 *)(p + 4);
        const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        parts_of<NQ>(x, out);
    }
}

// the sum of a word's two bf16 values and c
__device__ __forceinline__ float add_pair(uint32_t w, float c) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), __builtin_bit_cast(bf16x2, 0x3f803f80u), c, false);
}

// Parts of q (NQ) and of a weight (NP).  bf16 rows take their weights to bf16, 2^-8 as their output's own rounding, and divide by
// the sum of the rounded ones, so that equal values come out whole.  In two parts small items are off by no more than the output's
// rounding (64 rows of 1 k to 4 k keys 1.62e-3 instead of 1.68e-3) but 71.3 us instead of 67.3, and tiles would have half as
// many products again.
template <typename T> struct Rows8;
template <> struct Rows8<bf16> { static constexpr int NQ = 1, NP = 1; };
template <> struct Rows8<float> { static constexpr int NQ = 3, NP = 3; };

__device__ __forceinline__ void store4(float *p, float a, float b, float c, float d) { *(float4 *)p = float4{a, b, c, d}; }
__device__ __forceinline__ void store4(bf16 *p, float a, float b, float c, float d) {
    *(uint2 *)p = uint2{pack_bf16x2(a, b), pack_bf16x2(c, d)};
}

// A pair whose every score is minus infinity has no weights: its output is not a number, unlike that of a pair
// without keys.  Its sum of weights, which would be zero, is marked.
constexpr float kNoWeights = -1.f;
__device__ __forceinline__ float inverse(float l) { return l == 0.f ? 0.f : l < 0.f ? NAN : 1.f / l; }
// whether row `row` of the item at `at` of the plan has a key in the item's range (both read again: this is rare, registers are not)
__device__ __forceinline__ bool has_key(const Attend8 &a, int at, int row) {
    const int32_t *it = a.p.meta + at, *table = a.p.table + (size_t)it[A8_SEQ] * a.p.max_blocks;
    for (int k = it[A8_KEY0]; k < min(it[A8_KEY1], it[A8_POS] + row + 1); k += kPage8) {
        const int id = table[k / kPage8];
        if (id >= 0 && id < a.p.n_pages) return true;
    }
    return false;
}

// The last position among the keys of the item at `at` of the plan that not all of its rows see, whose value is not finite (-1:
// none); by one wave.  Sums that are not finite for another reason are what they should be.
template <int HD> __device__ int last_odd_value(const Attend8 &a, int at) {
    const int32_t *it = a.p.meta + at, *table = a.p.table + (size_t)it[A8_SEQ] * a.p.max_blocks;
    const int first = max(it[A8_KEY0], it[A8_POS] + 1), end = it[A8_KEY1], lane = threadIdx.x & 63;
    int found = -1;
    for (int b = first / kPage8; b * kPage8 < end; ++b) {
        const int id = table[b];
        if (id < 0 || id >= a.p.n_pages) continue;
        const size_t head = (size_t)id * a.p.nkv + it[A8_HEAD];
        const uint32_t *words = (const uint32_t *)(a.p.v + head * (kPage8 * HD));
        const bool all = !(fabsf(a.p.vs[head]) * 448.f < INFINITY);
        for (int i = lane; i < kPage8 * HD / 4; i += 64) {            // four slots of a dim
            const uint32_t w = words[i];
            for (int e = 0; e < 4; ++e) {
                const int pos = b * kPage8 + i / HD * 4 + e;
                if (pos >= first && pos < end && (all || (w >> (8 * e) & 0x7f) == 0x7f)) found = max(found, pos);
            }
        }
    }
#pragma unroll
    for (int o = 1; o < 64; o *= 2) found = max(found, __shfl_xor(found, o, 64));
    return found;
}

// One (row, query head) pair, by one wave, key after key, so that nothing the row does not see enters its
// sums: for pairs whose sums met something not finite in a masked place (zero times it is not zero).
// Lane l holds dims l (and l + 64).
template <typename T, int HD>
__device__ void pair_key_by_key(const Attend8 &a, int seq, int head, int pos, int key0, int key1, const T *qp, float &m_out,
                                float &l_out, float (&o)[HD / 64]) {
    constexpr int N = HD / 64;
    const int lane = threadIdx.x & 63;
    const int32_t *table = a.p.table + (size_t)seq * a.p.max_blocks;
    float q[N], m = -INFINITY, l = 0.f;
    bool any = false;
#pragma unroll
    for (int d = 0; d < N; ++d) {
        q[d] = to_f32(qp[lane + 64 * d]);
        o[d] = 0.f;
    }
    for (int key = key0; key < min(key1, pos + 1); ++key) {
        const int page = table[key / kPage8], slot = key % kPage8;
        if (page < 0 || page >= a.p.n_pages) continue;
        any = true;
        const size_t at = (size_t)page * a.p.nkv + head;
        const uint8_t *kp = a.p.k + at * (kPage8 * HD) + slot * HD, *vp = a.p.v + at * (kPage8 * HD) + (slot / 4) * (4 * HD) + slot % 4;
        float s = 0.f;
#pragma unroll
        for (int d = 0; d < N; ++d) s = fmaf(q[d], bf16_lo(codes_bf16<false>(kp[lane + 64 * d], a.p.ks[at])), s);
        s = wave_sum(s) * a.scale;
        const float mn = fmaxf(m, s);
        const float alpha = m == -INFINITY ? 0.f : exp2f(m - mn), p = s == -INFINITY ? 0.f : exp2f(s - mn);
        l = l * alpha + p;
#pragma unroll
        for (int d = 0; d < N; ++d) {
            const int dim = lane + 64 * d;
            const float v = bf16_lo(codes_bf16<false>(vp[(dim % 16) * (HD / 4) + (dim / 16) * 4], 1.f)) * a.p.vs[at];
            o[d] = fmaf(p, v, o[d] * alpha);
        }
        m = mn;
    }
    m_out = m;
    l_out = l == 0.f && any ? kNoWeights : l;
}

// ------------------------------------------------------------------ pieces of a key range
template <int HD> __device__ __forceinline__ float *partial_of(const Attend8 &a, int slot, int col) {
    return a.partials + ((size_t)slot * 16 + col) * (HD + kPartialPad);
}

// blockIdx.x: merge entry, blockIdx.y: 16 of its (row, head) pairs; the pieces in their order
template <typename T, int HD> __global__ __launch_bounds__(256) void attend8_merge_kernel(Attend8 a) {
    constexpr int TPC = 256 / kSmallCols;                 // threads a pair for its factors
    __shared__ float f[kSmallCols][kMaxPieces + 1], inv[kSmallCols];
    Entry8<kMerge8Ints> entry;
    if (!entry8(a.p, a.off_merge + kMerge8Ints * (int)blockIdx.x, entry)) return;
    const int32_t *me = entry.v;
    const int n = me[M8_PIECES], slots = me[M8_SLOTS], c0 = blockIdx.y * kSmallCols, tid = threadIdx.x;
    const int cols = min(kSmallCols, me[M8_LEN] * a.p.group - c0);
    if (cols <= 0) return;
    const int slot0 = me[M8_SLOT] + (int)blockIdx.y;
    // the first pieces' sums are on their way while the factors are taken
    constexpr int UNITS = kSmallCols * HD / 4 / 256, FIRST = 4;
    const size_t step = (size_t)slots * 16 * (HD + kPartialPad);
    auto sums_of = [&](int u) { return partial_of<HD>(a, slot0, u / (HD / 4)) + kPartialPad + u % (HD / 4) * 4; };
    f32x4 early[UNITS][FIRST];
#pragma unroll
    for (int k = 0; k < UNITS; ++k) {
        const float *p = sums_of(min(tid + 256 * k, cols * (HD / 4) - 1));
#pragma unroll
        for (int i = 0; i < FIRST; ++i)
            if (i < n) early[k][i] = *(const f32x4 *)(p + i * step);
    }
    {
        const int col = tid / TPC;
        float M = -INFINITY, L = 0.f, least = 0.f;
        if (col < cols) {
            for (int i = tid % TPC; i < n; i += TPC) M = fmaxf(M, partial_of<HD>(a, slot0 + i * slots, col)[0]);
        }
#pragma unroll
        for (int o = 1; o < TPC; o *= 2) M = fmaxf(M, __shfl_xor(M, o, 64));
        if (col < cols) {
            for (int i = tid % TPC; i < n; i += TPC) {
                const float *p = partial_of<HD>(a, slot0 + i * slots, col);
                // (a piece whose every score was not a number has a sum but no maximum)
                const float w = p[0] == -INFINITY ? (p[1] == 0.f || p[1] == kNoWeights ? 0.f : 1.f) : __builtin_amdgcn_exp2f(p[0] - M);
                f[col][i] = w;
                least = fminf(least, p[1]);
                L = fmaf(p[1], w, L);
            }
        }
#pragma unroll
        for (int o = 1; o < TPC; o *= 2) {
            L += __shfl_xor(L, o, 64);
            least = fminf(least, __shfl_xor(least, o, 64));
        }
        if (tid % TPC == 0) inv[col] = inverse(L == 0.f ? least : L);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < UNITS; ++k) {
        const int u = tid + 256 * k, col = u / (HD / 4), d = u % (HD / 4) * 4;
        if (col >= cols) break;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < FIRST; ++i)
            if (i < n) sum += early[k][i] * f[col][i];
        const float *p = sums_of(u);
#pragma unroll 8
        for (int i = FIRST; i < n; ++i) sum += *(const f32x4 *)(p + i * step) * f[col][i];
        const int c = c0 + col, row = me[M8_ROW] + c / a.p.group, h = me[M8_HEAD] * a.p.group + c % a.p.group;
        store4((T *)a.out + (size_t)row * a.out_stride + (size_t)h * HD + d, sum[0] * inv[col], sum[1] * inv[col], sum[2] * inv[col],
               sum[3] * inv[col]);
    }
}

// ------------------------------------------------------------------ small items
// LDS of a small item of `cols` pairs
template <int HD, int NW> constexpr int small_lds(int cols) { return NW * (32 + cols * (HD + 4)) * 4; }

template <typename T, int HD, int NW> __device__ __forceinline__ void small_item(const Attend8 &a, int index, char *lds) {
    using R = Rows8<T>;
    constexpr int QD = HD / 4, KK = HD / 32, DB = HD / 16, STEP = 64, PG = 4;
    constexpr int LD = HD + 4;
    float *sm = (float *)lds, *sl = sm + NW * 16;      // [NW][16] maxima and sums
    float *so = sl + NW * 16;                          // [NW][pairs][LD] sums
    Entry8<kItem8Ints> entry;
    if (!entry8(a.p, a.off_small + kItem8Ints * index, entry)) return;
    const int32_t *it = entry.v;
    const int seq = it[A8_SEQ], row0 = it[A8_ROW], len = it[A8_LEN], pos0 = it[A8_POS], g = it[A8_HEAD];
    const int key0 = it[A8_KEY0], key1 = it[A8_KEY1], slot = it[A8_SLOT];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, qd = lane >> 4;
    const int cols = len * a.p.group;
    const int cc = min(c, cols - 1), tok = cc / a.p.group, h = g * a.p.group + cc % a.p.group;
    const int pos = pos0 + tok;
    const int32_t *table = a.p.table + (size_t)seq * a.p.max_blocks;
    const size_t head_bytes = kPage8 * HD;
    const T *qp = (const T *)a.q + (size_t)(row0 + tok) * a.q_stride + (size_t)h * HD;

    bf16x8 q[KK][R::NQ];
#pragma unroll
    for (int k = 0; k < KK; ++k) load_q<T, R::NQ>(qp + qd * QD + 8 * k, q[k]);

    f32x4 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    const int last = (key1 - 1) / kPage8;
    const int steps = (key1 - key0 + STEP - 1) / STEP;
    u32x4 kr[PG][QD / 16], vr[PG][QD / 16];
    float ks[PG], vs[PG];
    int valid[PG], pg[PG];
    auto pages_of = [&](int st) {
#pragma unroll
        for (int p = 0; p < PG; ++p) pg[p] = table[min(key0 / kPage8 + st * PG + p, last)];
    };
    // keys of the step's pages that the item has; bad and absent pages have none and read page 0
    int next_valid[PG];
    auto check = [&](int st) {
#pragma unroll
        for (int p = 0; p < PG; ++p) {
            const int k = key0 + st * STEP + p * kPage8;
            const bool ok = pg[p] >= 0 && pg[p] < a.p.n_pages;
            next_valid[p] = ok ? max(0, min(kPage8, key1 - k)) : 0;
            if (!ok && k < key1 && lane == 0) flag_error(a.p.err, ORTHRUS_DEVERR_PAGE);
            pg[p] = ok ? pg[p] : 0;
        }
    };
    auto load = [&](const uint8_t *pool, const float *scales, u32x4 (&r)[PG][QD / 16], float (&s)[PG], int at) {
#pragma unroll
        for (int p = 0; p < PG; ++p) {
            const size_t head = (size_t)pg[p] * a.p.nkv + g;
#pragma unroll
            for (int j = 0; j < QD / 16; ++j) r[p][j] = *(const u32x4 *)(pool + head * head_bytes + at + 16 * j);
            s[p] = scales[head];
        }
    };
    const int k_at = c * HD + qd * QD;                 // lane (quarter, key): the quarter's dims
    const int v_at = qd * (4 * HD) + c * (HD / 4);     // lane (quarter, dim % 16): 4 slots of every 16th dim

    // the next step's keys are on their way once this step's scores are taken, its values once this
    // step's are used; its page ids were read a step ahead
    float ks_next[PG];
    if (wave < steps) {
        pages_of(wave);
        check(wave);
        load(a.p.k, a.p.ks, kr, ks_next, k_at);
        load(a.p.v, a.p.vs, vr, vs, v_at);
        pages_of(min(wave + NW, steps - 1));
    }
    for (int st = wave; st < steps; st += NW) {
        const bool more = st + NW < steps;
        f32x4 s[PG];
#pragma unroll
        for (int p = 0; p < PG; ++p) {
            valid[p] = next_valid[p];
            ks[p] = ks_next[p];
            s[p] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KK; ++k) {
                const bf16x8 kf = as_bf16x8(word_bf16(kr[p][k / 2][2 * (k % 2)], ks[p]), word_bf16(kr[p][k / 2][2 * (k % 2) + 1], ks[p]));
#pragma unroll
                for (int n = 0; n < R::NQ; ++n) s[p] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[k][n], s[p], 0, 0, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (more) {
            check(st + NW);
            load(a.p.k, a.p.ks, kr, ks_next, k_at);
        }
        __builtin_amdgcn_sched_barrier(0);
        const int kbase = key0 + st * STEP;
        float mloc = -INFINITY;
#pragma unroll
        for (int p = 0; p < PG; ++p) {
            const int seen = min(valid[p], pos + 1 - kbase - p * kPage8);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[p][r] = 4 * qd + r < seen ? s[p][r] * a.scale : -INFINITY;
                mloc = fmaxf(mloc, s[p][r]);
            }
            vs[p] = valid[p] > 0 ? vs[p] : 1.f;
        }
        mloc = quarters_max(mloc);
        // the maximum follows in jumps of more than 2^8, so that the sums are rarely rescaled
        if (__ballot(mloc > m + 8.f) != 0) {
            const float mn = fmaxf(m, mloc), alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
            l *= alpha;
#pragma unroll
            for (int d = 0; d < DB; ++d) acc[d] *= alpha;
            m = mn;
        }
        const float sub = m == -INFINITY ? 0.f : m;
        float w[PG][4];
#pragma unroll
        for (int p = 0; p < PG; ++p)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                w[p][r] = __builtin_amdgcn_exp2f(s[p][r] - sub);
                if (R::NP > 1) l += w[p][r];
            }
        // values of slots the item does not have may be anything: zero them
        bool whole = true;
#pragma unroll
        for (int p = 0; p < PG; ++p) whole &= valid[p] == kPage8;
        if (!whole) {
#pragma unroll
            for (int p = 0; p < PG; ++p) {
                const int n = min(4, max(0, valid[p] - 4 * qd));
                const uint32_t keep = n == 4 ? 0xffffffffu : (1u << (8 * n)) - 1;
#pragma unroll
                for (int j = 0; j < QD / 16; ++j) vr[p][j] &= keep;
            }
        }
#pragma unroll
        for (int p = 0; p < PG; p += 2) {
            const float x[8] = {w[p][0], w[p][1], w[p][2], w[p][3], w[p + 1][0], w[p + 1][1], w[p + 1][2], w[p + 1][3]};
            bf16x8 pf[R::NP];
            parts_of<R::NP>(x, pf);
            if (R::NP == 1) {                      // the sum of the weights as they are used
                const u32x4 u = __builtin_bit_cast(u32x4, pf[0]);
#pragma unroll
                for (int k = 0; k < 4; ++k) l = add_pair(u[k], l);
            }
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const bf16x8 vf = as_bf16x8(word_bf16(vr[p][d / 4][d % 4], vs[p]), word_bf16(vr[p + 1][d / 4][d % 4], vs[p + 1]));
#pragma unroll
                for (int n = 0; n < R::NP; ++n) acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[n], acc[d], 0, 0, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (more) {
            load(a.p.v, a.p.vs, vr, vs, v_at);
            pages_of(min(st + 2 * NW, steps - 1));
        }
    }
    l = quarters_sum(l);
    if (qd == 0) {
        sm[wave * 16 + c] = m;
        sl[wave * 16 + c] = l;
    }
    auto sums = [&](int w, int col) { return so + (w * cols + col) * LD; };
    if (c < cols) {
#pragma unroll
        for (int d = 0; d < DB; ++d) *(f32x4 *)(sums(wave, c) + 16 * d + 4 * qd) = acc[d];
    }
    __syncthreads();
    int group = a.p.group;
    asm("" : "+v"(group));       // its reciprocal is taken anew: kept through the loop it would cost a spill
    // Pairs of an earlier row of several: a later row's value that is not finite is masked, not absent.  Their sums are taken
    // again here, ahead of any store to rows that may be q's own.
    if (len > 1) {
        int last_odd = -2;     // (not looked for)
        for (int col = wave; col < cols; col += NW) {
            bool bad = false;
#pragma unroll
            for (int w = 0; w < NW; ++w)
                for (int d = lane; d < HD; d += 64) bad |= !(fabsf(sums(w, col)[d]) < INFINITY);
            if (__ballot(bad) == 0) continue;
            const int t = col / group, hh = g * group + col % group;
            if (pos0 + t + 1 >= key1) continue;        // nothing masked
            if (last_odd == -2) last_odd = last_odd_value<HD>(a, a.off_small + kItem8Ints * index);
            if (last_odd <= pos0 + t) continue;
            float o[HD / 64], mm, ll;
            pair_key_by_key<T, HD>(a, seq, g, pos0 + t, key0, key1, (const T *)a.q + (size_t)(row0 + t) * a.q_stride + (size_t)hh * HD, mm, ll, o);
            // as the first wave's sums, the others without keys
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                if (lane == 0) {
                    sm[w * 16 + col] = w == 0 ? mm : -INFINITY;
                    sl[w * 16 + col] = w == 0 && !(ll < 0.f) ? ll : 0.f;
                }
#pragma unroll
                for (int d = 0; d < HD / 64; ++d) sums(w, col)[lane + 64 * d] = w == 0 ? o[d] : 0.f;
            }
        }
        __syncthreads();
    }
    // merge the waves in order; four dims a thread
    for (int o = tid; o < cols * (HD / 4); o += 64 * NW) {
        const int col = o / (HD / 4), d = o % (HD / 4) * 4;
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) M = fmaxf(M, sm[w * 16 + col]);
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float mw = sm[w * 16 + col], lw = sl[w * 16 + col];
            const float f = mw == -INFINITY ? (lw == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(mw - M);
            L += lw * f;
            sum += *(const f32x4 *)(sums(w, col) + d) * f;
        }
        if (L == 0.f && has_key(a, a.off_small + kItem8Ints * index, col / group)) L = kNoWeights;
        if (slot >= 0) {
            float *pp = partial_of<HD>(a, slot, col);
            if (d == 0) {
                pp[0] = M;
                pp[1] = L;
            }
            *(f32x4 *)(pp + kPartialPad + d) = sum;
        } else {
            const float inv = inverse(L);
            T *dst = (T *)a.out + (size_t)(row0 + col / group) * a.out_stride + (size_t)(g * group + col % group) * HD + d;
            store4(dst, sum[0] * inv, sum[1] * inv, sum[2] * inv, sum[3] * inv);
        }
    }
}

// ------------------------------------------------------------------ tiles of longer segments
constexpr int kWindow = 256;      // pages
// exponents from which a tile takes the difference first (up to there the rounding of the maximum times the scale leaves at
// most 2^-4 in a weight's exponent, no more than the fp32 score's own error)
constexpr float kLargeScore = 0x1p20f;

template <int HD> struct Stage8 {
    static constexpr int KEYS = 64, KRB = HD * 2, KCH = KRB / 16;
    static constexpr int KBYTES = KEYS * KRB, VPAGE = HD * kPage8 * 2, BYTES = KBYTES + 4 * VPAGE;
    // physical 16-byte chunk of chunk c of key row r, and of half c (8 slots) of a value dim: lanes that
    // read one chunk of consecutive rows reach different banks
    static __device__ __forceinline__ int kchunk(int r, int c) { return c ^ ((r / (256 / KRB)) % KCH); }
    static __device__ __forceinline__ int vchunk(int d, int c) { return c ^ ((d >> 3) & 1); }
};

template <typename T, int HD> __device__ __forceinline__ void tile_item(const Attend8 &a, int index, char *smem) {
    using R = Rows8<T>;
    using St = Stage8<HD>;
    constexpr int KS = HD / 16, DB = HD / 32;
    constexpr int KL = HD / 64;              // 16-byte loads of codes a thread and block, keys and values each
    // Page ids (-1: bad) and scales of a run of pages.  Scalar loads would do, but they share a counter with LDS: the barrier
    // of every step would wait for their memory latency.
    float2 *win_scale = (float2 *)(smem + 2 * St::BYTES);
    int *win_page = (int *)(win_scale + kWindow);
    Entry8<kItem8Ints> entry;
    if (!entry8(a.p, a.off_tiles + kItem8Ints * index, entry)) return;
    const int32_t *it = entry.v;
    const int seq = it[A8_SEQ], row0 = it[A8_ROW], len = it[A8_LEN], pos0 = it[A8_POS], g = it[A8_HEAD];
    const int key0 = it[A8_KEY0], key1 = it[A8_KEY1], slot = it[A8_SLOT];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int cols = len * a.p.group;
    const int c = wave * 32 + col, cc = min(c, cols - 1);
    const int tok = cc / a.p.group, h = g * a.p.group + cc % a.p.group;
    const int pos = pos0 + tok;
    const int first_pos = pos0 + min(wave * 32, cols - 1) / a.p.group;     // of this wave's pairs
    const int32_t *table = a.p.table + (size_t)seq * a.p.max_blocks;
    const int nkb = (key1 - key0 + St::KEYS - 1) / St::KEYS, last = (key1 - 1) / kPage8;

    int w0 = key0 / kPage8;            // first page of the window (a multiple of 4)
    auto window_id = [&]() { return table[min(w0 + tid, last)]; };        // (places past the last page repeat it)
    auto load_window = [&](int id) {
        const bool ok = id >= 0 && id < a.p.n_pages;
        const size_t head = (size_t)(ok ? id : 0) * a.p.nkv + g;
        win_page[tid] = ok ? id : -1;
        win_scale[tid] = ok ? float2{a.p.ks[head], a.p.vs[head]} : float2{1.f, 1.f};
        if (!ok) flag_error(a.p.err, ORTHRUS_DEVERR_PAGE);
    };
    static_assert(kWindow == 256, "a page a thread");
    auto window_bad = [&]() {
        bool bad = false;
#pragma unroll
        for (int i = 0; i < kWindow; i += 64) bad |= win_page[i + lane] < 0;
        return __ballot(bad) != 0;
    };

    // Wave w takes page w of each block: lane (key, part) reads KL x 16 dims of a key, lane (dim % 16, quad) KL x 16
    // bytes of the page's values.
    u32x4 kr[KL], vr[KL];
    float ksc, vsc, vsc_next;
    int kvalid, vvalid, page, vpage;        // keys of the page that the item has; pages of the keys' and the values' block
    const int krow = tid / 4, kpart = tid % 4;
    const int vquad = lane % 4, vlane = lane / 4;      // (16 lanes then write 128 contiguous bytes of LDS)
    auto keys_in = [&](int b, int pg) {
        return pg >= 0 ? max(0, min(kPage8, key1 - (key0 + b * St::KEYS + wave * kPage8))) : 0;
    };
    // the keys' page of block b, from the window: read, and in use
    int page_read;
    float2 scale_read;
    auto look_up = [&](int b) {
        const int i = min(key0 / kPage8 + 4 * b + wave, last) - w0;
        page_read = win_page[i];
        scale_read = win_scale[i];
    };
    auto use_page = [&]() {
        page = __builtin_amdgcn_readfirstlane(page_read);
        ksc = first_lane(scale_read.x);
        vsc_next = first_lane(scale_read.y);
    };
    // codes of block b's keys (its page looked up), and of the block's values whose keys were fetched before
    auto fetch_k = [&](int b) {
        kvalid = keys_in(b, page);
        const uint8_t *kp = a.p.k + ((size_t)max(page, 0) * a.p.nkv + g) * (kPage8 * HD) + (krow % kPage8) * HD + kpart * (HD / 4);
#pragma unroll
        for (int j = 0; j < KL; ++j) kr[j] = *(const u32x4 *)(kp + 16 * j);
    };
    auto fetch_v = [&](int b) {
        vvalid = keys_in(b, vpage);
        const uint8_t *vp = a.p.v + ((size_t)max(vpage, 0) * a.p.nkv + g) * (kPage8 * HD) + vquad * (4 * HD) + vlane * (HD / 4);
#pragma unroll
        for (int j = 0; j < KL; ++j) vr[j] = *(const u32x4 *)(vp + 16 * j);
    };
    auto next_v = [&]() {
        vpage = page;
        vsc = vsc_next;
    };

    // 16-byte chunk i of the thread's keys, word i of its values, as bf16 into buffer buf; what the item does not have
    // is zero (keep_k, keep_v, once the codes are here)
    float k_mul, v_mul;
    const int k_dst = krow * St::KRB + St::kchunk(krow, kpart * (KL * 2)) * 16;      // chunk i enters by exclusive or
    const int v_dst = St::KBYTES + wave * St::VPAGE + vlane * 32 + St::vchunk(vlane, vquad / 2) * 16 + (vquad % 2) * 8;
    auto put_k = [&](int buf, int i, const u32x4 (&r)[KL]) {
        const uint2 lo = word_bf16(r[i / 2][2 * (i % 2)], k_mul), hi = word_bf16(r[i / 2][2 * (i % 2) + 1], k_mul);
        *(u32x4 *)(smem + buf * St::BYTES + (k_dst ^ (i * 16))) = u32x4{lo.x, lo.y, hi.x, hi.y};
    };
    auto put_v = [&](int buf, int i, const u32x4 (&r)[KL]) {
        *(uint2 *)(smem + buf * St::BYTES + i * 512 + v_dst) = word_bf16(r[i / 4][i % 4], v_mul);       // dim 16 i + vlane
    };
    auto keep_k = [&](int valid, u32x4 (&r)[KL]) {
        if (valid == 0) {          // (wave-uniform, as the next)
#pragma unroll
            for (int j = 0; j < KL; ++j) r[j] = u32x4{0u, 0u, 0u, 0u};
        }
    };
    auto keep_v = [&](int valid, u32x4 (&r)[KL]) {
        if (valid < kPage8) {
            const int n = max(0, min(4, valid - 4 * vquad));
            const uint32_t keep = n == 4 ? 0xffffffffu : (1u << (8 * n)) - 1;
#pragma unroll
            for (int j = 0; j < KL; ++j) r[j] &= keep;
        }
    };
    auto scales = [&]() {
        k_mul = ksc;
        v_mul = vsc;
    };

    f32x16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[d][e] = 0.f;
    float m = -INFINITY, l = 0.f;

    // S^T = K Q^T: operand row r holds key r with bits 2 and 3 swapped, so that the eight weights a lane packs for
    // one page are its slots 8 half .. 8 half + 7
    const int kcol = col ^ ((((col >> 2) ^ (col >> 3)) & 1) * 12);
    const int k_at = kcol * St::KRB + St::kchunk(kcol, half) * 16;       // step k's chunk 2 k + half: k enters by exclusive or
    const int v_at = St::KBYTES + col * 32 + St::vchunk(col, half) * 16;
    // operand i of the scores (k = i / 2, keys 32 (i % 2) ..) and of the products (page i / DB, dims 32 (i % DB) ..)
    auto k_frag = [&](int buf, int i) { return *(const bf16x8 *)(smem + buf * St::BYTES + (i % 2) * (32 * St::KRB) + (k_at ^ (i / 2 * 32))); };
    auto v_frag = [&](int buf, int i) { return *(const bf16x8 *)(smem + buf * St::BYTES + (i / DB) * St::VPAGE + (i % DB) * 1024 + v_at); };
    // masks block b's scores, whose maximum is mx if none is masked, and raises the running maximum; bit p of `bad`:
    // page p is bad (its keys are masked, their codes were zeroed)
    float neg = 0.f;               // minus the maximum times the scale, or zero
    float neg_now = 0.f;           // what the step at hand adds
    auto raise = [&](int b, uint32_t bad, f32x16 (&s)[2], float mx) {
        const int base = key0 + b * St::KEYS;
        if (base + St::KEYS > first_pos || base + St::KEYS > key1 || bad) {
            mx = -INFINITY;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int k = 32 * j + (e >> 3) * 16 + half * 8 + ((e >> 2) & 1) * 4 + (e & 3);
                    if (base + k > pos || base + k >= key1 || (bad >> (k / kPage8) & 1)) s[j][e] = -INFINITY;
                    mx = fmaxf(mx, s[j][e]);
                }
        }
        const float2 p = partner32(mx);
        const float mloc = fmaxf(p.x, p.y);
        // the maximum (of scores before their scale) follows in jumps of more than 2^8, so that the sums are rarely rescaled
        if (__ballot((mloc - m) * a.scale > 8.f) != 0) {
            const float mn = fmaxf(m, mloc), alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - mn) * a.scale);
            l *= alpha;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[d][e] *= alpha;
            m = mn;
            neg = m == -INFINITY ? 0.f : -m * a.scale;
        }
        // What rounding `neg` left out stays in the fused exponents: nothing beside the scores' own errors, but weights out of
        // range where the exponents are large.  Then the difference is taken first.
        neg_now = neg;
        if (__ballot(fabsf(neg) > kLargeScore) != 0) {
            const float sub = m == -INFINITY ? 0.f : m;
            neg_now = 0.f;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[j][e] -= sub;
        }
    };
    auto bad_pages = [&](int b) {
        uint32_t bad = 0;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const int id = table[min(key0 / kPage8 + 4 * b + p, last)];
            if (id < 0 || id >= a.p.n_pages) bad |= 1u << p;
        }
        return (uint32_t)__builtin_amdgcn_readfirstlane(bad);
    };

    // The codes of the first keys and values start before their scales are known (their pages straight from the table), the
    // query rows behind them: everything is on its way after one read of the table.  (One by one as in the loop the first
    // scores were there 5 us after the start, now after 3.5; 4 fresh prompts of 400 to 623 tokens 26.5 -> 24.9 us.)
    const int ids = window_id();
    auto first_page = [&](int b) {
        const int id = table[min(key0 / kPage8 + 4 * b + wave, last)];
        return id >= 0 && id < a.p.n_pages ? id : -1;
    };
    const int first_pages[3] = {first_page(0), first_page(1), first_page(2)};
    u32x4 k0[KL], k1[KL], v0[KL];
    int k_valid[2], v_valid;
    auto keep = [&](u32x4 (&to)[KL], const u32x4 (&from)[KL]) {
#pragma unroll
        for (int j = 0; j < KL; ++j) to[j] = from[j];
    };
    page = vpage = first_pages[0];
    fetch_k(0);
    keep(k0, kr);
    k_valid[0] = kvalid;
    fetch_v(0);
    keep(v0, vr);
    v_valid = vvalid;
    page = vpage = first_pages[1];
    fetch_k(1);
    keep(k1, kr);
    k_valid[1] = kvalid;
    fetch_v(1);
    page = first_pages[2];
    fetch_k(2);
    __builtin_amdgcn_sched_barrier(0);
    load_window(ids);
    const T *qp = (const T *)a.q + (size_t)(row0 + tok) * a.q_stride + (size_t)h * HD;
    bf16x8 q[KS][R::NQ];
#pragma unroll
    for (int k = 0; k < KS; ++k) load_q<T, R::NQ>(qp + 16 * k + 8 * half, q[k]);
    lds_barrier();
    bool any_bad = window_bad();               // then each block's pages are looked at again

    // Block b's weights run beside block b + 1's scores, and its products beside the next codes' way into LDS (keys one
    // block ahead of values): the compiler keeps no such order by itself, so every product is a slot with its share of the
    // vector work, operands read three slots ahead, and nothing moves between slots.
    constexpr int NA = 2 * KS, NB = 4 * DB, AHEAD = 3, EA = 32 / NA, EB = 32 / NB;
    f32x16 sa[2], sb[2];
    float mx = -INFINITY;          // maximum of the scores at hand
    auto step = [&](int b, auto parity, f32x16 (&s)[2], f32x16 (&next)[2]) {
        constexpr int P = decltype(parity)::value;           // b % 2
        bf16x8 ring[AHEAD], pf[4][R::NP];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) ring[i] = k_frag(P ^ 1, i);
        raise(b, any_bad ? bad_pages(b) : 0, s, mx);
        // (no branch between the slots: the compiler would move their work past it)
        keep_v(vvalid, vr);
        keep_k(kvalid, kr);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) next[j][e] = 0.f;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NA; ++i) {
#pragma unroll
            for (int n = 0; n < R::NQ; ++n) next[i % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[i % AHEAD], q[i / 2][n], next[i % 2], 0, 0, 0);
            ring[i % AHEAD] = i + AHEAD < NA ? k_frag(P ^ 1, i + AHEAD) : v_frag(P, i + AHEAD - NA);
#pragma unroll
            for (int e = EA * i; e < EA * (i + 1); ++e) {
                s[e / 16][e % 16] = __builtin_amdgcn_exp2f(fmaf(s[e / 16][e % 16], a.scale, neg_now));
                if (R::NP > 1) l += s[e / 16][e % 16];
            }
            if ((EA * (i + 1)) % 8 == 0) {
                const int t = EA * (i + 1) / 8 - 1;          // page t of the block
                const float x[8] = {s[t / 2][8 * (t % 2)], s[t / 2][8 * (t % 2) + 1], s[t / 2][8 * (t % 2) + 2], s[t / 2][8 * (t % 2) + 3],
                                    s[t / 2][8 * (t % 2) + 4], s[t / 2][8 * (t % 2) + 5], s[t / 2][8 * (t % 2) + 6], s[t / 2][8 * (t % 2) + 7]};
                parts_of<R::NP>(x, pf[t]);
                if (R::NP == 1) {                            // the sum of the weights as they are used
                    const u32x4 w = __builtin_bit_cast(u32x4, pf[t][0]);
#pragma unroll
                    for (int k = 0; k < 4; ++k) l = add_pair(w[k], l);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        scales();
        next_v();
        mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < NB; ++i) {
#pragma unroll
            for (int n = 0; n < R::NP; ++n) acc[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[(NA + i) % AHEAD], pf[i / DB][n], acc[i % DB], 0, 0, 0);
            if (i + AHEAD < NB) ring[(NA + i) % AHEAD] = v_frag(P, i + AHEAD);
            // into the buffers that iteration b - 1 read; the registers take the next ones, most of a step ahead
            if (i < NB / 2) put_v(P ^ 1, i, vr);
            else if (i % 2 == 1) put_k(P, (i - NB / 2) / 2, kr);
            if (i == NB / 4) look_up(b + 3);
            if (i == NB / 2) fetch_v(b + 2);
            if (i == NB - 2) use_page();
#pragma unroll
            for (int e = EB * i; e < EB * (i + 1); ++e) mx = fmaxf(mx, next[e / 16][e % 16]);
            __builtin_amdgcn_sched_barrier(0);
        }
        fetch_k(b + 3);
        if (4 * (b + 4) + key0 / kPage8 - w0 >= kWindow && w0 + kWindow <= last) {
            lds_barrier();             // everyone has looked up block b + 3
            w0 += kWindow;
            load_window(window_id());
            lds_barrier();
            any_bad |= window_bad();
        }
        lds_barrier();
    };
    keep_k(k_valid[0], k0);
    keep_v(v_valid, v0);
    look_up(0);
    use_page();
    next_v();
    scales();
#pragma unroll
    for (int i = 0; i < 2 * KL; ++i) put_k(0, i, k0);
#pragma unroll
    for (int i = 0; i < 4 * KL; ++i) put_v(0, i, v0);
    keep_k(k_valid[1], k1);
    look_up(1);
    use_page();
    next_v();
    scales();
#pragma unroll
    for (int i = 0; i < 2 * KL; ++i) put_k(1, i, k1);
    look_up(2);
    use_page();
    lds_barrier();
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) sa[j][e] = 0.f;
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int n = 0; n < R::NQ; ++n) sa[i % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(0, i), q[i / 2][n], sa[i % 2], 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 32; ++e) mx = fmaxf(mx, sa[e / 16][e % 16]);
    lds_barrier();
    for (int b = 0; b < nkb; b += 2) {
        step(b, std::integral_constant<int, 0>{}, sa, sb);
        if (b + 1 < nkb) step(b + 1, std::integral_constant<int, 1>{}, sb, sa);
    }
    {
        const float2 p = partner32(l);
        l = p.x + p.y;
        if (l == 0.f && has_key(a, a.off_tiles + kItem8Ints * index, tok)) l = kNoWeights;
    }
    // sums that are not finite: from what the pair sees, or from zero weights times something that is not finite
    // in a masked place; told apart key by key
    bool odd = false;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) odd |= !(fabsf(acc[d][e]) < INFINITY);
    uint64_t oddb = __ballot(odd && c < cols && pos + 1 < key1);     // (a pair that sees every key has nothing masked)
    if (oddb) {
        const int last_odd = last_odd_value<HD>(a, a.off_tiles + kItem8Ints * index);
        oddb = __ballot(odd && c < cols && pos < last_odd);
    }
    const uint32_t odd_cols = (uint32_t)oddb | (uint32_t)(oddb >> 32);
    for (int k = 0; k < 32; ++k) {
        if (!(odd_cols >> k & 1)) continue;
        const int ck = wave * 32 + k, t = ck / a.p.group, hh = g * a.p.group + ck % a.p.group;
        float o[HD / 64], mm, ll;
        pair_key_by_key<T, HD>(a, seq, g, pos0 + t, key0, key1, (const T *)a.q + (size_t)(row0 + t) * a.q_stride + (size_t)hh * HD, mm, ll, o);
        float *pp = partial_of<HD>(a, max(slot, 0), ck);
        if (slot >= 0 && lane == 0) {
            pp[0] = mm;
            pp[1] = ll;
        }
#pragma unroll
        for (int d = 0; d < HD / 64; ++d) {
            if (slot >= 0) pp[kPartialPad + lane + 64 * d] = o[d];
            else ((T *)a.out)[(size_t)(row0 + t) * a.out_stride + (size_t)hh * HD + lane + 64 * d] = from_f32<T>(o[d] * inverse(ll));
        }
    }
    if (c < cols && !(odd_cols >> col & 1)) {
        if (slot >= 0) {
            float *pp = partial_of<HD>(a, slot, c);
            if (half == 0) {
                pp[0] = m * a.scale;
                pp[1] = l;
            }
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    *(f32x4 *)(pp + kPartialPad + d * 32 + k * 8 + half * 4) =
                        f32x4{acc[d][4 * k], acc[d][4 * k + 1], acc[d][4 * k + 2], acc[d][4 * k + 3]};
        } else {
            const float inv = inverse(l);
            T *dst = (T *)a.out + (size_t)(row0 + tok) * a.out_stride + (size_t)h * HD;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    store4(dst + d * 32 + k * 8 + half * 4, acc[d][4 * k] * inv, acc[d][4 * k + 1] * inv, acc[d][4 * k + 2] * inv,
                           acc[d][4 * k + 3] * inv);
        }
    }
}

// ------------------------------------------------------------------ launches
template <typename T, int HD, int NW>
__global__ __launch_bounds__(64 * NW, sizeof(T) == 2 ? 3 : 2) void attend8_small_kernel(Attend8 a) {
    extern __shared__ __attribute__((aligned(16))) char dyn[];
    small_item<T, HD, NW>(a, blockIdx.x, dyn);
}

template <int HD> constexpr int kTileLds = 2 * Stage8<HD>::BYTES + kWindow * 12;

// Tiles, and behind them the small items of a batch that has both: one launch after another left the chip to the tail
// of the first (2 x 512 rows after 7680 keys beside 14 rows of 2048: 163 us apart, 152 jointly; 64 rows after 512 keys
// beside 64 rows of 2048: 68 and 53; 256 rows of 4096 beside 4 fresh prompts of 512: 399 and 400).  Jointly a small item has four
// waves, also where apart it would have eight and the chip is mostly idle (64 fresh rows beside one of 4000 keys 22.4 us apart,
// 15.3 jointly; 2 x 100 beside 4 of 900 19.9 and 10.8; 12 small fp32 segments 24.5 and 16.3).
template <typename T, int HD, bool SMALL>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void attend8_tile_kernel(Attend8 a) {
    __shared__ __attribute__((aligned(16))) char smem[kTileLds<HD>];
    static_assert(small_lds<HD, 4>(kSmallCols) <= kTileLds<HD>, "a small item's sums");
    if (!SMALL || (int)blockIdx.x < a.n_tiles) tile_item<T, HD>(a, blockIdx.x, smem);
    else if constexpr (SMALL) small_item<T, HD, 4>(a, (int)blockIdx.x - a.n_tiles, smem);
}

template <typename T, int HD, int NW> void small_of(const Attend8 &a, hipStream_t s) {
    const int lds = small_lds<HD, NW>(a.small_cols);
    hipLaunchKernelGGL((attend8_small_kernel<T, HD, NW>), dim3(a.n_small), dim3(64 * NW), lds, s, a);
}
template <typename T, int HD> hipError_t attend_of(const Attend8 &a, hipStream_t s) {
    if (a.joint) {
        hipLaunchKernelGGL((attend8_tile_kernel<T, HD, true>), dim3(a.n_tiles + a.n_small), dim3(256), 0, s, a);
    } else {
        if (a.n_small > 0) {
            if (a.wide && a.small_cols <= 8) small_of<T, HD, 8>(a, s);      // (more pairs' sums would take over 64 KB of LDS)
            else small_of<T, HD, 4>(a, s);
        }
        if (a.n_tiles > 0) hipLaunchKernelGGL((attend8_tile_kernel<T, HD, false>), dim3(a.n_tiles), dim3(256), 0, s, a);
    }
    if (a.n_merge > 0) hipLaunchKernelGGL((attend8_merge_kernel<T, HD>), dim3(a.n_merge, a.merge_slots), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attend8(const Attend8 &a, hipStream_t s) {
    if (a.dtype == ORTHRUS_BF16) return a.p.hd == 64 ? attend_of<bf16, 64>(a, s) : attend_of<bf16, 128>(a, s);
    return a.p.hd == 64 ? attend_of<float, 64>(a, s) : attend_of<float, 128>(a, s);
}

}  // namespace orthrus
