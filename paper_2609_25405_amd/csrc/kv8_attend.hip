// Causal attention of ragged rows over the 8-bit paged cache.
//
// Both kernels turn codes into bf16 by v_cvt_scalef32_pk_bf16_fp8 (two codes an instruction, exact) and
// multiply on bf16 MFMA, with an online softmax in fp32 (exp2 domain).  fp32 rows go through the
// same products in parts: q as three bf16 parts (exact), the weights as two (16 bits), each part a
// product of its own into the same sums.
//
// Small items ((rows, query heads of one KV head) pairs of a segment, at most 16): the pairs are the 16 columns
// of a 16x16x32 MFMA, so all query heads and rows that share a key read it once, and the arithmetic
// hides behind the cache's bytes.  A wave walks steps of 64 keys (4 pages): a page's keys are one
// 2-KB run (head_dim 128) of which lane (quarter, key) reads the quarter's dims; the scores then lie
// with lane (quarter, column) holding keys 4 quarter .. + 3 of each page, which is also how the
// cache lays out its values (slot / 4 outermost), so weights feed the second product without
// moving between lanes.
//
// Tiles (128 pairs of a longer segment): four waves of 32 pairs; 64-key blocks are turned into bf16 once
// per workgroup on their way into LDS (two buffers, the next block's codes in flight in registers).
//
// Long key ranges come as pieces that leave (max, sum, unnormalised output) to a merge launch.
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

template <typename T> struct Rows8;
template <> struct Rows8<bf16> { static constexpr int NQ = 1, NP = 1; };
template <> struct Rows8<float> { static constexpr int NQ = 3, NP = 2; };

__device__ __forceinline__ void store4(float *p, float a, float b, float c, float d) { *(float4 *)p = float4{a, b, c, d}; }
__device__ __forceinline__ void store4(bf16 *p, float a, float b, float c, float d) {
    *(uint2 *)p = uint2{pack_bf16x2(a, b), pack_bf16x2(c, d)};
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
#pragma unroll
    for (int d = 0; d < N; ++d) {
        q[d] = to_f32(qp[lane + 64 * d]);
        o[d] = 0.f;
    }
    for (int key = key0; key < min(key1, pos + 1); ++key) {
        const int page = table[key / kPage8], slot = key % kPage8;
        if (page < 0 || page >= a.p.n_pages) continue;
        const size_t at = (size_t)page * a.p.nkv + head;
        const uint8_t *kp = a.p.k + at * (kPage8 * HD) + slot * HD, *vp = a.p.v + at * (kPage8 * HD) + (slot / 4) * (4 * HD) + slot % 4;
        float s = 0.f;
#pragma unroll
        for (int d = 0; d < N; ++d) s = fmaf(q[d], bf16_lo(codes_bf16<false>(kp[lane + 64 * d], 1.f)), s);
        s = wave_sum(s) * (a.scale * a.p.ks[at]);
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
    l_out = l;
}

// ------------------------------------------------------------------ small items
template <typename T, int HD, int NW>
__global__ __launch_bounds__(64 * NW) void attend8_small_kernel(Attend8 a) {
    using R = Rows8<T>;
    constexpr int QD = HD / 4, KK = HD / 32, DB = HD / 16, STEP = 64, PG = 4;
    constexpr int LD = HD + 4;
    __shared__ float sm[NW][16], sl[NW][16];
    __shared__ __attribute__((aligned(16))) float so[NW][16][LD];
    if (stale8(a.p)) return;
    const int32_t *it = a.p.meta + a.off_small + kItem8Ints * (int)blockIdx.x;
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
    int valid[PG];
    auto pages_of = [&](int st, int (&pg)[PG]) {
#pragma unroll
        for (int p = 0; p < PG; ++p) pg[p] = table[min(key0 / kPage8 + st * PG + p, last)];
    };
    // keys of the step's pages that the item has; bad and absent pages have none and read page 0
    auto check = [&](int st, int (&pg)[PG]) {
#pragma unroll
        for (int p = 0; p < PG; ++p) {
            const int k = key0 + st * STEP + p * kPage8;
            const bool ok = pg[p] >= 0 && pg[p] < a.p.n_pages;
            valid[p] = ok ? max(0, min(kPage8, key1 - k)) : 0;
            if (!ok && k < key1 && lane == 0) flag_error(a.p.err, ORTHRUS_DEVERR_PAGE);
            pg[p] = ok ? pg[p] : 0;
        }
    };
    auto load = [&](const uint8_t *pool, const float *scales, const int (&pg)[PG], u32x4 (&r)[PG][QD / 16], float (&s)[PG], int at) {
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

    for (int st = wave; st < steps; st += NW) {
        int pg[PG];
        pages_of(st, pg);
        check(st, pg);
        load(a.p.k, a.p.ks, pg, kr, ks, k_at);
        load(a.p.v, a.p.vs, pg, vr, vs, v_at);
        f32x4 s[PG];
#pragma unroll
        for (int p = 0; p < PG; ++p) {
            s[p] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KK; ++k) {
                const bf16x8 kf = as_bf16x8(word_bf16(kr[p][k / 2][2 * (k % 2)], 1.f), word_bf16(kr[p][k / 2][2 * (k % 2) + 1], 1.f));
#pragma unroll
                for (int n = 0; n < R::NQ; ++n) s[p] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[k][n], s[p], 0, 0, 0);
            }
        }
        const int kbase = key0 + st * STEP;
        float mloc = -INFINITY;
#pragma unroll
        for (int p = 0; p < PG; ++p) {
            const float f = ks[p] * a.scale;
            const int seen = min(valid[p], pos + 1 - kbase - p * kPage8);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[p][r] = 4 * qd + r < seen ? s[p][r] * f : -INFINITY;
                mloc = fmaxf(mloc, s[p][r]);
            }
            vs[p] = valid[p] > 0 ? vs[p] : 0.f;
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
                const float e = __builtin_amdgcn_exp2f(s[p][r] - sub);
                l += e;
                w[p][r] = e * vs[p];
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
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const bf16x8 vf = as_bf16x8(word_bf16(vr[p][d / 4][d % 4], 1.f), word_bf16(vr[p + 1][d / 4][d % 4], 1.f));
#pragma unroll
                for (int n = 0; n < R::NP; ++n) acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[n], acc[d], 0, 0, 0);
            }
        }
    }
    l = quarters_sum(l);
    if (qd == 0) {
        sm[wave][c] = m;
        sl[wave][c] = l;
    }
#pragma unroll
    for (int d = 0; d < DB; ++d) *(f32x4 *)&so[wave][c][16 * d + 4 * qd] = acc[d];
    __syncthreads();
    // merge the waves in order; four dims a thread
    for (int o = tid; o < cols * (HD / 4); o += 64 * NW) {
        const int col = o / (HD / 4), d = o % (HD / 4) * 4;
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) M = fmaxf(M, sm[w][col]);
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float f = sm[w][col] == -INFINITY ? (sl[w][col] == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(sm[w][col] - M);
            L += sl[w][col] * f;
            sum += *(const f32x4 *)&so[w][col][d] * f;
        }
        if (slot >= 0) {
            float *pp = a.partials + ((size_t)slot * 16 + col) * (HD + 2);
            if (d == 0) {
                pp[0] = M;
                pp[1] = L;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) pp[2 + d + e] = sum[e];
        } else {
            const float inv = L != 0.f ? 1.f / L : 0.f;
            T *dst = (T *)a.out + (size_t)(row0 + col / a.p.group) * a.out_stride + (size_t)(g * a.p.group + col % a.p.group) * HD + d;
            store4(dst, sum[0] * inv, sum[1] * inv, sum[2] * inv, sum[3] * inv);
        }
    }
    // pairs of an earlier row of several: a later row's key or value that is not finite is masked, not absent
    if (len == 1) return;
    __syncthreads();       // after the stores above, which it may replace
    for (int col = wave; col < cols; col += NW) {
        float L = 0.f;
        bool bad = false;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            L += sl[w][col];
            for (int d = lane; d < HD; d += 64) bad |= !(fabsf(so[w][col][d]) < INFINITY);
        }
        if (__ballot(bad) == 0) continue;
        const int t = col / a.p.group, hh = g * a.p.group + col % a.p.group;
        float o[HD / 64], mm, ll;
        pair_key_by_key<T, HD>(a, seq, g, pos0 + t, key0, key1, (const T *)a.q + (size_t)(row0 + t) * a.q_stride + (size_t)hh * HD, mm, ll, o);
        float *pp = a.partials + ((size_t)max(slot, 0) * 16 + col) * (HD + 2);
        if (slot >= 0 && lane == 0) {
            pp[0] = mm;
            pp[1] = ll;
        }
#pragma unroll
        for (int d = 0; d < HD / 64; ++d) {
            if (slot >= 0) pp[2 + lane + 64 * d] = o[d];
            else ((T *)a.out)[(size_t)(row0 + t) * a.out_stride + (size_t)hh * HD + lane + 64 * d] = from_f32<T>(ll != 0.f ? o[d] / ll : 0.f);
        }
    }
}

// ------------------------------------------------------------------ tiles of longer segments
template <int HD> struct Stage8 {
    static constexpr int KEYS = 64, KRB = HD * 2, KCH = KRB / 16;
    static constexpr int KBYTES = KEYS * KRB, VPAGE = HD * kPage8 * 2, BYTES = KBYTES + 4 * VPAGE;
    // physical 16-byte chunk of chunk c of key row r, and of half c (8 slots) of a value dim: lanes that
    // read one chunk of consecutive rows reach different banks
    static __device__ __forceinline__ int kchunk(int r, int c) { return c ^ ((r / (256 / KRB)) % KCH); }
    static __device__ __forceinline__ int vchunk(int d, int c) { return c ^ ((d >> 3) & 1); }
};

template <typename T, int HD>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void attend8_tile_kernel(Attend8 a) {
    using R = Rows8<T>;
    using St = Stage8<HD>;
    constexpr int KS = HD / 16, DB = HD / 32;
    constexpr int KL = HD / 64;              // 16-byte loads of codes a thread and block, keys and values each
    __shared__ __attribute__((aligned(16))) char smem[2 * St::BYTES];
    if (stale8(a.p)) return;
    const int32_t *it = a.p.meta + a.off_tiles + kItem8Ints * (int)blockIdx.x;
    const int seq = it[A8_SEQ], row0 = it[A8_ROW], len = it[A8_LEN], pos0 = it[A8_POS], g = it[A8_HEAD];
    const int key0 = it[A8_KEY0], key1 = it[A8_KEY1], slot = it[A8_SLOT];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int cols = len * a.p.group;
    const int c = wave * 32 + col, cc = min(c, cols - 1);
    const int tok = cc / a.p.group, h = g * a.p.group + cc % a.p.group;
    const int pos = pos0 + tok;
    const bool idle = wave * 32 >= cols;                                     // no pairs for this wave
    const int first_pos = pos0 + min(wave * 32, cols - 1) / a.p.group, last_pos = pos0 + min(wave * 32 + 31, cols - 1) / a.p.group;
    const int32_t *table = a.p.table + (size_t)seq * a.p.max_blocks;
    const int nkb = (key1 - key0 + St::KEYS - 1) / St::KEYS, last = (key1 - 1) / kPage8;

    const T *qp = (const T *)a.q + (size_t)(row0 + tok) * a.q_stride + (size_t)h * HD;
    bf16x8 q[KS][R::NQ];
#pragma unroll
    for (int k = 0; k < KS; ++k) load_q<T, R::NQ>(qp + 16 * k + 8 * half, q[k]);

    // a block's codes: thread (key, part) reads KL x 16 dims of a key; thread (page, quad, 4 lanes of dims) KL x 16
    // bytes of a page's values
    u32x4 kr[KL], vr[KL];
    float ksc, vsc;
    int kvalid, vvalid;
    const int krow = tid / 4, kpart = tid % 4;
    const int vpage = tid / 64, vquad = (tid / 16) % 4, vlane = tid % 16;
    auto fetch = [&](int b) {
        const int base = key0 + b * St::KEYS;
        auto page_of = [&](int p, bool &ok) {
            const int pg = table[min(base / kPage8 + p, last)];
            ok = pg >= 0 && pg < a.p.n_pages;
            if (!ok && base + p * kPage8 < key1 && (tid & 15) == 0) flag_error(a.p.err, ORTHRUS_DEVERR_PAGE);
            return ok ? pg : 0;
        };
        bool ok;
        size_t head = (size_t)page_of(krow / kPage8, ok) * a.p.nkv + g;
        kvalid = ok ? 1 : 0;
        ksc = a.p.ks[head];
#pragma unroll
        for (int j = 0; j < KL; ++j) kr[j] = *(const u32x4 *)(a.p.k + head * (kPage8 * HD) + (krow % kPage8) * HD + kpart * (HD / 4) + 16 * j);
        head = (size_t)page_of(vpage, ok) * a.p.nkv + g;
        vvalid = ok ? max(0, min(4, key1 - base - vpage * kPage8 - 4 * vquad)) : 0;
        vsc = a.p.vs[head];
#pragma unroll
        for (int j = 0; j < KL; ++j) vr[j] = *(const u32x4 *)(a.p.v + head * (kPage8 * HD) + vquad * (4 * HD) + vlane * (HD / 4) + 16 * j);
    };
    // as bf16 into buffer buf; what the item does not have is zero
    auto put = [&](int buf) {
        char *kl = smem + buf * St::BYTES, *vl = kl + St::KBYTES;
#pragma unroll
        for (int j = 0; j < KL; ++j) {
            if (!kvalid) kr[j] = u32x4{0u, 0u, 0u, 0u};
            const float s = kvalid ? ksc : 1.f;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint2 lo = word_bf16(kr[j][2 * e], s), hi = word_bf16(kr[j][2 * e + 1], s);
                const int ch = kpart * (KL * 2) + 2 * j + e;
                *(u32x4 *)(kl + krow * St::KRB + St::kchunk(krow, ch) * 16) = u32x4{lo.x, lo.y, hi.x, hi.y};
            }
        }
        const uint32_t keep = vvalid == 4 ? 0xffffffffu : (1u << (8 * vvalid)) - 1;
        const float s = vvalid > 0 ? vsc : 1.f;
#pragma unroll
        for (int j = 0; j < KL; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int dim = 16 * (4 * j + e) + vlane;
                *(uint2 *)(vl + vpage * St::VPAGE + dim * 32 + St::vchunk(dim, vquad / 2) * 16 + (vquad % 2) * 8) =
                    word_bf16(vr[j][e] & keep, s);
            }
    };

    f32x16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[d][e] = 0.f;
    float m = -INFINITY, l = 0.f;

    // bit p: page p of the block is bad (its keys are masked; their codes were zeroed)
    auto compute = [&](int b, uint32_t bad) {
        const int base = key0 + b * St::KEYS;
        if (idle || base > last_pos) return;
        const char *kl = smem + (b & 1) * St::BYTES, *vl = kl + St::KBYTES;
        // S^T = K Q^T; operand row r holds key r with bits 2 and 3 swapped, so that the eight weights a lane
        // packs for one page are its slots 8 half .. 8 half + 7
        f32x16 s[2];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[j][e] = 0.f;
        const int kcol = col ^ ((((col >> 2) ^ (col >> 3)) & 1) * 12);
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int row = 32 * j + kcol;
                const bf16x8 kf = *(const bf16x8 *)(kl + row * St::KRB + St::kchunk(row, 2 * k + half) * 16);
#pragma unroll
                for (int n = 0; n < R::NQ; ++n) s[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[k][n], s[j], 0, 0, 0);
            }
        if (base + St::KEYS > first_pos || base + St::KEYS > key1 || bad) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int k = 32 * j + (e >> 3) * 16 + half * 8 + ((e >> 2) & 1) * 4 + (e & 3);
                    if (base + k > pos || base + k >= key1 || (bad >> (k / kPage8) & 1)) s[j][e] = -INFINITY;
                }
        }
        float mloc = s[0][0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mloc = fmaxf(mloc, s[0][e]);
#pragma unroll
        for (int e = 0; e < 16; ++e) mloc = fmaxf(mloc, s[1][e]);
        {
            const float2 p = partner32(mloc);
            mloc = fmaxf(p.x, p.y) * a.scale;
        }
        if (__ballot(mloc > m + 8.f) != 0) {
            const float mn = fmaxf(m, mloc), alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
            l *= alpha;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[d][e] *= alpha;
            m = mn;
        }
        const float neg = m == -INFINITY ? 0.f : -m;
        bf16x8 pf[2][2][R::NP];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int k2 = 0; k2 < 2; ++k2) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] = __builtin_amdgcn_exp2f(fmaf(s[j][8 * k2 + e], a.scale, neg));
                    l += x[e];
                }
                parts_of<R::NP>(x, pf[j][k2]);
            }
        // O^T[dim][pair] += V^T P^T
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const int dim = d * 32 + col;
                    const bf16x8 vf = *(const bf16x8 *)(vl + (2 * j + k2) * St::VPAGE + dim * 32 + St::vchunk(dim, half) * 16);
#pragma unroll
                    for (int n = 0; n < R::NP; ++n) acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[j][k2][n], acc[d], 0, 0, 0);
                }
    };
    auto bad_pages = [&](int b) {
        uint32_t bad = 0;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const int pg = table[min(key0 / kPage8 + 4 * b + p, last)];
            if (pg < 0 || pg >= a.p.n_pages) bad |= 1u << p;
        }
        return (uint32_t)__builtin_amdgcn_readfirstlane(bad);
    };

    fetch(0);
    put(0);
    for (int b = 0; b < nkb; ++b) {
        __syncthreads();       // block b is whole; everyone is done with block b - 1, whose buffer b + 1 takes
        if (b + 1 < nkb) fetch(b + 1);
        compute(b, bad_pages(b));
        if (b + 1 < nkb) put((b + 1) & 1);
    }
    {
        const float2 p = partner32(l);
        l = p.x + p.y;
    }
    // sums that are not finite: from what the pair sees, or from zero weights times something that is not finite
    // in a masked place; told apart key by key
    bool odd = false;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) odd |= !(fabsf(acc[d][e]) < INFINITY);
    const uint64_t oddb = __ballot(odd && c < cols);
    const uint32_t odd_cols = (uint32_t)oddb | (uint32_t)(oddb >> 32);
    for (int k = 0; k < 32; ++k) {
        if (!(odd_cols >> k & 1)) continue;
        const int ck = wave * 32 + k, t = ck / a.p.group, hh = g * a.p.group + ck % a.p.group;
        float o[HD / 64], mm, ll;
        pair_key_by_key<T, HD>(a, seq, g, pos0 + t, key0, key1, (const T *)a.q + (size_t)(row0 + t) * a.q_stride + (size_t)hh * HD, mm, ll, o);
        float *pp = a.partials + ((size_t)max(slot, 0) * 16 + ck) * (HD + 2);
        if (slot >= 0 && lane == 0) {
            pp[0] = mm;
            pp[1] = ll;
        }
#pragma unroll
        for (int d = 0; d < HD / 64; ++d) {
            if (slot >= 0) pp[2 + lane + 64 * d] = o[d];
            else ((T *)a.out)[(size_t)(row0 + t) * a.out_stride + (size_t)hh * HD + lane + 64 * d] = from_f32<T>(ll != 0.f ? o[d] / ll : 0.f);
        }
    }
    if (c >= cols || (odd_cols >> col & 1)) return;
    if (slot >= 0) {
        float *pp = a.partials + ((size_t)slot * 16 + c) * (HD + 2);
        if (half == 0) {
            pp[0] = m;
            pp[1] = l;
        }
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float2 *dst = (float2 *)(pp + 2 + d * 32 + k * 8 + half * 4);
                dst[0] = float2{acc[d][4 * k], acc[d][4 * k + 1]};
                dst[1] = float2{acc[d][4 * k + 2], acc[d][4 * k + 3]};
            }
        return;
    }
    const float inv = l != 0.f ? 1.f / l : 0.f;
    T *dst = (T *)a.out + (size_t)(row0 + tok) * a.out_stride + (size_t)h * HD;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            store4(dst + d * 32 + k * 8 + half * 4, acc[d][4 * k] * inv, acc[d][4 * k + 1] * inv, acc[d][4 * k + 2] * inv,
                   acc[d][4 * k + 3] * inv);
}

// ------------------------------------------------------------------ merge of pieces, in their order
// blockIdx.x: merge entry, blockIdx.y: eight of its (row, head) pairs, 32 lanes each
template <typename T, int HD> __global__ __launch_bounds__(256) void attend8_merge_kernel(Attend8 a) {
    constexpr int N = HD / 32;
    if (stale8(a.p)) return;
    const int32_t *me = a.p.meta + a.off_merge + kMerge8Ints * (int)blockIdx.x;
    const int col = blockIdx.y * 8 + threadIdx.x / 32, d0 = threadIdx.x % 32 * N;
    if (col >= me[M8_LEN] * a.p.group) return;
    const int n = me[M8_PIECES];
    const float *pp = a.partials + ((size_t)me[M8_SLOT] * 16 + col) * (HD + 2);
    const size_t step = (size_t)me[M8_SLOTS] * 16 * (HD + 2);
    float M = -INFINITY, L = 0.f, o[N];
    for (int i = 0; i < n; ++i) M = fmaxf(M, pp[i * step]);
#pragma unroll
    for (int d = 0; d < N; ++d) o[d] = 0.f;
    for (int i = 0; i < n; ++i) {
        const float *p = pp + i * step;
        // (a piece whose every score was not a number has a sum but no maximum)
        const float f = p[0] == -INFINITY ? (p[1] == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(p[0] - M);
        L += p[1] * f;
#pragma unroll
        for (int d = 0; d < N; ++d) o[d] += p[2 + d0 + d] * f;
    }
    const float inv = L != 0.f ? 1.f / L : 0.f;
    const int row = me[M8_ROW] + col / a.p.group, h = me[M8_HEAD] * a.p.group + col % a.p.group;
    T *dst = (T *)a.out + (size_t)row * a.out_stride + (size_t)h * HD + d0;
#pragma unroll
    for (int d = 0; d < N; ++d) dst[d] = from_f32<T>(o[d] * inv);
}

template <typename T, int HD> hipError_t attend_of(const Attend8 &a, hipStream_t s) {
    if (a.n_small > 0) hipLaunchKernelGGL((attend8_small_kernel<T, HD, 4>), dim3(a.n_small), dim3(256), 0, s, a);
    if (a.n_tiles > 0) hipLaunchKernelGGL((attend8_tile_kernel<T, HD>), dim3(a.n_tiles), dim3(256), 0, s, a);
    if (a.n_merge > 0)
        hipLaunchKernelGGL((attend8_merge_kernel<T, HD>), dim3(a.n_merge, (a.most_merge_cols + 7) / 8), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attend8(const Attend8 &a, hipStream_t s) {
    if (a.dtype == ORTHRUS_BF16) return a.p.hd == 64 ? attend_of<bf16, 64>(a, s) : attend_of<bf16, 128>(a, s);
    return a.p.hd == 64 ? attend_of<float, 64>(a, s) : attend_of<float, 128>(a, s);
}

}  // namespace orthrus
