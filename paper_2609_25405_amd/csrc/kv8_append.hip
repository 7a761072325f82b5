// Head norms, rotation and append into the 8-bit cache, and the read-back of what it holds.
//
// One workgroup serves one append unit (the tokens of one segment that share a page) and one KV
// head: that head's keys and values, and the query heads that read it.  A page's scale needs the
// largest magnitude of all its tokens, and here they are all in one workgroup: keys and values go
// from their rows to codes in registers, and only the values' tile, whose layout crosses tokens,
// passes through LDS.
//
// A head row of HD dims lies over HD / 16 lanes; lane i holds dims 8 i .. 8 i + 7 and HD / 2 + 8 i ..
// + 7, two 16-byte loads of bf16, so that the pairs (i, i + HD / 2) of a head that turns whole, and
// the pairs (2 i, 2 i + 1), are in one lane; pairs of a head that turns in part meet through LDS.
//
// Bound by the rows' bytes: 8.8 k bf16 rows of 32 + 2 x 8 heads of 128 dims in 42 us, 4.7 TB/s of 110 MB read and 90
// written; 256 decode rows with norms in 6.8 us, one round of waves that wait for two dependent reads.  The read-back of the
// same rows takes 13.0 and 5.0 us (18 MB in, 36 out).
#include <type_traits>

#include "kv8.hpp"

namespace orthrus {
namespace {

template <int CTRL> __device__ __forceinline__ float dpp(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
// over the LPR = 4 or 8 lanes of a head row (quad permutations, then the mirror of 8 lanes)
template <int LPR> __device__ __forceinline__ float row_sum(float v) {
    v += dpp<0xB1>(v);
    v += dpp<0x4E>(v);
    if (LPR == 8) v += dpp<0x141>(v);
    return v;
}
template <int LPR> __device__ __forceinline__ float row_max(float v) {
    v = fmaxf(v, dpp<0xB1>(v));
    v = fmaxf(v, dpp<0x4E>(v));
    if (LPR == 8) v = fmaxf(v, dpp<0x141>(v));
    return v;
}

// Magnitudes from here on would round to 2^128 (248 * 2^120, half-way between two codes under the largest scale): not a number
// as infinities are, so that every held value is finite in fp32 and bfloat16.
constexpr float kPastRange = 0x1.fp127f;

// the least power of two s with amax <= 448 s = 1.75 * 2^8 s, from amax's exponent and mantissa
__device__ __forceinline__ float scale_of(float amax) {
    const uint32_t b = __float_as_uint(amax);
    int e = (int)(b >> 23) - 127 - 8;
    if ((b & 0x7fffffu) > 0x600000u) ++e;
    return __uint_as_float((uint32_t)(max(e, kLeastExp8) + 127) << 23);
}

template <typename T> __device__ __forceinline__ void load8(const T *p, float (&x)[8]);
template <> __device__ __forceinline__ void load8<float>(const float *p, float (&x)[8]) {
    const float4 a = *(const float4 *)p, b = *(const float4 *)(p + 4);
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
template <> __device__ __forceinline__ void load8<bf16>(const bf16 *p, float (&x)[8]) {
    const u32x4 w = *(const u32x4 *)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = bf16_lo(w[i]);
        x[2 * i + 1] = bf16_hi(w[i]);
    }
}
__device__ __forceinline__ void store8(float *p, const float (&x)[8]) {
    *(float4 *)p = float4{x[0], x[1], x[2], x[3]};
    *(float4 *)(p + 4) = float4{x[4], x[5], x[6], x[7]};
}
__device__ __forceinline__ void store8(bf16 *p, const float (&x)[8]) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
    *(u32x4 *)p = w;
}

// e4m3 codes of four values, rounded to nearest even; |x| <= 448 by the choice of the scale, what is
// not finite becomes not a number
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// the codes of a word times `ratio`, rounded again
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float ratio) {
    const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return encode4(lo[0] * ratio, lo[1] * ratio, hi[0] * ratio, hi[1] * ratio);
}

// NT threads serve units of up to N tokens
template <typename TI, typename TO, int HD, int NT, int N>
__global__ __launch_bounds__(NT) void append8_kernel(Append8 a) {
    constexpr int LPR = HD / 16;             // lanes of a head row
    constexpr int GROUPS = NT / LPR;         // head rows in flight
    constexpr int DB = HD / 16;
    static_assert(GROUPS >= 2 * N, "keys and values of a unit in one round");
    __shared__ float2 turn[N][HD / 2];                 // (cos, sin) of each token and pair
    __shared__ float amax[2][N];
    __shared__ __attribute__((aligned(16))) uint8_t tile[kPage8 * HD];
    extern __shared__ __attribute__((aligned(16))) float swap[];       // [GROUPS][HD + 4], where half the pairs meet through it
    const int tid = threadIdx.x, g = blockIdx.x % a.p.nkv;
    Entry8<kUnit8Ints> entry;
    if (!entry8(a.p, kUnitsInt + kUnit8Ints * (int)(blockIdx.x / a.p.nkv), entry)) return;
    const int32_t *u = entry.v;
    const int seq = u[U8_SEQ], block = u[U8_BLOCK], first = u[U8_FIRST], n = u[U8_LEN], row0 = u[U8_ROW];
    const int page = a.p.table[(size_t)seq * a.p.max_blocks + block];
    const bool ok = page >= 0 && page < a.p.n_pages;
    if (!ok && tid == 0) flag_error(a.p.err, ORTHRUS_DEVERR_PAGE);

    // a thread's pair, the same for each of its tokens; its turns are read ahead of the rows, for which loads return in order
    constexpr int PAIRS = HD / 2;
    const int half = a.rot / 2, pair = tid % PAIRS;
    const double rate = ((const double *)(a.p.meta + kTurnsInt))[min(pair, max(half - 1, 0))];
    const int grp = tid / LPR, i = tid % LPR;
    // head row `h` of token t: this lane's 16 dims (x[0]: 8 i .., x[1]: HD / 2 + 8 i ..)
    auto load_row = [&](int t, int h, float (&x)[2][8]) {
        const TI *src = (const TI *)a.qkv + (size_t)(row0 + t) * a.stride + (size_t)h * HD + 8 * i;
        load8(src, x[0]);
        load8(src + HD / 2, x[1]);
        if constexpr (std::is_same<TI, float>::value) {
            if (a.slab) {                      // a projection in two parts: their sum
                float y[2][8];
                load8(src + a.slab, y[0]);
                load8(src + a.slab + HD / 2, y[1]);
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[c][j] += y[c][j];
            }
        }
    };
    // keys and values: group t holds token t's key, group N + t its value; on their way while the angles are taken
    const int which = grp / N, t = grp % N;      // 0 key, 1 value
    const bool live = which < 2 && t < n;
    float x[2][8];
    if (live) load_row(t, a.p.nq + which * a.p.nkv + g, x);
    // so are the first round's query heads
    const int rows = n * a.p.group;
    float xq[2][8];
    if (grp < rows) load_row(grp / a.p.group, g * a.p.group + grp % a.p.group, xq);
    // and what a page that was begun before holds: its scales, and the values' words that new ones go into.  The values'
    // tile is served by fours of slots, a wave one (or, one wave of few tokens, the two that these can touch).
    constexpr int W = HD / 64, QUADS = NT == 64 ? 2 : 1;       // words a lane
    const size_t head = (size_t)(ok ? page : 0) * a.p.nkv + g;
    uint8_t *kp = a.p.k + head * (kPage8 * HD), *vp = a.p.v + head * (kPage8 * HD);
    const int lane = tid % 64, wave = tid / 64;
    auto quad_of = [&](int k) { return NT == 64 ? first / 4 + k : wave; };
    auto words_of = [&](int q) { return (uint32_t *)(vp + q * (4 * HD)) + W * lane; };
    float was[2] = {0.f, 0.f};
    uint32_t old[QUADS][W] = {};
    if (first > 0) {
        was[0] = a.p.ks[head];
        was[1] = a.p.vs[head];
    }
#pragma unroll
    for (int k = 0; k < QUADS; ++k) {
        const int q = quad_of(k), lo = first - 4 * q, hi = first + n - 4 * q;      // new slots of the four, before clamping
        if (q < 4 && lo < 4 && hi > 0 && (lo > 0 || hi < 4)) {
#pragma unroll
            for (int j = 0; j < W; ++j) old[k][j] = words_of(q)[j];
        }
    }

    for (int tk = tid / PAIRS; tk < n; tk += NT / PAIRS) {
        if (pair >= half) break;
        // turns modulo one in double: far positions keep their angle
        const double c = (double)(block * kPage8 + first + tk) * rate;
        const double r = 2.0 * (c - rint(c));
        const float f = (float)r, rest = (float)(r - (double)f) * (float)M_PI;     // what fp32 leaves of the angle
        float sn, cs;
        sincospif(f, &sn, &cs);
        turn[tk][pair] = float2{fmaf(-sn, rest, cs) * a.magnitude, fmaf(cs, rest, sn) * a.magnitude};
    }
    __syncthreads();

    // norm and turn of a head row
    auto head_row = [&](int t, const float *gain, bool turns, float (&x)[2][8]) {
        if (gain) {
            float ss = 0.f;
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) ss = fmaf(x[c][j], x[c][j], ss);
            const float inv = 1.0f / sqrtf(row_sum<LPR>(ss) / (float)HD + a.eps);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float gv[8];
                load8(gain + c * (HD / 2) + 8 * i, gv);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[c][j] = x[c][j] * inv * gv[j];
            }
        }
        if (!turns || half == 0) return;
        if (a.interleaved) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int d = c * (HD / 2) + 8 * i;
                if (d < a.rot) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 cs = turn[t][d / 2 + j];
                        const float p = x[c][2 * j], q = x[c][2 * j + 1];
                        x[c][2 * j] = p * cs.x - q * cs.y;
                        x[c][2 * j + 1] = q * cs.x + p * cs.y;
                    }
                }
            }
        } else if (a.rot == HD) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float2 cs = turn[t][8 * i + j];
                const float p = x[0][j], q = x[1][j];
                x[0][j] = p * cs.x - q * cs.y;
                x[1][j] = q * cs.x + p * cs.y;
            }
        } else {
            // pairs (d, d + rot / 2): the partner's eight dims from another lane of the row
            float *mine = swap + grp * (HD + 4);
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            store8(mine + 8 * i, x[0]);
            store8(mine + HD / 2 + 8 * i, x[1]);
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int d = c * (HD / 2) + 8 * i;
                if (d < a.rot) {
                    const bool low = d < half;
                    const int pr = low ? d : d - half;
                    float other[8];
                    load8((const float *)mine + (low ? d + half : d - half), other);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float2 cs = turn[t][pr + j];
                        x[c][j] = low ? x[c][j] * cs.x - other[j] * cs.y : x[c][j] * cs.x + other[j] * cs.y;
                    }
                }
            }
        }
    };

    if (live) {
        head_row(t, which == 0 ? a.k_gain : nullptr, which == 0, x);
        float m = 0.f;
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float v = fabsf(x[c][j]);
                if (v < kPastRange) m = fmaxf(m, v);
                else x[c][j] = NAN;
            }
        m = row_max<LPR>(m);
        if (i == 0) amax[which][t] = m;
    }
    __syncthreads();
    float scale[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        float m = 0.f;
        for (int s = 0; s < n; ++s) m = fmaxf(m, amax[w][s]);
        scale[w] = scale_of(m);
        if (first > 0) scale[w] = fmaxf(scale[w], was[w]);
        else was[w] = scale[w];
    }
    if (live && ok) {
        const float inv = 1.0f / scale[which];             // a power of two: exact
        uint32_t c[2][2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                c[h][j] = encode4(x[h][4 * j] * inv, x[h][4 * j + 1] * inv, x[h][4 * j + 2] * inv, x[h][4 * j + 3] * inv);
        const int slot = first + t;
        if (which == 0) {
            *(uint2 *)(kp + slot * HD + 8 * i) = uint2{c[0][0], c[0][1]};
            *(uint2 *)(kp + slot * HD + HD / 2 + 8 * i) = uint2{c[1][0], c[1][1]};
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int d = h * (HD / 2) + 8 * i + j;
                    tile[(slot / 4) * (4 * HD) + (d % 16) * (4 * DB) + (d / 16) * 4 + slot % 4] = (uint8_t)(c[h][j / 4] >> (8 * (j % 4)));
                }
        }
    }
    __syncthreads();
    if (ok) {
        // the values' tile; slots outside the unit keep their codes (rounded again where they came before it and the scale
        // grew)
        const bool again_v = scale[1] > was[1];
#pragma unroll
        for (int k = 0; k < QUADS; ++k) {
            const int q = quad_of(k), lo = max(first - 4 * q, 0), hi = min(first + n - 4 * q, 4);
            if (q >= 4 || hi <= 0 || lo >= 4) continue;
            const uint32_t below = (1u << (8 * lo)) - 1;           // slots before the unit
            const uint32_t fresh = (hi == 4 ? 0xffffffffu : (1u << (8 * hi)) - 1) & ~below;
            const uint32_t *src = (const uint32_t *)(tile + q * (4 * HD)) + W * lane;
#pragma unroll
            for (int j = 0; j < W; ++j) {
                uint32_t w = src[j];
                if (fresh != 0xffffffffu) {
                    const uint32_t kept = again_v ? rescale4(old[k][j], was[1] / scale[1]) : old[k][j];
                    w = (w & fresh) | (kept & below) | (old[k][j] & ~(fresh | below));
                }
                words_of(q)[j] = w;
            }
        }
        if (again_v) {
            for (int q = wave; q < first / 4; q += NT / 64)
#pragma unroll
                for (int j = 0; j < W; ++j) words_of(q)[j] = rescale4(words_of(q)[j], was[1] / scale[1]);
        }
        if (scale[0] > was[0]) {
            uint32_t *dst = (uint32_t *)kp;
            for (int j = tid; j < first * HD / 4; j += NT) dst[j] = rescale4(dst[j], was[0] / scale[0]);
        }
        if (tid == 0) {
            a.p.ks[head] = scale[0];
            a.p.vs[head] = scale[1];
        }
    }

    // the query heads of this KV head, the next round's on their way while one is turned
    for (int r = grp; r < rows; r += GROUPS) {
        const int tq = r / a.p.group, h = g * a.p.group + r % a.p.group, rn = r + GROUPS;
        float next[2][8];
        if (rn < rows) load_row(rn / a.p.group, g * a.p.group + rn % a.p.group, next);
        head_row(tq, a.q_gain, true, xq);
        TO *dst = (TO *)a.q_out + (size_t)(row0 + tq) * a.q_stride + (size_t)h * HD + 8 * i;
        store8(dst, xq[0]);
        store8(dst + HD / 2, xq[1]);
        if (rn < rows) {
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) xq[c][j] = next[c][j];
        }
    }
}

template <int HD, int NT> __global__ __launch_bounds__(NT) void read8_kernel(Read8 a) {
    constexpr int PT = HD / 16, DB = HD / 16;              // dims a thread
    __shared__ __attribute__((aligned(16))) uint8_t tile[kPage8 * HD];
    const int tid = threadIdx.x, g = blockIdx.x % a.p.nkv;
    Entry8<kUnit8Ints> entry;
    if (!entry8(a.p, kUnitsInt + kUnit8Ints * (int)(blockIdx.x / a.p.nkv), entry)) return;
    const int32_t *u = entry.v;
    const int seq = u[U8_SEQ], block = u[U8_BLOCK], first = u[U8_FIRST], n = u[U8_LEN], row0 = u[U8_ROW];
    const int page = a.p.table[(size_t)seq * a.p.max_blocks + block];
    const bool ok = page >= 0 && page < a.p.n_pages;
    if (!ok && tid == 0) flag_error(a.p.err, ORTHRUS_DEVERR_PAGE);
    const size_t head = (size_t)(ok ? page : 0) * a.p.nkv + g;
    const uint8_t *kp = a.p.k + head * (kPage8 * HD), *vp = a.p.v + head * (kPage8 * HD);
    // 16 threads a token, each PT dims of its key (and value, from the page's tile in LDS)
    static_assert(NT == 64 || NT == 16 * kPage8, "a unit's tokens in one round");
    const int t = tid / 16, d0 = (tid % 16) * PT, slot = first + t;
    const bool live = t < n;
    uint32_t kw[PT / 4] = {};
    if (live && ok) {
#pragma unroll
        for (int j = 0; j < PT / 4; ++j) kw[j] = *(const uint32_t *)(kp + slot * HD + d0 + 4 * j);
    }
    for (int i = tid; i < kPage8 * HD / 8; i += NT) ((uint2 *)tile)[i] = ((const uint2 *)vp)[i];
    const float ks = ok ? a.p.ks[head] : 1.f, vs = ok ? a.p.vs[head] : 1.f;
    __syncthreads();
    if (!live) return;
    uint32_t ow[2][PT / 2];
#pragma unroll
    for (int j = 0; j < PT / 4; ++j) {
        const uint2 w = word_bf16(kw[j], ks);
        ow[0][2 * j] = w.x;
        ow[0][2 * j + 1] = w.y;
        uint32_t c = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int d = d0 + 4 * j + e;
            c |= (uint32_t)tile[(slot / 4) * (4 * HD) + (d % 16) * (4 * DB) + (d / 16) * 4 + slot % 4] << (8 * e);
        }
        const uint2 v = word_bf16(ok ? c : 0u, vs);
        ow[1][2 * j] = v.x;
        ow[1][2 * j + 1] = v.y;
    }
    const size_t at = (size_t)(row0 + t) * ((size_t)a.p.nkv * HD) + (size_t)g * HD + d0;
    if constexpr (PT == 8) {
        *(u32x4 *)(a.k_out + at) = u32x4{ow[0][0], ow[0][1], ow[0][2], ow[0][3]};
        *(u32x4 *)(a.v_out + at) = u32x4{ow[1][0], ow[1][1], ow[1][2], ow[1][3]};
    } else {
        *(uint2 *)(a.k_out + at) = uint2{ow[0][0], ow[0][1]};
        *(uint2 *)(a.v_out + at) = uint2{ow[1][0], ow[1][1]};
    }
}

// Units of a few tokens (decode rows) take one wave each: four would mostly wait (256 rows over 8 KV heads 10.4 us with 256
// threads a unit).
constexpr int kFewTokens = 4;

template <typename TI, typename TO, int HD, int NT, int N> void append_of(const Append8 &a, hipStream_t s) {
    // half pairs of a head that turns in part meet through LDS, in NT / (HD / 16) rows
    const int lds = !a.interleaved && a.rot > 0 && a.rot < HD ? NT / (HD / 16) * (HD + 4) * 4 : 0;
    hipLaunchKernelGGL((append8_kernel<TI, TO, HD, NT, N>), dim3(a.n_units * a.p.nkv), dim3(NT), lds, s, a);
}
template <typename TI, typename TO, int HD> void append_of(const Append8 &a, hipStream_t s) {
    if (a.most <= kFewTokens) append_of<TI, TO, HD, 64, kFewTokens>(a, s);
    else append_of<TI, TO, HD, 256, kPage8>(a, s);
}
template <int HD> void append_of(const Append8 &a, hipStream_t s) {
    if (a.in_dtype == ORTHRUS_BF16) append_of<bf16, bf16, HD>(a, s);
    else if (a.out_dtype == ORTHRUS_BF16) append_of<float, bf16, HD>(a, s);
    else append_of<float, float, HD>(a, s);
}

}  // namespace

hipError_t launch_append8(const Append8 &a, hipStream_t s) {
    if (a.p.hd == 64) append_of<64>(a, s);
    else append_of<128>(a, s);
    return hipGetLastError();
}

hipError_t launch_read8(const Read8 &a, hipStream_t s) {
    const dim3 grid(a.n_units * a.p.nkv);
    const bool few = a.most <= kFewTokens;
    if (a.p.hd == 64) {
        if (few) hipLaunchKernelGGL((read8_kernel<64, 64>), grid, dim3(64), 0, s, a);
        else hipLaunchKernelGGL((read8_kernel<64, 256>), grid, dim3(256), 0, s, a);
    } else {
        if (few) hipLaunchKernelGGL((read8_kernel<128, 64>), grid, dim3(64), 0, s, a);
        else hipLaunchKernelGGL((read8_kernel<128, 256>), grid, dim3(256), 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace orthrus
