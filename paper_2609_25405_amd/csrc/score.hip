// Scores of tokens under logits: log probability, entropy, rank and the largest entries of each row.
//
// A row is read once: a workgroup holds its slice of up to kSliceMost entries in registers; each thread sums its own under the
// largest of them so far, eight at a time as they arrive, and the sums meet under the slice's (1999 rows of 131072 entries
// 169 us, 6.2 TB/s; 256 rows of 32000 with 20 alternatives 11.6 us).  Longer rows are several slices, joined by a second
// launch of one wave a row.
//
// Order.  An entry's key is its value as an order-preserving integer (NaN above everything, -0 equal to +0) over the
// complement of its index, so all keys differ and equal values rank by index.
// The n largest of a slice: the n-th largest of the maxima of 64 groups of threads is a bound that n entries reach;
// the few that reach it (24 on average for n = 20) go to LDS as keys and one wave puts them in order.
// Rank: entries of a lower index count where they are not smaller than the token's, the others where they are larger.
//
// Slices with a NaN, an infinite maximum, nothing but -inf, fewer finite entries than alternatives, more candidates than LDS
// holds (long ties) or a token whose own logit is not finite take slice_by_keys: the same results from keys alone, read again,
// slower (256 rows of 32000 with 20 alternatives: five finite entries a row 113 us, all equal 117, a NaN 176).
#include <algorithm>

#include "score.hpp"

// a weight's exponent is a rounded difference times L wherever it is taken: no contraction but the written fused operations
#pragma clang fp contract(off)

namespace orthrus {
namespace {

constexpr int kSliceMost = 32768;

typedef unsigned long long u64;

__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return x != x ? 0xffffffffu : b ^ (uint32_t)((int32_t)b >> 31 | (int32_t)0x80000000);
}
__device__ __forceinline__ float value_of(uint32_t o) {
    if (o == 0xffffffffu) return NAN;
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ u64 key_of(uint32_t order, int idx) { return (u64)order << 32 | (uint32_t)~idx; }
__device__ __forceinline__ int index_of(u64 key) { return (int)~(uint32_t)key; }

// lane ^ M by DPP and half-swaps (no LDS permutes)
template <int CTRL> __device__ __forceinline__ uint32_t dpp(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false);
}
template <int M> __device__ __forceinline__ uint32_t lane_xor(uint32_t v) {
    if constexpr (M == 1) return dpp<0xB1>(v);                    // quad permutations
    else if constexpr (M == 2) return dpp<0x4E>(v);
    else if constexpr (M == 4) return dpp<0x1B>(dpp<0x141>(v));   // mirror of 8 (xor 7), then of 4 (xor 3)
    else if constexpr (M == 8) return dpp<0x128>(v);              // rotation by 8 within 16
    else if constexpr (M == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return (threadIdx.x & 16) ? r[0] : r[1];
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return (threadIdx.x & 32) ? r[0] : r[1];
    }
}
template <int M> __device__ __forceinline__ u64 lane_xor64(u64 v) {
    return (u64)lane_xor<M>((uint32_t)(v >> 32)) << 32 | lane_xor<M>((uint32_t)v);
}
template <int M> __device__ __forceinline__ float lane_xorf(float v) { return __uint_as_float(lane_xor<M>(__float_as_uint(v))); }
__device__ __forceinline__ u64 wave_max64(u64 v) {
    u64 o;
    o = lane_xor64<1>(v), v = o > v ? o : v;
    o = lane_xor64<2>(v), v = o > v ? o : v;
    o = lane_xor64<4>(v), v = o > v ? o : v;
    o = lane_xor64<8>(v), v = o > v ? o : v;
    o = lane_xor64<16>(v), v = o > v ? o : v;
    o = lane_xor64<32>(v), v = o > v ? o : v;
    return v;
}
__device__ __forceinline__ float wave_addf(float v) {
    v += lane_xorf<1>(v);
    v += lane_xorf<2>(v);
    v += lane_xorf<4>(v);
    v += lane_xorf<8>(v);
    v += lane_xorf<16>(v);
    return v + lane_xorf<32>(v);
}
__device__ __forceinline__ int wave_addi(int v) {
    v += (int)lane_xor<1>((uint32_t)v);
    v += (int)lane_xor<2>((uint32_t)v);
    v += (int)lane_xor<4>((uint32_t)v);
    v += (int)lane_xor<8>((uint32_t)v);
    v += (int)lane_xor<16>((uint32_t)v);
    return v + (int)lane_xor<32>((uint32_t)v);
}
__device__ __forceinline__ float wave_maxf(float v) {
    v = fmaxf(v, lane_xorf<1>(v));
    v = fmaxf(v, lane_xorf<2>(v));
    v = fmaxf(v, lane_xorf<4>(v));
    v = fmaxf(v, lane_xorf<8>(v));
    v = fmaxf(v, lane_xorf<16>(v));
    return fmaxf(v, lane_xorf<32>(v));
}
// the larger of two, not a number above all, and that of a wave
__device__ __forceinline__ float larger_of(float a, float b) { return b > a || b != b ? b : a; }
template <int M> __device__ __forceinline__ float lane_larger(float v) { return larger_of(v, lane_xorf<M>(v)); }
__device__ __forceinline__ float wave_larger(float v) {
    v = lane_larger<1>(v);
    v = lane_larger<2>(v);
    v = lane_larger<4>(v);
    v = lane_larger<8>(v);
    v = lane_larger<16>(v);
    return lane_larger<32>(v);
}
__device__ __forceinline__ u64 reversed64(u64 v) {
    const int lane = 63 - (threadIdx.x & 63);
    return (u64)__shfl((uint32_t)(v >> 32), lane, 64) << 32 | __shfl((uint32_t)v, lane, 64);
}
// 64 keys, one a lane, in descending order: the whole bitonic sort, or its last stage (of a bitonic sequence)
template <int J> __device__ __forceinline__ u64 wave_step(u64 v, int k, int lane) {
    const u64 o = lane_xor64<J>(v);
    return (v > o) == (((lane & J) == 0) == ((lane & k) == 0)) ? v : o;
}
template <int K> __device__ __forceinline__ u64 wave_stage(u64 v, int lane) {
    if constexpr (K >= 64) v = wave_step<32>(v, K, lane);
    if constexpr (K >= 32) v = wave_step<16>(v, K, lane);
    if constexpr (K >= 16) v = wave_step<8>(v, K, lane);
    if constexpr (K >= 8) v = wave_step<4>(v, K, lane);
    if constexpr (K >= 4) v = wave_step<2>(v, K, lane);
    return wave_step<1>(v, K, lane);
}
__device__ __forceinline__ u64 wave_sort(u64 v, int lane) {
    v = wave_stage<2>(v, lane);
    v = wave_stage<4>(v, lane);
    v = wave_stage<8>(v, lane);
    v = wave_stage<16>(v, lane);
    v = wave_stage<32>(v, lane);
    return wave_stage<64>(v, lane);
}
// the 64 largest of two descending runs of 64 (`other` read in reverse)
__device__ __forceinline__ u64 wave_merge(u64 mine, u64 other_reversed, int lane) {
    return wave_stage<64>(mine > other_reversed ? mine : other_reversed, lane);
}

// Sums are held in base 2^L, L = log2(e) as an fp32 number, under a reference m that is one of the entries: with
// t = (x - m) L, z = sum 2^t and s = sum t 2^t, log Z = m + log2(z) / L and the entropy is (log2 z - s / z) / L.  The difference
// x - m is taken first, and a token's log probability as (x - m) - log2(z) / L, so that no size of the logits costs
// digits: of L x - r for a rounded r = L m, r's own rounding is left, 2^6 and more from logits of 1e9 on.  What L differs from
// log2(e) by is a factor 1 + 1.3e-8 on the differences.
constexpr float kL = 1.4426950408889634f;
constexpr float kNoTop = -3.4028234663852886e38f;      // the reference before any entry: the least finite number
constexpr float kLeastT = -300.f;      // exponents below it weigh nothing, and minus infinity must not meet that zero

// what a slice leaves to the merge launch, in the workspace: one Part, then n_top keys
struct Part {
    float m, z, s;      // the maximum and the sums under it
    int rank;
};
__host__ __device__ __forceinline__ size_t part_bytes(int n_top) { return sizeof(Part) + 8 * (size_t)n_top; }

// (xt: the token's logit, if it has one)
__device__ void write_row(const Score &a, int r, int tok, float xt, const Part &p, u64 key, int lane) {
    const double logz = (double)log2f(p.z) * (1.0 / (double)kL);         // beside the maximum
    auto log_probability = [&](float v) { return (float)(((double)v - (double)p.m) - logz); };
    if (lane == 0) {
        const bool has = a.tokens && tok >= 0 && tok < a.vocab;
        if (a.logprob) a.logprob[r] = has ? log_probability(xt) : NAN;
        if (a.rank) a.rank[r] = has ? p.rank : -1;
        if (a.entropy) a.entropy[r] = (log2f(p.z) - p.s / p.z) / kL;
    }
    if (lane < a.n_top) {
        if (a.top_ids) a.top_ids[(size_t)r * a.n_top + lane] = index_of(key);
        if (a.top_logprobs) a.top_logprobs[(size_t)r * a.n_top + lane] = log_probability(value_of((uint32_t)(key >> 32)));
    }
}

constexpr int kCands = 1024;

template <int NT> struct ScoreShared {
    static constexpr int NW = NT / 64;
    u64 cand[kCands];
    u64 best[NW];                 // slice_by_keys
    float group[64];
    int larger[64];
    float red[2][NW];
    int red_rank[NW], n_cand;
};

// a sum over the workgroup in the waves' order, for every thread
template <int NT> __device__ __forceinline__ float block_total(const float *red) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) t += red[w];
    return t;
}

// The slice [e0, e1) of row x by keys alone: the sums under the largest, then the n largest one at a time, each the largest of
// what the threads have next.
template <int NT>
__device__ void slice_by_keys(ScoreShared<NT> &sh, const float *x, int e0, int e1, int n, bool has, int tok, bool alone, Part &p,
                              u64 &key) {
    constexpr int NW = NT / 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const u64 tok_key = has ? key_of(order_of(x[tok]), tok) : 0;
    u64 top = 0;
    int before = 0;
    for (int e = e0 + tid; e < e1; e += NT) {
        const u64 k = key_of(order_of(x[e]), e);
        top = k > top ? k : top;
        before += has && k > tok_key ? 1 : 0;
    }
    auto largest_of = [&](u64 mine) {      // the workgroup's largest (its first barrier: the fast path is done with what follows)
        mine = wave_max64(mine);
        __syncthreads();
        if (lane == 0) sh.best[wave] = mine;
        __syncthreads();
        u64 all = 0;
        for (int w = 0; w < NW; ++w) all = sh.best[w] > all ? sh.best[w] : all;
        return all;
    };
    const float m = value_of((uint32_t)(largest_of(top) >> 32));
    const bool none = m == -INFINITY;      // nothing but -inf in the slice
    float z = 0.f, s = 0.f;
    for (int e = e0 + tid; e < e1; e += NT) {
        const float v = x[e], t = (v - m) * kL;
        const float w = v == -INFINITY && !(none && alone) ? 0.f : __builtin_amdgcn_exp2f(t);
        z += w;
        s = fmaf(w, fmaxf(t, kLeastT), s);
    }
    z = wave_addf(z);
    s = wave_addf(s);
    before = wave_addi(before);
    if (lane == 0) {
        sh.red[0][wave] = z;
        sh.red[1][wave] = s;
        sh.red_rank[wave] = before;
    }
    // n rounds: the largest key below the last one
    u64 last = ~0ull;                      // (the first is below or at it: a NaN at index 0 has that key)
    key = 0;
    for (int i = 0; i < n; ++i) {
        const bool taken = i > 0 && top >= last && top != 0;
        u64 mine = taken ? 0 : top;
        if (taken) {                       // this thread's largest is taken: its next
            for (int e = e0 + tid; e < e1; e += NT) {
                const u64 k = key_of(order_of(x[e]), e);
                if (k < last && k > mine) mine = k;
            }
        }
        last = largest_of(mine);
        if (lane == i) key = last;
        if (last == 0) break;              // fewer entries than n
    }
    __syncthreads();
    p.m = m;
    p.z = block_total<NT>(sh.red[0]);
    p.s = block_total<NT>(sh.red[1]);
    p.rank = 0;
    for (int w = 0; w < NW; ++w) p.rank += sh.red_rank[w];
}

template <int NT, int E>
__global__ __launch_bounds__(NT, NT == 1024 ? 8 : 4) void score_kernel(Score a, int slices) {
    constexpr int NW = NT / 64, EV = E / 4, GL = NT / 64;      // GL lanes a group
    constexpr int CH = E < 8 ? E : 8;
    __shared__ ScoreShared<NT> sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = blockIdx.x / slices, slice = blockIdx.x % slices;
    const float *x = a.logits + (size_t)row * a.stride;
    // 16-byte loads from the aligned address at or before the row; elements outside the row are not read
    const int off = (int)(((uintptr_t)x >> 2) & 3);
    const int nvec = (a.vocab + off + 3) / 4;
    const int v0 = (int)((int64_t)slice * nvec / slices), v1 = (int)((int64_t)(slice + 1) * nvec / slices);
    const int tok = a.tokens ? a.tokens[row] : -1;
    const bool has = tok >= 0 && tok < a.vocab;
    // Vectors [qa, qb) lie wholly in the row.  One before and one after them may lie in it in part: a thread of wave 1 and one
    // of wave 2 take these as four entries more, read first; the other loads then stand in no branch, so that the first are
    // used while the last are on their way (in branches each use waits for all: 256 rows of 32000 entries 12.7 us).
    const int qa = off > 0, qb = (a.vocab + off) / 4;
    const bool head = wave == 1 && off > 0 && slice == 0, tail = wave == 2 && qb >= v0 && qb < v1 && !(qb == 0 && off > 0);
    const int ex = head ? -off : 4 * qb - off;
    float v[E + 4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[E + j] = (head || tail) && lane == 0 && ex + j >= 0 && ex + j < a.vocab ? x[ex + j] : -INFINITY;
    const int whole0 = max(v0, qa), whole1 = min(v1, qb);
    if (qb > qa) {
#pragma unroll
        for (int i = 0; i < EV; ++i) {
            const float4 f = *(const float4 *)(x + (4 * min(max(v0 + i * NT + tid, qa), qb - 1) - off));
            v[4 * i] = f.x, v[4 * i + 1] = f.y, v[4 * i + 2] = f.z, v[4 * i + 3] = f.w;
        }
    }
    auto entry_of = [&](int vec) { return vec < EV ? 4 * (v0 + vec * NT + tid) - off : ex; };
    const float xt = has ? x[tok] : INFINITY;
    if (tid == 0) sh.n_cand = 0;
    if (tid < 64) sh.larger[tid] = 0;
    // eight entries at a time, as they arrive, under a reference of the thread's own
    float top = kNoTop, z = 0.f, s = 0.f;
    // entries before the token: the next smaller float turns "not smaller" into "larger"
    const uint32_t tb = __float_as_uint(xt);
    const float below = xt > 0.f ? __uint_as_float(tb - 1) : xt < 0.f ? __uint_as_float(tb + 1) : __uint_as_float(0x80000001u);
    int before = 0;
    auto take = [&](int c, int count) {
        float mc = v[c];
#pragma unroll
        for (int j = 1; j < count; ++j) mc = fmaxf(mc, v[c + j]);
        if (mc > top) {
            const float d = (top - mc) * kL, f = __builtin_amdgcn_exp2f(d);
            s = f * fmaf(z, fmaxf(d, kLeastT), s);
            z *= f;
            top = mc;
        }
#pragma unroll
        for (int j = 0; j < count; ++j) {
            const float t = (v[c + j] - top) * kL, w = __builtin_amdgcn_exp2f(t);
            z += w;
            s = fmaf(w, fmaxf(t, kLeastT), s);
        }
        if (has) {
#pragma unroll
            for (int i = c / 4; i < (c + count) / 4; ++i) {
                const int e = entry_of(i);
                const float limit = e + 3 < tok ? below : xt;
#pragma unroll
                for (int j = 0; j < 4; ++j) before += v[4 * i + j] > limit ? 1 : 0;
                if (e < tok && e + 3 >= tok) {                   // the vector that holds the token
#pragma unroll
                    for (int j = 0; j < 4; ++j) before += e + j < tok && v[4 * i + j] == xt ? 1 : 0;
                }
            }
        }
    };
#pragma unroll
    for (int c = 0; c < E; c += CH) {
#pragma unroll
        for (int i = c / 4; i < (c + CH) / 4; ++i) {
            const int q = v0 + i * NT + tid;
            const bool in = q >= whole0 && q < whole1;
            if (__ballot(!in)) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[4 * i + j] = in ? v[4 * i + j] : -INFINITY;
            }
        }
        take(c, CH);
    }
    if (head || tail) take(E, 4);
    float gm = top;
    if constexpr (GL >= 2) gm = fmaxf(gm, lane_xorf<1>(gm));
    if constexpr (GL >= 4) gm = fmaxf(gm, lane_xorf<2>(gm));
    if constexpr (GL >= 8) gm = fmaxf(gm, lane_xorf<4>(gm));
    if constexpr (GL >= 16) gm = fmaxf(gm, lane_xorf<8>(gm));
    if (lane % GL == 0) sh.group[tid / GL] = gm;
    __syncthreads();
    gm = sh.group[lane];
    const float m = wave_maxf(gm);
    {
        const float d = (top - m) * kL, f = __builtin_amdgcn_exp2f(d);
        s = f * fmaf(z, fmaxf(d, kLeastT), s);
        z *= f;
    }
    z = wave_addf(z);
    s = wave_addf(s);
    before = wave_addi(before);
    if (lane == 0) {
        sh.red[0][wave] = z;
        sh.red[1][wave] = s;
        sh.red_rank[wave] = before;
    }
    if (a.n_top > 1) {
        // how many group maxima are larger (equal ones in group order): each wave compares with its share of the 64
        int larger = 0;
#pragma unroll
        for (int o = wave * (64 / NW); o < (wave + 1) * (64 / NW); ++o) {
            const float g = sh.group[o];
            larger += g > gm || (g == gm && o < lane) ? 1 : 0;
        }
        if (larger) atomicAdd(&sh.larger[lane], larger);
    }
    __syncthreads();
    if (a.n_top > 0) {
        float bound = m;
        if (a.n_top > 1) {
            const uint64_t nth = __ballot(sh.larger[lane] == a.n_top - 1);
            bound = __shfl(gm, nth ? __builtin_ctzll(nth) : 0, 64);
        }
        if (top >= bound) {
            // (their places as bits, the entries read again: unrolled over registers this would be 4 KB of code to fetch)
            u64 hits = 0;
#pragma unroll
            for (int i = 0; i < E + 4; ++i) hits |= v[i] >= bound ? 1ull << i : 0ull;
            while (hits) {
                const int i = __builtin_ctzll(hits), e = entry_of(i / 4) + i % 4;
                hits &= hits - 1;
                const int c = atomicAdd(&sh.n_cand, 1);
                if (c < kCands) sh.cand[c] = key_of(order_of(x[e]), e);
            }
        }
        __syncthreads();
    }
    Part p{m, block_total<NT>(sh.red[0]), 0.f, 0};
    u64 key = 0;
    const int nc = __builtin_amdgcn_readfirstlane(sh.n_cand);
    // (block-uniform: every thread has read the same sums)
    const bool odd = !(p.z > 0.f && p.z < INFINITY) || (has && !(fabsf(xt) < INFINITY)) || nc > kCands || nc < a.n_top;
    if (__builtin_expect(odd, false)) {
        slice_by_keys<NT>(sh, x, max(4 * v0 - off, 0), min(4 * v1 - off, a.vocab), a.n_top, has, tok, slices == 1, p, key);
        if (wave != 0) return;
    } else {
        if (wave != 0) return;
        p.s = block_total<NT>(sh.red[1]);
#pragma unroll
        for (int w = 0; w < NW; ++w) p.rank += sh.red_rank[w];
        if (a.n_top > 0 && nc <= 64) {
            // a candidate's place is the number of larger ones (1999 rows of 131072 entries 175 us with a sort, 171)
            const u64 mine = lane < nc ? sh.cand[lane] : 0;
            int place = 0;
#pragma unroll 8
            for (int o = 0; o < nc; ++o) place += sh.cand[o] > mine ? 1 : 0;
            if (lane < nc) sh.cand[64 + place] = mine;
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            key = lane < nc ? sh.cand[64 + lane] : 0;
        } else if (a.n_top > 0) {
            for (int c = 0; c < nc; c += 64) {
                const u64 k = wave_sort(c + lane < nc ? sh.cand[c + lane] : 0, lane);
                key = c == 0 ? k : wave_merge(key, reversed64(k), lane);
            }
        }
    }
    if (slices == 1) {
        write_row(a, row, tok, xt, p, key, lane);
        return;
    }
    char *pp = a.ws + (size_t)blockIdx.x * part_bytes(a.n_top);
    if (lane == 0) *(Part *)pp = p;
    if (lane < a.n_top) ((u64 *)(pp + sizeof(Part)))[lane] = key;
}

// one wave a row: its slices' sums under the common maximum, and the largest of their entries
__global__ __launch_bounds__(64) void score_merge_kernel(Score a, int slices) {
    const int r = blockIdx.x, lane = threadIdx.x;
    const char *pp = a.ws + (size_t)r * slices * part_bytes(a.n_top);
    auto part = [&](int s) { return (const Part *)(pp + s * part_bytes(a.n_top)); };
    const int total = slices * a.n_top;
    auto key_at = [&](int i) { return i < total ? ((const u64 *)(part(i / a.n_top) + 1))[i % a.n_top] : 0; };
    // a lane a slice (and every 64th after it); all that a few slices left is on its way at once
    const Part none{-INFINITY, 0.f, 0.f, 0};
    Part q = lane < slices ? *part(lane) : none, p = none;
    const u64 first_key = key_at(lane);
    const int tok = a.tokens ? a.tokens[r] : -1;
    const float xt = tok >= 0 && tok < a.vocab ? a.logits[(size_t)r * a.stride + tok] : 0.f;
    p.m = q.m;
    for (int s = lane + 64; s < slices; s += 64) p.m = larger_of(p.m, part(s)->m);
    p.m = wave_larger(p.m);
    for (int s = lane; s < slices; s += 64) {
        if (s > lane) q = *part(s);
        p.rank += q.rank;
        if (q.m == -INFINITY) continue;                // nothing but -inf in the slice
        const float d = (q.m - p.m) * kL, f = __builtin_amdgcn_exp2f(d);
        p.z += q.z * f;
        p.s += f * (q.s + q.z * fmaxf(d, kLeastT));
    }
    p.z = wave_addf(p.z);
    p.s = wave_addf(p.s);
    p.rank = wave_addi(p.rank);
    if (p.m == -INFINITY) p.z = NAN;
    u64 key = 0;
    for (int c = 0; c < total; c += 64) {
        const u64 k = c == 0 ? first_key : key_at(c + lane);
        const u64 sorted = wave_sort(k, lane);
        key = c == 0 ? sorted : wave_merge(key, reversed64(sorted), lane);
    }
    write_row(a, r, tok, xt, p, key, lane);
}

}  // namespace

namespace {
// slices of a row that starts `off` entries past a 16-byte boundary
int slices_of(int vocab, int off) { return (vocab + off + kSliceMost - 1) / kSliceMost; }
}  // namespace

int score_slices(int vocab) { return slices_of(vocab, 3); }

size_t score_bytes(int rows, int vocab, int n_top) {
    const int s = score_slices(vocab);
    return s == 1 ? 0 : (size_t)rows * s * part_bytes(n_top);
}

hipError_t launch_score(const Score &a, hipStream_t s) {
    const bool aligned = ((uintptr_t)a.logits & 15) == 0 && a.stride % 4 == 0;
    const int off = aligned ? 0 : 3, slices = slices_of(a.vocab, off);
    const int entries = ((a.vocab + off + 3) / 4 + slices - 1) / slices * 4;       // of the longest slice
    const dim3 grid(a.rows * slices);
    if (entries <= 1024) hipLaunchKernelGGL((score_kernel<256, 4>), grid, dim3(256), 0, s, a, slices);
    else if (entries <= 8192) hipLaunchKernelGGL((score_kernel<1024, 8>), grid, dim3(1024), 0, s, a, slices);
    else if (entries <= 16384) hipLaunchKernelGGL((score_kernel<1024, 16>), grid, dim3(1024), 0, s, a, slices);
    else hipLaunchKernelGGL((score_kernel<1024, 32>), grid, dim3(1024), 0, s, a, slices);
    if (slices > 1) hipLaunchKernelGGL(score_merge_kernel, dim3(a.rows), dim3(64), 0, s, a, slices);
    return hipGetLastError();
}

}  // namespace orthrus

using namespace orthrus;

extern "C" {

size_t orthrus_logprobs_bytes(int32_t rows, int32_t vocab, int32_t n_top) {
    if (rows < 1 || vocab < 1 || n_top < 0 || n_top > std::min(vocab, ORTHRUS_MAX_TOP)) return 0;
    return score_bytes(rows, vocab, n_top);
}

int orthrus_logprobs(const float *logits, int64_t row_stride, int32_t rows, int32_t vocab, const int32_t *tokens,
                     int32_t n_top, float *logprob, float *entropy, int32_t *rank, int32_t *top_ids, float *top_logprobs,
                     void *workspace, size_t ws_bytes, void *stream) {
    if (rows < 0 || vocab < 1 || n_top < 0 || n_top > std::min(vocab, ORTHRUS_MAX_TOP) || row_stride < vocab) return ORTHRUS_EINVAL;
    if (rows == 0) return ORTHRUS_OK;
    if (!logits || ((logprob || rank) && !tokens) || (n_top == 0 && (top_ids || top_logprobs))) return ORTHRUS_EINVAL;
    if ((uintptr_t)logits & 3) return ORTHRUS_EINVAL;
    // a launch has fewer than 2^32 threads, up to 1024 for each slice
    if (vocab > (1 << 30) || (int64_t)rows * score_slices(vocab) >= (1 << 22)) return ORTHRUS_ECAPACITY;
    const size_t need = score_bytes(rows, vocab, n_top);
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 15))) return ORTHRUS_EINVAL;
    if (ws_bytes < need) return ORTHRUS_ECAPACITY;
    Score a{logits, row_stride, rows, vocab, n_top, tokens, logprob, entropy, rank, top_ids, top_logprobs, (char *)workspace};
    return launch_score(a, (hipStream_t)stream) == hipSuccess ? ORTHRUS_OK : ORTHRUS_EHIP;
}

}  // extern "C"
