// Scores of tokens under logits: log probability, entropy, rank and the largest entries of each row.
//
// A row is read once: a workgroup holds its slice of up to kSliceMost entries in registers, so the maximum is
// known before the first exponential and nothing is rescaled.  Longer rows are several slices, joined by a
// second launch of one wave a row.
//
// Order.  An entry's key is its value as an order-preserving integer (NaN above everything, -0 equal to +0) over the
// complement of its index, so all keys differ and equal values rank by index.
// The n largest of a slice: the n-th largest of the maxima of 64 groups of threads is a bound that n entries reach;
// the few that reach it (24 on average for n = 20) go to LDS as keys and one wave sorts them.
// Rank: entries of a lower index count where they are not smaller than the token's, the others where they are larger.
//
// Slices with a NaN, an infinite maximum, more candidates than LDS holds (long ties) or a token whose own logit is not
// finite take slice_by_keys: the same results from keys alone, read again, slower.
#include <algorithm>

#include "score.hpp"

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

__device__ __forceinline__ u64 shfl_xor64(u64 v, int m) {
    const uint32_t lo = __shfl_xor((uint32_t)v, m, 64), hi = __shfl_xor((uint32_t)(v >> 32), m, 64);
    return (u64)hi << 32 | lo;
}
__device__ __forceinline__ u64 shfl64(u64 v, int lane) {
    const uint32_t lo = __shfl((uint32_t)v, lane, 64), hi = __shfl((uint32_t)(v >> 32), lane, 64);
    return (u64)hi << 32 | lo;
}
// 64 keys, one a lane, in descending order: the whole bitonic sort, or its last stage (of a bitonic sequence)
__device__ __forceinline__ u64 wave_stage(u64 v, int k, int lane) {
    for (int j = k / 2; j > 0; j /= 2) {
        const u64 o = shfl_xor64(v, j);
        const bool high = ((lane & j) == 0) == ((lane & k) == 0);
        v = (v > o) == high ? v : o;
    }
    return v;
}
__device__ __forceinline__ u64 wave_sort(u64 v, int lane) {
    for (int k = 2; k <= 64; k *= 2) v = wave_stage(v, k, lane);
    return v;
}
// the 64 largest of two descending runs of 64 (`other` read in reverse)
__device__ __forceinline__ u64 wave_merge(u64 mine, u64 other_reversed, int lane) {
    return wave_stage(mine > other_reversed ? mine : other_reversed, 64, lane);
}

// what a slice leaves to the merge launch, in the workspace: one Part, then n_top keys
struct Part {
    float m, z, s1;
    int rank;
};
__host__ __device__ __forceinline__ size_t part_bytes(int n_top) { return sizeof(Part) + 8 * (size_t)n_top; }

__device__ void write_row(const Score &a, int r, int tok, float m, float z, float s1, int rank, u64 key, int lane) {
    const float logz = logf(z);
    if (lane == 0) {
        const bool has = a.tokens && tok >= 0 && tok < a.vocab;
        if (a.logprob) a.logprob[r] = has ? a.logits[(size_t)r * a.stride + tok] - m - logz : NAN;
        if (a.rank) a.rank[r] = has ? rank : -1;
        if (a.entropy) a.entropy[r] = logz - s1 / z;
    }
    if (lane < a.n_top) {
        if (a.top_ids) a.top_ids[(size_t)r * a.n_top + lane] = index_of(key);
        if (a.top_logprobs) a.top_logprobs[(size_t)r * a.n_top + lane] = value_of((uint32_t)(key >> 32)) - m - logz;
    }
}

constexpr int kCands = 1024;

template <int NT> struct ScoreShared {
    static constexpr int NW = NT / 64;
    u64 cand[kCands];
    u64 best[NT];                 // slice_by_keys
    float group[64];
    float red[3][NW];
    int red_rank[NW], n_cand;
};

// a sum over the workgroup in the waves' order, for every thread
template <int NT> __device__ __forceinline__ float block_total(const float *red) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) t += red[w];
    return t;
}

// The slice [e0, e1) of row x by keys alone: every thread's largest key, the 64 largest of those (sorted in each wave, merged
// over the waves), whose n-th is a bound; the at most 64 threads that reach it then pass their keys in
// descending order, one at a time.
template <int NT>
__device__ void slice_by_keys(ScoreShared<NT> &sh, const float *x, int e0, int e1, int n, bool has, int tok, bool alone, float &m, float &z,
                              float &s1, int &rank, u64 &key) {
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
    __syncthreads();              // the fast path is done with what follows
    u64 sorted = wave_sort(top, lane);
    sh.best[tid] = sorted;
    for (int half = NW / 2; half >= 1; half /= 2) {
        __syncthreads();
        if (wave < half) {
            sorted = wave_merge(sorted, sh.best[(wave + half) * 64 + 63 - lane], lane);
            sh.best[tid] = sorted;
        }
    }
    __syncthreads();
    m = value_of((uint32_t)(sh.best[0] >> 32));
    const bool none = m == -INFINITY;      // nothing but -inf in the slice
    z = s1 = 0.f;
    for (int e = e0 + tid; e < e1; e += NT) {
        const float v = x[e], d = v - m;
        const float w = v == -INFINITY && !(none && alone) ? 0.f : __builtin_amdgcn_exp2f(d * 1.4426950408889634f);
        z += w;
        s1 += w > 0.f ? w * d : 0.f;
    }
    z = wave_sum(z);
    s1 = wave_sum(s1);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) before += __shfl_xor(before, o, 64);
    if (lane == 0) {
        sh.red[0][wave] = z;
        sh.red[1][wave] = s1;
        sh.red_rank[wave] = before;
    }
    // n rounds: the largest key below the last one
    u64 last = ~0ull;
    key = 0;
    for (int i = 0; i < n; ++i) {
        u64 mine = top < last ? top : 0;
        if (top >= last && top != 0) {     // this thread's largest is taken: its next
            for (int e = e0 + tid; e < e1; e += NT) {
                const u64 k = key_of(order_of(x[e]), e);
                if (k < last && k > mine) mine = k;
            }
        }
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) {
            const u64 p = shfl_xor64(mine, o);
            mine = p > mine ? p : mine;
        }
        __syncthreads();
        if (lane == 0) sh.best[wave] = mine;
        __syncthreads();
        last = 0;
        for (int w = 0; w < NW; ++w) last = sh.best[w] > last ? sh.best[w] : last;
        if (lane == i) key = last;
        if (last == 0) break;              // fewer entries than n
    }
    __syncthreads();
    z = block_total<NT>(sh.red[0]);
    s1 = block_total<NT>(sh.red[1]);
    rank = 0;
    for (int w = 0; w < NW; ++w) rank += sh.red_rank[w];
}

template <int NT, int E>
__global__ __launch_bounds__(NT, NT == 1024 ? 8 : 4) void score_kernel(Score a, int slices) {
    constexpr int NW = NT / 64, EV = E / 4, GL = NT / 64;      // GL lanes a group
    __shared__ ScoreShared<NT> sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int r = blockIdx.x / slices, slice = blockIdx.x % slices;
    const float *x = a.logits + (size_t)r * a.stride;
    // 16-byte loads from the aligned address at or before the row; elements outside the row are not read
    const int off = (int)(((uintptr_t)x >> 2) & 3);
    const int nvec = (a.vocab + off + 3) / 4;
    const int v0 = (int)((int64_t)slice * nvec / slices), v1 = (int)((int64_t)(slice + 1) * nvec / slices);
    const int tok = a.tokens ? a.tokens[r] : -1;
    const bool has = tok >= 0 && tok < a.vocab;
    float v[E];
#pragma unroll
    for (int i = 0; i < EV; ++i) {
        const int q = v0 + i * NT + tid, e = 4 * q - off;
        if (q < v1 && e >= 0 && e + 3 < a.vocab) {
            const float4 f = *(const float4 *)(x + e);
            v[4 * i] = f.x, v[4 * i + 1] = f.y, v[4 * i + 2] = f.z, v[4 * i + 3] = f.w;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * i + j] = q < v1 && e + j >= 0 && e + j < a.vocab ? x[e + j] : -INFINITY;
        }
    }
    const float xt = has ? x[tok] : INFINITY;
    if (tid == 0) sh.n_cand = 0;
    float top = v[0];
#pragma unroll
    for (int i = 1; i < E; ++i) top = fmaxf(top, v[i]);
    float gm = top;
#pragma unroll
    for (int o = 1; o < GL; o *= 2) gm = fmaxf(gm, __shfl_xor(gm, o, 64));
    if (lane % GL == 0) sh.group[tid / GL] = gm;
    __syncthreads();
    gm = sh.group[lane];
    const float m = wave_max(gm);
    // entries before the token: the next smaller float turns "not smaller" into "larger"
    const uint32_t tb = __float_as_uint(xt);
    const float below = xt > 0.f ? __uint_as_float(tb - 1) : xt < 0.f ? __uint_as_float(tb + 1) : __uint_as_float(0x80000001u);
    int before = 0;
    float z = 0.f, s1 = 0.f;
#pragma unroll
    for (int i = 0; i < EV; ++i) {
        const int e = 4 * (v0 + i * NT + tid) - off;
        const bool lower = e + 3 < tok;
        const float limit = lower ? below : xt;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float f = v[4 * i + j], d = f - m;
            const float w = __builtin_amdgcn_exp2f(d * 1.4426950408889634f);
            z += w;
            s1 = fmaf(w, fmaxf(d, -200.f), s1);        // (a weight of zero may have an infinite distance)
            before += f > limit ? 1 : 0;
            if (!lower && e + j < tok && f == xt) ++before;       // the vector that holds the token
        }
    }
    if (a.n_top > 0) {
        // the n-th largest group maximum: its rank among the 64 (equal ones in lane order)
        int larger = 0;
#pragma unroll 8
        for (int o = 0; o < 64; ++o) {
            const float g = sh.group[o];
            larger += g > gm || (g == gm && o < lane) ? 1 : 0;
        }
        const uint64_t nth = __ballot(larger == a.n_top - 1);
        const float bound = __shfl(gm, nth ? __builtin_ctzll(nth) : 0, 64);
        if (top >= bound) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const int e = 4 * (v0 + i / 4 * NT + tid) - off + i % 4;
                if (v[i] >= bound && v[i] > -INFINITY) {
                    const int c = atomicAdd(&sh.n_cand, 1);
                    if (c < kCands) sh.cand[c] = key_of(order_of(v[i]), e);
                }
            }
        }
    }
    z = wave_sum(z);
    s1 = wave_sum(s1);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) before += __shfl_xor(before, o, 64);
    if (lane == 0) {
        sh.red[0][wave] = z;
        sh.red[1][wave] = s1;
        sh.red_rank[wave] = before;
    }
    __syncthreads();
    z = block_total<NT>(sh.red[0]);
    float mm = m;
    u64 key = 0;
    const int nc = sh.n_cand;
    // (block-uniform: every thread has read the same sums)
    if (!(z < INFINITY) || (has && !(fabsf(xt) < INFINITY)) || nc > kCands || nc < a.n_top) {
        slice_by_keys<NT>(sh, x, max(4 * v0 - off, 0), min(4 * v1 - off, a.vocab), a.n_top, has, tok, slices == 1, mm, z, s1, before, key);
        if (wave != 0) return;
    } else {
        if (wave != 0) return;
        s1 = block_total<NT>(sh.red[1]);
        before = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) before += sh.red_rank[w];
        if (a.n_top > 0) {
            for (int c = 0; c < nc; c += 64) {
                const u64 k = wave_sort(c + lane < nc ? sh.cand[c + lane] : 0, lane);
                key = c == 0 ? k : wave_merge(key, shfl64(k, 63 - lane), lane);
            }
        }
    }
    if (slices == 1) {
        write_row(a, r, tok, mm, z, s1, before, key, lane);
        return;
    }
    char *pp = a.ws + (size_t)blockIdx.x * part_bytes(a.n_top);
    if (lane == 0) *(Part *)pp = Part{mm, z, s1, before};
    if (lane < a.n_top) ((u64 *)(pp + sizeof(Part)))[lane] = key;
}

// one wave a row: its slices' sums under the common maximum, and the largest of their entries
__global__ __launch_bounds__(64) void score_merge_kernel(Score a, int slices) {
    const int r = blockIdx.x, lane = threadIdx.x;
    const char *pp = a.ws + (size_t)r * slices * part_bytes(a.n_top);
    auto part = [&](int s) { return (const Part *)(pp + s * part_bytes(a.n_top)); };
    float m = -INFINITY;
    for (int s = 0; s < slices; ++s) m = part(s)->m > m || part(s)->m != part(s)->m ? part(s)->m : m;
    float z = 0.f, s1 = 0.f;
    int before = 0;
    for (int s = 0; s < slices; ++s) {
        const Part p = *part(s);
        const float d = p.m - m, f = __builtin_amdgcn_exp2f(d * 1.4426950408889634f);
        if (p.m != -INFINITY) {
            z += p.z * f;
            s1 += f > 0.f ? f * (p.s1 + p.z * d) : 0.f;
        }
        before += p.rank;
    }
    if (m == -INFINITY) z = NAN;
    u64 key = 0;
    const int total = slices * a.n_top;
    for (int c = 0; c < total; c += 64) {
        const int i = c + lane;
        const u64 k = i < total ? ((const u64 *)(part(i / a.n_top) + 1))[i % a.n_top] : 0;
        const u64 sorted = wave_sort(k, lane);
        key = c == 0 ? sorted : wave_merge(key, shfl64(sorted, 63 - lane), lane);
    }
    write_row(a, r, a.tokens ? a.tokens[r] : -1, m, z, s1, before, key, lane);
}

}  // namespace

int score_slices(int rows, int vocab) { return (vocab + 3 + kSliceMost - 1) / kSliceMost; }

size_t score_bytes(int rows, int vocab, int n_top) {
    const int s = score_slices(rows, vocab);
    return s == 1 ? 0 : (size_t)rows * s * part_bytes(n_top);
}

hipError_t launch_score(const Score &a, hipStream_t s) {
    const int slices = score_slices(a.rows, a.vocab);
    const int entries = ((a.vocab + 6) / 4 + slices - 1) / slices * 4;       // of the longest slice, with the row's misalignment
    const dim3 grid(a.rows * slices);
    if (entries <= 1024) hipLaunchKernelGGL((score_kernel<256, 4>), grid, dim3(256), 0, s, a, slices);
    else if (entries <= 8192) hipLaunchKernelGGL((score_kernel<1024, 8>), grid, dim3(1024), 0, s, a, slices);
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
    if (vocab > (1 << 30) || (int64_t)rows * score_slices(rows, vocab) > INT32_MAX) return ORTHRUS_ECAPACITY;
    const size_t need = score_bytes(rows, vocab, n_top);
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 15))) return ORTHRUS_EINVAL;
    if (ws_bytes < need) return ORTHRUS_ECAPACITY;
    Score a{logits, row_stride, rows, vocab, n_top, tokens, logprob, entropy, rank, top_ids, top_logprobs, (char *)workspace};
    return launch_score(a, (hipStream_t)stream) == hipSuccess ? ORTHRUS_OK : ORTHRUS_EHIP;
}

}  // extern "C"
