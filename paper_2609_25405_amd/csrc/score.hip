// Scores of tokens under logits: log probability, entropy, rank and the largest entries of each row.
//
// A row is read once: a workgroup holds its slice in registers, so the maximum is known before the first
// exponential and nothing is rescaled.  Rows of up to kSliceMost entries are one slice; longer ones,
// and rows too few to fill the chip, are several, joined by a second launch of one wave a row.
//
// Order.  An entry's key is its value as an order-preserving integer (NaN above everything, -0 equal to +0) over the
// complement of its index, so all keys differ and equal values rank by index.  The n largest of a
// slice: every thread's best entry, sorted within each wave and merged over the waves (64 at a time,
// bitonic), gives a bound that n entries reach; the n threads that reach it hold every entry that
// can be among the n largest, and those few are sorted.
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

template <int NT, int E>
__global__ __launch_bounds__(NT) void score_kernel(Score a, int slices) {
    constexpr int NW = NT / 64, EV = E / 4;
    __shared__ u64 best[NT];
    __shared__ u64 cand[64 * E];
    __shared__ float red[3][NW];
    __shared__ int red_rank[NW], n_cand;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int r = blockIdx.x / slices, slice = blockIdx.x % slices;
    const float *x = a.logits + (size_t)r * a.stride;
    // 16-byte loads from the aligned address at or before the row; elements outside the row are not read
    const int off = (int)(((uintptr_t)x >> 2) & 3);
    const int nvec = (a.vocab + off + 3) / 4;
    const int v0 = (int)((int64_t)slice * nvec / slices), v1 = (int)((int64_t)(slice + 1) * nvec / slices);
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
    auto index = [&](int i) { return 4 * (v0 + i / 4 * NT + tid) - off + i % 4; };
    auto real = [&](int i) { return v0 + i / 4 * NT + tid < v1 && index(i) >= 0 && index(i) < a.vocab; };
    const int tok = a.tokens ? a.tokens[r] : -1;
    const bool has = tok >= 0 && tok < a.vocab;
    const uint32_t tok_order = has ? order_of(x[tok]) : 0;
    u64 top = 0;
    int before = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const uint32_t o = order_of(v[i]);
        const u64 k = real(i) ? key_of(o, index(i)) : 0;
        top = k > top ? k : top;
        before += has && k > key_of(tok_order, tok) ? 1 : 0;
    }
    if (tid == 0) n_cand = 0;
    u64 sorted = 0;
    if (a.n_top > 0) {
        sorted = wave_sort(top, lane);
        best[tid] = sorted;
        for (int half = NW / 2; half >= 1; half /= 2) {
            __syncthreads();
            if (wave < half) {
                sorted = wave_merge(sorted, best[(wave + half) * 64 + 63 - lane], lane);
                best[tid] = sorted;
            }
        }
        __syncthreads();
    } else {
        u64 m = top;
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) {
            const u64 p = shfl_xor64(m, o);
            m = p > m ? p : m;
        }
        if (lane == 0) best[wave] = m;
        __syncthreads();
        m = best[0];
        for (int w = 1; w < NW; ++w) m = best[w] > m ? best[w] : m;
        __syncthreads();
        if (tid == 0) best[0] = m;
        __syncthreads();
    }
    const float m = value_of((uint32_t)(best[0] >> 32));
    const bool none = m == -INFINITY;      // nothing but -inf in the slice
    if (a.n_top > 0) {
        const u64 bound = best[a.n_top - 1];
        if (top >= bound && top != 0) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const u64 k = real(i) ? key_of(order_of(v[i]), index(i)) : 0;
                if (k >= bound && k != 0) cand[atomicAdd(&n_cand, 1)] = k;
            }
        }
    }
    float z = 0.f, s1 = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const float d = v[i] - m;
        const float e = v[i] == -INFINITY && !(none && slices == 1) ? 0.f : __builtin_amdgcn_exp2f(d * 1.4426950408889634f);
        z += e;
        s1 += e > 0.f ? e * d : 0.f;       // (a weight of zero may have an infinite distance)
    }
    z = wave_sum(z);
    s1 = wave_sum(s1);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) before += __shfl_xor(before, o, 64);
    if (lane == 0) {
        red[0][wave] = z;
        red[1][wave] = s1;
        red_rank[wave] = before;
    }
    __syncthreads();
    if (wave != 0) return;
    z = s1 = 0.f;
    before = 0;
    for (int w = 0; w < NW; ++w) {
        z += red[0][w];
        s1 += red[1][w];
        before += red_rank[w];
    }
    u64 key = 0;
    if (a.n_top > 0) {
        for (int c = 0; c < n_cand; c += 64) {
            const u64 k = wave_sort(c + lane < n_cand ? cand[c + lane] : 0, lane);
            key = c == 0 ? k : wave_merge(key, shfl64(k, 63 - lane), lane);
        }
    }
    if (slices == 1) {
        write_row(a, r, tok, m, z, s1, before, key, lane);
        return;
    }
    char *pp = a.ws + (size_t)blockIdx.x * part_bytes(a.n_top);
    if (lane == 0) *(Part *)pp = Part{m, z, s1, before};
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

int score_slices(int rows, int vocab) {
    const int least = (vocab + 3 + kSliceMost - 1) / kSliceMost;
    // few rows: slices of at least 4096 entries until the chip's 256 CUs have one each
    const int more = std::min((256 + rows - 1) / rows, vocab / 4096);
    return std::max({1, least, more});
}

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
