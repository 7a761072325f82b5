// The 8-bit paged cache: host plan of ragged rows, kernel arguments and the launchers.
#pragma once

#include <cstdint>
#include <vector>

#include "orthrus/kv8.h"

namespace orthrus {

constexpr int kPage8 = 16;         // positions of a page
constexpr int kLeastExp8 = -100;   // least exponent of a page's scale
constexpr int kSmallCols = 16;     // (row, query head) pairs of one small item: the columns of a 16x16 MFMA
constexpr int kTileRows8 = 128;    // (row, query head) pairs of one tile of a longer segment

// int32 fields of an attention item and of a merge entry: the rows and head of a range that comes in pieces, how many,
// the first partial slot and the slots of a piece
enum Item8 { A8_SEQ = 0, A8_ROW, A8_LEN, A8_POS, A8_HEAD, A8_KEY0, A8_KEY1, A8_SLOT, kItem8Ints };
enum Merge8 { M8_ROW = 0, M8_LEN, M8_HEAD, M8_PIECES, M8_SLOT, M8_SLOTS, kMerge8Ints };
// a partial slot holds 16 (row, head) pairs: maximum, sum, two words of padding, head_dim sums
constexpr int kPartialPad = 4;
// int32 fields of an append unit: the tokens of one segment that share a page
enum Unit8 { U8_SEQ = 0, U8_BLOCK, U8_FIRST, U8_LEN, U8_ROW, kUnit8Ints };

// pieces of long key ranges: at most so many a plan, and of one range
constexpr int kMaxSmallPieces = 2048, kMaxTilePieces = 1024, kMaxPieces = 128;

// The uploaded plan, from ws + kPlanOffset on: int32 stamp, padding to 64 bytes, turns[64] (double:
// turns per position of each pair, f_i / 2 pi), then units, small items, tile items, merges.
constexpr size_t kPlanOffset = 256;
constexpr int kTurnsInt = 16, kUnitsInt = kTurnsInt + 128;

struct RowsPlan {
    int T = 0, n_units = 0, n_small = 0, n_tiles = 0, n_merge = 0, n_slots = 0;
    int most_unit = 0;                          // tokens of the longest unit
    int merge_slots = 0;                        // slots of a piece, the most of any merge entry
    int small_cols = 0;                         // (row, head) pairs of the largest small item
    int wide = 0;                               // few small items alone: more waves each
    int joint = 0;                              // small items behind the tiles in one launch
    int need_seq = 0, need_blocks = 0;          // what a cache must have
    std::vector<int32_t> meta;                  // uploaded verbatim
    int off_small = 0, off_tiles = 0, off_merge = 0;
};

int validate_shape8(const orthrus_head_shape &s);
int plan_rows8(const orthrus_head_shape &s, const std::vector<double> &turns, const orthrus_kv8 &kv,
               const orthrus_segment *seg, int n, RowsPlan &out);
// The two halves of planning: validate and plan on the host (which also gives the workspace bytes that it takes), then
// upload.  err: the device error word that the plan's kernels flag.
int rows_prepare(const orthrus_rows *r, const orthrus_kv8 *kv, const orthrus_segment *segments, int n, RowsPlan &p, size_t &bytes);
int rows_upload(orthrus_rows *r, RowsPlan &&p, void *workspace, int *err, void *stream);
// orthrus_kv8_append of fp32 rows that come in two parts, `slab` elements apart (0: one part)
int append_rows8(const orthrus_rows *r, const orthrus_kv8 *kv, int32_t layer, const void *qkv, int32_t qkv_dtype, int64_t row_stride,
                 int64_t slab, const float *q_gain, const float *k_gain, void *q_out, int64_t q_stride, void *stream);
// most meta ints and partial slots that a plan of these sizes can have
void bound_rows8(const orthrus_head_shape &s, int64_t max_rows, int64_t max_segs, int64_t max_keys, size_t &meta_ints, size_t &slots);

}  // namespace orthrus

#ifdef __HIPCC__
#include <hip/hip_runtime.h>

#include "common.hpp"

namespace orthrus {

// what every kernel of a plan reads
struct Plan8 {
    const int32_t *meta;     // the uploaded plan
    int stamp;               // the plan these arguments were made for
    int *err;
    uint8_t *k, *v;          // the layer's pools and scales
    float *ks, *vs;
    const int32_t *table;
    int n_pages, max_blocks, nq, nkv, hd, group;
};

struct Append8 {
    Plan8 p;
    const void *qkv;
    int64_t stride;
    int64_t slab;            // elements to a second part of the rows (fp32), to be added; 0: none
    const float *q_gain, *k_gain;
    void *q_out;
    int64_t q_stride;
    int n_units, most, rot, interleaved, in_dtype, out_dtype;      // most: tokens of the longest unit
    float magnitude, eps;
};
hipError_t launch_append8(const Append8 &a, hipStream_t s);

struct Read8 {
    Plan8 p;
    int n_units, most;
    bf16 *k_out, *v_out;
};
hipError_t launch_read8(const Read8 &a, hipStream_t s);

struct Attend8 {
    Plan8 p;
    const void *q;
    void *out;
    int64_t q_stride, out_stride;
    int dtype, n_small, n_tiles, n_merge, merge_slots, small_cols, wide, joint, off_small, off_tiles, off_merge;
    float scale;             // log2(e) times the softmax scale
    float *partials;
};
hipError_t launch_attend8(const Attend8 &a, hipStream_t s);

// The entry at `at` of the plan, or false where the workspace holds another plan by now (replayed graphs): then the workgroup
// ends.  The entry is read before the comparison, so that the two latencies overlap; in any plan it is in bounds.
template <int N> struct Entry8 { int32_t v[N]; };
template <int N> __device__ __forceinline__ bool entry8(const Plan8 &p, int at, Entry8<N> &e) {
    // (a lane read keeps each load ahead of the branch, and its value in a scalar register)
#pragma unroll
    for (int i = 0; i < N; ++i) e.v[i] = __builtin_amdgcn_readfirstlane(p.meta[at + i]);
    const int stamp = p.meta[0];
    if (stamp == p.stamp) return true;
    if (threadIdx.x == 0) flag_error(p.err, ORTHRUS_DEVERR_STALE);
    return false;
}

typedef float f32x2_t __attribute__((ext_vector_type(2)));
// two codes (the low or the high half of a word) as bf16 values times a power of two: exact
template <bool HIGH> __device__ __forceinline__ uint32_t codes_bf16(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HIGH));
}
// four codes as four bf16 values
__device__ __forceinline__ uint2 word_bf16(uint32_t w, float scale) {
    return uint2{codes_bf16<false>(w, scale), codes_bf16<true>(w, scale)};
}

}  // namespace orthrus
#endif
