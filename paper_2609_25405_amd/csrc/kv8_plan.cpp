// Host planning of ragged rows over the 8-bit cache: validation of the segments, the append units
// and the attention work lists.  Plain C++17, no HIP calls.
#include "kv8.hpp"

#include <algorithm>
#include <array>
#include <climits>
#include <cmath>
#include <cstring>
#include <utility>

namespace orthrus {

namespace {
// Key ranges.  An item walks its keys in steps, so one long range can outlast the launch while CUs are
// idle: ranges longer than their share of the launch's workgroup slots are cut into pieces of about that share, on
// multiples of kCut keys.  A piece costs its partial sums' way through memory and, with the others, a merge launch (5 us for
// 64 rows, 11 for two chunks of 512), so it has a least length.
constexpr int kCut = 64;
// Small items run three workgroups of four waves a CU (8 KV heads, cut for 512, 768 and 1024 slots: 64 rows of 2560 keys
// 62.8, 62.8 and 68.8 us, of 1024 to 4096 71.2, 67.0 and 69.4, 100 rows of 3000 123 each, 40 of 6000 100.9, 100.9 and 97.8).
constexpr int kSlotsSmall = 768, kMinPieceSmall = 1024;
// Few of them run with eight waves each, cut for fewer workgroups (one row of 4000 keys over 8 KV heads 12.5 us in
// pieces of at least 512 keys, 14.5 of 1024; 16 rows of 2000 17.6 us in 192 slots, 18.8 in 256, 21.9 in 384).
constexpr int kWideItems = 256, kSlotsWide = 192, kMinPieceWide = 512;
// ... but not at all where none has more than two steps a wave (one row of 1000 keys 9.5 us whole, 11.0 in two pieces; of 1300 12.3
// and 10.2; 4 rows of 1400 13.6 and 11.6).
constexpr int kMostWhole = 1024;
// Tiles run two workgroups a CU; items i and kCus + i of a launch share one, so the second round comes shortest first
// (4 fresh prompts of 400 to 623 tokens 26.9 -> 26.5 us).  The least piece (32 query heads over 8, pieces from 256, 512, 1024
// and 2048 keys on): 64 rows after 900 keys 18, 22, 26 and 26 us, 128 after 4000 34, 30, 33 and 49, 512 after 2000 40, 40, 41
// and 53, four prompts of 512 33, 22, 23 and 23, 2 x 512 after 7680 152 each; fp32, 2 x 256 after 1000, 59, 49, 64 and 64.  512
// is the better one for a chunk or two alone.
constexpr int kCus = 256, kSlotsTile = 2 * kCus, kMinPieceTile = 1024;

int64_t piece_keys(int64_t total, int slots, int least) {
    const int64_t mean = (total + slots - 1) / slots;
    return std::max<int64_t>(least, (mean + kCut - 1) / kCut * kCut);
}
}  // namespace

int validate_shape8(const orthrus_head_shape &s) {
    if (s.n_q_heads <= 0 || s.n_kv_heads <= 0 || s.head_dim <= 0 || s.page_size <= 0) return ORTHRUS_EINVAL;
    if (s.dtype != ORTHRUS_F32 && s.dtype != ORTHRUS_BF16) return ORTHRUS_EINVAL;
    if (s.n_q_heads % s.n_kv_heads) return ORTHRUS_EINVAL;
    if (s.rot_dims < 0 || s.rot_dims > s.head_dim || (s.interleaved != 0 && s.interleaved != 1)) return ORTHRUS_EINVAL;
    if (!(s.norm_eps >= 0.f) || !std::isfinite(s.norm_eps) || !std::isfinite(s.rope_magnitude)) return ORTHRUS_EINVAL;
    if (s.rope_freq) {
        for (int i = 0; i < s.rot_dims / 2; ++i)
            if (!std::isfinite(s.rope_freq[i])) return ORTHRUS_EINVAL;
    } else if (s.rot_dims > 0 && !(s.rope_base > 1.f && std::isfinite(s.rope_base))) {
        return ORTHRUS_EINVAL;
    }
    if (s.head_dim != 64 && s.head_dim != 128) return ORTHRUS_EUNSUPPORTED;
    if (s.page_size != kPage8 || s.rot_dims % 16) return ORTHRUS_EUNSUPPORTED;
    if (s.n_q_heads / s.n_kv_heads > kSmallCols) return ORTHRUS_EUNSUPPORTED;
    if (s.n_q_heads > 65535) return ORTHRUS_EUNSUPPORTED;
    return ORTHRUS_OK;
}

void bound_rows8(const orthrus_head_shape &s, int64_t max_rows, int64_t max_segs, int64_t max_keys, size_t &meta_ints, size_t &slots) {
    const int64_t nkv = s.n_kv_heads, group = s.n_q_heads / nkv, per_tile = kTileRows8 / group;
    max_segs = std::min(max_segs, max_rows);
    const int64_t units = max_rows / kPage8 + 2 * max_segs;
    const int64_t small = max_segs * nkv, tiles = (max_rows / per_tile + max_segs) * nkv;
    // a range of k keys makes at most min(k / least, pieces allowed) pieces
    const int64_t ps = std::min<int64_t>(kMaxSmallPieces, small * (max_keys / kMinPieceWide + 1));
    const int64_t pt = std::min<int64_t>(kMaxTilePieces, tiles * (max_keys / kMinPieceTile + 1));
    meta_ints = (size_t)(kUnitsInt + units * kUnit8Ints + (small + ps + tiles + pt) * kItem8Ints + (ps + pt) / 2 * kMerge8Ints);
    slots = (size_t)(ps + pt * (kTileRows8 / kSmallCols));
}

int plan_rows8(const orthrus_head_shape &s, const std::vector<double> &turns, const orthrus_kv8 &kv,
               const orthrus_segment *seg, int n, RowsPlan &p) {
    if (n < 0 || (n > 0 && !seg)) return ORTHRUS_EINVAL;
    p = RowsPlan();
    const int nkv = s.n_kv_heads, group = s.n_q_heads / nkv, per_tile = kTileRows8 / group;
    std::vector<uint8_t> seen((size_t)kv.n_seq, 0);
    int64_t T = 0;
    for (int i = 0; i < n; ++i) {
        const orthrus_segment &g = seg[i];
        if (g.seq < 0 || g.seq >= kv.n_seq || g.offset < 0 || g.len < 1) return ORTHRUS_EDESC;
        const int64_t end = (int64_t)g.offset + g.len;
        if (end > (int64_t)kv.max_blocks * kPage8) return ORTHRUS_ECAPACITY;
        // positions are 32-bit in the kernels, the last block's end included
        if (end > INT32_MAX - 4 * kCut) return ORTHRUS_ECAPACITY;
        if (seen[g.seq]) return ORTHRUS_EDUPSEQ;
        seen[g.seq] = 1;
        T += g.len;
        p.need_seq = std::max(p.need_seq, g.seq + 1);
        p.need_blocks = std::max(p.need_blocks, (int)((end + kPage8 - 1) / kPage8));
    }
    // a launch has fewer than 2^32 threads, up to 256 for each row and KV head
    if (T * nkv > (1LL << 23)) return ORTHRUS_ECAPACITY;
    p.T = (int)T;

    std::vector<int32_t> units;
    struct Range { int64_t work; int seq, row, len, pos, head, key1; };
    std::vector<Range> small, tiles;
    int64_t keys_small = 0, keys_tiles = 0;
    int row = 0;
    for (int i = 0; i < n; ++i) {
        const orthrus_segment &g = seg[i];
        for (int t = 0; t < g.len;) {
            const int pos = g.offset + t, first = pos % kPage8, len = std::min(kPage8 - first, g.len - t);
            p.most_unit = std::max(p.most_unit, len);
            units.insert(units.end(), {g.seq, pos / kPage8, first, len, row + t});
            t += len;
        }
        const bool few = (int64_t)g.len * group <= kSmallCols;
        if (few) p.small_cols = std::max(p.small_cols, g.len * group);
        const int step = few ? g.len : per_tile;
        for (int t = 0; t < g.len; t += step) {
            const int len = std::min(step, g.len - t), key1 = g.offset + t + len;
            (few ? keys_small : keys_tiles) += (int64_t)key1 * nkv;
            for (int h = 0; h < nkv; ++h)
                (few ? small : tiles).push_back({(int64_t)key1, g.seq, row + t, len, g.offset + t, h, key1});
        }
        row += g.len;
    }
    p.n_units = (int)(units.size() / kUnit8Ints);

    std::vector<std::array<int32_t, kMerge8Ints>> merges;
    using Item = std::array<int32_t, kItem8Ints>;
    // longest first, so that the launch does not end on a long item; equal ones in the rows' order
    auto cut = [&](std::vector<Range> &ranges, int64_t piece, int64_t whole, int most_pieces, int slots_each) {
        std::vector<std::pair<int64_t, Item>> items;
        int pieces = 0;
        std::stable_sort(ranges.begin(), ranges.end(), [](const Range &a, const Range &b) { return a.work > b.work; });
        if (!ranges.empty() && ranges[0].work <= whole) piece = whole;       // none is worth a merge
        for (const Range &r : ranges) {
            // (the nearest count: one piece too many for some ranges would be a second round of the launch)
            int m = (int)std::max<int64_t>(1, std::min<int64_t>(kMaxPieces, (r.work + piece / 2) / piece));
            if (pieces + m > most_pieces) m = 1;
            int slot = -1;
            if (m > 1) {
                slot = p.n_slots;
                merges.push_back({r.row, r.len, r.head, m, slot, slots_each});
                p.merge_slots = std::max(p.merge_slots, slots_each);
                p.n_slots += m * slots_each;
                pieces += m;
            }
            int k0 = 0;
            for (int j = 0; j < m; ++j) {
                const int k1 = j + 1 == m ? r.key1 : (int)((int64_t)(j + 1) * r.key1 / m / kCut * kCut);
                items.push_back({k1 - k0, Item{r.seq, r.row, r.len, r.pos, r.head, k0, k1, m > 1 ? slot + j * slots_each : -1}});
                k0 = k1;
            }
        }
        std::stable_sort(items.begin(), items.end(), [](const auto &a, const auto &b) { return a.first > b.first; });
        return items;
    };
    p.joint = !small.empty() && !tiles.empty();
    p.wide = !p.joint && (int)small.size() <= kWideItems;
    const auto is = p.wide ? cut(small, piece_keys(keys_small, kSlotsWide, kMinPieceWide), kMostWhole, kMaxSmallPieces, 1)
                           : cut(small, piece_keys(keys_small, kSlotsSmall, kMinPieceSmall), 0, kMaxSmallPieces, 1);
    auto it = cut(tiles, piece_keys(keys_tiles, kSlotsTile, kMinPieceTile), 0, kMaxTilePieces, kTileRows8 / kSmallCols);
    if (it.size() > (size_t)kCus) std::reverse(it.begin() + kCus, it.begin() + std::min<size_t>(it.size(), 2 * kCus));
    p.n_small = (int)is.size();
    p.n_tiles = (int)it.size();
    p.n_merge = (int)merges.size();

    p.meta.assign(kUnitsInt, 0);
    std::memcpy(p.meta.data() + kTurnsInt, turns.data(), std::min<size_t>(turns.size(), 64) * sizeof(double));
    p.meta.insert(p.meta.end(), units.begin(), units.end());
    auto put = [&](const auto &items) {
        const int off = (int)p.meta.size();
        for (const auto &x : items) p.meta.insert(p.meta.end(), x.second.begin(), x.second.end());
        return off;
    };
    p.off_small = put(is);
    p.off_tiles = put(it);
    p.off_merge = (int)p.meta.size();
    for (const auto &m : merges) p.meta.insert(p.meta.end(), m.begin(), m.end());
    return ORTHRUS_OK;
}

}  // namespace orthrus
