// Host rules of the drafted rows' attention: how a call is cut, and its launch.
#pragma once

#include "common.h"

#include <algorithm>

namespace lvlm {

// Runs dealt out by the lengths (long calls): pairs at most; runs of one pair at most (that the fold takes).
constexpr int kSharePairs = 512, kShareRuns = 64;

// How a call is cut: rows of a workgroup (32, 64, 128 or 256, by how its waves share entries and rows), and runs of a pair's
// entries.  Many rows to a workgroup read an entry for all of them at once; few rows make many workgroups of few tiles each; runs
// make more still, and cost a second launch that folds their sums.  What a cut takes is put together from the numbers below, and
// the cut that takes least is done.  The numbers are a fit to the times of 766 shapes (4 to 512 pairs, 1 to 1536 rows, 64 to
// 16384 entries, both types and head dimensions) in all forms and up to 64 runs.  Of 778 timed once more with the present kernels the cut
// they choose takes 2.8 % longer than the shape's best on average, more than 10 % in 46 and 50 % at most (16 x 1024 rows x 4500 entries of 64
// channels).  Against splitting until there are 512 workgroups and 256 rows where there are more than
// 128, us: 4 pairs x 28 rows x 512 entries of 128 channels 12.6 -> 7.8, 8 x 384 x 2048 35 -> 17, 32 x 384 x 512 32 -> 13, 64 x 1 x
// 2048 23 -> 16, 128 x 192 x 2048 72 -> 44, 512 x 768 x 128 117 -> 70; with 256 rows where they are right 32 x 384 x 16384
// 160 -> 134.
constexpr int kFewRows = 4;
constexpr double kDealUs = 25;   // calls that take longer deal their runs out by the lengths
inline int few_rows(long long M) { return M <= 1 ? 1 : M <= 2 ? 2 : kFewRows; }
struct TreeForm {
    int rb, kw, tps;        // blocks of 32 rows to a wave; waves side by side over entries; tiles of a wave in a step
    float workgroup, tile;  // us: a workgroup without entries; a tile of 32 entries in one of its waves
    float shared;           // workgroups that share a compute unit, of what they would take in turn (1: they do not share)
    float alone;            // bytes per us that a workgroup gets from memory (1.6 times as many where the cache holds all entries)
    float busy;             // us of a compute unit for a tile of one row block, on a chip that has all it can do
    int rows() const { return rb == 0 ? kFewRows : 32 * rb * (4 / kw); }     // (rb 0: fp32, few rows on the vector ALUs; a workgroup takes 0.6 us more for each,
                                                                        // a tile as long again)
    int threads() const { return rb == 0 ? 512 : 256; }
};
constexpr int kTreeForms = 4;
inline const TreeForm *tree_forms(const lvlm_tree_desc &d, int &n) {
    static constexpr TreeForm kBf16[2][kTreeForms] = {
        {{1, 4, 1, 3.6f, 0.69f, 0.66f, 180e3f, 0.07f}, {1, 2, 1, 3.6f, 0.75f, 0.63f, 52e3f, 0.29f},
         {1, 1, 1, 3.7f, 0.69f, 0.62f, 8.5e3f, 0.11f}, {2, 1, 2, 8.9f, 0.58f, 1.f, 92e3f, 0.74f}},
        {{1, 4, 1, 4.2f, 0.77f, 1.f, 53e3f, 0.14f}, {1, 2, 1, 3.9f, 0.69f, 0.81f, 20e3f, 0.39f},
         {1, 1, 1, 4.5f, 0.82f, 0.62f, 14.5e3f, 0.68f}, {2, 1, 2, 8.6f, 0.92f, 1.f, 92e3f, 0.71f}}};
    static constexpr TreeForm kF32[2][kTreeForms] = {
        {{0, 4, 1, 3.3f, 0.25f, 0.6f, 50e3f, 0.05f}, {1, 4, 1, 4.1f, 2.8f, 1.f, 34e3f, 0.78f}, {1, 2, 1, 4.3f, 2.5f, 1.f, 14e3f, 1.5f},
         {1, 1, 1, 4.4f, 2.4f, 1.f, 29e3f, 2.8f}},
        {{0, 2, 1, 3.3f, 0.25f, 0.6f, 50e3f, 0.05f}, {1, 2, 1, 5.7f, 5.0f, 1.f, 52e3f, 2.8f}, {1, 1, 1, 6.9f, 4.4f, 1.f, 56e3f, 5.3f}, {}}};
    n = d.dtype == LVLM_BF16 || d.hd == 64 ? kTreeForms : 3;
    return d.dtype == LVLM_BF16 ? kBf16[d.hd == 128] : kF32[d.hd == 128];
}

inline TreeWs tree_cut(const lvlm_tree_desc &d) {
    constexpr int kUnits = 256;             // compute units
    const long long M = (long long)(d.Hq / d.Hkv) * d.T, pairs = (long long)d.B * d.Hkv;
    const int bound = d.len_bound > 0 ? d.len_bound : d.Lmax, es = d.dtype == LVLM_BF16 ? 2 : 4;
    const double bytes = (double)pairs * bound * d.hd * es * 2, tiles = (double)pairs * bound / 32 / kUnits;
    int n_forms;
    const TreeForm *forms = tree_forms(d, n_forms);
    TreeWs w{};
    double best = 0;
    for (int i = 0; i < n_forms; ++i) {
        const TreeForm &f = forms[i];
        if (f.rb == 0 && M > kFewRows) continue;
        const float begin = f.rb == 0 ? f.workgroup + 0.6f * (float)(few_rows(M) - 1) : f.workgroup;
        const float tile = f.rb == 0 ? f.tile * (float)(few_rows(M) + 1) : f.tile;
        const int step = 32 * f.kw * f.tps;
        const long long blocks = (M + f.rows() - 1) / f.rows(), steps = ((long long)bound + step - 1) / step;
        for (int wanted : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
            if (wanted > steps) break;
            const long long run = (steps + wanted - 1) / wanted, split = (steps + run - 1) / run;
            // a launch's most, half of 2^32 threads (the fold's: by pairs)
            if (pairs * blocks * split * f.threads() >= (1ll << 31) || (split > 1 && pairs > 65535)) break;
            const double per_unit = (double)(pairs * blocks * split) / kUnits, whole = (double)((pairs * blocks * split + kUnits - 1) / kUnits);
            const double rounds = per_unit > 8 ? per_unit : whole;
            double t = (begin + tile * (double)(run * f.tps)) * (rounds <= 1 ? 1.0 : rounds * f.shared);
            t = std::max(t, begin + (double)std::min<long long>(run * step, bound) * d.hd * es * 2 / (f.alone * (bytes > 200e6 ? 1.0 : 1.6)));
            t = std::max(t, begin + std::max(bytes / 14e6, tiles * f.busy) * (double)blocks);      // 14 TB/s from the L2s
            t = std::max(t, 1.0 + bytes / 7e6);                                                          // ... 7 from memory
            if (split > 1) t += 6.0 + (double)pairs * split * M * d.hd * 8 / 5.5e6;
            const bool dealt = split > 1 && pairs <= kSharePairs && t > kDealUs;
            if (!dealt && t > kDealUs) t *= 1.1;    // (its lengths may be as uneven as they like)
            if (w.n_split == 0 || t < best) {
                best = t;
                w.form = i;
                w.n_split = (int)split;
                w.run = (int)(run * step);
                w.step = step;
                w.dealt = dealt;
                w.row_blocks = (int)blocks;
            }
        }
    }
    if (w.n_split > 1) {
        w.part_ml = align_up((size_t)(pairs * w.n_split * M) * d.hd * 4, 256);
        w.places = w.part_ml + align_up((size_t)(pairs * w.n_split * M) * 8, 256);
        w.total = w.places + (w.dealt ? align_up((size_t)pairs * 8, 256) : 0);
    }
    return w;
}

// Workgroups of the launch.  Numbers with the same remainder modulo 8 run on one XCD: the row blocks of a run of entries follow each
// other there and share its L2.  per_xcd: too few runs for that are dealt out evenly, row block by row block, so many to an XCD (else 0).
inline long long tree_workgroups(const lvlm_tree_desc &d, const TreeWs &w, long long &per_xcd) {
    const long long units = (long long)d.B * d.Hkv * w.n_split, even = (units * w.row_blocks + 7) / 8, by_unit = (units + 7) / 8 * w.row_blocks;
    per_xcd = by_unit > even + even / 8 ? even : 0;
    return 8 * (per_xcd ? even : by_unit);
}

}  // namespace lvlm
