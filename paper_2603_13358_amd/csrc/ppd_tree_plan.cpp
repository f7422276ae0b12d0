// Tile list of tree and weighted attention: which columns of which sequence meet which keys in which workgroup.
#include <algorithm>

#include "ppd_ops.h"

namespace ppd {

bool build_tree_plan(const ppd_shape& s, const int32_t* L, const int32_t* n, int32_t B, bool weighted, int num_cus, TreePlan* plan) {
    const int G = s.num_q_heads / s.num_kv_heads, Hkv = s.num_kv_heads, D = s.head_dim;
    plan->items.clear();
    plan->groups.clear();
    plan->weighs.clear();
    plan->partial_floats = 0;
    // Two workgroups are resident on a compute unit.  A tile costs its keys and a start of about kTileKeys keys' time; the launch
    // lasts as long as its even share and, for what the last tiles stick out, half a tile.
    constexpr int kTileKeys = 256;
    const double slots = 2.0 * num_cus;
    double keys = 0, fewest = 0;
    int32_t longest = 1;
    for (int i = 0; i < B; ++i) {
        const int64_t blocks = ((int64_t)n[i] * G + kTreeCols - 1) / kTreeCols;
        keys += (double)blocks * Hkv * ((double)L[i] + n[i]);
        fewest += (double)blocks * Hkv * (((double)L[i] + n[i]) / kMaxTreeChunk + 1);
        longest = std::max(longest, L[i] + n[i]);
    }
    if (fewest > kMaxTiles) return false;
    int32_t chunk = kMaxTreeChunk;
    double best = -1;
    for (int32_t c = kMaxTreeChunk; c >= kTreeStep; c /= 2) {
        double tiles = 0;
        for (int i = 0; i < B; ++i) {
            const int64_t total = (int64_t)L[i] + n[i];
            tiles += (double)(((int64_t)n[i] * G + kTreeCols - 1) / kTreeCols) * Hkv * (double)((total + c - 1) / c);
        }
        if (tiles > kMaxTiles) break;
        const double est = (keys + tiles * kTileKeys) / slots + 0.5 * (std::min(c, longest) + kTileKeys);
        const double rounds_floor = std::min(c, longest) + kTileKeys;  // no launch is shorter than its longest tile
        const double cost = std::max(est, rounds_floor);
        if (best < 0 || cost < best) {
            best = cost;
            chunk = c;
        }
    }
    int32_t grow0 = 0;
    for (int i = 0; i < B; ++i) {
        const int32_t total = L[i] + n[i];
        const int64_t cols = (int64_t)n[i] * G;
        const int32_t nsplit = (total + chunk - 1) / chunk;
        for (int h = 0; h < Hkv; ++h) {
            for (int64_t c0 = 0; c0 < cols; c0 += kTreeCols) {
                const int32_t nc = (int32_t)std::min<int64_t>(kTreeCols, cols - c0);
                const int64_t stride = (int64_t)nc * (D + 2);
                if (nsplit > 1) plan->groups.push_back({h, grow0, (int32_t)c0, nc, nsplit, 0, plan->partial_floats, stride});
                for (int32_t p = 0; p < nsplit; ++p) {
                    TreeItem it{};
                    it.seq = i;
                    it.kvh = h;
                    it.grow0 = grow0;
                    it.col0 = (int32_t)c0;
                    it.ncols = nc;
                    it.L = L[i];
                    it.kv_total = total;
                    it.kv_begin = p * chunk;
                    it.kv_end = std::min(total, (p + 1) * chunk);
                    it.split = nsplit > 1;
                    it.part_off = plan->partial_floats + p * stride;
                    plan->items.push_back(it);
                }
                if (nsplit > 1) plan->partial_floats += stride * nsplit;
            }
            if (weighted)
                for (int32_t t = 0; t < total; t += kWeighKeys) plan->weighs.push_back({i, h, grow0, (int32_t)cols, L[i], total, t, 0});
        }
        grow0 += n[i];
    }
    plan->rows = grow0;
    std::stable_sort(plan->items.begin(), plan->items.end(), [](const TreeItem& a, const TreeItem& b) { return a.kv_end - a.kv_begin > b.kv_end - b.kv_begin; });
    return true;
}

}  // namespace ppd
