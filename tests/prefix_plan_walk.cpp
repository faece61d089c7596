// Host walk of the shared-prefix work partition: every key block of every item exactly once, every piece where the
// merge looks for it.  Returns 0, or the number of the first check that failed.
#include <map>
#include <tuple>
#include <vector>
#include "prefix_plan.cuh"
using namespace dcut_prefix;

extern "C" int walk(int G, const int* tokens, const int* lens, int group_size, int n_kv_heads, int n_seg, long long* most, long long* least) {
    std::vector<Group> groups(G + 1);
    std::vector<long long> cost(G + 1, 0);
    int q0 = 0;
    for (int g = 0; g < G; ++g) {
        groups[g] = Group{q0, tokens[g], lens[g], 0};
        q0 += tokens[g];
        cost[g + 1] = cost[g] + n_kv_heads * head_cost(groups[g], group_size);
    }
    std::vector<Seg> segs(n_seg + 1);
    for (int s = 0; s <= n_seg; ++s) segs[s] = boundary(s, n_seg, groups.data(), cost.data(), G, group_size, n_kv_heads);
    std::map<std::tuple<int, int, int>, int> done;           // blocks of each item so far
    std::map<std::tuple<int, int, int>, std::vector<int>> pieces;
    std::map<int, std::tuple<int, int, int>> slots;
    std::map<std::tuple<int, int, int>, Item> items;
    *most = 0;
    *least = 1ll << 60;
    for (int s = 0; s < n_seg; ++s) {
        Walk w = {segs[s], segs[s + 1], G, group_size, n_kv_heads};
        Item it;
        long long c = 0;
        for (int n = 0; next_item(w, groups.data(), &it); ++n) {
            if (n > 1000000) return 1;
            const auto key = std::make_tuple(it.g, it.h, it.u);
            if (it.g < 0 || it.g >= G || it.h < 0 || it.h >= n_kv_heads || it.tokens < 1) return 2;
            if (it.q0 < groups[it.g].q0 || it.q0 + it.tokens > groups[it.g].q0 + groups[it.g].tokens) return 3;
            if (it.dual != (it.tokens > tile_tokens(group_size))) return 4;
            if (it.b0 != (done.count(key) ? done[key] : 0) || it.b1 < it.b0 || it.b1 > it.blocks) return 5;
            if (it.blocks > 0 && it.b1 == it.b0) return 6;   // a piece without blocks
            if (it.blocks == 0 && done.count(key)) return 7; // an item without blocks, twice
            done[key] = it.b1;
            items[key] = it;
            if (!is_whole(it)) {
                const int slot = slot_of(it, s);
                if (slot < 0 || slot >= 2 * n_seg || slots.count(slot)) return 8;
                slots[slot] = key;
                pieces[key].push_back(slot);
            }
            c += kCostItem + (it.b1 - it.b0) * (it.dual ? kCostDual : kCostSingle);
        }
        if (c > *most) *most = c;
        if (c < *least) *least = c;
    }
    for (int g = 0; g < G; ++g)
        for (int h = 0; h < n_kv_heads; ++h)
            for (int u = 0; u < n_units(groups[g], group_size); ++u) {
                const auto key = std::make_tuple(g, h, u);
                if (!done.count(key) || done[key] != n_blocks(groups[g])) return 9;
            }
    std::map<std::tuple<int, int, int>, int> merged;
    for (int b = 1; b < n_seg; ++b) {
        const Cut c = cut_at(b, n_seg, segs.data(), groups.data(), G, group_size);
        if (c.pieces == 0) continue;
        const auto key = std::make_tuple(segs[b].g, segs[b].h, segs[b].u);
        if (merged[key]++) return 10;
        if (c.pieces != (int)pieces[key].size() || c.pieces < 2) return 11;
        for (int i = 0; i < c.pieces; ++i)
            if (pieces[key][i] != (i == 0 ? 2 * (b - 1) + 1 : 2 * (b + i - 1))) return 12;
        if (c.kv_head != segs[b].h || c.q0 != items[key].q0 || c.tokens != items[key].tokens) return 13;
    }
    for (auto& p : pieces)
        if (!merged.count(p.first)) return 14;
    return 0;
}
