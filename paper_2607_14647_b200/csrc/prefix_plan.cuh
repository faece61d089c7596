// Work partition of the shared-prefix attention: plain integer arithmetic, compiled for the device (prefix_attn.cu) and
// for the host (the tests walk every segment of it on the CPU).
//
// A group of requests with a shared prefix is a matrix of query rows per kv head: its tokens x the q heads of the kv
// head, row R = token * group_size + head.  A tile is floor(128 / group_size) whole tokens (at most 128 rows, the lanes
// of tensor memory); a unit is two tiles (dual: both see every key block) or the last odd tile (single: its key blocks
// are dealt to the CTA's two softmax teams in turn).  An item is (group, kv head, unit): `blocks` blocks of kBlock keys.
// The items of a call, in this order, are a stream of known cost that is cut into one segment of equal cost per CTA; a
// cut may fall inside an item, between two key blocks.  An item cut m times is computed in m + 1 pieces: the first in
// slot 2 s + 1 of the segment s it begins in, every other in slot 2 s of its segment.
#pragma once

#ifdef __CUDACC__
#define DCUT_HD __host__ __device__ __forceinline__
#else
#define DCUT_HD static inline
#endif

namespace dcut_prefix {

constexpr int kBlock = 64;            // keys per block: four pages (why 64: prefix_attn.cu)
constexpr int kTileRows = 128;
constexpr int kSlotRows = 2 * kTileRows;
constexpr int kMaxSegs = 256;

// Cost of a key block and of an item beyond its blocks; only the ratios matter.  A block of a single lasts as long as one of a
// dual (both are a chain of hand-overs), and an item costs about six blocks beyond its own: filling the chain, draining
// it and writing 256 rows.  Measured, (dual, single, item) on 48 requests of 64q/8kv heads in three groups, one of them
// without a prefix / on 64 requests of 32q/8kv behind 4099 keys (no other batch was tried): (16, 10, 30) 257 / 166 us, (16, 10, 100) 179 / 170,
// (16, 13, 100) 161 / 158, (16, 16, 60) 185 / 158, (16, 16, 100) 157 / 157, (16, 20, 80) 161 / 159.
constexpr long long kCostDual = 16, kCostSingle = 16, kCostItem = 100;

struct Group {                        // 16 bytes
    int q0;                           // first packed token
    int tokens;
    int len;                          // shared positions
    int pad;
};
struct Seg {                          // a boundary: before block b of item (g, h, u)
    int g, h, u, b;
};
struct Cut {                          // what is merged at a boundary (pieces = 0: nothing)
    int pieces, kv_head, q0, tokens;  // q0, tokens: the unit's packed tokens
};
struct Item {
    int g, h, u;
    int b0, b1, blocks;               // this piece's key blocks, the item's in all
    int dual;
    int q0, tokens;                   // first packed token of the unit, its tokens
    int len;                          // shared positions
};

DCUT_HD int tile_tokens(int group_size) { return kTileRows / group_size; }
DCUT_HD int n_tiles(const Group& g, int group_size) { return (g.tokens + tile_tokens(group_size) - 1) / tile_tokens(group_size); }
DCUT_HD int n_units(const Group& g, int group_size) { return (n_tiles(g, group_size) + 1) >> 1; }
DCUT_HD int n_blocks(const Group& g) { return (g.len + kBlock - 1) / kBlock; }
DCUT_HD long long unit_cost(const Group& g, int dual) { return kCostItem + n_blocks(g) * (dual ? kCostDual : kCostSingle); }
DCUT_HD long long head_cost(const Group& g, int group_size) {
    const int t = n_tiles(g, group_size);
    return (t >> 1) * unit_cost(g, 1) + (t & 1) * unit_cost(g, 0);
}

// segments that get work: no more than leave each at least one dual block's worth
DCUT_HD int n_active(long long total, int n_seg) {
    const long long most = total / kCostDual;
    return most < 1 ? 1 : most < n_seg ? (int)most : n_seg;
}

// Boundary s of n_seg: cost[g] = cost of the stream before group g, cost[G] = total.
DCUT_HD Seg boundary(int s, int n_seg, const Group* groups, const long long* cost, int G, int group_size, int n_kv_heads) {
    Seg r = {G, 0, 0, 0};
    const long long total = cost[G];
    if (s == 0) {
        r.g = 0;
        return r;
    }
    const int n = n_active(total, n_seg);
    if (s >= n) return r;
    const long long pos = (total / n) * s + (total % n) * s / n;
    int lo = 0, hi = G;               // largest g with cost[g] <= pos: a group that costs nothing is never found
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cost[mid] <= pos) lo = mid; else hi = mid;
    }
    r.g = lo;
    const Group g = groups[lo];
    const long long hc = head_cost(g, group_size), dc = unit_cost(g, 1);
    long long rem = pos - cost[lo];
    r.h = (int)(rem / hc);
    if (r.h >= n_kv_heads) r.h = n_kv_heads - 1;
    rem -= r.h * hc;
    const int t = n_tiles(g, group_size), last = n_units(g, group_size) - 1;
    r.u = (int)(rem / dc);
    if (r.u > last) r.u = last;
    rem -= r.u * dc + kCostItem;
    const int dual = 2 * r.u + 1 < t, nb = n_blocks(g);
    long long b = rem <= 0 ? 0 : rem / (dual ? kCostDual : kCostSingle);
    r.b = b >= nb ? (nb > 0 ? nb - 1 : 0) : (int)b;
    return r;
}

DCUT_HD bool same_item(const Seg& a, const Seg& b) { return a.g == b.g && a.h == b.h && a.u == b.u; }

DCUT_HD void unit_tokens(const Group& g, int u, int group_size, int* q0, int* tokens) {
    const int first = 2 * u * tile_tokens(group_size), left = g.tokens - first, most = 2 * tile_tokens(group_size);
    *q0 = g.q0 + first;
    *tokens = left < most ? left : most;
}

// The merge at boundary b (1 .. n_seg - 1): the item that it cuts, if it is the first boundary inside that item.
DCUT_HD Cut cut_at(int b, int n_seg, const Seg* segs, const Group* groups, int G, int group_size) {
    Cut c = {0, 0, 0, 0};
    const Seg s = segs[b];
    if (b < 1 || s.b <= 0 || s.g >= G) return c;
    if (same_item(segs[b - 1], s) && segs[b - 1].b > 0) return c;
    int m = 1;
    while (b + m < n_seg && same_item(segs[b + m], s) && segs[b + m].b > 0) ++m;
    c.pieces = m + 1;
    c.kv_head = s.h;
    unit_tokens(groups[s.g], s.u, group_size, &c.q0, &c.tokens);
    return c;
}

// Walks the items of one segment.
struct Walk {
    Seg at, end;
    int G, group_size, n_kv_heads;
};
DCUT_HD bool next_item(Walk& w, const Group* groups, Item* it) {
    for (;;) {
        if (w.at.g >= w.G || w.at.g > w.end.g) return false;
        const bool in_last = same_item(w.at, w.end);
        if (in_last && w.at.b >= w.end.b) return false;
        if (w.at.g == w.end.g && (w.at.h > w.end.h || (w.at.h == w.end.h && w.at.u > w.end.u))) return false;
        const Group g = groups[w.at.g];
        const int units = n_units(g, w.group_size);
        if (units == 0) {             // a group without tokens has no items
            ++w.at.g;
            continue;
        }
        it->g = w.at.g;
        it->h = w.at.h;
        it->u = w.at.u;
        it->blocks = n_blocks(g);
        it->b0 = w.at.b;
        it->b1 = in_last ? w.end.b : it->blocks;
        it->dual = 2 * w.at.u + 1 < n_tiles(g, w.group_size);
        it->len = g.len;
        unit_tokens(g, w.at.u, w.group_size, &it->q0, &it->tokens);
        w.at.b = 0;
        if (in_last) {
            w.at = w.end;
        } else if (++w.at.u == units) {
            w.at.u = 0;
            if (++w.at.h == w.n_kv_heads) {
                w.at.h = 0;
                ++w.at.g;
            }
        }
        return true;
    }
}
DCUT_HD bool is_whole(const Item& it) { return it.b0 == 0 && it.b1 == it.blocks; }
DCUT_HD int slot_of(const Item& it, int seg) { return 2 * seg + (it.b0 > 0 ? 0 : 1); }

}  // namespace dcut_prefix
