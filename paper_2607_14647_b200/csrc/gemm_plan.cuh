// How a GEMM launch runs (layer.cu): tile width, one SM or a pair per tile, K whole or cut between the SMs of a pair.  Plain
// integer arithmetic, for the device code and for the host (the tests check the choices on the CPU).
#pragma once
#include <limits.h>

#ifdef __CUDACC__
#define DCUT_GEMM_HD __host__ __device__
#else
#define DCUT_GEMM_HD
#endif

namespace dcut_gemm {

constexpr int BM = 128, BN = 256, BK = 64;

// Widths of the output tile that the one-SM mode may use: 256, 224, ..., 64 columns.  A narrower tile costs a little
// efficiency per flop and buys more tiles, which is what a GEMM with fewer than one wave of 128 x 256 tiles needs
// (T = 600, N = 4096: 80 tiles for 148 SMs at width 256, 130 at width 160).  One tensor map of the weight per width
// (box = half the width in rows: a B tile is loaded as two halves, which is also how the SwiGLU tile is put together).
constexpr int kNumBn = 7;
DCUT_GEMM_HD constexpr int bn_of(int i) { return BN - 32 * i; }
constexpr unsigned kBnMaskAll = (1u << kNumBn) - 1;
constexpr unsigned kBnMaskSwiGLU = 0x55;   // widths whose halves are whole 32-column epilogue steps: 256, 192, 128, 64
constexpr int kPlanRows = 72;
constexpr int kSplitCost = 50;             // what the exchange of partial sums between the two SMs costs
// dcut_linear with few k-blocks: one SM per tile only.  The costs are fitted to K of 4096 and more; with up to 512 a tile's cost is
// its epilogue and the start, which pairs and split K make dearer.  One SM against the plan's choice with them, us, no
// activation: K = 64, 8 x 6147 6.0 / 8.1, 333 x 6147 9.1 / 12.3; K = 384, 333 x 2048 6.0 / 7.0, 8 x 2048 5.6 / 5.2; K = 640,
// 8 x 2048 6.5 / 5.7, 700 x 6147 18.2 / 19.0.
// e4m3 operands have twice the elements in as many k-blocks, so the rule holds up to K = 1024 there.  The same comparison, geometric mean over 25 shapes
// of 8 to 1088 rows and 1024 to 12288 columns: pairs take 1.20 of the time of one SM per tile at K = 256 (gated 1.14), 1.14 at 512 (1.14), 1.11 at 768
// (1.13), 1.08 at 1024 (1.12); at K = 1024 8 x 2048 6.1 / 5.7, 64 x 1024 6.0 / 5.7 (the most that the rule loses), 333 x 6144 8.3 / 10.9, 1088 x 2048 8.4 / 10.8.
constexpr int kShortK = 512;
constexpr int kPlanPair = 8, kPlanSplit = 16;

struct Shape {
    int N_out, K, T_cap;
    bool gated;                  // two weights share a tile: a tile has half its width in output columns
    bool may_split;              // the epilogue can take its sums in two halves of K
    bool short_k_alone;          // kShortK applies
};
struct Device {
    int sm_count, n_clusters;    // n_clusters: clusters of two CTAs that run at once (0: launch without clusters)
    bool pair_mode;
    int force;                   // -1, or the plan that every length takes where it can
    unsigned bn_mask;            // widths that may be chosen (bit i: bn_of(i)); bit 0 is always added
};
struct Launch {
    int grid;
    bool pairs;                  // the pair modes may be chosen
    unsigned bn_mask;
    unsigned char by_m[kPlanRows];   // the plan for 1, 2, ... row blocks of 128; the last entry serves all larger counts
};

inline int tiles_of(const Shape& s, int i) {
    const int per = s.gated ? bn_of(i) >> 1 : bn_of(i);
    return (s.N_out + per - 1) / per;
}

// The cheapest way to run m1 row blocks under a model fitted to measurements on the four projections of an 8B-class
// layer at 17 packed lengths from 64 to 1088 (every width, every mode): time = waves x (4 bn + 1664) on one SM per
// tile, waves x (7 bn + 800) on a pair, half a one-SM tile + kSplitCost for a pair splitting K.  (A pair tile moves two
// thirds of the bytes per flop from L2 and its MMAs are issued at about 0.57 of the one-SM rate per column; the
// constants stand for what a tile costs whatever its width.)  Over those 68 cases the pick reaches the best measured
// single choice to within a percent (geometric mean).  Returns the width index, + kPlanPair or + kPlanSplit; the
// wider tile wins ties.
inline int choose(const Shape& s, int m1, unsigned bn_mask, int n_pairs, bool may_split, int grid) {
    const int m2 = (m1 + 1) / 2;
    int best = 0, best_cost = INT_MAX;
    for (int i = 0; i < kNumBn; ++i) {
        if (!((bn_mask >> i) & 1)) continue;
        const int bn = bn_of(i), n_tiles = tiles_of(s, i);
        const int cost1 = ((m1 * n_tiles + grid - 1) / grid) * (4 * bn + 1664);
        if (cost1 < best_cost) {
            best_cost = cost1;
            best = i;
        }
        if (n_pairs > 0) {
            const int cost2 = ((m2 * n_tiles + n_pairs - 1) / n_pairs) * (7 * bn + 800);
            if (cost2 < best_cost) {
                best_cost = cost2;
                best = kPlanPair + i;
            }
            // both SMs of a pair on one 128-row tile, half of K each (only as a single wave: a tile per pair)
            if (may_split && m1 * n_tiles <= n_pairs) {
                const int cost3 = (4 * bn + 1664) / 2 + kSplitCost;
                if (cost3 < best_cost) {
                    best_cost = cost3;
                    best = kPlanSplit + i;
                }
            }
        }
    }
    return best;
}

// The choice depends on T only through the number of 128-row blocks, so the host tabulates it per launch and the kernel
// looks it up after reading T.
inline Launch plan(const Shape& s, const Device& d) {
    Launch l;
    l.bn_mask = d.bn_mask | 1u;
    // work items at the narrowest width that may be chosen (the widest has the fewest per row block)
    int narrow = 0;
    for (int i = 0; i < kNumBn; ++i)
        if ((l.bn_mask >> i) & 1) narrow = i;
    const int m_cap = (s.T_cap + BM - 1) / BM, n_work = m_cap * ((tiles_of(s, 0) * BN + bn_of(narrow) - 1) / bn_of(narrow));
    l.pairs = d.n_clusters > 0 && d.pair_mode && !(s.short_k_alone && s.K <= kShortK);
    // persistent: at most one CTA per SM; with clusters always an even number (the kernel holds cta_group::2 instructions),
    // with room for either mode
    l.grid = d.n_clusters > 0 ? 2 * (n_work < d.n_clusters ? n_work : d.n_clusters) : n_work < d.sm_count ? n_work : d.sm_count;
    const int n_pairs = l.pairs ? l.grid >> 1 : 0;
    const bool two_halves = l.pairs && s.may_split && s.K >= 2 * BK;
    for (int m = 1; m <= kPlanRows; ++m) {
        if (m > m_cap && m > 1) {                    // no launch has more row blocks than that: the rest of the table repeats
            l.by_m[m - 1] = l.by_m[m - 2];
            continue;
        }
        // A pair that splits K has one tile and is done: the tiles have to fit one wave of pairs, at every length that takes
        // this entry.  The last entry's lengths have no bound here.
        const bool may_split = two_halves && !(m == kPlanRows && m_cap > kPlanRows);
        const int f = d.force, i = f & 7;
        bool forced = f >= 0 && f < kPlanSplit + kNumBn && i < kNumBn && ((l.bn_mask >> i) & 1);
        if (f >= kPlanPair) forced = forced && l.pairs;
        if (f >= kPlanSplit) forced = forced && may_split && m * tiles_of(s, i) <= n_pairs;
        l.by_m[m - 1] = (unsigned char)(forced ? f : choose(s, m, l.bn_mask, n_pairs, may_split, l.grid));
    }
    return l;
}

}  // namespace dcut_gemm
