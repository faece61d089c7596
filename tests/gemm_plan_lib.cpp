// Host build of the GEMM's choice of tiles, for test_gemm_plan.py.
#include "gemm_plan.cuh"

extern "C" void gemm_plan(int N, int K, int T_cap, int gated, int may_split, int short_k_alone, int sm_count, int n_clusters, int pair_mode, int force,
                          unsigned bn_mask, unsigned char* by_m, int* grid) {
    const dcut_gemm::Launch l = dcut_gemm::plan(dcut_gemm::Shape{N, K, T_cap, gated != 0, may_split != 0, short_k_alone != 0},
                                                dcut_gemm::Device{sm_count, n_clusters, pair_mode != 0, force, bn_mask});
    for (int m = 0; m < dcut_gemm::kPlanRows; ++m) by_m[m] = l.by_m[m];
    *grid = l.grid;
}
