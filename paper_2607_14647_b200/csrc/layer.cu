// dcut_layer_forward: one pre-norm decoder layer over the ragged packed batch (full-layer workload).
//
//   h1 = x + Wo . Attn(RoPE(Wqkv . RMSNorm(x)))        y = h1 + Wd . (SiLU(Wg . n2) * (Wu . n2)),  n2 = RMSNorm(h1)
//
// Kernels in this file
//   rmsnorm_kernel        one CTA per packed token, fp32 sum of squares, bf16 out
//   rope_append_kernel    rotate-half RoPE on q and k heads, K/V of the new tokens written into the paged cache at
//                         position L_i + t, q written as the attention kernel's [T, Hq, Dh] input
//   gemm_tcgen05_kernel   C[M, N] = A[M, K] . B[N, K]^T on the 5th-generation tensor cores.  Persistent; launched as
//                         clusters of two CTAs.  After reading the packed length it looks up how to run: 128-row
//                         tiles on single SMs (tcgen05.mma M128 K16), 256-row tiles on pairs of SMs (cta_group::2,
//                         M256, each CTA loading half of B), or a pair sharing one 128-row tile with half of K each;
//                         and how wide the tile is (256, 224, ..., 64 columns = the MMA's N).  Operands
//                         are staged by TMA as 128-byte-swizzled K-major tiles (BK = 64); one elected lane issues the
//                         MMAs and releases stages with tcgen05.commit; two accumulators in tensor memory let the four
//                         epilogue warps (tcgen05.ld) work on one tile while the next is being multiplied.
//                         Operands are bf16 or (dcut_linear8) e4m3: a k-block is 128 bytes of a row either way, so tiles, stages,
//                         swizzle and descriptors are the same and an MMA takes twice the elements.
//                         Epilogues: plain bf16, + residual, SwiGLU (the B tile is 128 gate rows and the 128 matching
//                         up rows, so silu(g) * u is formed in registers and the [T, 2I] intermediate never exists),
//                         row argmax (the LM head fused with acceptance: the logits are never stored), or dcut_linear's:
//                         bias, activation, gate and residual in fp32 for any N, K and row strides (the tensor maps' zero
//                         fill completes the last tile and the last k-block).  Measured: 7 rows, K = 4096, N = 6144 with
//                         bias 15 us (50 MB of weights: 8 us at the copy rate, the rest is fixed: launch, first loads, the
//                         pair's exchange); 1088 rows to N = 12288 with gelu_tanh 110 us (its products alone 88; operands
//                         from L2 bound them: 92 bytes per clock and SM at the full MMA rate, about 60 to be had).
// M is ragged and known only on the device (T = cu_q[B]): grids are sized for T_cap, CTAs without work fall through,
// rows past T are computed on whatever the buffers hold and never stored.  Every kernel is launched with programmatic
// dependent launch and waits for its predecessor before touching global memory.
#include <cstddef>
#include <cuda.h>
#include <cuda_bf16.h>
#include <limits.h>
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include "activation.cuh"
#include "dcut_internal.h"
#include "gemm_plan.cuh"
#include "tcgen05.cuh"

namespace {

using namespace dcut_gemm;

constexpr int kGemmStages = 4;
constexpr int kATile = BM * BK * 2;            // 16 KB
constexpr int kBTile = BN * BK * 2;            // 32 KB
constexpr int kGemmStageBytes = kATile + kBTile;
constexpr int kGemmThreads = 192;              // warp 0: TMA, warp 1: MMA + TMEM owner, warps 2-5: epilogue
constexpr int kTmemCols = 512;              // two 128 x 256 fp32 accumulators
constexpr int kMaxStages = 12;                 // a narrow tile's stage is smaller: more of them fit the same operand area
constexpr int kGemmSmem = kGemmStages * kGemmStageBytes + 1024 /* align */ + 512 /* two sets of barriers, tmem ptr */;
constexpr int kLinearSmem = kGemmSmem + 4 * (32 * 33 + 32 + 2 * BN) * 4;   // + LinearShared of four epilogue warps

enum GemmMode { kPlain = 0, kResidual = 1, kSwiGLU = 2, kArgmax = 3, kLinear = 4, kLinearGated = 5, kLinear8 = 6, kLinear8Gated = 7 };
__host__ __device__ constexpr bool is_fp8(int mode) { return mode == kLinear8 || mode == kLinear8Gated; }        // e4m3 operands with scales
__host__ __device__ constexpr bool is_gated(int mode) { return mode == kSwiGLU || mode == kLinearGated || mode == kLinear8Gated; }   // two weights share a tile
__host__ __device__ constexpr bool is_linear(int mode) { return mode == kLinear || mode == kLinearGated || is_fp8(mode); }
__host__ __device__ constexpr bool may_split_k(int mode) { return mode == kPlain || mode == kResidual || mode == kLinear || mode == kLinear8; }
__host__ __device__ constexpr bool is_split_linear(int mode) { return is_linear(mode) && may_split_k(mode); }
// A k-block is 128 bytes of a row of either operand: 64 bf16 or 128 e4m3 elements.
__host__ __device__ constexpr int kb_elements(int mode) { return is_fp8(mode) ? 2 * BK : BK; }

struct BMaps {
    CUtensorMap m[kNumBn];
};
// The activations' tensor map with the full 128-row box and with a 64-row box: with at most 64 packed rows a tile's
// lower half would only be fetched to be ignored (at T = 64 the A tiles were more than half of what the SMs took in).
struct AMaps {
    CUtensorMap full, half;
};
// ------------------------------------------------------------------------------------------------ GEMM

struct GemmArgs {
    const int* cu_q;   // T = cu_q[B]
    int B;
    int N_out;         // columns of the output (kSwiGLU: the intermediate size I; otherwise N)
    int K;
    __nv_bfloat16* out;
    const __nv_bfloat16* residual;   // [T, N_out] or null
    unsigned long long* row_key;     // kArgmax: one packed (ordered maximum, ~column) word per row
    int V;                           // kArgmax: live columns (rows of the weight)
    const __nv_bfloat16 *bias, *bias2;   // kLinear*: [N_out] or null
    const float *a_scale, *w_scale, *w2_scale;   // kLinear8*: [T], [N_out], [N_out]
    long long ldo, ldr;              // kLinear*: elements from one row of out / residual to the next
    int T_cap;                       // kLinear*: rows that out has
    int act;                         // kLinear*: dcut_act
    int vec;                         // kLinear*: out and residual take 16-byte accesses at multiples of 8 columns
    unsigned char plan_by_m[kPlanRows];   // gemm_plan.cuh: for 1, 2, ... row blocks of 128 (the last entry serves all larger counts)
    int* status;
};

// the map of width index i; every address is formed statically (kernel parameter space)
__device__ __forceinline__ const CUtensorMap* pick_map(const BMaps& s, int i) {
    switch (i) {
        case 1: return &s.m[1];
        case 2: return &s.m[2];
        case 3: return &s.m[3];
        case 4: return &s.m[4];
        case 5: return &s.m[5];
        case 6: return &s.m[6];
        default: return &s.m[0];
    }
}

// ------------------------------------------------------------------------------------------------ dcut_linear's epilogue

// Shared memory of one epilogue warp: 32 rows x 32 columns of results on their way to rows that take no vectors, and the
// biases of the tile's columns.
constexpr int kStageRow = 33;
struct LinearShared {
    float stage[32 * kStageRow];
    float pad[32];                       // (16-byte alignment of what follows, whatever the row)
    float bias[BN];                      // gated: bias, then bias2, half each
    float scale[BN];                     // e4m3 operands: the columns' scales, in the same places
};
static_assert(sizeof(LinearShared) % 16 == 0 && offsetof(LinearShared, bias) % 16 == 0, "read in vectors");
static_assert(kLinearSmem - kGemmSmem == 4 * sizeof(LinearShared), "one per epilogue warp");

// Before the accumulator is complete: the biases (and scales) of a tile's columns, zeros where there are none.
template <int MODE>
__device__ __forceinline__ void linear_stage_bias(const GemmArgs& g, int n_tile, int bn, LinearShared& sh) {
    constexpr bool GATED = is_gated(MODE);
    const int lane = threadIdx.x & 31, width = GATED ? bn >> 1 : bn, col0 = n_tile * width;
    __syncwarp();                                                      // (the previous tile's have been read)
    for (int c = lane; c < width; c += 32) {
        const bool there = col0 + c < g.N_out;
        sh.bias[c] = there && g.bias ? __bfloat162float(g.bias[col0 + c]) : 0.0f;
        if (GATED) sh.bias[BN / 2 + c] = there && g.bias2 ? __bfloat162float(g.bias2[col0 + c]) : 0.0f;
        if (is_fp8(MODE)) sh.scale[c] = there ? g.w_scale[col0 + c] : 0.0f;
        if (is_fp8(MODE) && GATED) sh.scale[BN / 2 + c] = there ? g.w2_scale[col0 + c] : 0.0f;
    }
    __syncwarp();
}
__device__ __forceinline__ bool linear_by_vector(const GemmArgs& g, int col) { return g.vec && col + 32 <= g.N_out; }
// The residual that linear_finish32 adds in 32 columns of the warp's 32 rows, fetched before the accumulators are read: 32 columns
// of this thread's row, or column `lane` of every row.
struct LinearAhead {
    uint32_t r[32];
};
__device__ __forceinline__ void linear_fetch(const GemmArgs& g, int T, int row0, int col, LinearAhead& f) {
    const int lane = threadIdx.x & 31;
    if (!g.residual) return;
    if (linear_by_vector(g, col)) {
        if (row0 + lane >= T) return;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const uint4 r = *reinterpret_cast<const uint4*>(g.residual + (size_t)(row0 + lane) * g.ldr + col + 8 * v);
            f.r[4 * v] = r.x, f.r[4 * v + 1] = r.y, f.r[4 * v + 2] = r.z, f.r[4 * v + 3] = r.w;
        }
    } else if (col + lane < g.N_out) {
        const unsigned short* r = reinterpret_cast<const unsigned short*>(g.residual) + (size_t)row0 * g.ldr + col + lane;
#pragma unroll
        for (int i = 0; i < 32; ++i, r += g.ldr) f.r[i] = row0 + i < T ? *r : 0;
    }
}
// x (and, gated, u): 32 columns of this thread's row as the MMAs left them; a whole warp calls with its 32 rows; c = the
// first column within the tile.  Everything in fp32, one rounding at the store.  Rows of out and residual that take 16-byte
// accesses are read and written by the thread that owns the row.  Others (an odd N, say) would be 2-byte accesses to 32
// rows at a time, 32 lines each: they go through shared memory, so that a warp reads and writes 32 columns of one row at a
// time (333 x 2051 with a residual, K = 1003: 21.1 us without that, 12.3 with it).
// a_scale: the row's (e4m3 operands; the column's scale is applied first).
template <int MODE>
__device__ __forceinline__ void linear_finish32(const GemmArgs& g, int T, int row0, int col, int c, LinearShared& sh, const LinearAhead& f,
                                                float a_scale, const float (&x)[32], const float (&u)[32]) {
    constexpr bool GATED = is_gated(MODE), FP8 = is_fp8(MODE);
    const int lane = threadIdx.x & 31, row = row0 + lane;
    const bool by_vector = linear_by_vector(g, col);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        float4 y[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int e = 8 * v + 4 * h;
            const float4 b = *reinterpret_cast<const float4*>(sh.bias + c + e);
            if (FP8) {
                const float4 w = *reinterpret_cast<const float4*>(sh.scale + c + e);
                y[h] = make_float4(fmaf(x[e] * w.x, a_scale, b.x), fmaf(x[e + 1] * w.y, a_scale, b.y), fmaf(x[e + 2] * w.z, a_scale, b.z),
                                   fmaf(x[e + 3] * w.w, a_scale, b.w));
            } else {
                y[h] = make_float4(x[e] + b.x, x[e + 1] + b.y, x[e + 2] + b.z, x[e + 3] + b.w);
            }
            if (g.act != DCUT_ACT_NONE) y[h] = activate4(g.act, y[h]);
            if (GATED) {
                const float4 b2 = *reinterpret_cast<const float4*>(sh.bias + BN / 2 + c + e);
                if (FP8) {
                    const float4 w = *reinterpret_cast<const float4*>(sh.scale + BN / 2 + c + e);
                    y[h].x *= fmaf(u[e] * w.x, a_scale, b2.x), y[h].y *= fmaf(u[e + 1] * w.y, a_scale, b2.y);
                    y[h].z *= fmaf(u[e + 2] * w.z, a_scale, b2.z), y[h].w *= fmaf(u[e + 3] * w.w, a_scale, b2.w);
                } else {
                    y[h].x *= u[e] + b2.x, y[h].y *= u[e + 1] + b2.y, y[h].z *= u[e + 2] + b2.z, y[h].w *= u[e + 3] + b2.w;
                }
            }
        }
        if (!by_vector) {
            float* s = sh.stage + lane * kStageRow + 8 * v;
            s[0] = y[0].x, s[1] = y[0].y, s[2] = y[0].z, s[3] = y[0].w, s[4] = y[1].x, s[5] = y[1].y, s[6] = y[1].z, s[7] = y[1].w;
        } else if (row < T) {
            if (g.residual) {
                const uint32_t* r = f.r + 4 * v;
                y[0].x += bf_lo(r[0]), y[0].y += bf_hi(r[0]), y[0].z += bf_lo(r[1]), y[0].w += bf_hi(r[1]);
                y[1].x += bf_lo(r[2]), y[1].y += bf_hi(r[2]), y[1].z += bf_lo(r[3]), y[1].w += bf_hi(r[3]);
            }
            *reinterpret_cast<uint4*>(g.out + (size_t)row * g.ldo + col + 8 * v) =
                make_uint4(pack_bf16(y[0].x, y[0].y), pack_bf16(y[0].z, y[0].w), pack_bf16(y[1].x, y[1].y), pack_bf16(y[1].z, y[1].w));
        }
    }
    if (by_vector) return;
    __syncwarp();
    if (col + lane < g.N_out) {
        __nv_bfloat16* o = g.out + (size_t)row0 * g.ldo + col + lane;
#pragma unroll
        for (int i = 0; i < 32; ++i, o += g.ldo)
            if (row0 + i < T) *o = __float2bfloat16_rn(sh.stage[i * kStageRow + lane] + (g.residual ? bf_lo(f.r[i]) : 0.0f));
    }
    __syncwarp();                                                      // the next step writes the stage again
}

// Epilogue of one 128 x bn accumulator (this thread: tensor-memory lane = output row `row`), for every mode.  Columns
// past N_out (a ragged last tile of a narrow width) were computed on zero weight rows and are not stored.
template <int MODE>
__device__ __forceinline__ void gemm_epilogue(const GemmArgs& g, int T, int row, int n_tile, uint32_t t_row, int bn, LinearShared& sh) {
    if (is_linear(MODE)) {
        constexpr bool GATED = is_gated(MODE);
        const int width = GATED ? bn >> 1 : bn, col0 = n_tile * width, row0 = row - (threadIdx.x & 31);
        if (row0 >= T) return;                                          // (the whole warp: none of its rows exists)
        const float a_scale = is_fp8(MODE) && row < T ? g.a_scale[row] : 0.0f;
        LinearAhead ahead;
        linear_fetch(g, T, row0, col0, ahead);
#pragma unroll 1
        for (int c = 0; c < width && col0 + c < g.N_out; c += 32) {
            uint32_t av[32], uv[32];
            tc_ld32(t_row + c, av);
            if (GATED) tc_ld32(t_row + width + c, uv);
            tc_wait_ld();
            float x[32], u[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                x[j] = __uint_as_float(av[j]);
                u[j] = GATED ? __uint_as_float(uv[j]) : 0.0f;
            }
            linear_finish32<MODE>(g, T, row0, col0 + c, c, sh, ahead, a_scale, x, u);
            if (c + 32 < width) linear_fetch(g, T, row0, col0 + c + 32, ahead);
        }
    } else if (MODE == kSwiGLU) {
        const int half = bn >> 1, col0 = n_tile * half;
        __nv_bfloat16* orow = g.out + (size_t)row * g.N_out + col0;
#pragma unroll 1
        for (int c = 0; c < half; c += 32) {
            uint32_t gt[32], up[32];
            tc_ld32(t_row + c, gt);
            tc_ld32(t_row + half + c, up);
            tc_wait_ld();
            if (row < T) {
#pragma unroll
                for (int e = 0; e < 32; e += 8) {
                    if (col0 + c + e >= g.N_out) break;
                    uint32_t o[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float g0 = __uint_as_float(gt[e + 2 * j]), g1 = __uint_as_float(gt[e + 2 * j + 1]);
                        const float u0 = __uint_as_float(up[e + 2 * j]), u1 = __uint_as_float(up[e + 2 * j + 1]);
                        o[j] = pack_bf16(g0 / (1.0f + __expf(-g0)) * u0, g1 / (1.0f + __expf(-g1)) * u1);
                    }
                    *reinterpret_cast<uint4*>(orow + c + e) = make_uint4(o[0], o[1], o[2], o[3]);
                }
            }
        }
    } else if (MODE == kArgmax) {
        // The bf16 logits an unfused path would store are formed in registers and reduced to the row's
        // (maximum, first column) over this tile; rows merge across tiles with a 64-bit atomicMax on
        // (ordered value << 32 | ~column): largest value, lowest column, whatever order the tiles finish in.
        float best = -INFINITY;
        int bidx = -1;
        const int col0 = n_tile * bn;
#pragma unroll 1
        for (int c = 0; c < bn; c += 32) {
            uint32_t av[32];
            tc_ld32(t_row + c, av);
            tc_wait_ld();
            if (col0 + c < g.V) {
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                    const uint32_t pk = pack_bf16(__uint_as_float(av[e]), __uint_as_float(av[e + 1]));
                    const float f0 = bf_lo(pk), f1 = bf_hi(pk);
                    const int col = col0 + c + e;
                    if (col < g.V && f0 > best) {        // strict: the first of equal values stays; NaN never passes
                        best = f0;
                        bidx = col;
                    }
                    if (col + 1 < g.V && f1 > best) {
                        best = f1;
                        bidx = col + 1;
                    }
                }
            }
        }
        if (row < T && bidx >= 0)
            atomicMax(g.row_key + row, ((unsigned long long)dcut_ordered_bits(best) << 32) | (0xffffffffu - (unsigned int)bidx));
    } else {
        const int col0 = n_tile * bn;
        __nv_bfloat16* orow = g.out + (size_t)row * g.N_out + col0;
        const __nv_bfloat16* rrow = MODE == kResidual ? g.residual + (size_t)row * g.N_out + col0 : nullptr;
#pragma unroll 1
        for (int c = 0; c < bn; c += 32) {
            uint32_t av[32];
            tc_ld32(t_row + c, av);
            tc_wait_ld();
            if (row < T) {
#pragma unroll
                for (int e = 0; e < 32; e += 8) {
                    if (col0 + c + e >= g.N_out) break;
                    uint4 res = make_uint4(0, 0, 0, 0);
                    if (MODE == kResidual) res = *reinterpret_cast<const uint4*>(rrow + c + e);
                    const uint32_t rw[4] = {res.x, res.y, res.z, res.w};
                    uint32_t o[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        o[j] = pack_bf16(__uint_as_float(av[e + 2 * j]) + bf_lo(rw[j]),
                                         __uint_as_float(av[e + 2 * j + 1]) + bf_hi(rw[j]));
                    *reinterpret_cast<uint4*>(orow + c + e) = make_uint4(o[0], o[1], o[2], o[3]);
                }
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------ GEMM, pair mode
//
// Pair mode of the GEMM kernel (a cluster of two SMs, tcgen05 cta_group::2): a pair owns a 256 x 256 output tile,
// each CTA its 128 rows.  Each CTA loads its own A tile and HALF of the B tile (128 of the 256 weight rows; for
// SwiGLU the leader's half is the gate rows, the peer's the up rows); the leader's MMA warp issues M256 N256 K16 MMAs
// that read both halves, so an MMA streams 8 KB per SM from shared memory instead of 12 KB and a stage is 32 KB
// instead of 48 KB (six stages fit).  Hand-overs: both CTAs' TMA loads complete on the LEADER's full barrier; the
// leader's commits are multicast to both CTAs' empty / accumulator-full barriers; the peer's epilogue threads arrive
// on the leader's accumulator-empty barrier through distributed shared memory.
// Measured against the one-CTA kernel: 74 us against 86 us for the down projection at T = 512-640 (K = 12288), 81 against
// 90 us for gate/up + SwiGLU at T = 512, but 135 against 92 us for the down projection at T = 1088, where 5 x 16 = 80
// pair tiles need two waves on 74 pairs (and 1280 padded rows are computed instead of 1152): the mode is therefore
// chosen per launch (gemm_plan.cuh).

constexpr int kG2Stages = 6;
constexpr int kG2StageBytes = kATile + kBTile / 2;     // 32 KB

__device__ __forceinline__ void mbar_arrive_remote(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// TMA tile load whose completion is signalled on a barrier of either CTA of the pair
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* map, int c0, int c1, uint32_t bar_cluster_addr) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(bar_cluster_addr) : "memory");
}
template <bool FP8>
__device__ __forceinline__ void tc_mma2(uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
    if (FP8)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, {%5, %5, %5, %5, %5, %5, %5, %5}, p;\n\t}"
            ::"r"(tmem_d), "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(accumulate), "r"(0u) : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, {%5, %5, %5, %5, %5, %5, %5, %5}, p;\n\t}"
            ::"r"(tmem_d), "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(accumulate), "r"(0u) : "memory");
}
// arrives on the barrier at the same offset in both CTAs of the pair once the MMAs issued so far have completed
__device__ __forceinline__ void tc_commit_pair(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((unsigned short)3) : "memory");
}

// One persistent kernel, three ways of running a GEMM and seven tile widths, looked up on the device from the packed
// length (the same answer in every CTA).
//   One SM per tile: a CTA walks the 128 x bn output tiles b, b + gridDim.x, ... (m fastest, so the CTAs running
//   together share weight tiles in L2); a stage holds the tile's A and B bytes, 4 (bn = 256) to 12 stages.
//   A pair of SMs per tile (see above): 256 x bn tiles, six 32 KB stages.  Fewer bytes per flop from L2, but rows
//   padded to 256 and half as many, larger work items.
//   A pair per 128 x bn tile, half of K each (below): for launches whose tiles all fit one wave of pairs.
// In the first two the operand ring and its barriers continue across tiles and the accumulator is double-buffered in
// tensor memory (2 x 256 columns), so the epilogue of one tile overlaps the main loop of the next.
// Which of them, and how wide a tile: gemm_plan.cuh, by the packed length.
static_assert(kGemmStages * kGemmStageBytes == kG2Stages * kG2StageBytes, "both modes use the same operand area");

template <int MODE>
__global__ void __launch_bounds__(kGemmThreads, 1)
gemm_tcgen05_kernel(const __grid_constant__ AMaps a_maps, const __grid_constant__ BMaps b_maps,
                    const __grid_constant__ BMaps b2_maps, GemmArgs g) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    unsigned long long* bars = reinterpret_cast<unsigned long long*>(smem + kGemmStages * kGemmStageBytes);
    unsigned long long* bars2 = bars + 2 * kMaxStages + 4;                  // the pair mode's set
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars2 + 2 * kG2Stages + 4);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    LinearShared& sh = reinterpret_cast<LinearShared*>(smem + kGemmSmem - 1024)[warp & 3];   // (linear modes only) behind the barriers
    constexpr int kKb = kb_elements(MODE);
    const int n_kb = g.K / kKb;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kMaxStages; ++s) {
            mbar_init(smem_u32(bars + s), 1);
            mbar_init(smem_u32(bars + kMaxStages + s), 1);
        }
        for (int s = 0; s < kG2Stages; ++s) {
            mbar_init(smem_u32(bars2 + s), 1);                 // the leader's expect_tx arrival (bytes of both CTAs)
            mbar_init(smem_u32(bars2 + kG2Stages + s), 1);     // the leader's multicast commit
        }
        for (int k = 0; k < 2; ++k) {
            mbar_init(smem_u32(bars + 2 * kMaxStages + k), 1);
            mbar_init(smem_u32(bars + 2 * kMaxStages + 2 + k), 128);   // the four epilogue warps
            mbar_init(smem_u32(bars2 + 2 * kG2Stages + k), 1);          // the leader's multicast commit
            mbar_init(smem_u32(bars2 + 2 * kG2Stages + 2 + k), 256);    // (leader's copy) the epilogue threads of both CTAs
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (threadIdx.x == 32) {                     // the tensor maps that the largest packed length would use
        const int m = g.plan_by_m[kPlanRows - 1];
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&a_maps.full)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&a_maps.half)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(pick_map(b_maps, m & 7))) : "memory");
        if (is_gated(MODE)) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(pick_map(b2_maps, m & 7))) : "memory");
    }
    __syncthreads();
    cluster_sync_all();                          // the peer's barriers exist before anything is signalled on them
    // everything above overlaps the previous kernel of the stream; nothing it wrote is read before this wait
    dcut_pdl_wait();
    dcut_pdl_launch_dependents();
    int T_packed = g.cu_q[g.B];
    if (is_linear(MODE) && T_packed > g.T_cap) {
        T_packed = g.T_cap;
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicExch(g.status, DCUT_DEV_BAD_ROWS);
    }
    const int T = T_packed;
    // rows 64..127 of the A tile are not loaded when no row of them exists: they hold whatever shared memory held, and
    // the accumulator rows computed from them are never stored (one-SM and split modes; a pair always loads full boxes)
    const bool a_half = T <= BM / 2;
    const CUtensorMap* a_map1 = a_half ? &a_maps.half : &a_maps.full;
    const uint32_t a_bytes = a_half ? kATile / 2 : kATile;
    const int m_blocks = (T + BM - 1) / BM;
    const int plan_all = m_blocks > 0 ? g.plan_by_m[(m_blocks < kPlanRows ? m_blocks : kPlanRows) - 1] : 0;
    const bool split = plan_all >= kPlanSplit;                      // the pair shares one 128-row tile, half of K each
    const bool pairs = plan_all >= kPlanPair && !split;
    const int plan = plan_all & 7;                                  // width index
    const int bn = bn_of(plan), half_rows = bn >> 1;                // tile width; a B tile is loaded as two halves
    const int per = is_gated(MODE) ? half_rows : bn;                // output columns per tile
    const int n_tiles = (g.N_out + per - 1) / per;
    // one-SM and split modes: a stage is this tile's A and B bytes, and as many stages as fit the operand area (a
    // 64-wide tile at T <= 64 moves 8 KB of weights per stage: with four stages too few bytes were in flight per SM to
    // cover the DRAM latency)
    const uint32_t stage_stride = a_bytes + (uint32_t)bn * BK * 2;                         // multiples of 1 KB
    const int n_stages = min(kMaxStages, (int)((uint32_t)(kGemmStages * kGemmStageBytes) / stage_stride));
    if (warp == 1) {   // tensor memory: two 128 x 256 fp32 accumulators (per CTA; allocated for the pair in pair mode)
        if (pairs) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "n"(kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "n"(kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    if (pairs) cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    bool failed = false;

    if (split) {
        // ------------------------------------------------------------------ one tile per pair of SMs, K cut in two
        // Each CTA runs the one-SM main loop over its half of the k-blocks into its own accumulator.  Then the two
        // exchange: a CTA sends the columns the other one will finish (fp32, through distributed shared memory into
        // the other's idle operand ring) and finishes its own columns with what it received.  Every thread of both
        // CTAs passes the same two cluster barriers whatever happened before, so a wait that gave up cannot strand
        // the peer.
        const int m_tiles = (T + BM - 1) / BM;
        const int w = blockIdx.x >> 1;                              // the pair's tile
        const bool has_tile = w < m_tiles * n_tiles;
        const uint32_t rank = cluster_ctarank();
        const int n_tile = has_tile ? w / m_tiles : 0, m0 = has_tile ? (w - n_tile * m_tiles) * BM : 0;
        const int kb_mid = (n_kb + 1) >> 1, kb0 = rank ? kb_mid : 0, kb1 = rank ? n_kb : kb_mid;
        const uint32_t full_bar = smem_u32(bars), empty_bar = smem_u32(bars + kMaxStages);
        const uint32_t acc_full = smem_u32(bars + 2 * kMaxStages);
        if (has_tile && warp == 0) {
            const CUtensorMap* b_map = pick_map(b_maps, plan);
            const uint32_t stage_tx = a_bytes + bn * BK * 2;
            for (int kb = kb0, kc = 0, s = 0, use = 0; kb < kb1; ++kb, ++kc) {
                if (use > 0 && !__all_sync(0xffffffffu, mbar_wait(empty_bar + 8 * s, (use - 1) & 1))) {
                    failed = true;
                    break;
                }
                if (elect_one()) {
                    const uint32_t a_dst = smem_u32(smem + s * stage_stride), b_dst = a_dst + a_bytes;
                    const uint32_t bar = full_bar + 8 * s;
                    mbar_arrive_expect_tx(bar, stage_tx);
                    tma_load_2d(a_dst, a_map1, kb * kKb, m0, bar);
                    tma_load_2d(b_dst, b_map, kb * kKb, n_tile * bn, bar);
                    tma_load_2d(b_dst + half_rows * BK * 2, b_map, kb * kKb, n_tile * bn + half_rows, bar);
                }
                __syncwarp();
                if (++s == n_stages) {
                    s = 0;
                    ++use;
                }
            }
        } else if (has_tile && warp == 1) {
            const uint32_t idesc = idesc_no_n<is_fp8(MODE)>(BM) | ((uint32_t)(bn >> 3) << 17);
            for (int kb = kb0, kc = 0, s = 0, use = 0; kb < kb1; ++kb, ++kc) {
                if (!__all_sync(0xffffffffu, mbar_wait(full_bar + 8 * s, use & 1))) {
                    failed = true;
                    break;
                }
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t a_addr = smem_u32(smem + s * stage_stride);
                    const uint64_t da = umma_desc_sw128(a_addr), db = umma_desc_sw128(a_addr + a_bytes);
#pragma unroll
                    for (int k = 0; k < BK / 16; ++k) tc_mma<is_fp8(MODE)>(tmem_base, da + 2 * k, db + 2 * k, idesc, (kc | k) ? 1u : 0u);
                    tc_commit(empty_bar + 8 * s);
                }
                __syncwarp();
                if (++s == n_stages) {
                    s = 0;
                    ++use;
                }
            }
            if (!failed && elect_one()) tc_commit(acc_full);    // this CTA's partial sums are complete
            __syncwarp();
        } else if (has_tile) {
            if (is_split_linear(MODE)) linear_stage_bias<MODE>(g, n_tile, bn, sh);
            if (!__all_sync(0xffffffffu, mbar_wait(acc_full, 0))) failed = true;   // ... and its operand ring is idle
            tc_fence_after();
        }
        // columns [0, cut) are finished by rank 0, [cut, bn) by rank 1
        const int cut = (bn >> 6) << 5;
        const int own0 = rank ? cut : 0, own1 = rank ? bn : cut, send0 = rank ? 0 : cut, send1 = rank ? cut : bn;
        const int quarter = warp & 3, row_in_tile = quarter * 32 + lane;
        const uint32_t t_row = tmem_base + ((uint32_t)(quarter * 32) << 16);
        const uint32_t stage_local = smem_u32(smem);              // [column / 4][row] vectors of four fp32: 64 KB at most
        LinearAhead ahead;                                        // (linear modes only)
        const int row0 = m0 + quarter * 32;
        const bool rows_here = row0 < T;                          // (a warp without rows has nothing to exchange)
        const float a_scale = is_fp8(MODE) && has_tile && warp >= 2 && row0 + lane < T ? g.a_scale[row0 + lane] : 0.0f;
        if (is_split_linear(MODE) && has_tile && warp >= 2 && rows_here) linear_fetch(g, T, row0, n_tile * bn + own0, ahead);
        tc_fence_before();
        cluster_sync_all();                                       // both accumulators complete, both rings idle
        tc_fence_after();
        if (has_tile && warp >= 2 && rows_here && !failed) {
            asm volatile("fence.proxy.async;" ::: "memory");      // the ring was last written and read through the async proxy
            const uint32_t stage_peer = mapa_rank(stage_local, rank ^ 1);
#pragma unroll 1
            for (int c = send0; c < send1; c += 32) {
                uint32_t av[32];
                tc_ld32(t_row + c, av);
                tc_wait_ld();
#pragma unroll
                for (int v = 0; v < 8; ++v) {
                    const uint32_t dst = stage_peer + (uint32_t)((((c - send0) >> 2) + v) * BM + row_in_tile) * 16;
                    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(av[4 * v]), "r"(av[4 * v + 1]),
                                 "r"(av[4 * v + 2]), "r"(av[4 * v + 3]) : "memory");
                }
            }
        }
        tc_fence_before();
        cluster_sync_all();                                       // the peer's partial sums have arrived
        tc_fence_after();
        if (has_tile && warp >= 2 && rows_here && !failed) {
            const int row = m0 + row_in_tile, col0 = n_tile * bn;
            __nv_bfloat16* orow = g.out + (size_t)row * g.N_out + col0;
            const __nv_bfloat16* rrow = MODE == kResidual ? g.residual + (size_t)row * g.N_out + col0 : nullptr;
#pragma unroll 1
            for (int c = own0; c < own1; c += 32) {
                if (is_split_linear(MODE) && col0 + c >= g.N_out) break;
                uint32_t av[32];
                tc_ld32(t_row + c, av);
                if (is_split_linear(MODE)) {
                    tc_wait_ld();
                    float x[32];
#pragma unroll
                    for (int v = 0; v < 8; ++v) {
                        float add[4];
                        const uint32_t src = stage_local + (uint32_t)((((c - own0) >> 2) + v) * BM + row_in_tile) * 16;
                        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(add[0]), "=f"(add[1]), "=f"(add[2]), "=f"(add[3]) : "r"(src));
#pragma unroll
                        for (int j = 0; j < 4; ++j)   // (rank 0's half of K) + (rank 1's)
                            x[4 * v + j] = rank ? add[j] + __uint_as_float(av[4 * v + j]) : __uint_as_float(av[4 * v + j]) + add[j];
                    }
                    linear_finish32<MODE>(g, T, row0, col0 + c, c, sh, ahead, a_scale, x, x);
                    if (c + 32 < own1) linear_fetch(g, T, row0, col0 + c + 32, ahead);
                    continue;
                }
                tc_wait_ld();
                if (row < T) {
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        if (col0 + c + e >= g.N_out) break;
                        float add[8];
#pragma unroll
                        for (int v = 0; v < 2; ++v) {
                            const uint32_t src = stage_local + (uint32_t)((((c - own0 + e) >> 2) + v) * BM + row_in_tile) * 16;
                            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                                         : "=f"(add[4 * v]), "=f"(add[4 * v + 1]), "=f"(add[4 * v + 2]), "=f"(add[4 * v + 3]) : "r"(src));
                        }
                        uint4 res = make_uint4(0, 0, 0, 0);
                        if (MODE == kResidual) res = *reinterpret_cast<const uint4*>(rrow + c + e);
                        const uint32_t rw[4] = {res.x, res.y, res.z, res.w};
                        uint32_t o[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j)   // (rank 0's half of K) + (rank 1's), then the residual
                            o[j] = pack_bf16((rank ? add[2 * j] + __uint_as_float(av[e + 2 * j]) : __uint_as_float(av[e + 2 * j]) + add[2 * j]) + bf_lo(rw[j]),
                                             (rank ? add[2 * j + 1] + __uint_as_float(av[e + 2 * j + 1]) : __uint_as_float(av[e + 2 * j + 1]) + add[2 * j + 1]) + bf_hi(rw[j]));
                        *reinterpret_cast<uint4*>(orow + c + e) = make_uint4(o[0], o[1], o[2], o[3]);
                    }
                }
            }
        }
    } else if (!pairs) {
        const int m_tiles = (T + BM - 1) / BM;
        const int n_work = m_tiles * n_tiles;                      // (a CTA without work falls through the loops below)
        const uint32_t full_bar = smem_u32(bars), empty_bar = smem_u32(bars + kMaxStages);
        const uint32_t acc_full = smem_u32(bars + 2 * kMaxStages), acc_empty = acc_full + 16;
        if (warp == 0) {
            // ---------------------------------------------------------------- TMA producer (whole warp walks, one lane issues)
            const CUtensorMap* b_map = pick_map(b_maps, plan);
            const CUtensorMap* b2_map = pick_map(b2_maps, plan);
            const uint32_t stage_tx = a_bytes + bn * BK * 2;
            int s = 0, use = 0;   // stage of the next k-block, and how often the ring has gone round (over all tiles)
            for (int w = blockIdx.x; w < n_work && !failed; w += gridDim.x) {
                const int n_tile = w / m_tiles, m0 = (w - n_tile * m_tiles) * BM;
                for (int kb = 0; kb < n_kb; ++kb) {
                    if (use > 0 && !__all_sync(0xffffffffu, mbar_wait(empty_bar + 8 * s, (use - 1) & 1))) {
                        failed = true;
                        break;
                    }
                    if (elect_one()) {
                        const uint32_t a_dst = smem_u32(smem + s * stage_stride), b_dst = a_dst + a_bytes;
                        const uint32_t bar = full_bar + 8 * s;
                        mbar_arrive_expect_tx(bar, stage_tx);
                        tma_load_2d(a_dst, a_map1, kb * kKb, m0, bar);
                        if (is_gated(MODE)) {    // the gate rows, then the up rows of the same features
                            tma_load_2d(b_dst, b_map, kb * kKb, n_tile * half_rows, bar);
                            tma_load_2d(b_dst + half_rows * BK * 2, b2_map, kb * kKb, n_tile * half_rows, bar);
                        } else {                 // (weight rows past N read as zeros)
                            tma_load_2d(b_dst, b_map, kb * kKb, n_tile * bn, bar);
                            tma_load_2d(b_dst + half_rows * BK * 2, b_map, kb * kKb, n_tile * bn + half_rows, bar);
                        }
                    }
                    __syncwarp();
                    if (++s == n_stages) {
                        s = 0;
                        ++use;
                    }
                }
            }
        } else if (warp == 1) {
            // ---------------------------------------------------------------- MMA issuer (whole warp walks, one lane issues)
            const uint32_t idesc = idesc_no_n<is_fp8(MODE)>(BM) | ((uint32_t)(bn >> 3) << 17);
            int s = 0, use = 0, it = 0;
            for (int w = blockIdx.x; w < n_work && !failed; w += gridDim.x, ++it) {
                const int acc = it & 1;
                // the epilogue must have drained this accumulator (used by tile it - 2)
                if (it >= 2 && !__all_sync(0xffffffffu, mbar_wait(acc_empty + 8 * acc, ((it >> 1) - 1) & 1))) {
                    failed = true;
                    break;
                }
                tc_fence_after();
                const uint32_t tmem_d = tmem_base + acc * BN;
                for (int kb = 0; kb < n_kb; ++kb) {
                    if (!__all_sync(0xffffffffu, mbar_wait(full_bar + 8 * s, use & 1))) {
                        failed = true;
                        break;
                    }
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t a_addr = smem_u32(smem + s * stage_stride);
                        const uint64_t da = umma_desc_sw128(a_addr), db = umma_desc_sw128(a_addr + a_bytes);
    #pragma unroll
                        for (int k = 0; k < BK / 16; ++k)   // 32 bytes along K per step = 2 descriptor address units
                            tc_mma<is_fp8(MODE)>(tmem_d, da + 2 * k, db + 2 * k, idesc, (kb | k) ? 1u : 0u);
                        tc_commit(empty_bar + 8 * s);       // the stage is free once these MMAs have read it
                    }
                    __syncwarp();
                    if (++s == n_stages) {
                        s = 0;
                        ++use;
                    }
                }
                if (failed) break;
                if (elect_one()) tc_commit(acc_full + 8 * acc);   // accumulator complete
                __syncwarp();
            }
        } else {
            // ---------------------------------------------------------------- epilogue warps
            const int quarter = warp & 3;               // tensor-memory lanes 32 * quarter .. + 31
            int it = 0;
            for (int w = blockIdx.x; w < n_work && !failed; w += gridDim.x, ++it) {
                const int n_tile = w / m_tiles, m0 = (w - n_tile * m_tiles) * BM;
                const int acc = it & 1;
                const int row = m0 + quarter * 32 + lane;
                if (is_linear(MODE)) linear_stage_bias<MODE>(g, n_tile, bn, sh);
                if (!__all_sync(0xffffffffu, mbar_wait(acc_full + 8 * acc, (it >> 1) & 1))) {
                    failed = true;
                    break;
                }
                tc_fence_after();
                const uint32_t t_row = tmem_base + ((uint32_t)(quarter * 32) << 16) + acc * BN;
                gemm_epilogue<MODE>(g, T, row, n_tile, t_row, bn, sh);
                // this accumulator may be overwritten once all four epilogue warps have read it
                tc_fence_before();
                mbar_arrive(acc_empty + 8 * acc);
            }
        }
    } else {
        const int m_tiles = (T + 2 * BM - 1) / (2 * BM);          // 256-row tiles of the pair
        const int n_work = m_tiles * n_tiles;
        const uint32_t rank = cluster_ctarank();                   // 0: leader
        const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
        const uint32_t full_bar = smem_u32(bars2), empty_bar = smem_u32(bars2 + kG2Stages);
        const uint32_t acc_full = smem_u32(bars2 + 2 * kG2Stages), acc_empty = acc_full + 16;
        if (warp == 0) {
            // ---------------------------------------------------------------- TMA producer (both CTAs)
            const uint32_t lead_full = mapa_rank(full_bar, 0);
            const CUtensorMap* b_map = pick_map(b_maps, plan);
            const CUtensorMap* b2_map = pick_map(b2_maps, plan);
            const uint32_t pair_tx = 2 * (kATile + half_rows * BK * 2);   // both CTAs' A tile and half of the B tile
            int kc = 0;
            for (int w = pair; w < n_work && !failed; w += n_pairs) {
                const int n_tile = w / m_tiles, m0 = (w - n_tile * m_tiles) * (2 * BM) + (int)rank * BM;
                for (int kb = 0; kb < n_kb; ++kb, ++kc) {
                    const int s = kc % kG2Stages;
                    if (kc >= kG2Stages && !__all_sync(0xffffffffu, mbar_wait(empty_bar + 8 * s, ((kc / kG2Stages) - 1) & 1))) {
                        failed = true;
                        break;
                    }
                    if (elect_one()) {
                        const uint32_t a_dst = smem_u32(smem + s * kG2StageBytes), b_dst = a_dst + kATile;
                        if (rank == 0) mbar_arrive_expect_tx(full_bar + 8 * s, pair_tx);
                        const uint32_t bar = lead_full + 8 * s;
                        tma_load_2d_pair(a_dst, &a_maps.full, kb * kKb, m0, bar);
                        if (is_gated(MODE))       // the leader's half: 128 gate rows; the peer's: the 128 up rows of the same features
                            tma_load_2d_pair(b_dst, rank == 0 ? b_map : b2_map, kb * kKb, n_tile * half_rows, bar);
                        else
                            tma_load_2d_pair(b_dst, b_map, kb * kKb, n_tile * bn + (int)rank * half_rows, bar);
                    }
                    __syncwarp();
                }
            }
        } else if (warp == 1) {
            // ---------------------------------------------------------------- MMA issuer (leader CTA only)
            if (rank == 0) {
                const uint32_t idesc2 = idesc_no_n<is_fp8(MODE)>(2 * BM) | ((uint32_t)(bn >> 3) << 17);
                int kc = 0, it = 0;
                for (int w = pair; w < n_work && !failed; w += n_pairs, ++it) {
                    const int acc = it & 1;
                    // the epilogues of both CTAs must have drained this accumulator (used by tile it - 2)
                    if (it >= 2 && !__all_sync(0xffffffffu, mbar_wait(acc_empty + 8 * acc, ((it >> 1) - 1) & 1))) {
                        failed = true;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t tmem_d = tmem_base + acc * BN;
                    for (int kb = 0; kb < n_kb; ++kb, ++kc) {
                        const int s = kc % kG2Stages;
                        if (!__all_sync(0xffffffffu, mbar_wait(full_bar + 8 * s, (kc / kG2Stages) & 1))) {
                            failed = true;
                            break;
                        }
                        tc_fence_after();
                        if (elect_one()) {
                            const uint32_t a_addr = smem_u32(smem + s * kG2StageBytes);
                            const uint64_t da = umma_desc_sw128(a_addr), db = umma_desc_sw128(a_addr + kATile);
    #pragma unroll
                            for (int k = 0; k < BK / 16; ++k)
                                tc_mma2<is_fp8(MODE)>(tmem_d, da + 2 * k, db + 2 * k, idesc2, (kb | k) ? 1u : 0u);
                            tc_commit_pair(empty_bar + 8 * s);     // the stage is free in both CTAs once these MMAs have read it
                        }
                        __syncwarp();
                    }
                    if (failed) break;
                    if (elect_one()) tc_commit_pair(acc_full + 8 * acc);   // accumulator complete, in both CTAs
                    __syncwarp();
                }
            }
        } else {
            // ---------------------------------------------------------------- epilogue warps (both CTAs)
            const int quarter = warp & 3;
            const uint32_t lead_acc_empty = mapa_rank(acc_empty, 0);
            int it = 0;
            for (int w = pair; w < n_work && !failed; w += n_pairs, ++it) {
                const int n_tile = w / m_tiles, m0 = (w - n_tile * m_tiles) * (2 * BM) + (int)rank * BM;
                const int acc = it & 1;
                const int row = m0 + quarter * 32 + lane;
                if (is_linear(MODE)) linear_stage_bias<MODE>(g, n_tile, bn, sh);
                if (!__all_sync(0xffffffffu, mbar_wait(acc_full + 8 * acc, (it >> 1) & 1))) {
                    failed = true;
                    break;
                }
                tc_fence_after();
                const uint32_t t_row = tmem_base + ((uint32_t)(quarter * 32) << 16) + acc * BN;
                gemm_epilogue<MODE>(g, T, row, n_tile, t_row, bn, sh);
                tc_fence_before();
                mbar_arrive_remote(lead_acc_empty + 8 * acc);
            }
        }
    }
    if (failed) atomicExch(g.status, DCUT_DEV_GEMM_WAIT_TIMEOUT);
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                          // nobody leaves while the other CTA may still signal its barriers
    if (warp == 1) {
        tc_fence_after();
        if (pairs)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "n"(kTmemCols) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "n"(kTmemCols) : "memory");
    }
}

// ------------------------------------------------------------------------------------------------ RMSNorm

__global__ void __launch_bounds__(256) rmsnorm_kernel(const __nv_bfloat16* __restrict__ x, const __nv_bfloat16* __restrict__ gain,
                                                      const int* __restrict__ cu_q, int B, int hidden, float eps,
                                                      __nv_bfloat16* __restrict__ y) {
    dcut_pdl_wait();
    dcut_pdl_launch_dependents();
    const int row = blockIdx.x;
    if (row >= cu_q[B]) return;
    const uint4* xr = reinterpret_cast<const uint4*>(x + (size_t)row * hidden);
    const uint4* gr = reinterpret_cast<const uint4*>(gain);
    uint4* yr = reinterpret_cast<uint4*>(y + (size_t)row * hidden);
    const int nvec = hidden >> 3;
    float ss = 0.0f;
    for (int v = threadIdx.x; v < nvec; v += 256) {
        const uint4 a = xr[v];
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) ss += bf_lo(w[j]) * bf_lo(w[j]) + bf_hi(w[j]) * bf_hi(w[j]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    __shared__ float wsum[8];
    if ((threadIdx.x & 31) == 0) wsum[threadIdx.x >> 5] = ss;
    __syncthreads();
    float tot = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; ++w) tot += wsum[w];
    const float inv = rsqrtf(tot / (float)hidden + eps);
    for (int v = threadIdx.x; v < nvec; v += 256) {
        const uint4 a = xr[v], gq = gr[v];
        const uint32_t w[4] = {a.x, a.y, a.z, a.w}, gw[4] = {gq.x, gq.y, gq.z, gq.w};
        uint32_t o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = pack_bf16(bf_lo(w[j]) * inv * bf_lo(gw[j]), bf_hi(w[j]) * inv * bf_hi(gw[j]));
        yr[v] = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

// ------------------------------------------------------------------------------------------------ RoPE + KV append

struct RopeArgs {
    const __nv_bfloat16* qkv;   // [T, (Hq + 2 Hkv) * Dh]: q heads, k heads, v heads
    const int* cu_q;
    const int* tok_req;
    const int* tok_pos;
    const int* block_table;
    int block_table_stride;
    const float* inv_freq;      // [Dh / 2] = theta^(-2e/Dh)
    int B, n_q_heads, n_kv_heads, head_dim;
    long long num_pages;
    __nv_bfloat16* q_out;       // [T, Hq, Dh]
    __nv_bfloat16* k_cache;
    __nv_bfloat16* v_cache;
    int* status;
};

__global__ void __launch_bounds__(256) rope_append_kernel(RopeArgs a) {
    dcut_pdl_wait();
    dcut_pdl_launch_dependents();
    const int tok = blockIdx.x;
    if (tok >= a.cu_q[a.B]) return;
    const int Dh = a.head_dim, half = Dh >> 1;
    const int req = a.tok_req[tok], pos = a.tok_pos[tok];
    int page = a.block_table[(size_t)req * a.block_table_stride + pos / 16];
    if (page < 0 || page >= a.num_pages) {
        if (threadIdx.x == 0) atomicExch(a.status, DCUT_DEV_BAD_PAGE);
        return;
    }
    const int slot = pos & 15;
    const int row_w = (a.n_q_heads + 2 * a.n_kv_heads) * Dh;
    const __nv_bfloat16* row = a.qkv + (size_t)tok * row_w;
    // A thread keeps its two rotation pairs (e, e + 1) and walks the heads: one sincos pair per thread, 4-byte accesses.
    // (head_dim is a multiple of 16, so half is even and rows are 4-byte aligned.)
    const int lanes_per_head = half >> 1;                      // threads that cover one head
    const int heads_per_pass = blockDim.x / lanes_per_head;
    const int e = (threadIdx.x % lanes_per_head) * 2;
    float sn0, cs0, sn1, cs1;
    sincosf((float)pos * a.inv_freq[e], &sn0, &cs0);
    sincosf((float)pos * a.inv_freq[e + 1], &sn1, &cs1);
    if ((int)threadIdx.x < heads_per_pass * lanes_per_head) {
        for (int h = threadIdx.x / lanes_per_head; h < a.n_q_heads + a.n_kv_heads; h += heads_per_pass) {
            const uint32_t lo = *reinterpret_cast<const uint32_t*>(row + h * Dh + e);
            const uint32_t hi = *reinterpret_cast<const uint32_t*>(row + h * Dh + e + half);
            const float a0 = bf_lo(lo), a1 = bf_hi(lo), b0 = bf_lo(hi), b1 = bf_hi(hi);
            const uint32_t y_lo = pack_bf16(a0 * cs0 - b0 * sn0, a1 * cs1 - b1 * sn1);
            const uint32_t y_hi = pack_bf16(b0 * cs0 + a0 * sn0, b1 * cs1 + a1 * sn1);
            __nv_bfloat16* dst = h < a.n_q_heads
                                     ? a.q_out + ((size_t)tok * a.n_q_heads + h) * Dh
                                     : a.k_cache + (((size_t)page * a.n_kv_heads + (h - a.n_q_heads)) * 16 + slot) * Dh;
            *reinterpret_cast<uint32_t*>(dst + e) = y_lo;
            *reinterpret_cast<uint32_t*>(dst + e + half) = y_hi;
        }
    }
    const uint4* vrow = reinterpret_cast<const uint4*>(row + (a.n_q_heads + a.n_kv_heads) * Dh);   // 16-byte aligned: Dh % 8 == 0
    const int vec_per_head = Dh >> 3;
    for (int idx = threadIdx.x; idx < a.n_kv_heads * vec_per_head; idx += blockDim.x) {
        const int h = idx / vec_per_head, v = idx - h * vec_per_head;
        reinterpret_cast<uint4*>(a.v_cache + (((size_t)page * a.n_kv_heads + h) * 16 + slot) * Dh)[v] = vrow[idx];
    }
}

// ------------------------------------------------------------------------------------------------ host

// K-major bf16 (or e4m3: bytes) matrix [rows, cols] as a 2-D tensor map with a {128 bytes, box_rows} box and 128-byte swizzle
dcut_status make_kmajor_map(dcut_ctx* ctx, CUtensorMap* map, const void* base, long long rows, long long cols, int box_rows, long long ld = 0, bool fp8 = false) {
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)(ld ? ld : cols) * (fp8 ? 1 : 2)};
    cuuint32_t box[2] = {(cuuint32_t)(fp8 ? 2 * BK : BK), (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1, 1};
    CUresult r = reinterpret_cast<EncodeTiledFn>(ctx->encode_tiled)(
        map, fp8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr,
        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return dcut_fail(ctx, DCUT_ECUDA, "cuTensorMapEncodeTiled failed for a GEMM operand (%d)", (int)r);
    return DCUT_OK;
}

dcut_status make_act_maps(dcut_ctx* ctx, AMaps* maps, const void* base, long long rows, long long cols, long long ld = 0, bool fp8 = false) {
    dcut_status st = make_kmajor_map(ctx, &maps->full, base, rows, cols, BM, ld, fp8);
    if (st != DCUT_OK) return st;
    return make_kmajor_map(ctx, &maps->half, base, rows, cols, BM / 2, ld, fp8);
}

// The weight's tensor maps for the tile widths in `mask` (box = half the width in rows)
dcut_status make_weight_maps(dcut_ctx* ctx, BMaps* maps, const void* w, long long rows, long long cols, unsigned mask) {
    for (int i = 0; i < kNumBn; ++i) {
        if (!((mask >> i) & 1)) continue;
        dcut_status st = make_kmajor_map(ctx, &maps->m[i], w, rows, cols, bn_of(i) / 2);
        if (st != DCUT_OK) return st;
    }
    return DCUT_OK;
}

// Fills in how a launch runs (gemm_plan.cuh); returns its grid
template <int MODE>
int plan_gemm(dcut_ctx* ctx, int T_cap, unsigned bn_mask, GemmArgs& ga) {
    const Shape shape = {ga.N_out, ga.K / kb_elements(MODE) * BK, T_cap, is_gated(MODE), may_split_k(MODE), is_linear(MODE)};   // (K in k-blocks)
    const Launch l = plan(shape, Device{ctx->sm_count, ctx->ly_gemm_pairs, ctx->ly_gemm_pair_mode != 0, ctx->ly_gemm_force, bn_mask});
    static_assert(sizeof(ga.plan_by_m) == sizeof(l.by_m), "one table");
    memcpy(ga.plan_by_m, l.by_m, sizeof(l.by_m));
    return l.grid;
}

template <int MODE>
dcut_status launch_planned_gemm(dcut_ctx* ctx, const AMaps& a, const BMaps& b, const BMaps& b2, int grid, const GemmArgs& ga, cudaStream_t stream) {
    const size_t smem = is_linear(MODE) ? kLinearSmem : kGemmSmem;
    if (ctx->ly_gemm_pairs > 0) {
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = 2;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[1].val.programmaticStreamSerializationAllowed = 1;
        cudaLaunchConfig_t lc = {};
        lc.gridDim = dim3(grid);
        lc.blockDim = dim3(kGemmThreads);
        lc.dynamicSmemBytes = smem;
        lc.stream = stream;
        lc.attrs = attr;
        lc.numAttrs = 2;
        return dcut_check_cuda(ctx, cudaLaunchKernelEx(&lc, gemm_tcgen05_kernel<MODE>, a, b, b2, ga), "launch gemm_tcgen05_kernel");
    }
    return dcut_check_cuda(ctx, dcut_launch_pdl(gemm_tcgen05_kernel<MODE>, dim3(grid), dim3(kGemmThreads), smem, stream, a, b, b2, ga),
                           "launch gemm_tcgen05_kernel");
}

template <int MODE>
dcut_status launch_gemm(dcut_ctx* ctx, const AMaps& a, const BMaps& b, const BMaps& b2, int T_cap, unsigned bn_mask, const GemmArgs& g, cudaStream_t stream) {
    GemmArgs ga = g;
    const int grid = plan_gemm<MODE>(ctx, T_cap, bn_mask, ga);
    return launch_planned_gemm<MODE>(ctx, a, b, b2, grid, ga, stream);
}

// dcut_linear: any N and K (the tensor maps' zero fill completes the last tile and the last k-block), rows of any stride.
// Encodes maps for the tile widths that the plan can pick only (about 0.3 us of host time each).  ARGS: dcut_linear_args or
// dcut_linear8_args.
template <int MODE, typename ARGS>
dcut_status launch_linear(dcut_ctx* ctx, const ARGS* l, int T_cap, GemmArgs& g, cudaStream_t stream) {
    const unsigned mask = (is_gated(MODE) ? ctx->ly_gemm_bn_mask & kBnMaskSwiGLU : ctx->ly_gemm_bn_mask) | 1u;
    const int grid = plan_gemm<MODE>(ctx, T_cap, mask, g);
    unsigned used = 0;
    for (int m = 0; m < kPlanRows && m <= (T_cap - 1) / BM; ++m) used |= 1u << (g.plan_by_m[m] & 7);
    AMaps am;
    BMaps bm = {}, b2m = {};
    dcut_status st;
    if ((st = make_act_maps(ctx, &am, l->a, T_cap, l->K, l->lda, is_fp8(MODE))) != DCUT_OK) return st;
    for (int i = 0; i < kNumBn; ++i) {
        if (!((used >> i) & 1)) continue;
        if ((st = make_kmajor_map(ctx, &bm.m[i], l->w, l->N, l->K, bn_of(i) / 2, l->ldw, is_fp8(MODE))) != DCUT_OK) return st;
        if (is_gated(MODE) && (st = make_kmajor_map(ctx, &b2m.m[i], l->w2, l->N, l->K, bn_of(i) / 2, l->ldw, is_fp8(MODE))) != DCUT_OK) return st;
    }
    return launch_planned_gemm<MODE>(ctx, am, bm, b2m, grid, g, stream);
}

// Tensor maps of the layers seen so far: the weights' (for every tile width) in a small direct-mapped cache keyed by the
// layer's w_qkv pointer, so that a model forward does not encode 36 x 31 maps on every call
struct WeightMaps {
    const void* w[5];
    BMaps m[5];         // w_qkv, w_o, w_gate, w_up, w_down
};
constexpr int kLayerCache = 64;
struct LayerMaps {
    AMaps act[4];       // norm out, attention out, norm-2 out, mlp activation
    bool act_ready;
    WeightMaps cache[kLayerCache];
};

}  // namespace

dcut_status dcut_init_layer(dcut_ctx* ctx) {
    cudaError_t e = cudaFuncSetAttribute(gemm_tcgen05_kernel<kPlain>, cudaFuncAttributeMaxDynamicSharedMemorySize, kGemmSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(gemm_tcgen05_kernel<kResidual>, cudaFuncAttributeMaxDynamicSharedMemorySize, kGemmSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(gemm_tcgen05_kernel<kSwiGLU>, cudaFuncAttributeMaxDynamicSharedMemorySize, kGemmSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(gemm_tcgen05_kernel<kArgmax>, cudaFuncAttributeMaxDynamicSharedMemorySize, kGemmSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(gemm_tcgen05_kernel<kLinear>, cudaFuncAttributeMaxDynamicSharedMemorySize, kLinearSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(gemm_tcgen05_kernel<kLinearGated>, cudaFuncAttributeMaxDynamicSharedMemorySize, kLinearSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(gemm_tcgen05_kernel<kLinear8>, cudaFuncAttributeMaxDynamicSharedMemorySize, kLinearSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(gemm_tcgen05_kernel<kLinear8Gated>, cudaFuncAttributeMaxDynamicSharedMemorySize, kLinearSmem);
    if (e != cudaSuccess) return dcut_check_cuda(ctx, e, "cudaFuncSetAttribute(gemm)");
    {
        // The GEMM is launched as clusters of two CTAs so that it can run tiles on pairs of SMs where that pays
        // (DCUT_GEMM_2CTA=0: never).  ly_gemm_pairs = how many such clusters the device runs at once.
        const char* env = getenv("DCUT_GEMM_2CTA");
        ctx->ly_gemm_pair_mode = (!env || atoi(env) != 0) ? 1 : 0;
        const char* envf = getenv("DCUT_GEMM_FORCE");
        ctx->ly_gemm_force = envf ? atoi(envf) : -1;
        const char* envw = getenv("DCUT_GEMM_WIDTHS");   // bit i allows tile width 256 - 32 i in the one-SM mode
        ctx->ly_gemm_bn_mask = ((envw ? (unsigned)strtoul(envw, nullptr, 0) : kBnMaskAll) & kBnMaskAll) | 1u;
        ctx->ly_gemm_pairs = 0;
        {
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = 2;
            attr[0].val.clusterDim.y = 1;
            attr[0].val.clusterDim.z = 1;
            cudaLaunchConfig_t lc = {};
            lc.gridDim = dim3(2 * ctx->sm_count);
            lc.blockDim = dim3(kGemmThreads);
            lc.dynamicSmemBytes = kGemmSmem;
            lc.attrs = attr;
            lc.numAttrs = 1;
            int n_clusters = 0;
            if (cudaOccupancyMaxActiveClusters(&n_clusters, gemm_tcgen05_kernel<kPlain>, &lc) == cudaSuccess && n_clusters > 0)
                ctx->ly_gemm_pairs = n_clusters;
            else
                (void)cudaGetLastError();
        }
    }
    ctx->layer_maps = calloc(1, sizeof(LayerMaps));
    return ctx->layer_maps ? DCUT_OK : dcut_fail(ctx, DCUT_EINVAL, "out of host memory");
}

void dcut_free_layer(dcut_ctx* ctx) { free(ctx->layer_maps); }

// x[t, :] = embed[tok_id[t], :] for the packed tokens (ids outside [0, V) read row 0 and set the status word)
__global__ void __launch_bounds__(128) embed_kernel(const __nv_bfloat16* __restrict__ embed, const int* __restrict__ tok_id,
                                                    const int* __restrict__ cu_q, int B, int hidden, int V,
                                                    __nv_bfloat16* __restrict__ x, int* __restrict__ status) {
    dcut_pdl_wait();
    dcut_pdl_launch_dependents();
    const int row = blockIdx.x;
    if (row >= cu_q[B]) return;
    int id = tok_id[row];
    if (id < 0 || id >= V) {
        if (threadIdx.x == 0) atomicExch(status, DCUT_DEV_BAD_TOKEN);
        id = 0;
    }
    const uint4* src = reinterpret_cast<const uint4*>(embed + (size_t)id * hidden);
    uint4* dst = reinterpret_cast<uint4*>(x + (size_t)row * hidden);
    for (int v = threadIdx.x; v < hidden / 8; v += 128) dst[v] = src[v];
}

// The whole verification forward of a small model: embedding, n_layers decoder layers (each with its own paged
// cache), final RMSNorm, LM head fused with acceptance.
dcut_status dcut_launch_model(dcut_ctx* ctx, const dcut_model* m, long long num_pages, const int* block_table,
                              int block_table_stride, const int* ctx_lens, const int* cu_q, const int* tok_req,
                              const int* tok_pos, const int* tok_id, const int* draft_ids, int B, int gamma, int T_cap,
                              int* accept_len, int* bonus, int* out_tokens, int* n_accepted_total, int* row_argmax,
                              void* hidden_out, cudaStream_t stream) {
    const int H = ctx->lim.hidden;
    __nv_bfloat16* user = static_cast<__nv_bfloat16*>(hidden_out);
    dcut_status st = dcut_check_cuda(ctx, dcut_launch_pdl(embed_kernel, dim3(T_cap), dim3(128), 0, stream,
                                                          static_cast<const __nv_bfloat16*>(m->embed), tok_id, cu_q, B, H, m->vocab,
                                                          (m->n_layers == 0 && user) ? user : ctx->ly_x[0], ctx->d_status),
                                     "launch embed_kernel");
    if (st != DCUT_OK) return st;
    __nv_bfloat16* x = (m->n_layers == 0 && user) ? user : ctx->ly_x[0];
    for (int l = 0; l < m->n_layers; ++l) {   // ping-pong between the context's two buffers; the last layer may write to the caller
        __nv_bfloat16* y = (l == m->n_layers - 1 && user) ? user : ctx->ly_x[(l + 1) & 1];
        st = dcut_launch_layer(ctx, &m->layers[l], x, y, m->k_caches[l], m->v_caches[l], num_pages,
                               block_table, block_table_stride, ctx_lens, cu_q, tok_req, tok_pos, B, T_cap,
                               l > 0 /* the attention work list of layer 0 serves every layer */, 0, stream);
        if (st != DCUT_OK) return st;
        x = y;
    }
    const float eps = m->n_layers > 0 ? m->layers[0].rms_eps : 1e-6f;
    if ((st = dcut_check_cuda(ctx, dcut_launch_pdl(rmsnorm_kernel, dim3(T_cap), dim3(256), 0, stream,
                                                   static_cast<const __nv_bfloat16*>(x),
                                                   static_cast<const __nv_bfloat16*>(m->g_final), cu_q, B, H, eps, ctx->ly_norm),
                              "launch rmsnorm_kernel")) != DCUT_OK) return st;
    if ((st = dcut_launch_lm_head_argmax(ctx, ctx->ly_norm, m->w_lm, m->vocab, H, cu_q, B, T_cap, ctx->d_row_key, stream)) != DCUT_OK) return st;
    return dcut_launch_accept_match(ctx, nullptr, m->vocab, draft_ids, cu_q, B, gamma, T_cap, accept_len, bonus, out_tokens,
                                    n_accepted_total, row_argmax, ctx->d_row_key, stream);
}

// logits = x . w_lm^T reduced on the fly to one (maximum, first column) word per row: the [T, V] logits never exist
dcut_status dcut_launch_lm_head_argmax(dcut_ctx* ctx, const void* x, const void* w_lm, int V, int K, const int* cu_q, int B,
                                       int T_cap, unsigned long long* row_key, cudaStream_t stream) {
    AMaps am;
    BMaps bm;
    dcut_status st = make_act_maps(ctx, &am, x, T_cap, K);
    if (st != DCUT_OK) return st;
    // rows past V read as zeros; hundreds of tiles per row block: only the full width is offered
    if ((st = make_weight_maps(ctx, &bm, w_lm, V, K, 1u)) != DCUT_OK) return st;
    for (int i = 1; i < kNumBn; ++i) bm.m[i] = bm.m[0];
    GemmArgs g;
    g.cu_q = cu_q;
    g.B = B;
    g.N_out = V;
    g.K = K;
    g.out = nullptr;
    g.residual = nullptr;
    g.row_key = row_key;
    g.V = V;
    g.status = ctx->d_status;
    return launch_gemm<kArgmax>(ctx, am, bm, bm, T_cap, 1u, g, stream);
}

dcut_status dcut_launch_gemm(dcut_ctx* ctx, const void* a, const void* w, const void* w2, int mode, int N, int K,
                             const int* cu_q, int B, int T_cap, void* out, const void* residual, cudaStream_t stream) {
    // generic entry used by dcut_gemm_bf16 (tests, benchmarks): encodes its maps on every call
    AMaps am;
    BMaps bm, b2m;
    dcut_status st = make_act_maps(ctx, &am, a, T_cap, K);
    if (st != DCUT_OK) return st;
    const unsigned mask = (mode == kSwiGLU ? ctx->ly_gemm_bn_mask & kBnMaskSwiGLU : ctx->ly_gemm_bn_mask) | 1u;
    for (int i = 0; i < kNumBn; ++i) bm.m[i] = am.full;   // entries outside the mask are never used; keep them defined
    if ((st = make_weight_maps(ctx, &bm, w, N, K, mask)) != DCUT_OK) return st;
    b2m = bm;
    if (mode == kSwiGLU && (st = make_weight_maps(ctx, &b2m, w2, N, K, mask)) != DCUT_OK) return st;
    GemmArgs g;
    g.cu_q = cu_q;
    g.B = B;
    g.N_out = N;
    g.K = K;
    g.out = static_cast<__nv_bfloat16*>(out);
    g.residual = static_cast<const __nv_bfloat16*>(residual);
    g.row_key = nullptr;
    g.V = 0;
    g.status = ctx->d_status;
    if (mode == kSwiGLU) return launch_gemm<kSwiGLU>(ctx, am, bm, b2m, T_cap, mask, g, stream);
    if (mode == kResidual) return launch_gemm<kResidual>(ctx, am, bm, b2m, T_cap, mask, g, stream);
    return launch_gemm<kPlain>(ctx, am, bm, b2m, T_cap, mask, g, stream);
}

namespace {
// What dcut_linear and dcut_linear8 share; whole k-blocks: the tail reads as zeros in both operands.
template <typename ARGS>
GemmArgs linear_args(dcut_ctx* ctx, const ARGS* l, int k_block, const int* cu_q, int B, int T_cap) {
    GemmArgs g = {};
    g.cu_q = cu_q;
    g.B = B;
    g.N_out = l->N;
    g.K = (l->K + k_block - 1) / k_block * k_block;
    g.out = static_cast<__nv_bfloat16*>(l->out);
    g.residual = static_cast<const __nv_bfloat16*>(l->residual);
    g.bias = static_cast<const __nv_bfloat16*>(l->bias);
    g.bias2 = static_cast<const __nv_bfloat16*>(l->bias2);
    g.ldo = l->ldo;
    g.ldr = l->ldr;
    g.act = l->act;
    g.T_cap = T_cap;
    auto vec = [](const void* p, long long ld) { return !(reinterpret_cast<uintptr_t>(p) & 15) && ld % 8 == 0; };
    g.vec = vec(l->out, l->ldo) && (!l->residual || vec(l->residual, l->ldr));
    g.status = ctx->d_status;
    return g;
}
}  // namespace

dcut_status dcut_launch_linear(dcut_ctx* ctx, const dcut_linear_args* l, const int* cu_q, int B, int T_cap, cudaStream_t stream) {
    GemmArgs g = linear_args(ctx, l, kb_elements(kLinear), cu_q, B, T_cap);
    return l->w2 ? launch_linear<kLinearGated>(ctx, l, T_cap, g, stream) : launch_linear<kLinear>(ctx, l, T_cap, g, stream);
}

dcut_status dcut_launch_linear8(dcut_ctx* ctx, const dcut_linear8_args* l, const int* cu_q, int B, int T_cap, cudaStream_t stream) {
    GemmArgs g = linear_args(ctx, l, kb_elements(kLinear8), cu_q, B, T_cap);
    g.a_scale = l->a_scale;
    g.w_scale = l->w_scale;
    g.w2_scale = l->w2_scale;
    return l->w2 ? launch_linear<kLinear8Gated>(ctx, l, T_cap, g, stream) : launch_linear<kLinear8>(ctx, l, T_cap, g, stream);
}

dcut_status dcut_launch_layer(dcut_ctx* ctx, const dcut_layer_weights* w, const void* x, void* y, void* k_cache,
                              void* v_cache, long long num_pages, const int* block_table, int block_table_stride,
                              const int* ctx_lens, const int* cu_q, const int* tok_req, const int* tok_pos, int B,
                              int T_cap, int reuse_plan, int part, cudaStream_t stream) {
    // part 0: the whole layer.  Tensor-parallel halves (a rank's shard of the heads / of the intermediate width, the
    // projections that close a half WITHOUT the residual, so that the ranks' outputs can be summed first):
    // part 1: y = Attn(RoPE(Wqkv . RMSNorm(x))) . Wo^T;  part 2: y = (SiLU(Wg . n) * (Wu . n)) . Wd^T with n = RMSNorm(x).
    const dcut_limits& l = ctx->lim;
    const int H = l.hidden, I = l.intermediate, Dh = l.head_dim;
    const int qkv_w = (l.n_q_heads + 2 * l.n_kv_heads) * Dh, q_w = l.n_q_heads * Dh;
    const int max_T = l.max_B * (l.max_gamma + 1);
    LayerMaps* lm = static_cast<LayerMaps*>(ctx->layer_maps);
    dcut_status st;
    if (!lm->act_ready) {
        if ((st = make_act_maps(ctx, &lm->act[0], ctx->ly_norm, max_T, H)) != DCUT_OK) return st;
        if ((st = make_act_maps(ctx, &lm->act[1], ctx->ly_attn, max_T, q_w)) != DCUT_OK) return st;
        if ((st = make_act_maps(ctx, &lm->act[2], ctx->ly_norm2, max_T, H)) != DCUT_OK) return st;
        if ((st = make_act_maps(ctx, &lm->act[3], ctx->ly_act, max_T, I)) != DCUT_OK) return st;
        lm->act_ready = true;
    }
    const void* wp[5] = {w->w_qkv, w->w_o, w->w_gate, w->w_up, w->w_down};
    const long long wr[5] = {qkv_w, H, I, I, H}, wc[5] = {H, q_w, H, H, I};
    const unsigned mask = ctx->ly_gemm_bn_mask, wmask[5] = {mask, mask, mask & kBnMaskSwiGLU, mask & kBnMaskSwiGLU, mask};
    WeightMaps* wm = &lm->cache[(reinterpret_cast<uintptr_t>(w->w_qkv) >> 8) % kLayerCache];
    for (int i = 0; i < 5; ++i)
        if (wm->w[i] != wp[i]) {
            if ((st = make_weight_maps(ctx, &wm->m[i], wp[i], wr[i], wc[i], wmask[i] | 1u)) != DCUT_OK) return st;
            wm->w[i] = wp[i];
        }
    GemmArgs g;
    g.cu_q = cu_q;
    g.B = B;
    g.row_key = nullptr;
    g.V = 0;
    g.status = ctx->d_status;

    if (part != 2) {
    // 1. n = RMSNorm(x)
    if ((st = dcut_check_cuda(ctx, dcut_launch_pdl(rmsnorm_kernel, dim3(T_cap), dim3(256), 0, stream, static_cast<const __nv_bfloat16*>(x),
                                                   static_cast<const __nv_bfloat16*>(w->g_attn), cu_q, B, H, w->rms_eps, ctx->ly_norm),
                              "launch rmsnorm_kernel")) != DCUT_OK) return st;
    // 2. qkv = n . Wqkv^T
    g.N_out = qkv_w; g.K = H; g.out = ctx->ly_qkv; g.residual = nullptr;
    if ((st = launch_gemm<kPlain>(ctx, lm->act[0], wm->m[0], wm->m[0], T_cap, wmask[0], g, stream)) != DCUT_OK) return st;
    // 3. RoPE, append the new K/V to the paged cache
    RopeArgs r;
    r.qkv = ctx->ly_qkv; r.cu_q = cu_q; r.tok_req = tok_req; r.tok_pos = tok_pos; r.block_table = block_table;
    r.block_table_stride = block_table_stride; r.inv_freq = ctx->ly_inv_freq; r.B = B; r.n_q_heads = l.n_q_heads;
    r.n_kv_heads = l.n_kv_heads; r.head_dim = Dh; r.num_pages = num_pages; r.q_out = ctx->ly_q;
    r.k_cache = static_cast<__nv_bfloat16*>(k_cache); r.v_cache = static_cast<__nv_bfloat16*>(v_cache); r.status = ctx->d_status;
    if ((st = dcut_check_cuda(ctx, dcut_launch_pdl(rope_append_kernel, dim3(T_cap), dim3(256), 0, stream, r), "launch rope_append_kernel")) != DCUT_OK) return st;
    // 4. attention
    st = dcut_launch_verify_attn(ctx, ctx->ly_q, k_cache, v_cache, num_pages, block_table, block_table_stride, ctx_lens,
                                 cu_q, B, T_cap, 1.0f / sqrtf((float)Dh), ctx->ly_attn, nullptr, reuse_plan, nullptr, nullptr, stream);
    if (st != DCUT_OK) return st;
    // 5. h1 = x + attn . Wo^T   (a tensor-parallel half: the rank's partial product alone, into y)
    g.N_out = H; g.K = q_w;
    if (part == 1) {
        g.out = static_cast<__nv_bfloat16*>(y); g.residual = nullptr;
        return launch_gemm<kPlain>(ctx, lm->act[1], wm->m[1], wm->m[1], T_cap, wmask[1], g, stream);
    }
    g.out = ctx->ly_h1; g.residual = static_cast<const __nv_bfloat16*>(x);
    if ((st = launch_gemm<kResidual>(ctx, lm->act[1], wm->m[1], wm->m[1], T_cap, wmask[1], g, stream)) != DCUT_OK) return st;
    }
    // 6. n2 = RMSNorm(h1)   (the MLP half of a tensor-parallel layer starts here, from the caller's h1)
    const __nv_bfloat16* h1 = part == 2 ? static_cast<const __nv_bfloat16*>(x) : ctx->ly_h1;
    if ((st = dcut_check_cuda(ctx, dcut_launch_pdl(rmsnorm_kernel, dim3(T_cap), dim3(256), 0, stream, h1,
                                                   static_cast<const __nv_bfloat16*>(w->g_mlp), cu_q, B, H, w->rms_eps, ctx->ly_norm2),
                              "launch rmsnorm_kernel")) != DCUT_OK) return st;
    // 7. act = SiLU(n2 . Wg^T) * (n2 . Wu^T)
    g.N_out = I; g.K = H; g.out = ctx->ly_act; g.residual = nullptr;
    if ((st = launch_gemm<kSwiGLU>(ctx, lm->act[2], wm->m[2], wm->m[3], T_cap, wmask[2], g, stream)) != DCUT_OK) return st;
    // 8. y = h1 + act . Wd^T
    g.N_out = H; g.K = I; g.out = static_cast<__nv_bfloat16*>(y);
    if (part == 2) {
        g.residual = nullptr;
        return launch_gemm<kPlain>(ctx, lm->act[3], wm->m[4], wm->m[4], T_cap, wmask[4], g, stream);
    }
    g.residual = ctx->ly_h1;
    return launch_gemm<kResidual>(ctx, lm->act[3], wm->m[4], wm->m[4], T_cap, wmask[4], g, stream);
}

namespace {
// out = a + b over the rows in use (bf16, one 16-byte vector per thread and step)
__global__ void __launch_bounds__(256) residual_add_kernel(const uint4* __restrict__ a, const uint4* __restrict__ b, uint4* __restrict__ out,
                                                           const int* __restrict__ cu_q, int B, int vec_per_row) {
    dcut_pdl_wait();
    dcut_pdl_launch_dependents();
    const long long n = (long long)cu_q[B] * vec_per_row;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
        const uint4 x = a[i], y = b[i];
        const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
        uint32_t r[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const __nv_bfloat162 u = *reinterpret_cast<const __nv_bfloat162*>(&xs[e]), v = *reinterpret_cast<const __nv_bfloat162*>(&ys[e]);
            const __nv_bfloat162 s = __floats2bfloat162_rn(__low2float(u) + __low2float(v), __high2float(u) + __high2float(v));
            r[e] = *reinterpret_cast<const uint32_t*>(&s);
        }
        out[i] = make_uint4(r[0], r[1], r[2], r[3]);
    }
}
}  // namespace

dcut_status dcut_launch_residual_add(dcut_ctx* ctx, const void* a, const void* b, void* out, int width, const int* cu_q, int B,
                                     int T_cap, cudaStream_t stream) {
    const long long cap = (long long)T_cap * (width / 8);
    int grid = (int)((cap + 255) / 256);
    if (grid > 4 * ctx->sm_count) grid = 4 * ctx->sm_count;
    if (grid < 1) grid = 1;
    return dcut_check_cuda(ctx, dcut_launch_pdl(residual_add_kernel, dim3(grid), dim3(256), 0, stream, static_cast<const uint4*>(a),
                                                static_cast<const uint4*>(b), static_cast<uint4*>(out), cu_q, B, width / 8),
                           "launch residual_add_kernel");
}
