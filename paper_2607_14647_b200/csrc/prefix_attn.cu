// dcut_prefix_attn: verification attention of a batch whose requests share prefixes.
//
//   out = softmax_j(q . k_j * scale) v_j  over the group's shared positions j < P and the request's own P <= j <= L + t
//
// The softmax is split at P.  Each part gives its normalised output and its log-sum-exp, and two such pairs merge into
// one (weights 2^(lse - max)), so the shared keys are read once for all rows of a group instead of once per request:
//
//   prefix_plan_kernel     two CTAs: the partition of the shared part (prefix_plan.cuh) and, for the own parts, the work
//                          list of dcut_verify_attn on own lengths L - P
//   attn_item_kernel, attn_combine_kernel   (verify_attn.cu) the own parts: bound by HBM; output kept in fp32
//   prefix_attn_kernel     the shared part on the tensor cores, its epilogue merging the own part's result and writing out
//   prefix_combine_kernel  merges the pieces of the items that a segment boundary cuts, and the own part's result
//
// prefix_attn_kernel, persistent, one CTA per SM, 384 threads.  An item is 256 query rows (two tiles of 128) of a kv head
// against a run of 64-key blocks:
//   warp 0      TMA: the item's Q tiles, and K and V of each block page by page into a ring of eight 64-key slots
//   warps 1-2   issue tcgen05.mma, one elected lane per tile t: S_t = Q_t K^T (A and B from shared memory), O_t += P_t V
//               (P from tensor memory, V read MN-major)
//   warps 4-11  two softmax teams, one per tile, a thread per row.  The running maximum only moves when it would grow by
//               more than 2^8 (then O is rescaled in tensor memory); row sums are kept in fp32 over the unrounded weights.
// Tensor memory holds, per tile, a 128 x DH fp32 O and two 128 x 64 fp32 S, each of which its P replaces in place: while a
// team exponentiates one block, the tensor cores fill its other buffer, and a step has two hand-overs only (S to the
// softmax, P to the MMAs), each of about 190 cycles between warps.
// An odd last tile is a single: both teams work on the one tile, taking its key blocks in turn, and merge at the end.
// P is rounded to bf16 (half a step, 2^-8 of the weight at most, as V's type asks of the MMA); everything else stays in fp32
// until the one rounding of the output.
//
// Measured: 2176 tokens of 32q/8kv heads behind 8192 keys (292 Gflop) 318 us of a call of 398 to 407; a pair of tiles takes 1900 to
// 2050 cycles per block, of which the tensor pipe is busy for 1544 (Q K^T with both operands in shared memory runs at half
// rate at N = 64), the MUFU for 1024; the softmax code alone takes 1300.  Blocks of 128 or 80 keys with one S buffer per
// tile: 317 and 297-338 us.  Rescaling by a stale maximum 636 (spills), warps taking turns 592.
//
// Every wait is bounded; on expiry a role sets the device status word, the others see the CTA's abort flag.
#include <cuda.h>
#include <cuda_bf16.h>

#include "attn_plan.cuh"
#include "dcut_internal.h"
#include "prefix_plan.cuh"

namespace {

using namespace dcut_prefix;

constexpr int kThreads = 384;
constexpr int kTeamThreads = 128;
// Ring of K and V blocks, in the order K V K V.  No role waits for a slot's load while the load before it in that slot may
// still be under way: the wait would return at once (tests/test_prefix_ring.py walks the roles' waits under delayed loads).
// K: an item's Q arrives after the last Q K^T of the item before.  V: the issuers wait for o_free first; a softmax warp that
// clears V rows has seen the item before end (both teams' o_full of a single, its own team's of a dual, which reads every V).
constexpr int kSlots = 8;
constexpr int kPage = dcut_plan::kPage;
constexpr int kPagesPerBlock = kBlock / kPage;
constexpr int kStageBytes = 2048;     // epilogue staging of a warp: 32 rows x 16 fp32
constexpr int kSpinLimit = 1 << 21;
constexpr int kTmemCols = 512, kColS = 256;    // tile t: O at 128 t, S / P buffer b at 256 + 128 t + 64 b
constexpr float kRescaleLog2 = 8.0f;
constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;

// ------------------------------------------------------------------------------------------------ PTX

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive_expect_tx(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// whether the phase is over, without waiting for it
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, const volatile int* abort_flag) {
    if (mbar_try_wait(bar, parity)) return true;
    if (abort_flag && *abort_flag) return false;
    for (int it = 0; it < kSpinLimit; ++it) {
        if (mbar_try_wait(bar, parity)) return true;
        if (it > 4096) {
            __nanosleep(128);
            if ((it & 255) == 0 && abort_flag && *abort_flag) return false;
        }
    }
    return false;
}
__device__ __forceinline__ bool elect_one() {
    uint32_t pred;
    asm volatile("{\n\t.reg .pred P;\n\telect.sync _|P, 0xffffffff;\n\tselp.u32 %0, 1, 0, P;\n\t}" : "=r"(pred));
    return pred != 0;
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// D[tmem] (+)= A[smem] . B[smem]
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, {%5, %5, %5, %5}, p;\n\t}"
        ::"r"(d), "l"(da), "l"(db), "r"(idesc), "r"(accumulate), "r"(0u) : "memory");
}
// D[tmem] (+)= A[tmem] . B[smem]
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t db, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, {%5, %5, %5, %5}, p;\n\t}"
        ::"r"(d), "r"(a), "l"(db), "r"(idesc), "r"(accumulate), "r"(0u) : "memory");
}
__device__ __forceinline__ void tc_ld32(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
}
__device__ __forceinline__ void tc_ld16(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
}
__device__ __forceinline__ void tc_st32(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]),
          "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]),
          "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t taddr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                 "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ float fast_exp2(float x) {     // 2 ulp; -inf -> 0
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ unsigned long long pack_f32x2(float lo, float hi) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpack_f32x2(unsigned long long v, float& lo, float& hi) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ unsigned long long fma_f32x2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ unsigned long long add_f32x2(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float fmax3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// Shared-memory descriptors (128-byte swizzle, version 1).  K-major: 8-row groups `sbo` bytes apart.  MN-major (V: rows =
// keys, 128 bytes = 64 head elements): the next 64 head elements 2048 bytes on, the next 8 keys 1024.
__device__ __forceinline__ uint64_t desc_kmajor(uint32_t addr, uint32_t sbo) {
    return (uint64_t)((addr & 0x3ffff) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(sbo >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ uint64_t desc_mnmajor(uint32_t addr) {
    return (uint64_t)((addr & 0x3ffff) >> 4) | ((uint64_t)(2048 >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
constexpr uint32_t kIdescBase = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 4) << 24);   // fp32 += bf16 x bf16, M = 128

// ------------------------------------------------------------------------------------------------ shared declarations

struct PrefixArgs {
    const int* prefix_table;
    int prefix_table_stride;
    const Group* groups;
    const Seg* segs;
    int n_groups, n_q_heads, n_kv_heads, group_size;
    long long num_pages;
    float scale_log2;
    const float* own_o;           // [T, Hq, DH], [T, Hq]: the own parts' outputs and log-sum-exps
    const float* own_lse;
    __nv_bfloat16* out;
    float* lse;                   // or null
    float* part_o;                // [2 n_seg][256][DH], [2 n_seg][256]
    float* part_lse;
    int* status;
};

struct __align__(16) Ctrl {
    unsigned long long kv_full[kSlots], kv_empty[kSlots];
    unsigned long long q_full, q_free;
    unsigned long long s_full[2][2], p_full[2][2], pv_done[2], o_full[2];   // [team][buffer], [team]
    unsigned long long o_free, x_ready, drain[2];
    float xm[2][kTileRows], xl[2][kTileRows];      // a single's teams: running maximum and sum of each row
    uint32_t tmem_base;
    int abort;
};

template <int DH>
struct Smem {
    static constexpr int kQTile = kTileRows * DH * 2;
    static constexpr int kBlockBytes = kBlock * DH * 2;
    static constexpr int kPageBytes = kPage * DH * 2;
    static constexpr int kRing = 2 * kQTile;
    static constexpr int kStage = kRing + kSlots * kBlockBytes;
    static constexpr int kCtrl = kStage + 8 * kStageBytes;
    static constexpr int kTotal = kCtrl + (int)sizeof(Ctrl) + 1024;
};
static_assert(Smem<128>::kTotal <= 232448, "shared memory of a CTA");

__device__ __forceinline__ int pages_of_block(int len, int blk) {
    const int keys = len - blk * kBlock;
    return keys >= kBlock ? kPagesPerBlock : (keys + kPage - 1) / kPage;
}

// ------------------------------------------------------------------------------------------------ roles

template <int DH>
__device__ __forceinline__ void produce(const CUtensorMap& q_map, const CUtensorMap& k_map, const CUtensorMap& v_map,
                                        const PrefixArgs& a, unsigned char* smem, Ctrl* c, Walk w) {
    using L = Smem<DH>;
    const int lane = threadIdx.x & 31;
    const uint32_t kv_full = smem_u32(c->kv_full), kv_empty = smem_u32(c->kv_empty);
    const int tpt = tile_tokens(a.group_size);
    const uint32_t q_bytes = (uint32_t)(tpt * a.group_size * DH * 2);
    Item it;
    int n_items = 0, pos = 0;             // pos: K and V blocks issued so far
    bool failed = false;
    while (!failed && next_item(w, a.groups, &it)) {
        if (it.blocks == 0) continue;
        const int* table = a.prefix_table + (size_t)it.g * a.prefix_table_stride;
        int page = 0;
        if (lane < pages_of_block(it.len, it.b0)) page = table[it.b0 * kPagesPerBlock + lane];
        for (int blk = it.b0; blk < it.b1 && !failed; ++blk) {
            const int np = pages_of_block(it.len, blk);
            if (lane < np && (page < 0 || page >= a.num_pages)) {
                atomicExch(a.status, DCUT_DEV_BAD_PAGE);
                page = 0;
            }
            const int row = (page * a.n_kv_heads + it.h) * kPage;
            int rows[kPagesPerBlock];
#pragma unroll
            for (int j = 0; j < kPagesPerBlock; ++j) rows[j] = __shfl_sync(0xffffffffu, row, j);
            if (blk + 1 < it.b1 && lane < pages_of_block(it.len, blk + 1)) page = table[(blk + 1) * kPagesPerBlock + lane];
#pragma unroll
            for (int kv = 0; kv < 2; ++kv, ++pos) {
                const int slot = pos % kSlots, use = pos / kSlots;
                if (use > 0 && !__all_sync(0xffffffffu, mbar_wait(kv_empty + 8 * slot, (use - 1) & 1, &c->abort))) {
                    failed = true;
                    break;
                }
                if (elect_one()) {
                    const uint32_t bar = kv_full + 8 * slot, dst = smem_u32(smem + L::kRing + slot * L::kBlockBytes);
                    mbar_arrive_expect_tx(bar, (uint32_t)np * L::kPageBytes);
#pragma unroll
                    for (int j = 0; j < kPagesPerBlock; ++j)
                        if (j < np) {
                            if (DH == 128 && kv == 0) tma_load_4d(dst + j * L::kPageBytes, &k_map, 0, 0, 0, rows[j] >> 3, bar);
                            else tma_load_3d(dst + j * L::kPageBytes, kv == 0 ? &k_map : &v_map, 0, rows[j], 0, bar);
                        }
                }
                __syncwarp();
                if (kv == 0 && blk == it.b0) {
                    // the item's Q tiles, once the last QK^T of the item before has read the old ones
                    if (n_items > 0 && !__all_sync(0xffffffffu, mbar_wait(smem_u32(&c->q_free), (n_items - 1) & 1, &c->abort))) {
                        failed = true;
                        ++pos;
                        break;
                    }
                    if (elect_one()) {
                        const uint32_t bar = smem_u32(&c->q_full);
                        mbar_arrive_expect_tx(bar, (it.dual ? 2 : 1) * q_bytes);
                        for (int t = 0; t <= it.dual; ++t)
#pragma unroll
                            for (int half = 0; half < DH / 64; ++half)
                                tma_load_4d(smem_u32(smem + t * L::kQTile + half * kTileRows * 128), &q_map, 0, it.h * a.group_size, it.q0 + t * tpt, half, bar);
                    }
                    __syncwarp();
                    ++n_items;
                }
            }
        }
    }
    if (failed) {
        atomicExch(a.status, DCUT_DEV_ATTN_WAIT_TIMEOUT);
        c->abort = 1;
        // nothing of this CTA's is in flight when it leaves
        for (int p = pos > kSlots ? pos - kSlots : 0; p < pos; ++p) mbar_wait(kv_full + 8 * (p % kSlots), (p / kSlots) & 1, nullptr);
        if (n_items > 0) mbar_wait(smem_u32(&c->q_full), (n_items - 1) & 1, nullptr);
    }
}

// The issuer of one team's products.  One elected lane (not `lane == 0`: the compiler then keeps the operands of
// tcgen05.mma in uniform registers) runs the whole role.  Each team has an issuer of its own: issuing an MMA lasts as long
// as the MMA (73 cycles for Q K^T of 64 keys and 16 of the head's elements, 65 for P V of 16 keys, at head size 128), a wait for
// a barrier about 150 even when its phase is over, and while one issuer waits the other feeds the tensor pipe.
template <int DH>
__device__ __forceinline__ void issue(const PrefixArgs& a, unsigned char* smem, Ctrl* c, Walk w, const int team) {
    using L = Smem<DH>;
    constexpr uint32_t kIdescPV = kIdescBase | (1u << 16) | ((uint32_t)(DH >> 3) << 17);
    const uint32_t kv_full = smem_u32(c->kv_full), kv_empty = smem_u32(c->kv_empty);
    const uint32_t s_full = smem_u32(c->s_full[team]), p_full = smem_u32(c->p_full[team]);
    const uint32_t pv_done = smem_u32(c->pv_done) + 8 * team, o_full = smem_u32(c->o_full) + 8 * team;
    const uint32_t t_o = c->tmem_base + 128 * team, t_s = c->tmem_base + kColS + 128 * team;
    const uint32_t ring = smem_u32(smem + L::kRing);
    Item it;
    int n_items = 0, n_qk = 0, n_pv = 0;  // this team's steps so far: step n uses buffer n % 2, for the (n / 2)th time
    int base = 0, base_phase = 0;         // ring slot of the item's first K block, and its phase
    bool ok = true;
    auto wait = [&](uint32_t bar, int parity) { return mbar_wait(bar, parity & 1, &c->abort); };
    while (ok && next_item(w, a.groups, &it)) {
        if (it.blocks == 0) continue;
        const int nblk = it.b1 - it.b0;
        const int steps = it.dual ? nblk : (nblk + 1 - team) >> 1;            // this team's blocks: all, or every other one
        const int last_pages = pages_of_block(it.len, it.b1 - 1);
        const bool ends_here = it.dual || ((nblk - 1) & 1) == team;           // the piece's last block is this team's
        const int ahead = it.dual ? 2 : 4;                                    // ring slots from one of its blocks to the next
        const uint32_t q_tile = smem_u32(smem) + (it.dual ? team * L::kQTile : 0);
        int k_slot = base, k_phase = base_phase;
        auto move = [&](int& slot, int& phase, int by) {
            slot += by;
            if (slot >= kSlots) {
                slot -= kSlots;
                phase ^= 1;
            }
        };
        if (!it.dual) move(k_slot, k_phase, 2 * team);
        int v_slot = k_slot, v_phase = k_phase;
        move(v_slot, v_phase, 1);
        if (!wait(smem_u32(&c->q_full), n_items)) {
            ok = false;
            break;
        }
        // S = Q K^T of the team's next block (the P V that read this buffer's last P has completed)
        auto qk = [&](bool last) {
            tc_fence_after();
            const uint32_t k_addr = ring + k_slot * L::kBlockBytes, d = t_s + 64 * (n_qk & 1);
            const int np = last && ends_here ? last_pages : kPagesPerBlock;
            const uint32_t idesc = kIdescBase | ((uint32_t)(np * kPage >> 3) << 17);
#pragma unroll
            for (int half = 0; half < DH / 64; ++half) {
                const uint64_t dq = desc_kmajor(q_tile + half * kTileRows * 128, 1024);
                const uint64_t dk = DH == 128 ? desc_kmajor(k_addr + half * 1024, 2048) : desc_kmajor(k_addr, 1024);
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) tc_mma_ss(d, dq + 2 * ks, dk + 2 * ks, idesc, (half | ks) ? 1u : 0u);
            }
            tc_commit(s_full + 8 * (n_qk & 1));
            if (last) tc_commit(smem_u32(&c->q_free));
            ++n_qk;
            move(k_slot, k_phase, ahead);
        };
        for (int s = 0; ok && s < 2 && s < steps; ++s)
            if ((ok = wait(kv_full + 8 * k_slot, k_phase))) qk(s == steps - 1);
        // The epilogues of the item before are over.  Before this wait the item has no wait for a V slot, no P V and no o_full:
        // a parity wait cannot tell two phases from none.  The V of the item before may have been the other team's (a single's
        // every other block), so its slot may be two phases behind; with o_free all of them have been loaded and read.  O is
        // overwritten by the first P V, and a warp that still has to look at o_full must not find it a phase ahead (a single's
        // second team may have no block).
        if (ok && n_items > 0) ok = wait(smem_u32(&c->o_free), n_items - 1);
        for (int s = 0; ok && s < steps; ++s) {
            if (!wait(kv_full + 8 * v_slot, v_phase) || !wait(p_full + 8 * (n_pv & 1), n_pv >> 1)) {
                ok = false;
                break;
            }
            tc_fence_after();
            const uint64_t dv = desc_mnmajor(ring + v_slot * L::kBlockBytes);
            const uint32_t p = t_s + 64 * (n_pv & 1);
            const int np = s == steps - 1 && ends_here ? last_pages : kPagesPerBlock;
            if (np == kPagesPerBlock) {
#pragma unroll
                for (int j = 0; j < kPagesPerBlock; ++j) tc_mma_ts(t_o, p + 8 * j, dv + (L::kPageBytes >> 4) * j, kIdescPV, (s || j) ? 1u : 0u);
            } else {
                for (int j = 0; j < np; ++j) tc_mma_ts(t_o, p + 8 * j, dv + (L::kPageBytes >> 4) * j, kIdescPV, (s || j) ? 1u : 0u);
            }
            tc_commit(pv_done);
            const bool more = s + 2 < steps;
            if (!wait(pv_done, n_pv) || (more && !wait(kv_full + 8 * k_slot, k_phase))) {
                ok = false;
                break;
            }
            mbar_arrive(kv_empty + 8 * v_slot);
            if (!it.dual) mbar_arrive(kv_empty + 8 * v_slot);     // (a slot waits for two arrivals)
            ++n_pv;
            move(v_slot, v_phase, ahead);
            if (more) qk(s + 2 == steps - 1);
        }
        if (!ok) break;
        if (steps == 0) tc_commit(smem_u32(&c->q_free));
        tc_commit(o_full);
        const int pos = base + 2 * nblk;
        base = pos % kSlots;
        base_phase ^= (pos / kSlots) & 1;
        ++n_items;
    }
    if (!ok) {
        atomicExch(a.status, DCUT_DEV_ATTN_WAIT_TIMEOUT);
        c->abort = 1;
        tc_commit(smem_u32(&c->drain) + 8 * team);                            // the MMAs issued so far end before tensor memory is freed
        mbar_wait(smem_u32(&c->drain) + 8 * team, 0, nullptr);
    }
}

// A softmax thread's steps over an item: its team's blocks of the piece, one after the other.  Not inlined: the loop then
// has the registers to itself (64 scores, 32 words of P), and what the caller keeps for the epilogue is saved once per item.
struct Steps {
    uint32_t t_s, t_o;            // this lane's S / P buffers and O in tensor memory
    uint32_t s_full, p_full, pv_done, kv_full, kv_empty;
    int steps, last_cols;         // blocks; columns of the last of them (kBlock unless the prefix ends in it)
    int n;                        // the team's steps before these
    int pos, ahead;               // ring position of the first K block, positions from one of the team's blocks to the next
    int live;                     // some of this warp's rows exist
    int releases;                 // arrivals this lane owes the ring for every K block: 0, 1, or 2 (a single's only reader)
    float cs;
    const volatile int* abort_flag;
};
template <int DH>
__device__ __noinline__ bool softmax_steps(const Steps p, unsigned char* smem_ring, float* m_out, float* l_out) {
    constexpr int kPageBytes = Smem<DH>::kPageBytes;
    const int lane = threadIdx.x & 31;
    auto warp_wait = [&](uint32_t bar, int parity) {              // one lane polls
        return __any_sync(0xffffffffu, lane == 0 && mbar_wait(bar, parity, p.abort_flag));
    };
    auto warp_arrive = [&](uint32_t bar) {                        // one arrival for the warp's 32
        __syncwarp();
        if (lane == 0) mbar_arrive(bar);
    };
    float m_run = -INFINITY, l_run = 0.0f;
    int n = p.n, pos = p.pos;
    bool s_over = false;                                          // (lane 0) the next S is known to be there
#pragma unroll 1
    for (int s = 0; s < p.steps; ++s, ++n, pos += p.ahead) {
        const uint32_t t_s = p.t_s + 64 * (n & 1), p_bar = p.p_full + 8 * (n & 1);
        if (!__any_sync(0xffffffffu, s_over) && !warp_wait(p.s_full + 8 * (n & 1), (n >> 1) & 1)) return false;
        s_over = false;
        // (a committed S: K has been read)
        if (p.releases > 0) mbar_arrive(p.kv_empty + 8 * (pos & (kSlots - 1)));
        if (p.releases > 1) mbar_arrive(p.kv_empty + 8 * (pos & (kSlots - 1)));
        if (s == p.steps - 1 && p.last_cols < kBlock) {
            if (p.last_cols & (kPage - 1)) {
                // The prefix ends inside this block's last page.  What lies behind it has weight 0, but 0 x NaN is NaN: the
                // V rows of the unused slots are cleared before the MMA reads them (in a dual by both teams, each for its own).
                const int slot = (pos + 1) & (kSlots - 1);
                if (!warp_wait(p.kv_full + 8 * slot, ((pos + 1) / kSlots) & 1)) return false;
                unsigned char* page = smem_ring + slot * Smem<DH>::kBlockBytes + (p.last_cols / kPage) * kPageBytes;
                const int r0 = p.last_cols & (kPage - 1), chunks = (kPage - r0) * 8;       // 16-byte chunks of a 64-element half
                for (int i = threadIdx.x & (kTeamThreads - 1); i < chunks * (DH / 64); i += kTeamThreads) {
                    const int half = i / chunks, rest = i - half * chunks;
                    *reinterpret_cast<uint4*>(page + half * (kPage * 128) + r0 * 128 + rest * 16) = make_uint4(0, 0, 0, 0);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            // the columns behind the prefix become -inf, in tensor memory: the common path has one version of the scores
            tc_fence_after();
#pragma unroll 1
            for (int cc = 0; cc < kBlock; cc += 16) {
                uint32_t x[16];
                tc_ld16(t_s + cc, x);
                tc_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] = cc + e < p.last_cols ? x[e] : 0xff800000u;
                tc_st16(t_s + cc, x);
            }
            tc_wait_st();
        }
        if (!p.live) {                                            // P keeps what it holds
            warp_arrive(p_bar);
            continue;
        }
        tc_fence_after();
        uint32_t sr[kBlock];
        tc_ld32(t_s, sr);
        tc_ld32(t_s + 32, sr + 32);
        tc_wait_ld();
        float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int e = 0; e < kBlock; e += 8)
#pragma unroll
            for (int k = 0; k < 4; ++k) mx4[k] = fmax3(mx4[k], __uint_as_float(sr[e + k]), __uint_as_float(sr[e + 4 + k]));
        const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3]));
        const bool grows = mx > m_run && (m_run == -INFINITY || (mx - m_run) * p.cs > kRescaleLog2);
        if (__any_sync(0xffffffffu, grows)) {
            const float alpha = grows ? fast_exp2((m_run - mx) * p.cs) : 1.0f;
            if (grows) m_run = mx;
            l_run *= alpha;
            if (s > 0) {
                if (!warp_wait(p.pv_done, (n - 1) & 1)) return false;              // the team's last P V: O is at rest
                tc_fence_after();
#pragma unroll 1
                for (int cc = 0; cc < DH; cc += 16) {             // (S is in registers: no more of O at once)
                    uint32_t o[16];
                    tc_ld16(p.t_o + cc, o);
                    tc_wait_ld();
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                    tc_st16(p.t_o + cc, o);
                }
                tc_wait_st();
            }
        }
        const float cs = p.cs, mc = (m_run == -INFINITY ? 0.0f : m_run) * cs;
        const unsigned long long cs2 = pack_f32x2(cs, cs), nmc2 = pack_f32x2(-mc, -mc);
        unsigned long long sum2[2] = {0ull, 0ull};                // four partial sums, two per register pair
        uint32_t pw[kBlock / 2];
#pragma unroll
        for (int e = 0; e < kBlock / 2; ++e) {
            float x0, x1;
            unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(sr[2 * e]), __uint_as_float(sr[2 * e + 1])), cs2, nmc2), x0, x1);
            const float p0 = fast_exp2(x0), p1 = fast_exp2(x1);
            sum2[e & 1] = add_f32x2(sum2[e & 1], pack_f32x2(p0, p1));
            pw[e] = pack_bf16(p0, p1);
        }
        tc_st32(t_s, pw);                                         // P over the first half of S
        // (asked for now, read at the next step's beginning: the answer takes more than 100 cycles)
        s_over = lane == 0 && s + 1 < p.steps && mbar_test(p.s_full + 8 * ((n + 1) & 1), ((n + 1) >> 1) & 1);
        float s0, s1, s2, s3;
        unpack_f32x2(sum2[0], s0, s1);
        unpack_f32x2(sum2[1], s2, s3);
        l_run += (s0 + s1) + (s2 + s3);
        tc_wait_st();
        tc_fence_before();
        warp_arrive(p_bar);
    }
    *m_out = m_run;
    *l_out = l_run;
    return true;
}

template <int DH>
__device__ __forceinline__ void softmax(const PrefixArgs& a, unsigned char* smem, Ctrl* c, Walk w) {
    using L = Smem<DH>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int team = (warp - 4) >> 2, quarter = warp & 3;
    const int R = quarter * 32 + lane;                            // tensor-memory lane = row of the tile
    const int gs = a.group_size, tpt = tile_tokens(gs), row_tok = R / gs, row_head = R - row_tok * gs;
    const uint32_t lanes = c->tmem_base + ((uint32_t)(quarter * 32) << 16);
    const uint32_t t_o = lanes + 128 * team, t_oo = lanes + 128 * (team ^ 1);
    const uint32_t o_full = smem_u32(c->o_full) + 8 * team;
    float* stage = reinterpret_cast<float*>(smem + L::kStage + (warp - 4) * kStageBytes);
    const float cs = a.scale_log2;
    Item it;
    int n_items = 0, n_s = 0, n_x = 0, first = 0;
    bool failed = false;
    auto warp_wait = [&](uint32_t bar, int parity) { return __any_sync(0xffffffffu, lane == 0 && mbar_wait(bar, parity, &c->abort)); };
    auto warp_arrive = [&](uint32_t bar) {
        __syncwarp();
        if (lane == 0) mbar_arrive(bar);
    };
    while (next_item(w, a.groups, &it)) {
        const int nblk = it.b1 - it.b0, tile = it.dual ? team : 0;
        const int tok = tile * tpt + row_tok;
        const bool valid = row_tok < tpt && tok < it.tokens;
        const bool live = __any_sync(0xffffffffu, valid);
        float m_run = -INFINITY, l_run = 0.0f;
        const int steps = it.dual ? nblk : (nblk + 1 - team) >> 1;
        if (steps > 0) {
            Steps p;
            p.t_s = lanes + kColS + 128 * team;
            p.t_o = t_o;
            p.s_full = smem_u32(c->s_full[team]);
            p.p_full = smem_u32(c->p_full[team]);
            p.pv_done = smem_u32(c->pv_done) + 8 * team;
            p.kv_full = smem_u32(c->kv_full);
            p.kv_empty = smem_u32(c->kv_empty);
            p.steps = steps;
            p.last_cols = it.dual || ((nblk - 1) & 1) == team ? min(kBlock, it.len - (it.b1 - 1) * kBlock) : kBlock;
            p.n = n_s;
            p.pos = 2 * (first + (it.dual ? 0 : team));
            p.ahead = it.dual ? 2 : 4;
            p.live = live;
            p.releases = quarter == 0 && lane == 0 ? (it.dual ? 1 : 2) : 0;
            p.cs = cs;
            p.abort_flag = &c->abort;
            if (!softmax_steps<DH>(p, smem + L::kRing, &m_run, &l_run)) {
                failed = true;
                break;
            }
            n_s += steps;
        }

        // ---------------------------------------------------------------- epilogue
        const bool has = it.blocks > 0, whole = is_whole(it);
        const bool other = !it.dual && (nblk + team) >> 1 > 0;    // the other team has blocks of the same rows
        float m_o = -INFINITY, l_o = 0.0f;                        // the other team's part of a single's row
        // 16 columns of the warp's 32 rows at a time go through shared memory, so that global memory sees 64 bytes of a row
        // at once; the own part is fetched a chunk ahead, the first while the last products run
        const int c0 = it.dual ? 0 : team * (DH / 2), c1 = it.dual ? DH : c0 + DH / 2;
        const int v = lane & 3, rsub = lane >> 2;                 // this lane's vector of four columns, its row of eight
        const int orow = valid ? (it.q0 + tok) * a.n_q_heads + it.h * gs + row_head : 0;
        int row[4];
        bool row_ok[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 8 * i + rsub;
            row[i] = __shfl_sync(0xffffffffu, orow, r);
            row_ok[i] = __shfl_sync(0xffffffffu, (int)valid, r);
        }
        float4 own[4];
        auto fetch = [&](float4 (&o)[4], int cc) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (whole && row_ok[i] && cc < c1) o[i] = *reinterpret_cast<const float4*>(a.own_o + (size_t)row[i] * DH + cc + 4 * v);
            }
        };
        const float ls = whole && valid ? a.own_lse[orow] * kLog2e : 0.0f;
        if (live) fetch(own, c0);
        if (has) {
            failed = !warp_wait(o_full, n_items & 1);
            if (!it.dual && !failed) failed = !warp_wait(smem_u32(c->o_full) + 8 * (team ^ 1), n_items & 1);
            if (!it.dual && !failed) {
                c->xm[team][R] = m_run;
                c->xl[team][R] = l_run;
                warp_arrive(smem_u32(&c->x_ready));
                failed = !warp_wait(smem_u32(&c->x_ready), n_x & 1);
                ++n_x;
                m_o = c->xm[team ^ 1][R];
                l_o = c->xl[team ^ 1][R];
            }
            if (failed) break;
            tc_fence_after();
        }
        const float m_all = fmaxf(m_run, m_o);
        const float w_s = m_run == -INFINITY ? 0.0f : fast_exp2((m_run - m_all) * cs), w_o = m_o == -INFINITY ? 0.0f : fast_exp2((m_o - m_all) * cs);
        const float l_all = l_run * w_s + l_o * w_o;
        // l_all is 0 without keys and NaN where a key's score is NaN or +inf, and so are all the sums below: maxima pass over a
        // NaN, weights and sums keep it
        const float lp = l_all == 0.0f ? -INFINITY : m_all * cs + log2f(l_all);            // in powers of two
        float f_s = l_all == 0.0f ? 0.0f : w_s / l_all, f_o = l_all == 0.0f ? 0.0f : w_o / l_all, f_own = 0.0f;
        if (whole) {
            const float top = fmaxf(lp, ls), wp = lp == -INFINITY ? 0.0f : exp2f(lp - top), wo = ls == -INFINITY ? 0.0f : exp2f(ls - top);
            const float inv = wp + wo == 0.0f ? 0.0f : 1.0f / (wp + wo);
            f_s *= wp * inv;
            f_o *= wp * inv;
            f_own = wo * inv;
            if (a.lse && valid && (it.dual || team == 0)) a.lse[orow] = wp + wo == 0.0f ? -INFINITY : (top + log2f(wp + wo)) * kLn2;
        }
        const size_t prow0 = whole ? 0 : (size_t)slot_of(it, blockIdx.x) * kSlotRows + tile * kTileRows;
        if (!whole && valid && (it.dual || team == 0)) a.part_lse[prow0 + R] = lp * kLn2;
        float f_row[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) f_row[i] = __shfl_sync(0xffffffffu, f_own, 8 * i + rsub);
        auto chunk = [&](const float4 (&o)[4], int cc) {
            if (has) {
                uint32_t os[16], oo[16];
                tc_ld16(t_o + cc, os);
                if (other) tc_ld16(t_oo + cc, oo);
                tc_wait_ld();
                float x[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {                    // the accumulator of a team without blocks may hold anything
                    x[e] = steps > 0 ? __uint_as_float(os[e]) * f_s : 0.0f;
                    if (other) x[e] += __uint_as_float(oo[e]) * f_o;
                }
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<float4*>(stage + lane * 16 + ((q ^ ((lane >> 1) & 3)) << 2)) = make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 8 * i + rsub;
                float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
                if (has) y = *reinterpret_cast<const float4*>(stage + r * 16 + ((v ^ ((r >> 1) & 3)) << 2));
                if (!row_ok[i]) continue;
                if (whole) {
                    *reinterpret_cast<uint2*>(a.out + (size_t)row[i] * DH + cc + 4 * v) =
                        make_uint2(pack_bf16(fmaf(o[i].x, f_row[i], y.x), fmaf(o[i].y, f_row[i], y.y)),
                                   pack_bf16(fmaf(o[i].z, f_row[i], y.z), fmaf(o[i].w, f_row[i], y.w)));
                } else {
                    *reinterpret_cast<float4*>(a.part_o + (prow0 + quarter * 32 + r) * DH + cc + 4 * v) = y;
                }
            }
            __syncwarp();
        };
        if (live) {
#pragma unroll 1
            for (int cc = c0; cc < c1; cc += 16) {
                chunk(own, cc);
                fetch(own, cc + 16);
            }
        }
        if (has) {
            tc_fence_before();
            warp_arrive(smem_u32(&c->o_free));
            first += nblk;
            ++n_items;
        }
    }
    if (failed) {
        atomicExch(a.status, DCUT_DEV_ATTN_WAIT_TIMEOUT);
        c->abort = 1;
    }
}

template <int DH>
__global__ void __launch_bounds__(kThreads, 1)
prefix_attn_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                   const __grid_constant__ CUtensorMap v_map, PrefixArgs a) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    Ctrl* c = reinterpret_cast<Ctrl*>(smem + Smem<DH>::kCtrl);
    const int warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kSlots; ++s) {
            mbar_init(smem_u32(&c->kv_full[s]), 1);
            mbar_init(smem_u32(&c->kv_empty[s]), 2);
        }
        mbar_init(smem_u32(&c->q_full), 1);
        mbar_init(smem_u32(&c->q_free), 2);
        for (int t = 0; t < 2; ++t) {
            for (int b = 0; b < 2; ++b) {
                mbar_init(smem_u32(&c->s_full[t][b]), 1);
                mbar_init(smem_u32(&c->p_full[t][b]), kTeamThreads / 32);
            }
            mbar_init(smem_u32(&c->pv_done[t]), 1);
            mbar_init(smem_u32(&c->o_full[t]), 1);
            mbar_init(smem_u32(&c->drain[t]), 1);

        }
        mbar_init(smem_u32(&c->o_free), 2 * kTeamThreads / 32);
        mbar_init(smem_u32(&c->x_ready), 2 * kTeamThreads / 32);
        c->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&c->tmem_base)), "n"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    dcut_pdl_wait();
    Walk w;
    w.at = a.segs[blockIdx.x];
    w.end = a.segs[blockIdx.x + 1];
    w.G = a.n_groups;
    w.group_size = a.group_size;
    w.n_kv_heads = a.n_kv_heads;
    if (warp == 0) produce<DH>(q_map, k_map, v_map, a, smem, c, w);
    else if (warp == 1 || warp == 2) {
        if (elect_one()) issue<DH>(a, smem, c, w, warp - 1);
    } else if (warp >= 4) softmax<DH>(a, smem, c, w);
    __syncwarp();
    dcut_pdl_launch_dependents();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(c->tmem_base), "n"(kTmemCols) : "memory");
    }
}

// ------------------------------------------------------------------------------------------------ plan

struct PrefixPlanArgs {
    const int* cu_group;
    const int* prefix_lens;
    int n_groups, prefix_table_stride, block_table_stride;
    int group_size, max_rows, T_cap;      // max_rows: tokens of a request
    Group* groups;                        // [n_groups + 1]
    Seg* segs;                            // [n_seg + 1]
    Cut* cuts;                            // [n_seg]
    int n_seg;
};

// The own parts' scan takes 2 B + 1 of the long longs; the partition G + 1 costs, a gap for alignment and, as far as that
// fits (every B up to 8192 has to), G groups of two.
constexpr int kSmemGroups = 4096;
__host__ __device__ inline int plan_longs(int B) { return B <= kSmemGroups ? 3 * (B + 1) : 2 * (B + 1); }
size_t plan_smem(int B) { return sizeof(long long) * plan_longs(B) + sizeof(int) * (2 * (size_t)B + 1); }

// Two CTAs, which check the batch alike: the first makes the own parts' work list, the second the shared part's partition
// (one after the other in one CTA they took 12 us, chains of dependent loads and scans both).  A batch that is not what the
// call's contract says (cu_q, cu_group, prefixes against their table and contexts, own positions against the block table) is
// reported and left alone: its partition is empty, so nothing behind the arrays' ends is read or written.
__global__ void __launch_bounds__(1024) prefix_plan_kernel(PrefixPlanArgs p, dcut_plan::PlanArgs a) {
    extern __shared__ long long prefix_s[];                   // cu_q [B + 1] and own lengths [B] lie behind plan_longs(B) of these
    __shared__ long long ws64[33], ws64b[33];
    __shared__ int ws32[33], ws32b[33];
    const int tid = threadIdx.x, nthr = blockDim.x, B = a.B, G = p.n_groups;
    __shared__ Seg segs_s[kMaxSegs + 1];                      // (dcut_create bounds the SMs)
    int* cu_s = reinterpret_cast<int*>(prefix_s + plan_longs(B));
    const bool own_part = blockIdx.x == 0;
    int* own_s = cu_s + B + 1;
    dcut_pdl_wait();
    dcut_pdl_launch_dependents();
    for (int i = tid; i <= B; i += nthr) cu_s[i] = a.cu_q[i];
    for (int i = tid; i < B; i += nthr) own_s[i] = a.ctx_lens[i];
    __syncthreads();
    bool packed = cu_s[0] == 0 && cu_s[B] <= p.T_cap;
    for (int i = tid; i < B; i += nthr) packed = packed && cu_s[i + 1] > cu_s[i] && cu_s[i + 1] - cu_s[i] <= p.max_rows;
    packed = __syncthreads_and(packed);
    bool sound = p.cu_group[0] == 0 && p.cu_group[G] == B;
    for (int g = tid; g < G; g += nthr) {
        const int len = p.prefix_lens[g];
        sound = sound && p.cu_group[g] <= p.cu_group[g + 1] && len >= 0 && len <= (long long)kPage * p.prefix_table_stride;
    }
    sound = __syncthreads_and(sound);
    if (packed && sound) {
        bool fits = true;
        for (int i = tid; i < B; i += nthr) {
            int lo = 0, hi = G;                               // largest g with cu_group[g] <= i (empty groups share a border: the last)
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (p.cu_group[mid] <= i) lo = mid; else hi = mid;
            }
            const long long own = (long long)own_s[i] - p.prefix_lens[lo];
            fits = fits && own >= 0 && own + (cu_s[i + 1] - cu_s[i]) <= (long long)kPage * p.block_table_stride;
            own_s[i] = (int)own;
        }
        sound = __syncthreads_and(fits);
    }
    if (!packed || !sound) {
        if (!own_part) {
            for (int s = tid; s <= p.n_seg; s += nthr) {
                p.segs[s] = Seg{G, 0, 0, 0};
                if (s < p.n_seg) p.cuts[s] = Cut{0, 0, 0, 0};
            }
            return;
        }
        if (tid == 0) atomicExch(a.status, packed ? DCUT_DEV_BAD_GROUPS : DCUT_DEV_BAD_CU_Q);
        a.B = 0;
    }
    if (own_part) {
        // dcut_verify_attn's work list on the own lengths
        a.cu_q = cu_s;
        a.ctx_lens = own_s;
        dcut_plan::attn_plan_body(a, prefix_s);
        return;
    }
    long long* cost = prefix_s;                               // [G + 1]
    Group* groups = B <= kSmemGroups ? reinterpret_cast<Group*>(prefix_s + ((B + 2) & ~1)) : p.groups;   // [G], 16-byte aligned
    // the groups and the cost of the stream before each
    const int per = (G + nthr - 1) / nthr, g0 = tid * per;
    long long mine = 0;
    for (int g = g0; g < g0 + per && g < G; ++g) {
        const int q0 = cu_s[p.cu_group[g]];
        const Group gr = {q0, cu_s[p.cu_group[g + 1]] - q0, p.prefix_lens[g], 0};
        groups[g] = gr;
        p.groups[g] = gr;
        mine += a.n_kv_heads * head_cost(gr, p.group_size);
    }
    dcut_plan::PlanScan4 o, t;
    dcut_plan::plan_block_exclusive_scan4(dcut_plan::PlanScan4{0, 0, mine, 0}, ws32, ws32b, ws64, ws64b, o, t);
    long long before = o.c0;
    for (int g = g0; g < g0 + per && g < G; ++g) {
        cost[g] = before;
        before += a.n_kv_heads * head_cost(groups[g], p.group_size);
    }
    if (tid == 0) cost[G] = t.c0;
    __syncthreads();
    for (int s = tid; s <= p.n_seg; s += nthr) p.segs[s] = segs_s[s] = boundary(s, p.n_seg, groups, cost, G, p.group_size, a.n_kv_heads);
    __syncthreads();
    for (int b = tid; b < p.n_seg; b += nthr) p.cuts[b] = cut_at(b, p.n_seg, segs_s, groups, G, p.group_size);
}

// ------------------------------------------------------------------------------------------------ merge of cut items

// grid: x: boundary b = blockIdx.x + 1; y: 16 of the unit's 256 rows; 16 threads per row.  One prefix in a small batch is a
// single item per kv head, cut into a segment for every SM: the pieces of 8 heads are then all there is to merge, and with
// one or two CTAs per boundary 8 or 16 SMs read everything (15 us for 16 single tokens of 32q/8kv heads).
constexpr int kCombineThreads = 256, kCombineY = kSlotRows / (kCombineThreads / 16);
template <int DH>
__global__ void __launch_bounds__(kCombineThreads) prefix_combine_kernel(PrefixArgs a, const Cut* cuts) {
    dcut_pdl_wait();
    dcut_pdl_launch_dependents();
    constexpr int kVec = DH / 64;                                        // float4 per thread
    const int b = blockIdx.x + 1, c0 = (threadIdx.x & 15) * (DH / 16);
    const Cut cut = cuts[b];
    if (cut.pieces == 0) return;
    const int gs = a.group_size, tpt = tile_tokens(gs);
    const int R = blockIdx.y * (kCombineThreads / 16) + (threadIdx.x >> 4);
    const int r = R & (kTileRows - 1), tok = (R / kTileRows) * tpt + r / gs;
    if (r / gs >= tpt || tok >= cut.tokens) return;
    const size_t orow = (size_t)(cut.q0 + tok) * a.n_q_heads + cut.kv_head * gs + r % gs;
    auto prow = [&](int i) { return (size_t)(i == 0 ? 2 * (b - 1) + 1 : 2 * (b + i - 1)) * kSlotRows + R; };
    const float own = a.own_lse[orow];
    float4 acc[kVec];
#pragma unroll
    for (int v = 0; v < kVec; ++v) acc[v] = *reinterpret_cast<const float4*>(a.own_o + orow * DH + c0 + 4 * v);
    float top = own;
#pragma unroll 4
    for (int i = 0; i < cut.pieces; ++i) top = fmaxf(top, a.part_lse[prow(i)]);
    float sum = own == -INFINITY ? 0.0f : exp2f((own - top) * kLog2e);       // (a NaN is no maximum, but its weight is NaN)
#pragma unroll
    for (int v = 0; v < kVec; ++v) acc[v].x *= sum, acc[v].y *= sum, acc[v].z *= sum, acc[v].w *= sum;
#pragma unroll 4
    for (int i = 0; i < cut.pieces; ++i) {
        const size_t pr = prow(i);
        const float l = a.part_lse[pr], wgt = l == -INFINITY ? 0.0f : exp2f((l - top) * kLog2e);
        sum += wgt;
#pragma unroll
        for (int v = 0; v < kVec; ++v) {
            const float4 x = *reinterpret_cast<const float4*>(a.part_o + pr * DH + c0 + 4 * v);
            acc[v].x += wgt * x.x, acc[v].y += wgt * x.y, acc[v].z += wgt * x.z, acc[v].w += wgt * x.w;
        }
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int v = 0; v < kVec; ++v)
        *reinterpret_cast<uint2*>(a.out + orow * DH + c0 + 4 * v) = make_uint2(pack_bf16(acc[v].x * inv, acc[v].y * inv), pack_bf16(acc[v].z * inv, acc[v].w * inv));
    if (a.lse && c0 == 0) a.lse[orow] = sum == 0.0f ? -INFINITY : top + logf(sum);
}

// ------------------------------------------------------------------------------------------------ host

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Packed queries as {64 columns, heads, tokens, column halves}: one {64, group, tokens of a tile, 1} box is half of a tile's
// columns and arrives as its rows of 128 bytes, in row order (token, head)
dcut_status make_q_map(dcut_ctx* ctx, CUtensorMap* map, const void* q, int T_cap) {
    const int Hq = ctx->lim.n_q_heads, DH = ctx->lim.head_dim, gs = Hq / ctx->lim.n_kv_heads;
    cuuint64_t dims[4] = {64, (cuuint64_t)Hq, (cuuint64_t)T_cap, (cuuint64_t)(DH / 64)};
    cuuint64_t strides[3] = {(cuuint64_t)DH * 2, (cuuint64_t)Hq * DH * 2, 128};
    cuuint32_t box[4] = {64, (cuuint32_t)gs, (cuuint32_t)tile_tokens(gs), 1}, estr[4] = {1, 1, 1, 1};
    CUresult r = reinterpret_cast<EncodeTiledFn>(ctx->encode_tiled)(
        map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(q), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
        CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return dcut_fail(ctx, DCUT_ECUDA, "cuTensorMapEncodeTiled failed for the queries (%d)", (int)r);
    return DCUT_OK;
}

template <int DH>
dcut_status launch_prefix(dcut_ctx* ctx, const CUtensorMap& qm, const CUtensorMap& km, const CUtensorMap& vm, const PrefixArgs& a,
                          const Cut* cuts, cudaStream_t stream) {
    dcut_status st = dcut_check_cuda(ctx, dcut_launch_pdl(prefix_attn_kernel<DH>, dim3(ctx->sm_count), dim3(kThreads), Smem<DH>::kTotal, stream,
                                                          qm, km, vm, a), "launch prefix_attn_kernel");
    if (st != DCUT_OK || ctx->sm_count < 2) return st;
    return dcut_check_cuda(ctx, dcut_launch_pdl(prefix_combine_kernel<DH>, dim3(ctx->sm_count - 1, kCombineY), dim3(kCombineThreads), 0, stream, a, cuts),
                           "launch prefix_combine_kernel");
}


// the context's scratch for these calls, one allocation
struct Scratch {
    float *own_o, *own_lse, *part_o, *part_lse;
    Group* groups;
    Seg* segs;
    Cut* cuts;
    AttnEntry* entries;           // the own parts' work list
    AttnSeg* own_segs;
    AttnCut* own_cuts;
    int* plan;
};
size_t carve(const dcut_ctx* c, unsigned char* base, Scratch* s) {
    size_t off = 0;
    auto take = [&](size_t bytes) {
        unsigned char* p = base + off;
        off += (bytes + 255) & ~size_t(255);
        return p;
    };
    const size_t max_T = (size_t)c->lim.max_B * (c->lim.max_gamma + 1), rows = max_T * c->lim.n_q_heads, slots = 2 * (size_t)c->sm_count * kSlotRows;
    s->own_o = reinterpret_cast<float*>(take(rows * c->lim.head_dim * sizeof(float)));
    s->own_lse = reinterpret_cast<float*>(take(rows * sizeof(float)));
    s->part_o = reinterpret_cast<float*>(take(slots * c->lim.head_dim * sizeof(float)));
    s->part_lse = reinterpret_cast<float*>(take(slots * sizeof(float)));
    s->groups = reinterpret_cast<Group*>(take(sizeof(Group) * ((size_t)c->lim.max_B + 1)));
    s->segs = reinterpret_cast<Seg*>(take(sizeof(Seg) * ((size_t)c->sm_count + 1)));
    s->cuts = reinterpret_cast<Cut*>(take(sizeof(Cut) * ((size_t)c->sm_count + 1)));
    s->entries = reinterpret_cast<AttnEntry*>(take(sizeof(AttnEntry) * (size_t)c->max_entries));
    s->own_segs = reinterpret_cast<AttnSeg*>(take(sizeof(AttnSeg) * ((size_t)c->sm_count + 1)));
    s->own_cuts = reinterpret_cast<AttnCut*>(take(sizeof(AttnCut) * ((size_t)c->sm_count + 1)));
    s->plan = reinterpret_cast<int*>(take(sizeof(int) * 16));
    return off;
}

}  // namespace

dcut_status dcut_enable_prefix(dcut_ctx* ctx, int max_groups) {
    if (max_groups > ctx->prefix_max_groups) ctx->prefix_max_groups = max_groups;
    if (ctx->prefix_scratch) return DCUT_OK;   // (it has room for max_B groups: captured graphs keep their pointers)
    ctx->prefix_max_groups = 0;
    cudaError_t e = cudaFuncSetAttribute(prefix_attn_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<128>::kTotal);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(prefix_attn_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<64>::kTotal);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(prefix_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)plan_smem(DCUT_MAX_KEYS));
    if (e != cudaSuccess) return dcut_check_cuda(ctx, e, "cudaFuncSetAttribute(prefix attention)");
    Scratch s;
    const size_t bytes = carve(ctx, nullptr, &s);
    dcut_status st = dcut_check_cuda(ctx, cudaMalloc(reinterpret_cast<void**>(&ctx->prefix_scratch), bytes), "cudaMalloc(prefix attention scratch)");
    if (st == DCUT_OK) ctx->prefix_max_groups = max_groups;
    return st;
}

dcut_status dcut_launch_prefix_attn(dcut_ctx* ctx, const void* q, const void* k_cache, const void* v_cache, long long num_pages,
                                    const int* block_table, int block_table_stride, const int* ctx_lens, const int* cu_q, int B,
                                    int T_cap, const dcut_prefix_groups* groups, float scale, void* out, float* lse, cudaStream_t stream) {
    const dcut_limits& l = ctx->lim;
    Scratch s;
    carve(ctx, ctx->prefix_scratch, &s);
    CUtensorMap qm, km, vm;
    dcut_status st = make_q_map(ctx, &qm, q, T_cap);
    if (st != DCUT_OK) return st;
    if ((st = dcut_make_cache_map(ctx, &vm, v_cache, num_pages)) != DCUT_OK) return st;
    if ((st = l.head_dim == 128 ? dcut_make_k_group_map(ctx, &km, k_cache, num_pages) : dcut_make_cache_map(ctx, &km, k_cache, num_pages)) != DCUT_OK) return st;

    PrefixPlanArgs pp;
    pp.cu_group = groups->cu_group;
    pp.prefix_lens = groups->prefix_lens;
    pp.n_groups = groups->n_groups;
    pp.prefix_table_stride = groups->prefix_table_stride;
    pp.block_table_stride = block_table_stride;
    pp.group_size = l.n_q_heads / l.n_kv_heads;
    pp.max_rows = l.max_gamma + 1;
    pp.T_cap = T_cap;
    pp.groups = s.groups;
    pp.segs = s.segs;
    pp.cuts = s.cuts;
    pp.n_seg = ctx->sm_count;
    dcut_plan::PlanArgs pa;
    dcut_fill_plan_args(ctx, ctx_lens, cu_q, B, &pa);
    // (a list of its own: the context's may be one that a selector has left for dcut_verify_attn, and a replayed graph could
    // not tell the host that it is gone)
    pa.entries = s.entries;
    pa.segs = s.own_segs;
    pa.cuts = s.own_cuts;
    pa.plan = s.plan;
    if ((st = dcut_check_cuda(ctx, dcut_launch_pdl(prefix_plan_kernel, dim3(2), dim3(B <= 256 ? 256 : 1024), plan_smem(B), stream, pp, pa),
                              "launch prefix_plan_kernel")) != DCUT_OK) return st;
    if ((st = dcut_launch_verify_attn(ctx, q, k_cache, v_cache, num_pages, block_table, block_table_stride, ctx_lens, cu_q, B, T_cap, scale,
                                      out, s.own_lse, 0, &pa, s.own_o, stream)) != DCUT_OK) return st;

    PrefixArgs a;
    a.prefix_table = groups->prefix_table;
    a.prefix_table_stride = groups->prefix_table_stride;
    a.groups = s.groups;
    a.segs = s.segs;
    a.n_groups = groups->n_groups;
    a.n_q_heads = l.n_q_heads;
    a.n_kv_heads = l.n_kv_heads;
    a.group_size = pp.group_size;
    a.num_pages = num_pages;
    a.scale_log2 = scale * kLog2e;
    a.own_o = s.own_o;
    a.own_lse = s.own_lse;
    a.out = static_cast<__nv_bfloat16*>(out);
    a.lse = lse;
    a.part_o = s.part_o;
    a.part_lse = s.part_lse;
    a.status = ctx->d_status;
    if (l.head_dim == 128) return launch_prefix<128>(ctx, qm, km, vm, a, s.cuts, stream);
    return launch_prefix<64>(ctx, qm, km, vm, a, s.cuts, stream);
}
