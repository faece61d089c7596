// dcut_lora: the low-rank adapters of many requests beside a shared projection.
//
//   d[r, n] = scale[i] sum_j s[r, j] B_i[n, j],   s = x[r, :] . A_i^T,   i the adapter of the row's request
//   out = act(base + d), or act(base_gate + d_gate) * (base_up + d_up)
//
// Two products with a rank between them; each byte of x, base and out moves once, A and B of an adapter once per tile of rows (from
// L2 but for the first).  A few multiplications per byte: the memory, and for few rows its latency, bounds it.  A tile is up to 16, 32 or 64 rows
// that share an adapter (of several requests, where those share it).
//   lora_low_kernel   s of a tile, by 1 to 8 CTAs (a cluster) that cut K between them: A by TMA, the rows of x, which lie anywhere, by asynchronous copies,
//                     the product on tcgen05 with its accumulator in tensor memory.  The partial sums meet through distributed shared memory,
//                     added in a fixed order.  s is scaled in fp32 and kept as the sum of two bf16 values (off by 2^-17 of it at most; a single one
//                     cost the result up to 1.7 times its error where d outweighs base).
//   lora_out_kernel   a few columns of a tile per warp, 16 rows at a time, on warp-level MMAs: the base, the sum and the result stay in one lane.
// Measured on the device (floors in brackets: bytes at the copy rate): 16 single tokens with an adapter each, rank 16, 4096 -> 6144 in three slices 10 us
// (1.4); 603 tokens of 64 requests with 24 adapters, 4096 -> 4096 14 us (3); gate and up projection of 1088 tokens, 8 adapters of rank 64,
// 4096 -> 2 x 12288 with SiLU 58 us (18); 8191 tokens of three prompts, rank 32, 4096 -> 6144 75 us (42).  The small ones are two launches and their
// chains of loads (find the tile 1.5 us, x and A 2.3, the sums' way between CTAs 2); at length the first product takes a third (L2 to shared memory),
// the second is bound by instructions and their latency (0.41 to 0.44 issued per active cycle and scheduler, two to three CTAs per SM by their registers).
// One kernel for both, whose clusters kept s to themselves and took an eighth of the columns per CTA each, took 200 and 175 us where these take 58
// and 75: 8 to 16 warps per SM, and every step waited for its loads.
#include <cuda_bf16.h>
#include <math.h>

#include <type_traits>

#include "activation.cuh"
#include "dcut_internal.h"
#include "tcgen05.cuh"

namespace {

constexpr int kMostSplit = 8, kWarps = 8, kThreads = 32 * kWarps;
constexpr int kMaxSlices = DCUT_LORA_MAX_SLICES;

struct LoraArgs {
    const __nv_bfloat16 *x, *a, *b, *base;
    long long ldx, lda, ldbase, ldo;
    const float* scale;                  // [n_adapters] or null
    const int* adapter;                  // [B]
    const int* cu_q;
    __nv_bfloat16* out;
    int n_adapters, rank, n_slices, K, N, B, T_cap, act, gated;
    int in_place;                        // rows without an adapter keep what they have
    int vec;                             // base and out take 16-byte accesses at columns that are multiples of 8
    int end[kMaxSlices];                 // last column + 1 of each slice
    int part_row;                        // floats from a row of s to the next in the partial sums
    int tile_rows;                       // rows of a tile: 16, 32 or 64
    int tile0, groups, blocks;           // first tile of this pass; groups of columns, and CTAs of the second product, per tile
    unsigned char* scratch;              // per tile: a Tile, then its s
    long long tile_bytes;
    int b_at;                            // where B follows the second product's s in shared memory
    int* status;
};

__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint4& a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}
// Asynchronous copies to shared memory; `bytes` of the 16 are read, the rest is filled with zeros.
__device__ __forceinline__ void copy16(uint32_t to, const void* from, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.commit_group;" ::: "memory"); }       // ends a group of copies
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }   // all but the last N groups
// what bf16 rounding took from two values (nothing from an infinity): `high` is their packed rounding
__device__ __forceinline__ uint32_t low_parts(float x, float y, uint32_t high) {
    const float hx = bf_lo(high), hy = bf_hi(high);
    return pack_bf16(fabsf(hx) < INFINITY ? x - hx : 0.0f, fabsf(hy) < INFINITY ? y - hy : 0.0f);
}
// 16 bytes where `there`, else zeros.  A predicate and no branch: the loads of a step leave together.
__device__ __forceinline__ uint4 load_if(const __nv_bfloat16* p, bool there) {
    uint4 v;
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
                 "@p ld.global.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}" : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w) : "l"(p), "r"((int)there));
    return v;
}
// the first `n` of 8 elements, one by one
__device__ __forceinline__ uint4 load_some(const __nv_bfloat16* p, int n) {
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) w[j >> 1] |= (uint32_t)reinterpret_cast<const unsigned short*>(p)[j] << (16 * (j & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// What a cluster works on: up to R rows of one adapter (of several requests, where they share it).
struct Tile {
    int rows, adapter;                   // rows = 0: there is no such tile
    int row[64];                         // (kMostRows)
    int pad[14];
};
static_assert(sizeof(Tile) % 64 == 0, "s follows in 16-byte pieces");
struct Search {
    int2 request[kThreads];              // adapter and rows
    int warp_sum[kWarps], before, adapter, offset;
};
__device__ __forceinline__ int up_to(int v, int* warp_sum, int& all) {                   // inclusive sum over the CTA
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += u;
    }
    __syncthreads();                     // (the sums of the pass before have been read)
    if (lane == 31) warp_sum[warp] = v;
    __syncthreads();
    all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) v += warp_sum[w];
        all += warp_sum[w];
    }
    return v;
}
// Tile number t of the batch.  Up to kThreads requests: the rows of an adapter, request after request, are cut into tiles, so that the
// requests of a tenant share A and B; the adapters come in the order of their first requests.  More requests: tiles of single requests.
// Rows that keep what they have are left out.
__device__ __forceinline__ void find_tile(const LoraArgs& g, int t, int R, Tile& tile, Search& f) {
    const int tid = threadIdx.x;
    const bool grouped = g.B <= kThreads;
    if (tid == 0) tile.rows = 0, f.adapter = -2;
    int before = 0;                      // tiles of the requests that earlier passes looked at
    for (int i0 = 0; i0 < g.B && (before <= t || t == 0); i0 += kThreads) {              // (tile 0 looks at every request)
        const int i = i0 + tid;
        int lo = 0, n = 0, id = -1;
        if (i < g.B) {
            lo = max(0, g.cu_q[i]), n = max(0, min(g.cu_q[i + 1], g.T_cap) - lo), id = max(g.adapter[i], -1);
            if (id >= g.n_adapters) {
                if (t == 0) atomicExch(g.status, DCUT_DEV_BAD_ADAPTER);
                id = -1;
            }
            if (i == g.B - 1 && t == 0 && g.cu_q[g.B] > g.T_cap) atomicExch(g.status, DCUT_DEV_BAD_ROWS);
            if (id < 0 && g.in_place) n = 0;
        }
        int mine = n, first = 0;         // rows of the unit that this request leads; rows of its adapter ahead of it
        if (grouped) {
            f.request[tid] = make_int2(id, n);
            __syncthreads();
            if (n > 0) {
#pragma unroll 8
                for (int j = 0; j < g.B; ++j) {
                    const int2 r = f.request[j];
                    const int same = r.x == id ? r.y : 0;
                    first += j < i ? same : 0;
                    mine += j > i ? same : 0;
                }
            }
            if (first > 0 || n == 0) mine = 0;                          // (the first request with rows leads)
        }
        const int tiles = (mine + R - 1) / R;
        int all;
        const int at = t - before - (up_to(tiles, f.warp_sum, all) - tiles);
        if (at >= 0 && at < tiles) {
            tile.rows = min(R, mine - at * R), tile.adapter = id;
            f.adapter = id, f.offset = at * R;
            if (!grouped)
                for (int k = 0; k < tile.rows; ++k) tile.row[k] = lo + at * R + k;
        }
        if (grouped) {
            __syncthreads();
            if (f.adapter == id) {       // this request's rows among the tile's
                const int k0 = max(0, f.offset - first), k1 = min(n, f.offset + tile.rows - first);
                for (int k = k0; k < k1; ++k) tile.row[first + k - f.offset] = lo + k;
            }
        }
        before += all;
    }
    __syncthreads();
}

// The columns of out that a warp works on at a time: 32 of one slice, or, gated, 16 of the gate and the same ones of the up projection.
struct Group {
    int col, end, slice;                 // first column; where the slice ends
};
template <bool GATED>
__device__ __forceinline__ Group group_of(const LoraArgs& g, int i) {
    if (GATED) return Group{16 * i, g.N / 2, 0};
    int first = 0, end = g.end[0], slice = 0;
    while (i >= (end - first + 31) / 32) {
        i -= (end - first + 31) / 32;
        first = end;
        end = g.end[++slice];
    }
    return Group{first + 32 * i, end, slice};
}

// How s lies in the scratch: as the fragments of the second product.  A step of that is 32 elements (two MMAs), 8 neighbouring ones in a lane.
// Ranks that are multiples of 32 take a step with the high parts and again with the low ones (parts = 2); others walk the high parts and then the
// low ones as one row, so that rank 16 fills a step.  Per slice, 16 rows, step, part and MMA: 16 bytes per lane, pairs of rows gr and gr + 8 in turn.
struct Low {
    int steps, parts;
    __host__ __device__ Low(int rank) : steps(rank % 32 ? (2 * rank + 31) / 32 : rank / 32), parts(rank % 32 ? 1 : 2) {}
    __host__ __device__ int pieces() const { return steps * parts * 2; }                 // of 512 bytes, per slice and 16 rows
    // the byte where the pair of elements (j, j + 1) (high or low parts) of row r lies; the next pair of the MMA is 8 bytes on
    __device__ __forceinline__ int at(int blocks16, int rank, int slice, int r, int j, int low) const {
        const int v = parts == 1 && low ? rank + j : j, part = parts == 1 ? 0 : low, pair = (v & 7) >> 1;
        return ((((slice * blocks16 + (r >> 4)) * steps + (v >> 5)) * parts + part) * 2 + (pair >> 1)) * 512 + (((r & 7) << 2) + ((v >> 3) & 3)) * 16 +
               ((pair & 1) * 2 + ((r >> 3) & 1)) * 4;
    }
};

constexpr int kChunk = 64;               // elements of K per step of the first product: rows of 128 bytes, 16-byte piece c of row r at c ^ (r & 7)
constexpr int kRowBytes = 2 * kChunk, kPieces = kRowBytes / 16, kCopiers = 128, kStrideRows = kCopiers / kPieces, kMostRows = 64;
constexpr int kEdgeRow = 80;             // bytes of a row of a group's results on their way to rows that take no vectors

// act(v), in place.  The common ones stand here: a call's cost is that of the registers that live across it.
template <int N>
__device__ __forceinline__ void activate(int act, float (&v)[N]) {
    if (act == DCUT_ACT_NONE) return;
    if (act == DCUT_ACT_SILU) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] *= sigmoid(v[j]);
    } else if (act == DCUT_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = v[j] < 0.0f ? 0.0f : v[j];
    } else {
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            const float4 y = activate4(act, make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]));
            v[j] = y.x, v[j + 1] = y.y, v[j + 2] = y.z, v[j + 3] = y.w;
        }
    }
}

// s of a tile of R rows: one accumulator of 128 x (columns of s) in tensor memory, of which R rows are used (tcgen05.mma has M = 128; what its other rows
// read is whatever follows the tile of x in shared memory, and nobody looks at them).  STAGES - 1 steps of K are on their way.
template <int STAGES>
__global__ void __launch_bounds__(kThreads, 2) lora_low_kernel(LoraArgs g, const __grid_constant__ CUtensorMap a_map) {
    extern __shared__ unsigned char smem_raw[];
    __shared__ Tile tile;
    __shared__ Search search;
    __shared__ unsigned long long bars[2 * STAGES + 1];                // a step has arrived; its products have been formed, its place is free; all are formed
    __shared__ uint32_t tmem_slot;
    const int R = g.tile_rows, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(smem_u32(bars + s), 1 + kCopiers);               // A's bytes, and the threads that copy x
            mbar_init(smem_u32(bars + STAGES + s), 1);
        }
        mbar_init(smem_u32(bars + 2 * STAGES), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    dcut_pdl_wait();
    dcut_pdl_launch_dependents();
    const int rank = (int)cluster_ctarank(), split = (int)cluster_size(), SR = g.n_slices * g.rank, number = blockIdx.x / split;
    find_tile(g, g.tile0 + number, R, tile, search);
    const int rows = tile.rows, adapter = tile.adapter;
    unsigned char* record = g.scratch + number * g.tile_bytes;
    if (rank == 0 && threadIdx.x < 2 + rows) reinterpret_cast<int*>(record)[threadIdx.x] = reinterpret_cast<const int*>(&tile)[threadIdx.x];
    if (rows == 0 || adapter < 0) return;                              // (the whole cluster)
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    float* sums = reinterpret_cast<float*>(smem);                      // in the ring's place, later: [R][part_row]

    const int chunks = (g.K + kChunk - 1) / kChunk, c0 = (int)((long long)chunks * rank / split), n_chunks = (int)((long long)chunks * (rank + 1) / split) - c0;
    const int stage = (R + SR) * kRowBytes;                            // (a multiple of 1024, as the swizzle wants: R of 16, SR of 8)
    const uint32_t ring_at = smem_u32(smem), full = smem_u32(bars), empty = smem_u32(bars + STAGES), done = smem_u32(bars + 2 * STAGES);
    const int n = (SR + 15) & ~15;                                     // the MMA's N; 8 columns beyond SR read what follows A
    const uint32_t columns = n <= 32 ? 32u : n <= 64 ? 64u : n <= 128 ? 128u : 256u;
    bool failed = false;
    if (warp == 1) {
        // ---- A, by TMA (zeros behind K)
        for (int c = 0, slot = 0; c < n_chunks; ++c) {
            if (c >= STAGES && !__all_sync(0xffffffffu, mbar_wait(empty + 8 * slot, (c / STAGES - 1) & 1))) {
                failed = true;
                break;
            }
            if (elect_one()) {
                mbar_arrive_expect_tx(full + 8 * slot, SR * kRowBytes);
                tma_load_2d(ring_at + slot * stage + R * kRowBytes, &a_map, (c0 + c) * kChunk, adapter * SR, full + 8 * slot);
            }
            __syncwarp();
            slot = slot + 1 == STAGES ? 0 : slot + 1;
        }
    } else if (warp >= kWarps - kCopiers / 32) {
        // ---- x, whose rows lie anywhere: a thread copies the same 16-byte piece of every 16th row
        const int t = threadIdx.x - (kThreads - kCopiers), piece = t % kPieces, r0 = t / kPieces;
        const uint32_t to0 = ring_at + r0 * kRowBytes + ((piece ^ (r0 & 7)) << 4);
        const __nv_bfloat16* from[kMostRows / kStrideRows];
#pragma unroll
        for (int i = 0; i < kMostRows / kStrideRows; ++i)
            from[i] = g.x + (size_t)tile.row[min(r0 + kStrideRows * i, rows - 1)] * g.ldx + (size_t)c0 * kChunk + 8 * piece;
        int left = g.K - c0 * kChunk - 8 * piece;                      // elements from this thread's piece to the end of its rows (their bytes may not fit 31 bits)
        for (int c = 0, slot = 0; c < n_chunks; ++c) {
            if (c >= STAGES && !mbar_wait(empty + 8 * slot, (c / STAGES - 1) & 1)) {
                failed = true;
                break;
            }
            const int bytes = 2 * min(8, max(0, left));                // (0: nothing is read, and the address is one that exists)
#pragma unroll
            for (int i = 0; i < kMostRows / kStrideRows; ++i) {
                if (r0 + kStrideRows * i < rows) copy16(to0 + slot * stage + i * kStrideRows * kRowBytes, bytes ? from[i] : g.x, bytes);
                from[i] += kChunk;
            }
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(full + 8 * slot) : "memory");
            left -= kChunk;
            slot = slot + 1 == STAGES ? 0 : slot + 1;
        }
    } else if (warp == 0) {
        // ---- the products (every earlier kernel has ended: whoever held tensor memory on this SM has given it back, or belongs to another stream
        // and will)
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&tmem_slot), idesc = idesc_no_n<false>(128) | ((uint32_t)(n >> 3) << 17);
        for (int c = 0, slot = 0; c < n_chunks; ++c) {
            if (!__all_sync(0xffffffffu, mbar_wait(full + 8 * slot, (c / STAGES) & 1))) {
                failed = true;
                break;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the copies of x, for the tensor core
            tc_fence_after();
            if (elect_one()) {
                const uint32_t at = ring_at + slot * stage;
                const uint64_t dx = umma_desc_sw128(at), da = umma_desc_sw128(at + R * kRowBytes);
#pragma unroll
                for (int k = 0; k < kChunk / 16; ++k) tc_mma<false>(tmem, dx + 2 * k, da + 2 * k, idesc, (c | k) ? 1u : 0u);
                tc_commit(empty + 8 * slot);
                if (c == n_chunks - 1) tc_commit(done);
            }
            __syncwarp();
            slot = slot + 1 == STAGES ? 0 : slot + 1;
        }
    }
    if (n_chunks > 0 && !failed && !mbar_wait(done, 0)) failed = true;
    copies_done();
    copies_wait<0>();
    if (failed) {
        atomicExch(g.status, DCUT_DEV_LORA_WAIT_TIMEOUT);
        if (warp == 1)                                                 // nothing is on its way to this CTA's memory when it leaves
            for (int s = 0; s < STAGES; ++s) (void)mbar_wait(full + 8 * s, 0), (void)mbar_wait(full + 8 * s, 1);
    }
    tc_fence_before();
    __syncthreads();                                                   // every product is formed, the ring is free
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    {
        const int quarter = warp & 3, r = 32 * quarter + lane;         // (a warp reads the 32 lanes of tensor memory that its number gives)
        if (32 * quarter < R) {
            for (int col = 8 * (warp >> 2); col < SR; col += 16) {
                uint32_t v[8];
                asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                             : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                             : "r"(tmem + ((uint32_t)(32 * quarter) << 16) + col));
                tc_wait_ld();
                if (r < R) {
                    uint4* p = reinterpret_cast<uint4*>(sums + r * g.part_row + col);
                    p[0] = n_chunks > 0 ? make_uint4(v[0], v[1], v[2], v[3]) : make_uint4(0, 0, 0, 0);      // (no share of K: nothing was written)
                    p[1] = n_chunks > 0 ? make_uint4(v[4], v[5], v[6], v[7]) : make_uint4(0, 0, 0, 0);
                }
            }
        }
    }
    tc_fence_before();
    cluster_sync_all();                                                // every CTA's share is complete
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
    }
    const float scale = g.scale ? g.scale[adapter] : 1.0f;
    const uint32_t sums_at = smem_u32(sums);
    const Low low(g.rank);
    unsigned char* s_out = record + sizeof(Tile);
    const int blocks16 = R / 16, quads = SR / 4, each = R * quads / split;               // (R is a multiple of 16, SR of 8, the split of 8 a divisor)
    for (int e = rank * each + threadIdx.x; e < (rank + 1) * each; e += kThreads) {
        const int r = e / quads, c = 4 * (e - r * quads), slice = c / g.rank, j = c - slice * g.rank;
        float4 s = make_float4(0, 0, 0, 0), v[kMostSplit];
#pragma unroll
        for (int p = 0; p < kMostSplit; ++p)
            if (p < split)
                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[p].x), "=f"(v[p].y), "=f"(v[p].z), "=f"(v[p].w)
                             : "r"(mapa_rank(sums_at + 4 * (r * g.part_row + c), p)) : "memory");
#pragma unroll
        for (int p = 0; p < kMostSplit; ++p)
            if (p < split) s.x += v[p].x, s.y += v[p].y, s.z += v[p].z, s.w += v[p].w;
        s.x *= scale, s.y *= scale, s.z *= scale, s.w *= scale;
        const uint32_t hi0 = pack_bf16(s.x, s.y), hi1 = pack_bf16(s.z, s.w);
        uint32_t* high = reinterpret_cast<uint32_t*>(s_out + low.at(blocks16, g.rank, slice, r, j, 0));
        uint32_t* rest = reinterpret_cast<uint32_t*>(s_out + low.at(blocks16, g.rank, slice, r, j, 1));
        high[0] = hi0, high[2] = hi1;
        rest[0] = low_parts(s.x, s.y, hi0), rest[2] = low_parts(s.z, s.w, hi1);
    }
    if (low.parts == 1 && rank == split - 1) {                         // what fills up the last step
        const int rest = (32 * low.steps - 2 * g.rank) / 4;
        for (int e = threadIdx.x; e < g.n_slices * R * rest; e += kThreads) {
            const int sr = e / rest, v = 2 * g.rank + 4 * (e - sr * rest);
            uint32_t* p = reinterpret_cast<uint32_t*>(s_out + low.at(blocks16, g.rank, sr / R, sr % R, v, 0));
            p[0] = p[2] = 0;
        }
    }
    cluster_sync_all();                                                // nobody leaves while its sums are read
}

// out of a tile: a warp has a group of columns, 16 rows at a time.  Column n of the MMA's tile t is column 8 (n >> 1) + 2 t + (n & 1) of the
// 32, so that a lane ends with the 8 neighbouring columns 8 q .. + 7 (gated: t = 0, 1 the gate's and t = 2, 3 the up projection's columns 4 (n >> 1) +
// 2 (t & 1) + (n & 1), 4 q .. + 3 of each); a lane's 8 neighbouring elements of s and of B serve as its fragments of two MMAs (the order of a
// sum's terms is free).  KEEP: the rank's steps, where B's fragments stay in registers for all rows; 0: they are read again for every 16.
// `early`: the CTA finds its tile itself and asks for B and its first rows of base while the first product runs (what that one waited for is
// complete once this grid has started); otherwise it reads the tile from the scratch.
// FEW: tiles of 16 rows, one block of them: a body without what the others need.  CTAs per SM (registers): of long tiles 2 with two steps in
// registers, else 3 (4 took 87 us where 3 take 75 for 8191 tokens).  Tiles of 16 rows have more to wait for and less to do: 4 against 3, 16 tokens with
// an adapter each, gated, 4096 -> 2 x 12288, rank 16 18.7 us against 20.2, 64 tokens of rank 96 93 against 104; two steps in registers 3 against 2, 64
// tokens of rank 64, 4096 -> 12288 37 against 42 (4: 46; gated 64 tokens 78 either way, 4: 84); B read again, no gate: 3, for at 4 it spills too much
// (16 tokens of rank 128, 4096 -> 6144 21 against 18).  These limits cost spills in every form but the one with two steps of long tiles: of long tiles with one
// step 44 bytes (gated 56), with B read again 152 (68), of tiles of 16 rows 8 to 16 (gated 24 to 88).
constexpr int out_ctas(bool gated, int keep, bool few) { return few ? (keep == 2 || (keep == 0 && !gated) ? 3 : 4) : keep == 2 ? 2 : 3; }
// STAGED: the kept B comes by way of shared memory (a lane's own pieces: nobody else looks at them).  For two steps of long tiles, of ranks that are
// multiples of 32: gated 1088 tokens of rank 64 63.1 us -> 57.9, 2800 tokens 4096 -> 2 x 4096 57.4 -> 53.7 (600 tokens 54.2 -> 54.7), both kernels
// together; the second one alone takes the same 50 us either way.  Other ranks ask for the same pieces twice: rank 24 52 us, staged 59 (55 with copies
// through L1, which cost rank 64 its gain and more).
template <bool GATED, int KEEP, bool FEW, bool STAGED>
__global__ void __launch_bounds__(kThreads, out_ctas(GATED, KEEP, FEW)) lora_out_kernel(LoraArgs g, int early) {
    constexpr int kCols = GATED ? 16 : 32, kPer = kCols / 4;           // columns of a group, of a lane
    const int blocks16 = g.tile_rows / 16;
    __shared__ __align__(16) unsigned char edges[kWarps][16 * kEdgeRow];
    __shared__ Tile tile;
    __shared__ Search search;
    __shared__ unsigned long long arrived;
    extern __shared__ __align__(128) unsigned char s_here[];           // s of the slices that this CTA's columns belong to, where the tile has several blocks of rows
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gr = lane >> 2, q = lane & 3;
    const int number = blockIdx.x / g.blocks;
    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&arrived), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    const unsigned char* record = g.scratch + number * g.tile_bytes;
    if (early) find_tile(g, g.tile0 + number, g.tile_rows, tile, search);
    else {
        dcut_pdl_wait();
        if (threadIdx.x < 2 + kMostRows) reinterpret_cast<int*>(&tile)[threadIdx.x] = reinterpret_cast<const int*>(record)[threadIdx.x];
        __syncthreads();
    }
    const int rows = tile.rows, adapter = tile.adapter, width = GATED ? g.N / 2 : g.N;       // columns of out
    const int i = (blockIdx.x - number * g.blocks) * kWarps + warp;
    const bool work = rows > 0 && i < g.groups, live = work && adapter >= 0;
    const Group at = group_of<GATED>(g, work ? i : 0);
    const Low low(g.rank);
    // base and out in 8- or 16-byte pieces (the same answer in the whole warp)
    const bool vec = g.vec && at.col + kCols <= at.end && !((at.col | (GATED ? width : 0)) & (kPer - 1));
    const int left = at.end - at.col;
    const __nv_bfloat16* b = g.b + ((size_t)max(adapter, 0) * g.N + at.col) * g.rank;
    // the place of a lane's piece t of a step in B, and whether there is one (behind both parts s is zero, and so is this)
    auto b_place = [&](int step, int t, bool& there) {
        const int v = 32 * step + 8 * q, k = v < g.rank ? v : v - g.rank, n = kPer * (gr >> 1) + 2 * (GATED ? t & 1 : t) + (gr & 1);
        there = n < left && v < 2 * g.rank;
        return b + (size_t)(GATED && t >= 2 ? width + n : n) * g.rank + k;
    };
    auto load_b = [&](int step, uint4 (&bv)[4]) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            bool there;
            const __nv_bfloat16* p = b_place(step, t, there);
            bv[t] = load_if(p, there);
        }
    };
    // base at this lane's columns of rows gr and gr + 8 of block m (those that do not exist: of the last one that does); `row`: twice their numbers,
    // so that an address is one 32 x 32 + 64 bit operation
    const unsigned char* base_at = reinterpret_cast<const unsigned char*>(g.base + at.col + kPer * q);
    unsigned char* out_at = reinterpret_cast<unsigned char*>(g.out + at.col + kPer * q);
    auto fetch = [&](auto vector, int m, int (&row)[2], uint4 (&v)[2]) {
        constexpr bool VEC = decltype(vector)::value;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            row[h] = 2 * tile.row[min(16 * m + 8 * h + gr, rows - 1)];
            const __nv_bfloat16* p = reinterpret_cast<const __nv_bfloat16*>(base_at + (unsigned long long)(unsigned)row[h] * (unsigned)g.ldbase);
            if (!GATED) {
                v[h] = VEC ? *reinterpret_cast<const uint4*>(p) : load_some(p, left - 8 * q);
            } else if (VEC) {
                const uint2 x = *reinterpret_cast<const uint2*>(p), y = *reinterpret_cast<const uint2*>(p + width);
                v[h] = make_uint4(x.x, x.y, y.x, y.y);
            } else {
                const uint4 x = load_some(p, min(4, left - 4 * q)), y = load_some(p + width, min(4, left - 4 * q));
                v[h] = make_uint4(x.x, x.y, y.x, y.y);
            }
        }
    };
    uint4 kept[KEEP ? KEEP : 1][4], base[2];
    int row[2];
    if (work && vec) fetch(std::true_type{}, 0, row, base);
    if (work && !vec) fetch(std::false_type{}, 0, row, base);
    const uint32_t b_here = smem_u32(s_here) + g.b_at + (warp * KEEP * 4 * 32 + lane) * 16;
    if (STAGED && live) {
#pragma unroll
        for (int e = 0; e < KEEP * 4; ++e) {
            bool there;
            const __nv_bfloat16* p = b_place(e / 4, e % 4, there);
            copy16(b_here + e * 512, there ? p : g.b, there ? 16 : 0);
        }
        copies_done();
    } else if (KEEP && live) {
#pragma unroll
        for (int step = 0; step < KEEP; ++step) load_b(step, kept[step]);
    }
    for (int r = 16 + lane; !FEW && work && r < rows; r += 32) {               // the other rows of base come to L2 meanwhile
        const __nv_bfloat16* p = g.base + (unsigned long long)(unsigned)tile.row[r] * (unsigned)g.ldbase + at.col;
        asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
        if (GATED) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + width));
    }
    if (early) dcut_pdl_wait();
    dcut_pdl_launch_dependents();
    // s comes to shared memory in one piece; a single block of rows reads it where it is
    const int slice_bytes = blocks16 * low.pieces() * 512, i0 = (blockIdx.x - number * g.blocks) * kWarps;
    const int first_slice = GATED ? 0 : group_of<GATED>(g, i0).slice, last_slice = GATED ? g.n_slices - 1 : group_of<GATED>(g, min(i0 + kWarps, g.groups) - 1).slice;
    const unsigned char* s_in = record + sizeof(Tile);
    if (!FEW && rows > 16 && adapter >= 0) {
        if (threadIdx.x == 0) {
            const uint32_t bytes = (last_slice - first_slice + 1) * slice_bytes;
            mbar_arrive_expect_tx(smem_u32(&arrived), bytes);
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                         ::"r"(smem_u32(s_here)), "l"(s_in + first_slice * slice_bytes), "r"(bytes), "r"(smem_u32(&arrived)) : "memory");
        }
        if (mbar_wait(smem_u32(&arrived), 0)) s_in = s_here - first_slice * slice_bytes;
        else atomicExch(g.status, DCUT_DEV_LORA_WAIT_TIMEOUT);
    }
    if (!work) return;
    if (STAGED && live) {
        copies_wait<0>();
#pragma unroll
        for (int e = 0; e < KEEP * 4; ++e) {
            uint4& v = kept[e / 4][e % 4];
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(b_here + e * 512) : "memory");
        }
    }

    s_in += 16 * lane;
    const int slice = at.slice, slice_up = GATED && g.n_slices == 2 ? 1 : slice;
    // (a body for either way of access: with both in one, the predicated single accesses were half of its instructions)
    auto all_rows = [&](auto vector) {
        constexpr bool VEC = decltype(vector)::value;
        for (int m = 0; FEW ? m < 1 : 16 * m < rows; ++m) {
            float d[4][4];
#pragma unroll
            for (int t = 0; t < 4; ++t) d[t][0] = d[t][1] = d[t][2] = d[t][3] = 0.0f;
            if (live) {
                const uint4* s_at = reinterpret_cast<const uint4*>(s_in + slice * slice_bytes + m * low.pieces() * 512);
                const uint4* s_up = reinterpret_cast<const uint4*>(s_in + slice_up * slice_bytes + m * low.pieces() * 512);
                auto multiply = [&](const uint4 (&bv)[4]) {
                    const uint4 s0 = s_at[0], s1 = s_at[32], u0 = GATED ? s_up[0] : s0, u1 = GATED ? s_up[32] : s1;       // (of its two MMAs)
                    s_at += 64, s_up += 64;
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        if (GATED && t >= 2) mma16816(d[t], u0, bv[t].x, bv[t].y);
                        else mma16816(d[t], s0, bv[t].x, bv[t].y);
                    }
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        if (GATED && t >= 2) mma16816(d[t], u1, bv[t].z, bv[t].w);
                        else mma16816(d[t], s1, bv[t].z, bv[t].w);
                    }
                };
                if (KEEP) {
#pragma unroll
                    for (int step = 0; step < KEEP; ++step) {
                        multiply(kept[step]);
                        if (low.parts == 2) multiply(kept[step]);
                    }
                } else {
#pragma unroll 1
                    for (int step = 0; step < low.steps; ++step) {
                        uint4 bv[4];
                        load_b(step, bv);
                        multiply(bv);
                        if (low.parts == 2) multiply(bv);
                    }
                }
            }
            const uint4 was[2] = {base[0], base[1]};
            const int now[2] = {row[0], row[1]};
            if (!FEW && 16 * (m + 1) < rows) fetch(vector, m + 1, row, base);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t w[4] = {was[h].x, was[h].y, was[h].z, was[h].w};
                float v[kPer], u[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const float x = bf_lo(w[t]) + d[t][2 * h], y = bf_hi(w[t]) + d[t][2 * h + 1];
                    if (GATED && t >= 2) u[2 * t - 4] = x, u[2 * t - 3] = y;
                    else v[2 * t] = x, v[2 * t + 1] = y;
                }
                activate(g.act, v);
                if (GATED) {
#pragma unroll
                    for (int j = 0; j < kPer; ++j) v[j] *= u[j & 3];
                }
                uint32_t o[kPer / 2];
#pragma unroll
                for (int j = 0; j < kPer / 2; ++j) o[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
                const int r = 8 * h + gr;
                unsigned char* to = VEC ? out_at + (unsigned long long)(unsigned)now[h] * (unsigned)g.ldo
                                        : edges[warp] + r * kEdgeRow + 2 * kPer * q;
                if (!VEC || 16 * m + r < rows) {
                    if (GATED) *reinterpret_cast<uint2*>(to) = make_uint2(o[0], o[1]);
                    else *reinterpret_cast<uint4*>(to) = make_uint4(o[0], o[1], o[kPer / 2 - 2], o[kPer / 2 - 1]);
                }
            }
            if (!VEC) {                                                    // a row's columns at a time
                __syncwarp();
                if (lane < min(kCols, left))
                    for (int r = 0; r < 16 && 16 * m + r < rows; ++r)
                        reinterpret_cast<unsigned short*>(g.out)[(size_t)tile.row[16 * m + r] * g.ldo + at.col + lane] =
                            *reinterpret_cast<const unsigned short*>(edges[warp] + r * kEdgeRow + 2 * lane);
                __syncwarp();
            }
        }
    };
    if (vec) all_rows(std::true_type{});
    else all_rows(std::false_type{});
}

// Two CTAs of the first product per SM, and never three: CTAs of several streams' launches may meet on an SM, and three could want more tensor memory
// than it has (256 columns at most each).  One would wait for another's, whose cluster might wait for the first one's.  The library's other kernels that
// hold tensor memory leave no room beside them.
constexpr int kStagedB = kWarps * 2 * 4 * 512;                        // two steps of a CTA's columns
constexpr int kMostShared = 110 * 1024, kLeastShared = 77 * 1024;

template <int STAGES>
dcut_status launch_low(dcut_ctx* ctx, const LoraArgs& g, const CUtensorMap& a_map, int grid, int split, size_t smem, cudaStream_t stream) {
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = split;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(grid);
    lc.blockDim = dim3(kThreads);
    lc.dynamicSmemBytes = smem;
    lc.stream = stream;
    lc.attrs = attr;
    lc.numAttrs = 2;
    return dcut_check_cuda(ctx, cudaLaunchKernelEx(&lc, lora_low_kernel<STAGES>, g, a_map), "launch lora_low_kernel");
}
template <bool GATED>
auto out_kernel(int rank, bool few) {
    const Low low(rank);
    if (few) return low.steps == 1 ? lora_out_kernel<GATED, 1, true, false> : low.steps == 2 ? lora_out_kernel<GATED, 2, true, false> : lora_out_kernel<GATED, 0, true, false>;
    if (low.steps == 2) return low.parts == 2 ? lora_out_kernel<GATED, 2, false, true> : lora_out_kernel<GATED, 2, false, false>;
    return low.steps == 1 ? lora_out_kernel<GATED, 1, false, false> : lora_out_kernel<GATED, 0, false, false>;
}
dcut_status launch(dcut_ctx* ctx, LoraArgs& g, const CUtensorMap& a_map, int R, int units, cudaStream_t stream) {
    const int SR = g.n_slices * g.rank, stage = (R + SR) * kRowBytes, sums = R * (SR + 8) * 4;
    // behind the last step: 128 rows from the beginning of its x on, 8 more rows of A; and the alignment
    const int slack = (stage < 128 * kRowBytes ? 128 * kRowBytes - stage : 0) + 1024 + 1024;
    const int stages = 8 * stage + slack <= kMostShared ? 8 : 4 * stage + slack <= kMostShared ? 4 : 2;
    const int need = (stages * stage > sums ? stages * stage : sums) + slack;
    const size_t smem = need > kLeastShared ? need : kLeastShared;
    g.tile_rows = R;
    g.part_row = SR + 8;
    g.tile_bytes = (long long)sizeof(Tile) + (long long)g.n_slices * (R / 16) * Low(g.rank).pieces() * 512;
    g.groups = g.gated ? (g.N / 2 + 15) / 16 : 0;
    for (int s = 0, lo = 0; s < (g.gated ? 0 : g.n_slices); ++s) {
        g.groups += (g.end[s] - lo + 31) / 32;
        lo = g.end[s];
    }
    g.blocks = (g.groups + kWarps - 1) / kWarps;
    // the sum of ceil(rows / R) over the units that are cut into tiles, at most; as many of them at a time as the scratch holds
    const long long tiles = ((long long)g.T_cap + (long long)units * (R - 1)) / R, room = DCUT_LORA_SCRATCH / g.tile_bytes;
    const Low low(g.rank);
    g.b_at = R > 16 ? (int)(g.tile_bytes - (long long)sizeof(Tile)) : 0;
    const size_t s_bytes = g.b_at + (R > 16 && low.steps == 2 && low.parts == 2 ? kStagedB : 0);
    auto* out = g.gated ? out_kernel<true>(g.rank, R == 16) : out_kernel<false>(g.rank, R == 16);
    for (long long t = 0; t < tiles; t += room) {
        const int n = (int)(tiles - t < room ? tiles - t : room);
        g.tile0 = (int)t;
        int split = kMostSplit;                                         // CTAs per tile: one wave of two per SM, where there are tiles for it
        while (split > 1 && (long long)n * split > 2 * ctx->sm_count) split >>= 1;
        dcut_status st = stages == 8   ? launch_low<8>(ctx, g, a_map, n * split, split, smem, stream)
                         : stages == 4 ? launch_low<4>(ctx, g, a_map, n * split, split, smem, stream)
                                       : launch_low<2>(ctx, g, a_map, n * split, split, smem, stream);
        if (st != DCUT_OK) return st;
        const int early = n * split <= ctx->sm_count;                    // there is room for this kernel's CTAs beside the first one's
        st = dcut_check_cuda(ctx, dcut_launch_pdl(out, dim3((unsigned)(n * g.blocks)), dim3(kThreads), s_bytes, stream, g, early), "launch lora_out_kernel");
        if (st != DCUT_OK) return st;
    }
    return DCUT_OK;
}

}  // namespace

dcut_status dcut_init_lora(dcut_ctx* ctx) {
    constexpr int M = DCUT_LORA_MAX_RANKS;
    static_assert(2 * (64 + M) * kRowBytes + 2048 <= kMostShared && 64 * (M + 8) * 4 + 2048 <= kMostShared, "two steps and the sums fit");
    cudaError_t e = cudaFuncSetAttribute(lora_low_kernel<8>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(lora_low_kernel<4>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(lora_low_kernel<2>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared);
    constexpr int kMostLow = 64 * 4 * (M + 96);                         // s of a tile: ranks that are no multiple of 32 fill up to 24 elements of two parts
    for (int rank : {8, 24, 64, 128})                                   // one for each form (tiles of 16 rows read s where it lies)
        for (auto* out : {out_kernel<false>(rank, false), out_kernel<true>(rank, false)})
            if (e == cudaSuccess) e = cudaFuncSetAttribute(out, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostLow + kStagedB);
    return dcut_check_cuda(ctx, e, "cudaFuncSetAttribute(lora)");
}

dcut_status dcut_launch_lora(dcut_ctx* ctx, const dcut_lora_args* l, const int* cu_q, int B, int T_cap, cudaStream_t stream) {
    LoraArgs g = {};
    g.x = static_cast<const __nv_bfloat16*>(l->x);
    g.a = static_cast<const __nv_bfloat16*>(l->a);
    g.b = static_cast<const __nv_bfloat16*>(l->b);
    g.base = static_cast<const __nv_bfloat16*>(l->base);
    g.out = static_cast<__nv_bfloat16*>(l->out);
    g.ldx = l->ldx, g.lda = l->lda, g.ldbase = l->ldbase, g.ldo = l->ldo;
    g.scale = l->scale, g.adapter = l->adapter, g.cu_q = cu_q;
    g.n_adapters = l->n_adapters, g.rank = l->rank, g.n_slices = l->n_slices, g.K = l->K, g.B = B, g.T_cap = T_cap;
    g.act = l->act, g.gated = l->gated != 0;
    for (int i = 0; i < l->n_slices; ++i) g.end[i] = l->slice_end[i];
    g.N = l->slice_end[l->n_slices - 1];
    g.in_place = l->out == l->base && l->act == DCUT_ACT_NONE && !g.gated;
    auto vec = [](const void* p, long long ld) { return !(reinterpret_cast<uintptr_t>(p) & 15) && ld % 8 == 0; };
    g.vec = vec(l->base, l->ldbase) && vec(l->out, l->ldo);
    g.status = ctx->d_status;
    g.scratch = ctx->lora_scratch;
    // units that are cut into tiles: adapters (and the rows without one), or requests
    const bool grouped = B <= kThreads && g.n_adapters < B;
    const int units = grouped ? g.n_adapters + 1 : B, mean = T_cap / (grouped ? g.n_adapters : B);     // rows of a unit on average, at most
    // A as a matrix of all the adapters' rows; a step takes 64 columns of one adapter's
    const cuuint64_t dims[2] = {(cuuint64_t)g.K, (cuuint64_t)g.n_adapters * g.n_slices * g.rank}, strides[1] = {(cuuint64_t)g.lda * 2};
    const cuuint32_t box[2] = {kChunk, (cuuint32_t)(g.n_slices * g.rank)}, ones[2] = {1, 1};
    CUtensorMap a_map;
    const CUresult r = reinterpret_cast<EncodeTiledFn>(ctx->encode_tiled)(&a_map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(l->a), dims, strides, box, ones,
                                                                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                                                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return dcut_fail(ctx, DCUT_ECUDA, "cuTensorMapEncodeTiled failed for the adapters (%d)", (int)r);
    // Rows of a tile.  The packed lengths are on the device: the mean is that of T_cap.  us on the device with 16 / 32 / 64 rows, requests with an adapter each, K = 4096:
    //                       64 of 16     64 of 17        24 of 40        16 of 64        16 of 65        8 of 136
    //   rank 16, 3 slices   26 / 27 / 28 34 / 31 / 32    24 / 23 / 21    23 / 19 / 19    27 / 23 / 25    23 / 22 / 21
    //   rank 64, gated     100 / 103 / 100 140 / 117 / 116 88 / 77 / 65  81 / 65 / 59    95 / 78 / 71    86 / 69 / 60
    //   rank 128            40 / 45 / 54 52 / 56 / 65    34 / 37 / 36    32 / 34 / 34    36 / 36 / 45    32 / 35 / 37
    // So 64 rows would do from some 33 on at ranks up to 64, and 16 rows are best for rank 128 up to 300 (3 of 2730: 165 / 139 / 133); the rule does not go by the rank.
    return launch(ctx, g, a_map, mean <= 16 ? 16 : mean <= 64 ? 32 : 64, units, stream);
}
