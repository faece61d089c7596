// dcut_lora: the low-rank adapters of many requests beside a shared projection.
//
//   d[r, n] = scale[i] sum_j s[r, j] B_i[n, j],   s = x[r, :] . A_i^T,   i the adapter of the row's request
//   out = act(base + d), or act(base_gate + d_gate) * (base_up + d_up)
//
// Two products with a rank between them; each byte of x, base and out moves once, A and B of an adapter once per tile of rows (from
// L2 but for the first).  A few multiplications per byte: the memory, and for few rows its latency, bounds it, so both products run on
// warp-level MMAs.  A tile is up to 16, 32 or 64 rows that share an adapter (of several requests, where those share it).
//   lora_low_kernel   s of a tile, by 1 to 8 CTAs (a cluster) that cut K between them: x and A come through asynchronous copies, several steps
//                     ahead; the partial sums meet through distributed shared memory, added in a fixed order.  s is scaled in fp32 and kept as
//                     the sum of two bf16 values (off by 2^-17 of it at most; a single one cost the result up to 1.7 times its error where
//                     d outweighs base), in the order in which the second product's lanes read it.
//   lora_out_kernel   32 columns of a tile per warp, 16 rows at a time: no shared memory, no barrier, many warps per SM.
// One kernel for both, whose clusters kept s to themselves and took an eighth of the columns per CTA each, was 1.5 to 3 times slower at length:
// with 8 to 16 warps per SM every step waited for its loads.
#include <cuda_bf16.h>
#include <math.h>

#include "activation.cuh"
#include "dcut_internal.h"

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
    int wn;                              // first product: warps side by side over the columns of s; the others of a row block split K
    int part_row;                        // floats from a row of s to the next in the partial sums
    int tile0, blocks;                   // first tile of this pass; CTAs of the second product per tile
    unsigned char* scratch;              // per tile: a Tile, then its s
    long long tile_bytes;
    int* status;
};

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Asynchronous copies to shared memory; `bytes` of the 16 are read, the rest is filled with zeros.
__device__ __forceinline__ void copy16(uint32_t to, const void* from, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.commit_group;" ::: "memory"); }       // ends a group of copies
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }   // all but the last N groups
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t shared_at(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

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
    int row[64];
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

// The columns of out that a warp works on at a time: 32 of one slice (gated: of the gate, with the same ones of the up projection).
struct Group {
    int col, end, slice;                 // first column; where the slice ends
};
__device__ __forceinline__ Group group_of(const LoraArgs& g, int i, bool gated) {
    int first = 0, end = gated ? g.N / 2 : g.end[0], slice = 0;
    if (!gated)
        while (i >= (end - first + 31) / 32) {
            i -= (end - first + 31) / 32;
            first = end;
            end = g.end[++slice];
        }
    return Group{first + 32 * i, end, slice};
}

// whether the group at column `col` is read and written in 16-byte pieces (the same answer in the whole warp)
__device__ __forceinline__ bool by_vector(const LoraArgs& g, int col, int end) { return g.vec && !(col & 7) && col + 32 <= end; }

// How s lies in the scratch.  A step of the second product is 32 elements, 8 in a lane.  Ranks that are multiples of 32 take a step with the high
// parts and again with the low ones (parts = 2); others walk the high parts and then the low ones as one row, so that rank 16 fills a step.
// Per slice, 16 rows, step and part: rows gr and gr + 8 of the 16, a 16-byte piece per lane each.
struct Low {
    int steps, parts;
    __host__ __device__ Low(int rank) : steps(rank % 32 ? (2 * rank + 31) / 32 : rank / 32), parts(rank % 32 ? 1 : 2) {}
    __host__ __device__ int pieces() const { return steps * parts * 2; }                 // of 512 bytes, per slice and 16 rows
    // the piece and the byte within it of element j (high or low part) of row r of a tile of MT blocks of 16 rows
    __device__ __forceinline__ int at(int blocks16, int rank, int slice, int r, int j, int low) const {
        const int v = parts == 1 && low ? rank + j : j, part = parts == 1 ? 0 : low;
        return ((((slice * blocks16 + (r >> 4)) * steps + (v >> 5)) * parts + part) * 2 + ((r >> 3) & 1)) * 512 + (((r & 7) << 2) + ((v >> 3) & 3)) * 16 + (v & 7) * 2;
    }
};

constexpr int kChunk = 64;               // elements of K per step of the first product: rows of 128 bytes, 16-byte piece c of row r at c ^ (r & 7)
constexpr int kRowBytes = 2 * kChunk, kPieces = kRowBytes / 16, kStrideRows = kThreads / kPieces;
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

// s of a tile of 16 MT rows.  A warp has 16 rows and up to 8 NT columns; STAGES - 1 steps of K are on their way.
template <int MT, int NT, int STAGES>
__global__ void __launch_bounds__(kThreads, 2) lora_low_kernel(LoraArgs g) {
    constexpr int R = 16 * MT, kSet = kWarps / MT;                     // kSet: warps that share 16 rows
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ Tile tile;
    __shared__ Search search;
    dcut_pdl_wait();
    dcut_pdl_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gr = lane >> 2, q = lane & 3;
    const int rank = (int)cluster_rank(), split = (int)cluster_size(), SR = g.n_slices * g.rank, number = blockIdx.x / split;
    find_tile(g, g.tile0 + number, R, tile, search);
    const int rows = tile.rows, adapter = tile.adapter;
    unsigned char* record = g.scratch + number * g.tile_bytes;
    if (rank == 0 && threadIdx.x < 2 + rows) reinterpret_cast<int*>(record)[threadIdx.x] = reinterpret_cast<const int*>(&tile)[threadIdx.x];
    if (rows == 0 || adapter < 0) return;                              // (the whole cluster)
    float* sums = reinterpret_cast<float*>(smem);                      // in the ring's place, later: [K split of the warps][R][part_row]; the total in the first

    const int chunks = (g.K + kChunk - 1) / kChunk, c0 = (int)((long long)chunks * rank / split), n_chunks = (int)((long long)chunks * (rank + 1) / split) - c0;
    const int stage = (R + SR) * kRowBytes;
    // a thread copies the same 16-byte piece of every 32nd row: of x (zeros where there is no row), then of A
    const int piece = threadIdx.x % kPieces, r0 = threadIdx.x / kPieces;
    const uint32_t ring_at = shared_at(smem), to0 = ring_at + r0 * kRowBytes + ((piece ^ (r0 & 7)) << 4);
    constexpr int kX = (R + kStrideRows - 1) / kStrideRows;
    const __nv_bfloat16* x_from[kX];                                   // (these two move along K with the steps that are asked for)
#pragma unroll
    for (int i = 0; i < kX; ++i) x_from[i] = g.x + (size_t)tile.row[min(r0 + kStrideRows * i, rows - 1)] * g.ldx + (size_t)c0 * kChunk + 8 * piece;
    const __nv_bfloat16* a_from = g.a + ((size_t)adapter * SR + r0) * g.lda + (size_t)c0 * kChunk + 8 * piece;
    const long long a_step = kStrideRows * g.lda;
    int left = 2 * (g.K - c0 * kChunk - 8 * piece), asked = 0;         // bytes from this thread's next piece to the end of its rows; steps asked for
    auto load = [&](int slot) {
        if (asked < n_chunks) {
            const uint32_t to = to0 + slot * stage;
            const int bytes = min(16, max(0, left));                   // (0: nothing is read, and the address is one that exists)
#pragma unroll
            for (int i = 0; i < kX; ++i)
                if (R % kStrideRows == 0 || r0 + kStrideRows * i < R)
                    copy16(to + i * kStrideRows * kRowBytes, bytes ? x_from[i] : g.x, r0 + kStrideRows * i < rows ? bytes : 0), x_from[i] += kChunk;
            const __nv_bfloat16* from = bytes ? a_from : g.a;
            const long long step = bytes ? a_step : 0;
            uint32_t to_a = to + R * kRowBytes;
#pragma unroll 4
            for (int r = r0; r < SR; r += kStrideRows, to_a += kStrideRows * kRowBytes, from += step) copy16(to_a, from, bytes);
            a_from += kChunk, left -= kRowBytes, ++asked;
        }
        copies_done();
    };
    const int wn = min(g.wn, kSet), wk = kSet / wn, m = warp / kSet, in_set = warp % kSet, my_n = in_set % wn, my_k = in_set / wn;
    const int tiles = SR / 8, per = (tiles + wn - 1) / wn, t0 = my_n * per, nt = min(per, tiles - t0);         // this warp's 8-column tiles of s
    // this lane's rows for ldmatrix: where they begin in a step, and the swizzle with the half of 16 elements that the lane points to
    const int x_row = 16 * m + (lane & 15), x_at = x_row * kRowBytes, x_flip = ((x_row & 7) ^ (lane >> 4)) << 4;
    const int a_flip = ((lane & 7) ^ ((lane >> 3) & 1)) << 4;          // (R and the tiles' first rows are multiples of 8)
    int a_at[(NT + 1) / 2];                                            // (a tile that does not exist: the last one that does)
#pragma unroll
    for (int n = 0; n < NT; n += 2) a_at[n / 2] = (R + 8 * min(t0 + n + (lane >> 4), tiles - 1) + (lane & 7)) * kRowBytes;
    float acc[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.0f;
#pragma unroll
    for (int c = 0; c < STAGES - 1; ++c) load(c);
    for (int c = 0, slot = 0, ahead = STAGES - 1; c < n_chunks; ++c) {
        copies_wait<STAGES - 2>();
        __syncthreads();                                               // step c has arrived, step c - 1 has been read
        load(ahead);
        const uint32_t at = ring_at + slot * stage;
        auto multiply = [&](int k) {                                   // 16 elements of K
            uint32_t xf[4];
            ldmatrix4(xf, at + x_at + ((32 * k) ^ x_flip));
#pragma unroll
            for (int n = 0; n < NT; n += 2) {
                if (n >= nt) break;
                uint32_t af[4];                                        // two tiles' fragments
                ldmatrix4(af, at + a_at[n / 2] + ((32 * k) ^ a_flip));
                mma16816(acc[n], xf[0], xf[1], xf[2], xf[3], af[0], af[1]);
                if (n + 1 < nt) mma16816(acc[n + 1], xf[0], xf[1], xf[2], xf[3], af[2], af[3]);
            }
        };
        if (wk == 1) {
#pragma unroll
            for (int k = 0; k < kChunk / 16; ++k) multiply(k);
        } else {                                                       // the warps of a set take turns
            for (int k = (my_k - c * (kChunk / 16)) & (wk - 1); k < kChunk / 16; k += wk) multiply(k);
        }
        slot = slot + 1 == STAGES ? 0 : slot + 1;
        ahead = ahead + 1 == STAGES ? 0 : ahead + 1;
    }
    copies_wait<0>();
    __syncthreads();                                                   // the ring is free
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (n >= nt) break;
        float* p = sums + (my_k * R + 16 * m + gr) * g.part_row + 8 * (t0 + n) + 2 * q;
        *reinterpret_cast<float2*>(p) = make_float2(acc[n][0], acc[n][1]);
        *reinterpret_cast<float2*>(p + 8 * g.part_row) = make_float2(acc[n][2], acc[n][3]);
    }
    const int quads = SR / 4;
    if (wk > 1) {
        __syncthreads();
        for (int e = threadIdx.x; e < R * quads; e += kThreads) {
            const int r = e / quads, c = 4 * (e - r * quads);
            float* p = sums + r * g.part_row + c;
            float4 s = *reinterpret_cast<const float4*>(p);
            for (int w = 1; w < wk; ++w) {
                const float4 v = *reinterpret_cast<const float4*>(p + w * R * g.part_row);
                s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
            }
            *reinterpret_cast<float4*>(p) = s;
        }
    }
    cluster_sync();                                                    // every CTA's share is complete
    const float scale = g.scale ? g.scale[adapter] : 1.0f;
    const uint32_t sums_at = shared_at(sums);
    const Low low(g.rank);
    unsigned char* s_out = record + sizeof(Tile);
    const int each = R * quads / split;                                // (R is a multiple of 16, SR of 8, the split of 8 a divisor)
    for (int e = rank * each + threadIdx.x; e < (rank + 1) * each; e += kThreads) {
        const int r = e / quads, c = 4 * (e - r * quads), slice = c / g.rank, j = c - slice * g.rank;
        float4 s = make_float4(0, 0, 0, 0), v[kMostSplit];
#pragma unroll
        for (int p = 0; p < kMostSplit; ++p)
            if (p < split)
                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[p].x), "=f"(v[p].y), "=f"(v[p].z), "=f"(v[p].w)
                             : "r"(in_cta(sums_at + 4 * (r * g.part_row + c), p)) : "memory");
#pragma unroll
        for (int p = 0; p < kMostSplit; ++p)
            if (p < split) s.x += v[p].x, s.y += v[p].y, s.z += v[p].z, s.w += v[p].w;
        s.x *= scale, s.y *= scale, s.z *= scale, s.w *= scale;
        const uint32_t hi0 = pack_bf16(s.x, s.y), hi1 = pack_bf16(s.z, s.w);
        *reinterpret_cast<uint2*>(s_out + low.at(MT, g.rank, slice, r, j, 0)) = make_uint2(hi0, hi1);
        *reinterpret_cast<uint2*>(s_out + low.at(MT, g.rank, slice, r, j, 1)) = make_uint2(low_parts(s.x, s.y, hi0), low_parts(s.z, s.w, hi1));
    }
    if (low.parts == 1 && rank == split - 1) {                         // what fills up the last step
        const int rest = (32 * low.steps - 2 * g.rank) / 4;
        for (int e = threadIdx.x; e < g.n_slices * R * rest; e += kThreads) {
            const int sr = e / rest, v = 2 * g.rank + 4 * (e - sr * rest);
            *reinterpret_cast<uint2*>(s_out + low.at(MT, g.rank, sr / R, sr % R, v, 0)) = make_uint2(0, 0);
        }
    }
    cluster_sync();                                                    // nobody leaves while its sums are read
}

// out of a tile: a warp has 32 columns, 16 rows at a time.  The MMA's column n of tile t is column 8 (n >> 1) + 2 t + (n & 1) of the 32, so that
// a lane ends with the 8 neighbouring columns 8 q .. + 7; its 8 neighbouring elements of s and of B serve as its fragments of two MMAs
// (the order of a sum's terms is free).  KEEP: the rank's steps, where B's fragments stay in registers for all rows; 0: they are read again.
// `early`: the CTA finds its tile itself and asks for B and its first rows of base while the first product runs (what that one waited for is
// complete once this grid has started); otherwise it reads the tile from the scratch.
template <bool GATED, int KEEP>
__global__ void __launch_bounds__(kThreads, GATED || KEEP > 1 ? 2 : 3) lora_out_kernel(LoraArgs g, int blocks16, int early) {
    constexpr int kParts = GATED ? 2 : 1;
    __shared__ __align__(16) unsigned char edges[kWarps][16 * kEdgeRow];
    __shared__ Tile tile;
    __shared__ Search search;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gr = lane >> 2, q = lane & 3;
    const int number = blockIdx.x / g.blocks;
    const unsigned char* record = g.scratch + number * g.tile_bytes;
    if (early) find_tile(g, g.tile0 + number, 16 * blocks16, tile, search);
    else {
        dcut_pdl_wait();
        if (threadIdx.x < 66) reinterpret_cast<int*>(&tile)[threadIdx.x] = reinterpret_cast<const int*>(record)[threadIdx.x];
        __syncthreads();
    }
    const int rows = tile.rows, adapter = tile.adapter;
    const int width = GATED ? g.N / 2 : g.N;                           // columns of out
    int groups = 0;
    if (GATED) groups = (width + 31) / 32;
    else
        for (int s = 0, lo = 0; s < g.n_slices; ++s) {
            groups += (g.end[s] - lo + 31) / 32;
            lo = g.end[s];
        }
    const int i = (blockIdx.x - number * g.blocks) * kWarps + warp;
    const bool work = rows > 0 && i < groups, live = work && adapter >= 0;
    const Group at = group_of(g, work ? i : 0, GATED);
    const Low low(g.rank);
    const bool vec = by_vector(g, at.col, at.end), vec_up = GATED && by_vector(g, width + at.col, g.N);
    // B: rows b_row + 2 t of a part's columns; elements from this lane's first one of a step on (behind both parts s is zero, and so is this)
    const int b_row = 8 * (gr >> 1) + (gr & 1);
    const __nv_bfloat16* b = g.b + ((size_t)max(adapter, 0) * g.N + at.col + b_row) * g.rank;
    const int left = at.end - at.col - b_row, left_up = g.N - width - at.col - b_row;
    auto load_b = [&](int part, int step, uint4 (&bv)[4]) {
        const int v = 32 * step + 8 * q, k = v < g.rank ? v : v - g.rank;
        const __nv_bfloat16* p = b + (part ? (size_t)width * g.rank : 0) + k;
#pragma unroll
        for (int t = 0; t < 4; ++t, p += 2 * g.rank) bv[t] = load_if(p, 2 * t < (part ? left_up : left) && v < 2 * g.rank);
    };
    // base at this lane's 8 columns of rows gr and gr + 8 of block m (those that do not exist: of the last one that does)
    auto fetch = [&](int m, int (&row)[2], uint4 (&v)[kParts][2]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            row[h] = tile.row[min(16 * m + 8 * h + gr, rows - 1)];
            const __nv_bfloat16* p = g.base + (unsigned long long)(unsigned)row[h] * (unsigned)g.ldbase + at.col + 8 * q;
            v[0][h] = vec ? *reinterpret_cast<const uint4*>(p) : load_some(p, at.end - at.col - 8 * q);
            if (GATED) v[kParts - 1][h] = vec_up ? *reinterpret_cast<const uint4*>(p + width) : load_some(p + width, at.end - at.col - 8 * q);
        }
    };
    uint4 kept[KEEP ? kParts * KEEP : 1][4], base[kParts][2];
    int row[2];
    if (work) fetch(0, row, base);
    if (KEEP && live) {
#pragma unroll
        for (int part = 0; part < kParts; ++part)
#pragma unroll
            for (int step = 0; step < KEEP; ++step) load_b(part, step, kept[part * KEEP + step]);
    }
    if (early) dcut_pdl_wait();
    dcut_pdl_launch_dependents();
    if (!work) return;

    const uint4* s_in = reinterpret_cast<const uint4*>(record + sizeof(Tile)) + lane;
    for (int m = 0; 16 * m < rows; ++m) {
        float y[2][8];
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
            float d[4][4];
#pragma unroll
            for (int t = 0; t < 4; ++t) d[t][0] = d[t][1] = d[t][2] = d[t][3] = 0.0f;
            if (live) {
                const uint4* s_at = s_in + ((GATED ? (g.n_slices == 2 ? part : 0) : at.slice) * blocks16 + m) * low.pieces() * 32;
                auto multiply = [&](const uint4 (&bv)[4]) {
                    const uint4 s0 = s_at[0], s1 = s_at[32];
                    s_at += 64;
#pragma unroll
                    for (int t = 0; t < 4; ++t) mma16816(d[t], s0.x, s1.x, s0.y, s1.y, bv[t].x, bv[t].y);
#pragma unroll
                    for (int t = 0; t < 4; ++t) mma16816(d[t], s0.z, s1.z, s0.w, s1.w, bv[t].z, bv[t].w);
                };
                if (KEEP) {
#pragma unroll
                    for (int step = 0; step < KEEP; ++step) {
                        multiply(kept[part * KEEP + step]);
                        if (low.parts == 2) multiply(kept[part * KEEP + step]);
                    }
                } else {
#pragma unroll 1
                    for (int step = 0; step < low.steps; ++step) {
                        uint4 bv[4];
                        load_b(part, step, bv);
                        multiply(bv);
                        if (low.parts == 2) multiply(bv);
                    }
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint4 w = base[part][h];
                float v[8] = {bf_lo(w.x) + d[0][2 * h], bf_hi(w.x) + d[0][2 * h + 1], bf_lo(w.y) + d[1][2 * h], bf_hi(w.y) + d[1][2 * h + 1],
                              bf_lo(w.z) + d[2][2 * h], bf_hi(w.z) + d[2][2 * h + 1], bf_lo(w.w) + d[3][2 * h], bf_hi(w.w) + d[3][2 * h + 1]};
                if (part == 0) activate(g.act, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) y[h][j] = part ? y[h][j] * v[j] : v[j];
            }
        }
        const int row_now[2] = {row[0], row[1]};
        if (16 * (m + 1) < rows) fetch(m + 1, row, base);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float(&v)[8] = y[h];
            const uint4 w = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
            const int r = 8 * h + gr;
            if (!vec) *reinterpret_cast<uint4*>(edges[warp] + r * kEdgeRow + 16 * q) = w;
            else if (16 * m + r < rows)
                *reinterpret_cast<uint4*>(g.out + (unsigned long long)(unsigned)row_now[h] * (unsigned)g.ldo + at.col + 8 * q) = w;
        }
        if (!vec) {                                                    // a row's 32 columns at a time
            __syncwarp();
            if (at.col + lane < at.end)
                for (int r = 0; r < 16 && 16 * m + r < rows; ++r)
                    reinterpret_cast<unsigned short*>(g.out)[(size_t)tile.row[16 * m + r] * g.ldo + at.col + lane] =
                        *reinterpret_cast<const unsigned short*>(edges[warp] + r * kEdgeRow + 2 * lane);
            __syncwarp();
        }
    }
}

constexpr int kMostShared = 110 * 1024;                                 // two CTAs of the first product per SM

template <int MT, int NT, int STAGES>
dcut_status launch_low(dcut_ctx* ctx, const LoraArgs& g, int grid, int split, size_t smem, cudaStream_t stream) {
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
    return dcut_check_cuda(ctx, cudaLaunchKernelEx(&lc, lora_low_kernel<MT, NT, STAGES>, g), "launch lora_low_kernel");
}
// How the first product of a launch runs
struct Plan {
    int wn, stages;
    size_t smem;
};
template <int MT>
Plan plan_low(int SR) {
    constexpr int R = 16 * MT, kSet = kWarps / MT;
    Plan p;
    for (p.wn = 1; p.wn < kSet && (SR / 8 + p.wn - 1) / p.wn > 4;) p.wn *= 2;             // up to 4 tiles of s per warp, where there are warps for it
    const int stage = (R + SR) * kRowBytes, sums = kSet / p.wn * R * (SR + 8) * 4;
    p.stages = 8 * stage <= kMostShared ? 8 : 4 * stage <= kMostShared ? 4 : 2;
    p.smem = p.stages * stage > sums ? p.stages * stage : sums;
    return p;
}
template <int MT>
dcut_status launch(dcut_ctx* ctx, LoraArgs& g, int units, cudaStream_t stream) {
    constexpr int R = 16 * MT, NT = 8;
    const int SR = g.n_slices * g.rank;
    const Plan p = plan_low<MT>(SR);
    g.wn = p.wn;
    g.part_row = SR + 8;
    g.tile_bytes = (long long)sizeof(Tile) + (long long)g.n_slices * MT * Low(g.rank).pieces() * 512;
    int groups = 0;
    for (int s = 0, lo = 0; s < (g.gated ? 1 : g.n_slices); ++s) {
        const int end = g.gated ? g.N / 2 : g.end[s];
        groups += (end - lo + 31) / 32;
        lo = end;
    }
    g.blocks = (groups + kWarps - 1) / kWarps;
    // the sum of ceil(rows / R) over the units that are cut into tiles, at most; as many of them at a time as the scratch holds
    const long long tiles = ((long long)g.T_cap + (long long)units * (R - 1)) / R, room = DCUT_LORA_SCRATCH / g.tile_bytes;
    for (long long t = 0; t < tiles; t += room) {
        const int n = (int)(tiles - t < room ? tiles - t : room);
        g.tile0 = (int)t;
        int split = kMostSplit;                                         // CTAs per tile: one wave of two per SM, where there are tiles for it
        while (split > 1 && (long long)n * split > 2 * ctx->sm_count) split >>= 1;
        dcut_status st = p.stages == 8   ? launch_low<MT, NT, 8>(ctx, g, n * split, split, p.smem, stream)
                         : p.stages == 4 ? launch_low<MT, NT, 4>(ctx, g, n * split, split, p.smem, stream)
                                         : launch_low<MT, NT, 2>(ctx, g, n * split, split, p.smem, stream);
        if (st != DCUT_OK) return st;
        const int steps = Low(g.rank).steps;
        auto* out = g.gated ? (steps == 1 ? lora_out_kernel<true, 1> : lora_out_kernel<true, 0>)
                            : (steps == 1 ? lora_out_kernel<false, 1> : steps == 2 ? lora_out_kernel<false, 2> : lora_out_kernel<false, 0>);
        const long long ctas = (long long)n * g.blocks;
        const int early = ctas <= 2 * ctx->sm_count;                     // all of them can wait beside the first product
        st = dcut_check_cuda(ctx, dcut_launch_pdl(out, dim3((unsigned)ctas), dim3(kThreads), 0, stream, g, MT, early), "launch lora_out_kernel");
        if (st != DCUT_OK) return st;
    }
    return DCUT_OK;
}
template <int MT>
cudaError_t allow() {
    constexpr int R = 16 * MT, M = MT > 2 ? DCUT_LORA_MAX_RANKS / 2 : DCUT_LORA_MAX_RANKS, NT = 8;
    static_assert(2 * (R + M) * kRowBytes <= kMostShared && R * (M + 8) * 4 <= kMostShared && 2 * R * (M / 2 + 8) * 4 <= kMostShared, "two steps and the sums fit");
    static_assert(M / 8 <= NT * (kWarps / MT), "a warp's tiles of s");
    cudaError_t e = cudaFuncSetAttribute(lora_low_kernel<MT, NT, 8>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(lora_low_kernel<MT, NT, 4>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared);
    return e == cudaSuccess ? cudaFuncSetAttribute(lora_low_kernel<MT, NT, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared) : e;
}

}  // namespace

dcut_status dcut_init_lora(dcut_ctx* ctx) {
    cudaError_t e = allow<1>();
    if (e == cudaSuccess) e = allow<2>();
    if (e == cudaSuccess) e = allow<4>();
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
    return mean <= 16 ? launch<1>(ctx, g, units, stream) : mean <= 64 || g.n_slices * g.rank > DCUT_LORA_MAX_RANKS / 2 ? launch<2>(ctx, g, units, stream) : launch<4>(ctx, g, units, stream);
}
