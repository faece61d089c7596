// dcut_lora: the low-rank adapters of many requests beside a shared projection.
//
//   d[r, n] = scale[i] sum_j s[r, j] B_i[n, j],   s = x[r, :] . A_i^T,   i the adapter of the row's request
//   out = act(base + d), or act(base_gate + d_gate) * (base_up + d_up)
//
// Two products with a rank between them; each byte of x, base and out moves once, A and B of an adapter once per tile of rows (from
// L2 but for the first).  A few multiplications per byte: the memory, and for few rows its latency, bounds it, so the products run
// on warp-level MMAs that take their operands from global memory in 16-byte pieces: the order of a sum's terms is free, so a
// lane's piece of 8 neighbouring elements serves as its fragments of two MMAs, and the columns of four MMAs are dealt so that
// a lane ends with 8 neighbouring results.
// One launch, no scratch: a tile is up to 16, 32 or 64 rows that share an adapter, done by a cluster of 8 CTAs.  Each takes an eighth of K
// for s (its warps again an eighth each); the partial sums meet through distributed shared memory (every CTA adds an eighth of s in a
// fixed order and hands it to all), then each takes an eighth of the columns.  s is scaled in fp32 and enters the second product as
// the sum of two bf16 values (off by 2^-17 of it at most; a single one cost the result up to 1.7 times its error where d outweighs base).
#include <cuda_bf16.h>
#include <math.h>

#include "activation.cuh"
#include "dcut_internal.h"

namespace {

constexpr int kCluster = 8, kWarps = 8, kThreads = 32 * kWarps;
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
    int wn;                              // warps side by side over the columns of s
    int part_row;                        // floats from a row of s to the next in the partial sums
    int s_row;                           // bytes from a row of s to the next (bf16)
    int front;                           // bytes of the partial sums
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
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 16 bytes where `there`, else zeros.  A predicate and no branch: the loads of a step leave together.  (Not volatile: what it reads does
// not change while the kernel runs, base excepted, which is read where the value that replaces it depends on it.)
__device__ __forceinline__ uint4 load_if(const __nv_bfloat16* p, bool there) {
    uint4 v;
    asm("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
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

// what bf16 rounding took from two values (nothing from an infinity): `high` is their packed rounding
__device__ __forceinline__ uint32_t low_parts(float x, float y, uint32_t high) {
    const float hx = bf_lo(high), hy = bf_hi(high);
    return pack_bf16(fabsf(hx) < INFINITY ? x - hx : 0.0f, fabsf(hy) < INFINITY ? y - hy : 0.0f);
}
__device__ __forceinline__ void with_base(const uint4& v, const float (&d)[4][4], int h, float4 (&y)[2]) {
    y[0] = make_float4(bf_lo(v.x) + d[0][2 * h], bf_hi(v.x) + d[0][2 * h + 1], bf_lo(v.y) + d[1][2 * h], bf_hi(v.y) + d[1][2 * h + 1]);
    y[1] = make_float4(bf_lo(v.z) + d[2][2 * h], bf_hi(v.z) + d[2][2 * h + 1], bf_lo(v.w) + d[3][2 * h], bf_hi(v.w) + d[3][2 * h + 1]);
}

// What a cluster works on: up to R rows of one adapter (of several requests, where they share it).
struct Tile {
    int rows, adapter;                   // rows = 0: there is no such tile
    int row[64];
};
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
            for (int j = 0; j < g.B; ++j) {
                const int2 r = f.request[j];
                if (r.x == id && j < i) first += r.y;
                if (r.x == id && j > i) mine += r.y;
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

// asks for `bytes` (a multiple of 16) from p on (aligned to 16) to come to L2
__device__ __forceinline__ void ahead_to_l2(const void* p, uint32_t bytes) {
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
}

// A tile has 16 MT WR rows: WR sets of warps with 16 MT rows each.  NT: 8-column MMA tiles of s that a warp takes at a time.
// With MT = 1 a step's loads leave one step early; with MT = 2 the registers hold one step, and two CTAs per SM hide its latency.
template <int WR, int MT, int NT, bool GATED>
__global__ void __launch_bounds__(kThreads, 2) __cluster_dims__(kCluster, 1, 1) lora_kernel(LoraArgs g) {
    constexpr int R = 16 * MT * WR, kSet = kWarps / WR, kParts = GATED ? 2 : 1;          // kSet: warps that share their rows
    constexpr bool kEarly = MT == 1;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ Tile tile;
    __shared__ Search search;
    dcut_pdl_wait();
    dcut_pdl_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gr = lane >> 2, q = lane & 3;
    const int rank = (int)cluster_rank(), SR = g.n_slices * g.rank;
    find_tile(g, blockIdx.x / kCluster, R, tile, search);
    const int rows = tile.rows, adapter = tile.adapter;
    if (rows == 0) return;                                             // (the whole cluster)
    const bool live = adapter >= 0;
    float* red = reinterpret_cast<float*>(smem);                       // [K split][R][part_row]: the warps' sums; their total in the first
    unsigned char* s_area = smem + g.front;                            // [R][s_row bytes]: per slice the rank's high parts, then the low ones
    const int row_set = warp / kSet, in_set = warp % kSet, row_w = 16 * MT * row_set;     // this warp's rows: row_w ..
    int row[MT][2];                                                    // rows that do not exist: the last one that does
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) row[m][h] = tile.row[min(row_w + 16 * m + 8 * h + gr, rows - 1)];

    const int width = GATED ? g.N / 2 : g.N;                           // columns of out
    int groups = 0;
    if (GATED) groups = (width + 31) / 32;
    else
        for (int s = 0, lo = 0; s < g.n_slices; ++s) {
            groups += (g.end[s] - lo + 31) / 32;
            lo = g.end[s];
        }
    const int g0 = (int)((long long)groups * rank / kCluster), g1 = (int)((long long)groups * (rank + 1) / kCluster);
    const __nv_bfloat16* b = g.b + (size_t)max(adapter, 0) * g.N * g.rank;
    if (live && warp == kWarps - 1 && lane < kParts && g0 < g1) {       // this CTA's rows of B
        const Group from = group_of(g, g0, GATED), to = group_of(g, g1 - 1, GATED);
        const int n = min(to.col + 32, to.end) - from.col;
        ahead_to_l2(b + (size_t)(lane * width + from.col) * g.rank, (uint32_t)n * g.rank * 2);
    }
    // s is kept as the sum of two bf16 values.  A step is 32 elements of the rank, 8 in a lane, and both parts take it (wide); ranks that
    // are no multiple of 32 walk the high parts and the low ones as one row of 2 rank elements instead, so that rank 16 fills a step.
    const bool wide = g.rank % 32 == 0;
    const int row_len = wide ? g.rank : 2 * g.rank, steps = live ? (row_len + 31) / 32 : 0;

    // rows col + 8 (n >> 1) + 2 t + (n & 1) of B, n the MMA's column: a lane ends with columns col + 8 q .. + 7 of the results
    auto load_b = [&](const Group& at, int part, int step, uint4 (&bv)[4]) {
        const int v = 32 * step + 8 * q, k = v >= g.rank ? v - g.rank : v;
        const int first = part ? width + at.col : at.col, end = part ? g.N : at.end;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int n = first + 8 * (gr >> 1) + 2 * t + (gr & 1);
            bv[t] = load_if(b + (size_t)n * g.rank + k, n < end && v < row_len);
        }
    };
    // base at this lane's 8 columns of its rows
    auto fetch = [&](const Group& at, int part, uint4 (&v)[MT][2]) {
        const int col = (part ? width + at.col : at.col) + 8 * q, end = part ? g.N : at.end;
        const bool vec = by_vector(g, col - 8 * q, end);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool there = row_w + 16 * m + 8 * h + gr < rows;
                const __nv_bfloat16* p = g.base + (size_t)row[m][h] * g.ldbase + col;
                v[m][h] = vec ? load_if(p, there) : load_some(p, there ? end - col : 0);
            }
    };

    Group at = {0, 0, 0};
    uint4 bv[4], base[MT][2];
    int i = g0 + in_set;
    if (i < g1) {
        at = group_of(g, i, GATED);
        if (kEarly) {                                                  // what the first columns need does not wait for s
            if (live) load_b(at, 0, 0, bv);
            fetch(at, 0, base);
        }
    }

    if (live) {
        // ---- s = x . A^T: this CTA's eighth of K; the warps of a set share the columns (wn of them) and then K (wk of them)
        const __nv_bfloat16* a = g.a + (size_t)adapter * SR * g.lda + 8 * q;
        const int chunks = (g.K + 31) / 32, c0 = (int)((long long)chunks * rank / kCluster), c1 = (int)((long long)chunks * (rank + 1) / kCluster);
        const int wn = min(g.wn, kSet), wk = kSet / wn, my_n = in_set % wn, my_k = in_set / wn;
        const __nv_bfloat16* xp[MT][2];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) xp[m][h] = g.x + (size_t)row[m][h] * g.ldx + 8 * q;
        for (int n0 = 8 * NT * my_n; n0 < SR; n0 += 8 * NT * wn) {
            float acc[MT][NT][4];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[m][n][0] = acc[m][n][1] = acc[m][n][2] = acc[m][n][3] = 0.0f;
            auto load = [&](int c, uint4 (&xv)[MT][2], uint4 (&av)[NT]) {
                const int left = g.K - 32 * c - 8 * q;                  // elements from this lane's first one on
                const bool there = left >= 8 && c < c1;
#pragma unroll
                for (int m = 0; m < MT; ++m) xv[m][0] = load_if(xp[m][0] + 32 * c, there), xv[m][1] = load_if(xp[m][1] + 32 * c, there);
#pragma unroll
                for (int n = 0; n < NT; ++n) av[n] = load_if(a + (size_t)(n0 + 8 * n + gr) * g.lda + 32 * c, there && n0 + 8 * n < SR);
                if ((g.K & 7) && c == chunks - 1 && c < c1 && left > 0 && left < 8) {
#pragma unroll
                    for (int m = 0; m < MT; ++m) xv[m][0] = load_some(xp[m][0] + 32 * c, left), xv[m][1] = load_some(xp[m][1] + 32 * c, left);
#pragma unroll
                    for (int n = 0; n < NT; ++n) av[n] = load_some(a + (size_t)(n0 + 8 * n + gr) * g.lda + 32 * c, n0 + 8 * n < SR ? left : 0);
                }
            };
            uint4 xv[MT][2], av[NT], xn[MT][2], an[NT];
            if (kEarly) load(c0 + my_k, xv, av);
            for (int c = c0 + my_k; c < c1; c += wk) {
                if (kEarly) load(c + wk, xn, an);
                else load(c, xv, av);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        mma16816(acc[m][n], xv[m][0].x, xv[m][1].x, xv[m][0].y, xv[m][1].y, av[n].x, av[n].y);
                        mma16816(acc[m][n], xv[m][0].z, xv[m][1].z, xv[m][0].w, xv[m][1].w, av[n].z, av[n].w);
                    }
                if (kEarly) {
#pragma unroll
                    for (int m = 0; m < MT; ++m) xv[m][0] = xn[m][0], xv[m][1] = xn[m][1];
#pragma unroll
                    for (int n = 0; n < NT; ++n) av[n] = an[n];
                }
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    if (n0 + 8 * n >= SR) continue;
                    float* p = red + (my_k * R + row_w + 16 * m + gr) * g.part_row + n0 + 8 * n + 2 * q;
                    *reinterpret_cast<float2*>(p) = make_float2(acc[m][n][0], acc[m][n][1]);
                    *reinterpret_cast<float2*>(p + 8 * g.part_row) = make_float2(acc[m][n][2], acc[m][n][3]);
                }
        }
        const int quads = SR / 4;
        if (wk > 1) {
            __syncthreads();
            for (int e = threadIdx.x; e < R * quads; e += kThreads) {
                const int r = e / quads, c = 4 * (e - r * quads);
                float* p = red + r * g.part_row + c;
                float4 s = *reinterpret_cast<const float4*>(p);
                for (int w = 1; w < wk; ++w) {
                    const float4 v = *reinterpret_cast<const float4*>(p + w * R * g.part_row);
                    s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
                }
                *reinterpret_cast<float4*>(p) = s;
            }
        }
        cluster_sync();                                                // every CTA's share is complete
        const float scale = g.scale ? g.scale[adapter] : 1.0f;
        const uint32_t red_at = static_cast<uint32_t>(__cvta_generic_to_shared(red)), s_at = static_cast<uint32_t>(__cvta_generic_to_shared(s_area));
        const int each = R * quads / kCluster;                         // (R is a multiple of 16, SR of 8)
        for (int e = rank * each + threadIdx.x; e < (rank + 1) * each; e += kThreads) {
            const int r = e / quads, c = 4 * (e - r * quads), slice = c / g.rank;
            float4 v[kCluster], s = make_float4(0, 0, 0, 0);
#pragma unroll
            for (int p = 0; p < kCluster; ++p)
                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[p].x), "=f"(v[p].y), "=f"(v[p].z), "=f"(v[p].w)
                             : "r"(in_cta(red_at + 4 * (r * g.part_row + c), p)) : "memory");
#pragma unroll
            for (int p = 0; p < kCluster; ++p) s.x += v[p].x, s.y += v[p].y, s.z += v[p].z, s.w += v[p].w;
            s.x *= scale, s.y *= scale, s.z *= scale, s.w *= scale;
            const uint32_t hi0 = pack_bf16(s.x, s.y), hi1 = pack_bf16(s.z, s.w);
            const uint32_t lo0 = low_parts(s.x, s.y, hi0), lo1 = low_parts(s.z, s.w, hi1);
            const uint32_t to = s_at + r * g.s_row + 2 * (c + slice * g.rank);
#pragma unroll
            for (int p = 0; p < kCluster; ++p) {
                const uint32_t there = in_cta(to, p);
                asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(there), "r"(hi0), "r"(hi1) : "memory");
                asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(there + 2 * g.rank), "r"(lo0), "r"(lo1) : "memory");
            }
        }
        cluster_sync();                                                // s is complete everywhere; nothing remote is read or written after this
    }

    // ---- this CTA's eighth of the columns
    for (; i < g1; i += kSet) {
        const Group next = i + kSet < g1 ? group_of(g, i + kSet, GATED) : at;
        float y[MT][2][8];                                             // this lane's results, row by row
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
            uint4 here[MT][2], bn[4];
            if (kEarly) {                                              // on their way: what follows this part
#pragma unroll
                for (int m = 0; m < MT; ++m) here[m][0] = base[m][0], here[m][1] = base[m][1];
                if (part + 1 < kParts) fetch(at, part + 1, base);
                else fetch(next, 0, base);
            } else {
                if (live) load_b(at, part, 0, bv);
                fetch(at, part, here);
            }
            float d[MT][4][4];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int t = 0; t < 4; ++t) d[m][t][0] = d[m][t][1] = d[m][t][2] = d[m][t][3] = 0.0f;
            const int slice = GATED ? (g.n_slices == 2 ? part : 0) : at.slice;
#pragma unroll 1
            for (int step = 0; step < steps; ++step) {
                if (step + 1 < steps) load_b(at, part, step + 1, bn);
                else if (kEarly) {
                    if (part + 1 < kParts) load_b(at, part + 1, 0, bn);
                    else load_b(next, 0, 0, bn);
                }
                const int v = 32 * step + 8 * q;
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const unsigned char* p = s_area + (row_w + 16 * m + gr) * g.s_row + 2 * (2 * slice * g.rank + v);
#pragma unroll
                    for (int low = 0; low < 2; ++low) {
                        if (low && !wide) break;
                        uint4 s0 = make_uint4(0, 0, 0, 0), s1 = s0;
                        if (v < row_len) {
                            s0 = *reinterpret_cast<const uint4*>(p + 2 * low * g.rank);
                            s1 = *reinterpret_cast<const uint4*>(p + 2 * low * g.rank + 8 * g.s_row);
                        }
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            mma16816(d[m][t], s0.x, s1.x, s0.y, s1.y, bv[t].x, bv[t].y);
                            mma16816(d[m][t], s0.z, s1.z, s0.w, s1.w, bv[t].z, bv[t].w);
                        }
                    }
                }
#pragma unroll
                for (int t = 0; t < 4; ++t) bv[t] = bn[t];
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float4 z[2];
                    with_base(here[m][h], d[m], h, z);
                    if (part == 0 && g.act != DCUT_ACT_NONE) z[0] = activate4(g.act, z[0]), z[1] = activate4(g.act, z[1]);
                    const float zs[8] = {z[0].x, z[0].y, z[0].z, z[0].w, z[1].x, z[1].y, z[1].z, z[1].w};
#pragma unroll
                    for (int j = 0; j < 8; ++j) y[m][h][j] = part == 0 ? zs[j] : y[m][h][j] * zs[j];
                }
        }
        const int mine = at.col + 8 * q;
        const bool vec = by_vector(g, at.col, at.end);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (row_w + 16 * m + 8 * h + gr >= rows) continue;
                __nv_bfloat16* o = g.out + (size_t)row[m][h] * g.ldo + mine;
                const float(&v)[8] = y[m][h];
                const uint32_t w[4] = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
                if (vec) *reinterpret_cast<uint4*>(o) = make_uint4(w[0], w[1], w[2], w[3]);
                else
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (mine + j < at.end) reinterpret_cast<unsigned short*>(o)[j] = (unsigned short)(w[j >> 1] >> (16 * (j & 1)));
            }
        at = next;
    }
}

template <int WR, int MT, int NT, bool GATED>
dcut_status launch(dcut_ctx* ctx, LoraArgs& g, cudaStream_t stream) {
    constexpr int R = 16 * MT * WR, kSet = kWarps / WR;
    const int SR = g.n_slices * g.rank, share = (SR + 8 * NT - 1) / (8 * NT);
    g.wn = share > 2 ? 4 : share;                                      // warps side by side over the columns of s; the others split K
    const int wk = kSet / (g.wn < kSet ? g.wn : kSet);
    g.front = (wk * R * g.part_row * 4 + 127) & ~127;
    const size_t smem = (size_t)g.front + (size_t)R * g.s_row;
    // the sum of ceil(rows / R) over the units that are cut into tiles, at most: adapters (and the rows without one), or requests
    const int units = g.B <= kThreads && g.n_adapters < g.B ? g.n_adapters + 1 : g.B;
    const long long tiles = ((long long)g.T_cap + (long long)units * (R - 1)) / R;
    return dcut_check_cuda(ctx, dcut_launch_pdl(lora_kernel<WR, MT, NT, GATED>, dim3((unsigned)(tiles * kCluster)), dim3(kThreads), smem, stream, g),
                           "launch lora_kernel");
}
template <int WR, int MT>
dcut_status launch(dcut_ctx* ctx, LoraArgs& g, cudaStream_t stream) {
    const bool few = g.n_slices * g.rank <= 16;
    if (g.gated) return few ? launch<WR, MT, 2, true>(ctx, g, stream) : launch<WR, MT, 4, true>(ctx, g, stream);
    return few ? launch<WR, MT, 2, false>(ctx, g, stream) : launch<WR, MT, 4, false>(ctx, g, stream);
}
template <int WR, int MT>
cudaError_t allow() {
    // as many splits of K as there can be with so many ranks: 8 / WR up to 32, half of that up to 64, then a quarter
    constexpr int R = 16 * MT * WR, kMost = 160 * 1024;
    constexpr int at32 = 8 / WR * R * 40 * 4 + R * 192, at256 = (2 / WR < 1 ? 1 : 2 / WR) * R * (DCUT_LORA_MAX_RANKS + 8) * 4 + R * (4 * DCUT_LORA_MAX_RANKS + 64);
    static_assert(at32 + 128 <= kMost && at256 + 128 <= kMost, "fits an SM");
    cudaError_t e = cudaFuncSetAttribute(lora_kernel<WR, MT, 2, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(lora_kernel<WR, MT, 4, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(lora_kernel<WR, MT, 2, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    return e == cudaSuccess ? cudaFuncSetAttribute(lora_kernel<WR, MT, 4, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost) : e;
}

}  // namespace

dcut_status dcut_init_lora(dcut_ctx* ctx) {
    cudaError_t e = allow<1, 1>();
    if (e == cudaSuccess) e = allow<1, 2>();
    if (e == cudaSuccess) e = allow<2, 2>();
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
    const int SR = g.n_slices * g.rank;
    g.part_row = SR + 8;
    g.s_row = (4 * SR + 127) / 128 * 128 + 64;                         // rows 64 bytes apart modulo 128: no two lanes of a 16-byte read meet in a bank
    g.status = ctx->d_status;
    const long long mean = T_cap / (B <= kThreads && g.n_adapters < B ? g.n_adapters : B);   // rows of a unit, at most, on average
    return mean <= 8 ? launch<1, 1>(ctx, g, stream) : mean <= 40 ? launch<1, 2>(ctx, g, stream) : launch<2, 2>(ctx, g, stream);
}
