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
// One launch, no scratch: a tile is up to 16, 32 or 64 rows of one request, done by a cluster of 8 CTAs.  Each takes an eighth of K
// for s (its warps again an eighth each); the partial sums meet through distributed shared memory (every CTA adds an eighth of s in a
// fixed order and hands it to all), then each takes an eighth of the columns.  s is scaled in fp32 and rounded once to bf16 for the
// second product (an error of 2^-8 of s at most, as in the weights of the attention; it reaches d, not base).
#include <cuda_bf16.h>

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
    int part_row;                        // floats from a row of s to the next in the partial sums
    int s_row;                           // bytes from a row of s to the next (bf16)
    int front;                           // bytes of the area that the warps' sums and then s occupy
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
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 8 elements of a row from element k on; zeros from K on and where the row does not exist
__device__ __forceinline__ uint4 load8(const __nv_bfloat16* row, int k, int K, bool there) {
    if (!there || k >= K) return make_uint4(0, 0, 0, 0);
    if (k + 8 <= K) return *reinterpret_cast<const uint4*>(row + k);
    uint32_t w[4] = {0, 0, 0, 0};
    const unsigned short* p = reinterpret_cast<const unsigned short*>(row) + k;
#pragma unroll
    for (int j = 0; j < 7; ++j)
        if (k + j < K) w[j >> 1] |= (uint32_t)p[j] << (16 * (j & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

struct Tile {
    int row0, rows, adapter;             // rows = 0: there is no such tile
};
// Tile number t of the batch (tiles of R rows, request by request).  Requests that keep what they have are left out.
__device__ __forceinline__ Tile find_tile(const LoraArgs& g, int t, int R, Tile* found, int* warp_sum) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) found->rows = 0;
    int before = 0;                      // tiles of the requests that earlier passes looked at
    for (int i0 = 0; i0 < g.B && (before <= t || t == 0); i0 += kThreads) {      // (tile 0 looks at every request)
        const int i = i0 + tid;
        int lo = 0, hi = 0, id = -1;
        if (i < g.B) {
            lo = max(0, g.cu_q[i]), hi = min(g.cu_q[i + 1], g.T_cap), id = g.adapter[i];
            if (id >= g.n_adapters) {
                if (t == 0) atomicExch(g.status, DCUT_DEV_BAD_ADAPTER);
                id = -1;
            }
            if (i == g.B - 1 && t == 0 && g.cu_q[g.B] > g.T_cap) atomicExch(g.status, DCUT_DEV_BAD_ROWS);
        }
        const int n = hi > lo && !(id < 0 && g.in_place) ? (hi - lo + R - 1) / R : 0;
        int upto = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        __syncthreads();                 // (the sums of the pass before have been read)
        if (lane == 31) warp_sum[warp] = upto;
        __syncthreads();
        int all = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) upto += warp_sum[w];
            all += warp_sum[w];
        }
        const int at = t - before - (upto - n);
        if (at >= 0 && at < n) *found = Tile{lo + at * R, min(R, hi - lo - at * R), id};
        before += all;
    }
    __syncthreads();
    return *found;
}

// MT: 16-row MMA tiles of a tile; NT: 8-column MMA tiles of s that a pass takes; WIDE: the rank is a multiple of 32.
template <int MT, int NT, bool WIDE>
__global__ void __launch_bounds__(kThreads) __cluster_dims__(kCluster, 1, 1) lora_kernel(LoraArgs g) {
    constexpr int R = 16 * MT, kRed = NT * 8 + 8;                      // kRed: floats of a row of the warps' sums (8 of padding: banks)
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ Tile found;
    __shared__ int warp_sum[kWarps];
    dcut_pdl_wait();
    dcut_pdl_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gr = lane >> 2, q = lane & 3;
    const int rank = (int)cluster_rank(), SR = g.n_slices * g.rank;
    const Tile tile = find_tile(g, blockIdx.x / kCluster, R, &found, warp_sum);
    if (tile.rows == 0) return;                                        // (the whole cluster)
    const bool live = tile.adapter >= 0;
    float* red = reinterpret_cast<float*>(smem);                       // [warp][R][kRed], later s in bf16 [R][s_row bytes]
    float* part = reinterpret_cast<float*>(smem + g.front);            // [R][part_row]: this CTA's share of s

    if (live) {
        const __nv_bfloat16* a = g.a + (size_t)tile.adapter * SR * g.lda;
        const __nv_bfloat16* x = g.x + (size_t)tile.row0 * g.ldx;
        const int chunks = (g.K + 31) / 32, c0 = (int)((long long)chunks * rank / kCluster), c1 = (int)((long long)chunks * (rank + 1) / kCluster);
        for (int n0 = 0; n0 < SR; n0 += 8 * NT) {                      // columns n0 .. of s
            float acc[MT][NT][4];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[m][n][0] = acc[m][n][1] = acc[m][n][2] = acc[m][n][3] = 0.0f;
#pragma unroll 2
            for (int c = c0 + warp; c < c1; c += kWarps) {
                const int k = 32 * c + 8 * q;
                uint4 xv[MT][2], av[NT];
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int r = 16 * m + 8 * h + gr;
                        xv[m][h] = load8(x + (size_t)r * g.ldx, k, g.K, r < tile.rows);
                    }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int j = n0 + 8 * n + gr;
                    av[n] = load8(a + (size_t)j * g.lda, k, g.K, j < SR);
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        mma16816(acc[m][n], xv[m][0].x, xv[m][1].x, xv[m][0].y, xv[m][1].y, av[n].x, av[n].y);
                        mma16816(acc[m][n], xv[m][0].z, xv[m][1].z, xv[m][0].w, xv[m][1].w, av[n].z, av[n].w);
                    }
            }
            if (n0 > 0) __syncthreads();                               // (the warps' sums of the pass before have been read)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float* p = red + (warp * R + 16 * m + gr) * kRed + 8 * n + 2 * q;
                    *reinterpret_cast<float2*>(p) = make_float2(acc[m][n][0], acc[m][n][1]);
                    *reinterpret_cast<float2*>(p + 8 * kRed) = make_float2(acc[m][n][2], acc[m][n][3]);
                }
            __syncthreads();
            const int cols = min(8 * NT, SR - n0), quads = cols / 4;
            for (int e = threadIdx.x; e < R * quads; e += kThreads) {
                const int r = e / quads, c = 4 * (e - r * quads);
                float4 s = make_float4(0, 0, 0, 0);
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    const float4 v = *reinterpret_cast<const float4*>(red + (w * R + r) * kRed + c);
                    s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
                }
                *reinterpret_cast<float4*>(part + r * g.part_row + n0 + c) = s;
            }
        }
        cluster_sync();                                                // every CTA's share is complete; the warps' sums are dead
        const float scale = g.scale ? g.scale[tile.adapter] : 1.0f;
        const uint32_t part_at = static_cast<uint32_t>(__cvta_generic_to_shared(part)), s_at = static_cast<uint32_t>(__cvta_generic_to_shared(smem));
        const int quads = SR / 4, each = R * quads / kCluster;         // (R is a multiple of 16, SR of 8)
        for (int e = rank * each + threadIdx.x; e < (rank + 1) * each; e += kThreads) {
            const int r = e / quads, c = 4 * (e - r * quads);
            float4 v[kCluster], s = make_float4(0, 0, 0, 0);
#pragma unroll
            for (int p = 0; p < kCluster; ++p)
                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[p].x), "=f"(v[p].y), "=f"(v[p].z), "=f"(v[p].w)
                             : "r"(in_cta(part_at + 4 * (r * g.part_row + c), p)) : "memory");
#pragma unroll
            for (int p = 0; p < kCluster; ++p) s.x += v[p].x, s.y += v[p].y, s.z += v[p].z, s.w += v[p].w;
            const uint32_t lo = pack_bf16(s.x * scale, s.y * scale), hi = pack_bf16(s.z * scale, s.w * scale);
#pragma unroll
            for (int p = 0; p < kCluster; ++p)
                asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(in_cta(s_at + r * g.s_row + 2 * c, p)), "r"(lo), "r"(hi) : "memory");
        }
        cluster_sync();                                                // s is complete everywhere; nothing remote is read or written after this
    }

    // ---- the columns: groups of 32 of one slice (gated: of the gate, with the same ones of the up projection)
    const int width = g.gated ? g.N / 2 : g.N;                         // columns of out
    int groups = 0;
    if (g.gated) groups = (width + 31) / 32;
    else
        for (int s = 0, lo = 0; s < g.n_slices; ++s) {
            groups += (g.end[s] - lo + 31) / 32;
            lo = g.end[s];
        }
    const int g0 = (int)((long long)groups * rank / kCluster), g1 = (int)((long long)groups * (rank + 1) / kCluster);
    const __nv_bfloat16* b = g.b + (size_t)max(tile.adapter, 0) * g.N * g.rank;

    // d[m][t]: rows 16 m + gr and + 8 of s times rows col + 8 (n >> 1) + 2 t + (n & 1) of B, n the MMA's column: a lane ends with
    // columns col + 8 q .. + 7
    auto product = [&](int col, int end, int s_col, float (&d)[MT][4][4]) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int t = 0; t < 4; ++t) d[m][t][0] = d[m][t][1] = d[m][t][2] = d[m][t][3] = 0.0f;
        constexpr int kStep = WIDE ? 32 : 16;                          // rank elements per step, 8 or 4 of them in a lane
        for (int k0 = 0; k0 < g.rank; k0 += kStep) {
            const int k = k0 + kStep / 4 * q;
            uint4 bv[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int n = col + 8 * (gr >> 1) + 2 * t + (gr & 1);
                bv[t] = make_uint4(0, 0, 0, 0);
                if (n < end && k < g.rank) {
                    const __nv_bfloat16* p = b + (size_t)n * g.rank + k;
                    if (WIDE) bv[t] = *reinterpret_cast<const uint4*>(p);
                    else {
                        const uint2 v = *reinterpret_cast<const uint2*>(p);
                        bv[t].x = v.x, bv[t].y = v.y;
                    }
                }
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                uint4 sv[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const unsigned char* p = smem + (16 * m + 8 * h + gr) * g.s_row + 2 * (s_col + k);
                    sv[h] = make_uint4(0, 0, 0, 0);
                    if (WIDE) sv[h] = *reinterpret_cast<const uint4*>(p);
                    else if (k < g.rank) {
                        const uint2 v = *reinterpret_cast<const uint2*>(p);
                        sv[h].x = v.x, sv[h].y = v.y;
                    }
                }
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    mma16816(d[m][t], sv[0].x, sv[1].x, sv[0].y, sv[1].y, bv[t].x, bv[t].y);
                    if (WIDE) mma16816(d[m][t], sv[0].z, sv[1].z, sv[0].w, sv[1].w, bv[t].z, bv[t].w);
                }
            }
        }
    };
    // the 8 values of base at this lane's columns of row r
    auto fetch = [&](int r, int col, int end, bool vec) {
        const __nv_bfloat16* p = g.base + (size_t)(tile.row0 + r) * g.ldbase + col;
        if (r >= tile.rows) return make_uint4(0, 0, 0, 0);
        if (vec) return *reinterpret_cast<const uint4*>(p);
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (col + j < end) w[j >> 1] |= (uint32_t)reinterpret_cast<const unsigned short*>(p)[j] << (16 * (j & 1));
        return make_uint4(w[0], w[1], w[2], w[3]);
    };
    auto values = [&](const uint4& v, const float (&d)[4][4], int h, float4 (&y)[2]) {
        y[0] = make_float4(bf_lo(v.x) + d[0][2 * h], bf_hi(v.x) + d[0][2 * h + 1], bf_lo(v.y) + d[1][2 * h], bf_hi(v.y) + d[1][2 * h + 1]);
        y[1] = make_float4(bf_lo(v.z) + d[2][2 * h], bf_hi(v.z) + d[2][2 * h + 1], bf_lo(v.w) + d[3][2 * h], bf_hi(v.w) + d[3][2 * h + 1]);
    };
    for (int i = g0 + warp; i < g1; i += kWarps) {
        int first = 0, end = width, slice = 0, in = i;                 // the slice of out's columns, and the group within it
        if (!g.gated) {
            end = g.end[0];
            while (in >= (end - first + 31) / 32) {
                in -= (end - first + 31) / 32;
                first = end;
                end = g.end[++slice];
            }
        }
        const int col = first + 32 * in, mine = col + 8 * q;
        const bool vec = g.vec && !(first & 7) && mine + 8 <= end, vec_up = vec && !(width & 7);
        uint4 base[MT][2], up[MT][2];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                base[m][h] = fetch(16 * m + 8 * h + gr, mine, end, vec);
                if (g.gated) up[m][h] = fetch(16 * m + 8 * h + gr, width + mine, g.N, vec_up);
            }
        float d[MT][4][4], u[MT][4][4];
        if (live) product(col, end, slice * g.rank, d);
        else
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int t = 0; t < 4; ++t) d[m][t][0] = d[m][t][1] = d[m][t][2] = d[m][t][3] = 0.0f;
        if (g.gated) {
            if (live) product(width + col, g.N, g.n_slices == 2 ? g.rank : 0, u);
            else
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int t = 0; t < 4; ++t) u[m][t][0] = u[m][t][1] = u[m][t][2] = u[m][t][3] = 0.0f;
        }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = 16 * m + 8 * h + gr;
                float4 y[2];
                values(base[m][h], d[m], h, y);
                if (g.act != DCUT_ACT_NONE) y[0] = activate4(g.act, y[0]), y[1] = activate4(g.act, y[1]);
                if (g.gated) {
                    float4 z[2];
                    values(up[m][h], u[m], h, z);
#pragma unroll
                    for (int j = 0; j < 2; ++j) y[j].x *= z[j].x, y[j].y *= z[j].y, y[j].z *= z[j].z, y[j].w *= z[j].w;
                }
                if (r >= tile.rows) continue;
                __nv_bfloat16* o = g.out + (size_t)(tile.row0 + r) * g.ldo + mine;
                const uint32_t w[4] = {pack_bf16(y[0].x, y[0].y), pack_bf16(y[0].z, y[0].w), pack_bf16(y[1].x, y[1].y), pack_bf16(y[1].z, y[1].w)};
                if (vec) *reinterpret_cast<uint4*>(o) = make_uint4(w[0], w[1], w[2], w[3]);
                else
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (mine + j < end) reinterpret_cast<unsigned short*>(o)[j] = (unsigned short)(w[j >> 1] >> (16 * (j & 1)));
            }
    }
}

template <int MT, int NT, bool WIDE>
dcut_status launch(dcut_ctx* ctx, LoraArgs& g, cudaStream_t stream) {
    constexpr int R = 16 * MT;
    const int warps = kWarps * R * (NT * 8 + 8) * 4, s = R * g.s_row;
    g.front = ((warps > s ? warps : s) + 127) & ~127;
    const size_t smem = (size_t)g.front + (size_t)R * g.part_row * 4;
    const long long tiles = ((long long)g.T_cap + (long long)g.B * (R - 1)) / R;         // sum of ceil(rows / R) over the requests, at most
    auto* kernel = lora_kernel<MT, NT, WIDE>;
    return dcut_check_cuda(ctx, dcut_launch_pdl(kernel, dim3((unsigned)(tiles * kCluster)), dim3(kThreads), smem, stream, g), "launch lora_kernel");
}
template <int MT, int NT>
dcut_status launch(dcut_ctx* ctx, LoraArgs& g, cudaStream_t stream) {
    return g.rank % 32 ? launch<MT, NT, false>(ctx, g, stream) : launch<MT, NT, true>(ctx, g, stream);
}
template <int MT, int NT>
cudaError_t allow() {
    constexpr int most = (kWarps * 16 * MT * (NT * 8 + 8) + 16 * MT * (DCUT_LORA_MAX_RANKS + 4)) * 4 + 128;
    static_assert(16 * MT * (2 * DCUT_LORA_MAX_RANKS + 192) <= kWarps * 16 * MT * (NT * 8 + 8) * 4 && most <= 227 * 1024, "s lies in the place of the warps' sums");
    cudaError_t e = cudaFuncSetAttribute(lora_kernel<MT, NT, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    return e == cudaSuccess ? cudaFuncSetAttribute(lora_kernel<MT, NT, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) : e;
}

}  // namespace

dcut_status dcut_init_lora(dcut_ctx* ctx) {
    cudaError_t e = allow<1, 8>();
    if (e == cudaSuccess) e = allow<2, 8>();
    if (e == cudaSuccess) e = allow<4, 4>();
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
    g.part_row = SR + 4;
    // rows of s 32 bytes (8-byte reads) or 64 (16-byte reads) apart modulo 128: no two lanes of a read meet in a bank
    g.s_row = (2 * SR + 127) / 128 * 128 + (g.rank % 32 ? 32 : 64);
    g.status = ctx->d_status;
    const long long mean = T_cap / B;                                  // rows of a request, at most, on average
    return mean <= 8 ? launch<1, 8>(ctx, g, stream) : mean <= 40 ? launch<2, 8>(ctx, g, stream) : launch<4, 4>(ctx, g, stream);
}
