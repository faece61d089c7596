// dcut_rms_norm: the residual's addition, the RMS norm and the 8-bit rows that dcut_linear8 reads, in one pass over a row.
//
//   h = x + residual;   y = (h * gain) * r,  r = 1 / sqrt(mean(h^2) + eps)   (or y = h);   scale = max(max|y|, 2^-100) / 448,
//   y8 = e4m3(y / scale)
//
// Every byte is read once and written once: bound by HBM for thousands of rows, by the launch and one trip to memory for few.
// A row stays in registers.  max|y| = r * max|h * gain| (rounding is monotone, r > 0), so the sum of squares and the maximum
// leave through one reduction and the row is finished behind a single barrier.  Sum and statistics are fp32, h is normalised
// before it is rounded to bf16; each output is rounded once.
// 8191 rows of 4096 with a residual and both outputs (302 MB) 53 us, 5.6 TB/s of reads and writes; 16 rows 2.6 us.  A thread has 1 to 8 pieces of 16 bytes, by
// the width: more of them mean fewer threads per row and more rows per SM, fewer a shorter chain for a single row.
// A sum of squares that overflows (|h| above about 10^18) is formed again from h * 2^-80.  Where it does, or h * gain does, h is normalised ahead of
// the gain (2^-80 would make the squares of ordinary values vanish).  The maximum keeps a NaN.
#include <cuda_bf16.h>
#include <math.h>

#include "dcut_internal.h"

namespace {

constexpr int kMaxThreads = 512;
constexpr float kE4m3Max = 448.0f;
constexpr float kLeast = 7.888609052210118e-31f;       // 2^-100: 448 / it and it / 448 are normal numbers

struct NormArgs {
    const __nv_bfloat16 *x, *residual, *gain;          // residual, gain may be null
    long long ldx, ldr, ldh, ldo, ld8;
    __nv_bfloat16 *h_out, *out;                        // may be null
    unsigned char* out8;                               // may be null (with scale8)
    float* scale8;
    const int* cu_q;                                   // or null: T_cap rows
    int B, T_cap, width, normed;
    float eps, gain_add;                               // gain_add: 0, or 1 (the factor is 1 + gain)
    int* status;
};

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ void unpack8(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) x[2 * j] = bf_lo(w[j]), x[2 * j + 1] = bf_hi(w[j]);
}
// the larger magnitude (its sign says nothing); NaN if either is
__device__ __forceinline__ float larger(float a, float b) {
    float r;
    asm("max.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// two values to e4m3, round to nearest even, saturating; the first goes to the low byte
__device__ __forceinline__ uint32_t e4m3x2(float first, float second) {
    unsigned short r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(second), "f"(first));
    return r;
}

// Quotients of neighbours by a scale, two at a time: a product with the scale's reciprocal and its remainder's correction (P. Markstein, 1990).  The product
// alone, half an ulp of the reciprocal off, put one code in 1500 to 4300 of bf16 rows beside the one of y / scale; an fp32 division for each element took
// 15 to 48 % longer than the product.  Scales below 2^-80 are lifted, so that the remainder of whatever e4m3 does not round to 0 is exact.  A zero keeps its sign.
struct Quotient {
    uint64_t factor, inv, by, plain;                   // both halves of each: -lift r, -1 / (lift scale), lift scale, r
    static __device__ __forceinline__ uint64_t pack(float lo, float hi) {
        uint64_t v;
        asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi));
        return v;
    }
    static __device__ __forceinline__ uint64_t mul(uint64_t a, uint64_t b) {
        uint64_t v;
        asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
        return v;
    }
    static __device__ __forceinline__ uint64_t fma(uint64_t a, uint64_t b, uint64_t c) {
        uint64_t v;
        asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
        return v;
    }
    __device__ __forceinline__ Quotient(float r, float scale) {
        const float lift = scale < 0x1p-80f ? 0x1p40f : 1.0f, s = scale * lift, i = -1.0f / s, f = -r * lift;
        factor = pack(f, f), inv = pack(i, i), by = pack(s, s), plain = pack(r, r);
    }
    // x r
    __device__ __forceinline__ void times(float x0, float x1, float& y0, float& y1) const {
        const uint64_t v = mul(pack(x0, x1), plain);
        asm("mov.b64 {%0, %1}, %2;" : "=f"(y0), "=f"(y1) : "l"(v));
    }
    // x r / scale
    __device__ __forceinline__ void of(float& x0, float& x1) const {
        const uint64_t z = mul(pack(x0, x1), factor), q = mul(z, inv), v = fma(fma(q, by, z), inv, q);
        asm("mov.b64 {%0, %1}, %2;" : "=f"(x0), "=f"(x1) : "l"(v));
    }
};

// How rows are read and written.  kVector: a slot of a thread is 8 neighbouring elements, a vector (the row's last one may be partly used).
// kShifted: the same, but bf16 outputs begin anywhere (rows of an odd width one after the other, say; 7698 x 2789 54 us, 69 with 2-byte stores; the code
// for it slows aligned rows down, so it is a form of its own).  kSingle: inputs begin anywhere too; element j of a slot is `threads` elements after
// element j - 1, so that a warp's 2-byte accesses are neighbours.
enum Access { kVector, kShifted, kSingle };
template <Access ACCESS>
struct Place {
    static constexpr bool VEC = ACCESS != kSingle;
    int first, step, live;                             // live: elements of the slot that exist
    __device__ __forceinline__ Place(int slot, int tid, int threads, int width) {
        if (VEC) {
            first = (slot * threads + tid) * 8, step = 1;
            live = min(8, max(0, width - first));
        } else {
            first = slot * 8 * threads + tid, step = threads;
            live = first < width ? min(8, (width - first + threads - 1) / threads) : 0;
        }
    }
    __device__ __forceinline__ uint4 load(const __nv_bfloat16* row) const {
        if (VEC && live == 8) return *reinterpret_cast<const uint4*>(row + first);
        uint32_t w[4] = {0, 0, 0, 0};
        const unsigned short* p = reinterpret_cast<const unsigned short*>(row) + first;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < live) w[j >> 1] |= (uint32_t)p[j * step] << (16 * (j & 1));
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    // (called by whole warps)
    __device__ __forceinline__ void store(__nv_bfloat16* row, const float (&v)[8]) const {
        const uint32_t w[4] = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
        unsigned short* p = reinterpret_cast<unsigned short*>(row) + first;
        auto some = [&](int from, int to) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j >= from && j < to) p[j * step] = (unsigned short)(w[j >> 1] >> (16 * (j & 1)));
        };
        const int s = ACCESS == kShifted ? (int)(reinterpret_cast<uintptr_t>(row) >> 1) & 7 : 0;      // elements from the 16-byte boundary before the row on
        if (ACCESS != kShifted || !__all_sync(0xffffffffu, live == 8)) {
            if (VEC && live == 8 && s == 0) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
            else some(0, live);
            return;
        }
        if (s == 0) {
            *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
            return;
        }
        // Rows that begin elsewhere: a lane stores the vector on the boundary before its first element, whose first s elements are the last ones of the
        // lane before it.  The warp's first lane has none before it, and its last lane's last s elements are nobody else's.
        uint32_t x[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = __shfl_up_sync(0xffffffffu, w[j], 1), x[4 + j] = w[j];
        const int skip = 8 - s, lane = threadIdx.x & 31;               // elements of x that are left out
#pragma unroll
        for (int bit = 4; bit >= 2; bit >>= 1)
            if (skip & bit) {
#pragma unroll
                for (int j = 0; j + bit / 2 < 8; ++j) x[j] = x[j + bit / 2];
            }
        if (skip & 1) {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = __funnelshift_r(x[j], x[j + 1], 16);
        }
        if (lane > 0) *reinterpret_cast<uint4*>(p - s) = make_uint4(x[0], x[1], x[2], x[3]);
        else some(0, skip);
        if (lane == 31) some(skip, 8);
    }
    __device__ __forceinline__ void store8(unsigned char* row, const float (&v)[8]) const {
        const uint32_t w[2] = {e4m3x2(v[0], v[1]) | e4m3x2(v[2], v[3]) << 16, e4m3x2(v[4], v[5]) | e4m3x2(v[6], v[7]) << 16};
        if (VEC && live == 8) {
            *reinterpret_cast<uint2*>(row + first) = make_uint2(w[0], w[1]);
            return;
        }
        unsigned char* p = row + first;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < live) p[j * step] = (unsigned char)(w[j >> 2] >> (8 * (j & 3)));
    }
};

struct Stats {
    float sum, top;
};
// Over the threads of a row, in a fixed order: a warp's by shuffles, then (ALONE: a row per CTA) the warps'.
template <bool ALONE, bool SUM>
__device__ __forceinline__ Stats over_row(Stats s, Stats* warps) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        if (SUM) s.sum += __shfl_xor_sync(0xffffffffu, s.sum, o);
        s.top = larger(s.top, __shfl_xor_sync(0xffffffffu, s.top, o));
    }
    if (!ALONE) return s;
    const int lane = threadIdx.x & 31, n_warps = blockDim.x >> 5;
    if (lane == 0) warps[threadIdx.x >> 5] = s;
    __syncthreads();
    s = lane < n_warps ? warps[lane] : Stats{0.0f, 0.0f};
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        if (SUM) s.sum += __shfl_xor_sync(0xffffffffu, s.sum, o);
        s.top = larger(s.top, __shfl_xor_sync(0xffffffffu, s.top, o));
    }
    return s;
}

// V slots per thread; ALONE: the CTA has one row, otherwise every warp its own.  kBare: neither residual nor gain (with their registers
// fewer CTAs fit an SM, 1088 x 12288 14 us against 11); kRows: no norm either, rows that are only quantised
// (without the sum of squares: 1088 x 12288 10.8 us against 11.4, 8191 x 4096 22.8 against 24.5).
enum Form { kFull, kBare, kRows };
template <int V, Access ACCESS, bool ALONE, Form FORM>
__global__ void __launch_bounds__(kMaxThreads) rms_norm_kernel(NormArgs a) {
    constexpr bool PLAIN = FORM != kFull, NORM = FORM != kRows;
    __shared__ Stats warps[3][32];
    dcut_pdl_wait();
    dcut_pdl_launch_dependents();
    const int T = a.cu_q ? a.cu_q[a.B] : a.T_cap;
    if (T > a.T_cap && blockIdx.x == 0 && threadIdx.x == 0) atomicExch(a.status, DCUT_DEV_BAD_ROWS);
    const int row = ALONE ? blockIdx.x : blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    const int tid = ALONE ? threadIdx.x : threadIdx.x & 31, threads = ALONE ? blockDim.x : 32;
    if (row >= min(T, a.T_cap)) return;

    const __nv_bfloat16* x_row = a.x + (size_t)row * a.ldx;
    const __nv_bfloat16* r_row = !PLAIN && a.residual ? a.residual + (size_t)row * a.ldr : nullptr;
    const bool has_gain = !PLAIN && a.gain;
    uint4 xv[V], rv[PLAIN ? 1 : V], gv[PLAIN ? 1 : V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const Place<ACCESS> at(i, tid, threads, a.width);
        xv[i] = at.load(x_row);
        if (r_row) rv[PLAIN ? 0 : i] = at.load(r_row);
        if (has_gain) gv[PLAIN ? 0 : i] = at.load(a.gain);
    }
    float h[V][8];
    Stats s = {0.0f, 0.0f};
    auto factor = [&](int i, float (&g)[8]) {
        if (!has_gain) return;
        unpack8(gv[PLAIN ? 0 : i], g);
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] += a.gain_add;
    };
    auto take = [&](int i) {                           // elements that do not exist are zeros
        float g[8];
        factor(i, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (NORM) s.sum = fmaf(h[i][j], h[i][j], s.sum);
            s.top = larger(s.top, has_gain ? h[i][j] * g[j] : h[i][j]);
        }
    };
#pragma unroll
    for (int i = 0; i < V; ++i) {
        unpack8(xv[i], h[i]);
        if (r_row) {
            float r[8];
            unpack8(rv[PLAIN ? 0 : i], r);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[i][j] += r[j];
        }
        if (a.h_out) Place<ACCESS>(i, tid, threads, a.width).store(a.h_out + (size_t)row * a.ldh, h[i]);
        take(i);
    }
    s = over_row<ALONE, NORM>(s, warps[0]);
    float r = 1.0f;
    if (NORM && a.normed) {
        float eps = a.eps;
        auto again = [&](float by, Stats* at) {                        // the statistics of h * by
            s = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < V; ++i) {
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] *= by;
                take(i);
            }
            s = over_row<ALONE, NORM>(s, at);
        };
        const bool far = !(s.sum < INFINITY) || !(fabsf(s.top) < INFINITY);          // (the same answer in every thread of the row)
        if (!(s.sum < INFINITY)) {
            again(0x1p-80f, warps[1]);
            eps = eps * 0x1p-80f * 0x1p-80f;
        }
        r = 1.0f / sqrtf(s.sum / (float)a.width + eps);
        if (far) {
            again(r, warps[2]);
            r = 1.0f;
        }
    }
    const float top = fabsf(s.top) * r;
    const float most = top < INFINITY ? fmaxf(top, kLeast) : NAN;     // a row with a value that is no number has no scale
    const float scale = most / kE4m3Max;
    if (a.out8 && tid == 0) a.scale8[row] = scale;
    const Quotient over(r, scale);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const Place<ACCESS> at(i, tid, threads, a.width);
        float g[8], y[8];
        factor(i, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) h[i][j] = has_gain ? h[i][j] * g[j] : h[i][j];
        if (a.out) {
#pragma unroll
            for (int j = 0; j < 8; j += 2) over.times(h[i][j], h[i][j + 1], y[j], y[j + 1]);
            at.store(a.out + (size_t)row * a.ldo, y);
        }
        if (a.out8) {
#pragma unroll
            for (int j = 0; j < 8; j += 2) over.of(h[i][j], h[i][j + 1]);
            at.store8(a.out8 + (size_t)row * a.ld8, h[i]);
        }
    }
}

template <int V, bool ALONE, Access ACCESS>
cudaError_t launch(const NormArgs& a, int rows_per_cta, int threads, cudaStream_t stream) {
    const dim3 grid((a.T_cap + rows_per_cta - 1) / rows_per_cta), block(threads);
    return a.residual || a.gain ? dcut_launch_pdl(rms_norm_kernel<V, ACCESS, ALONE, kFull>, grid, block, 0, stream, a)
           : a.normed           ? dcut_launch_pdl(rms_norm_kernel<V, ACCESS, ALONE, kBare>, grid, block, 0, stream, a)
                                : dcut_launch_pdl(rms_norm_kernel<V, ACCESS, ALONE, kRows>, grid, block, 0, stream, a);
}
template <int V, bool ALONE>
cudaError_t launch(const NormArgs& a, Access access, int rows_per_cta, int threads, cudaStream_t stream) {
    return access == kVector    ? launch<V, ALONE, kVector>(a, rows_per_cta, threads, stream)
           : access == kShifted ? launch<V, ALONE, kShifted>(a, rows_per_cta, threads, stream)
                                : launch<V, ALONE, kSingle>(a, rows_per_cta, threads, stream);
}

}  // namespace

dcut_status dcut_launch_rms_norm(dcut_ctx* ctx, const dcut_norm_args* n, const int* cu_q, int B, int T_cap, cudaStream_t stream) {
    NormArgs a;
    a.x = static_cast<const __nv_bfloat16*>(n->x);
    a.residual = static_cast<const __nv_bfloat16*>(n->residual);
    a.gain = static_cast<const __nv_bfloat16*>(n->gain);
    a.ldx = n->ldx, a.ldr = n->ldr, a.ldh = n->ldh, a.ldo = n->ldo, a.ld8 = n->ld8;
    a.h_out = static_cast<__nv_bfloat16*>(n->h_out);
    a.out = static_cast<__nv_bfloat16*>(n->out);
    a.out8 = static_cast<unsigned char*>(n->out8);
    a.scale8 = n->scale8;
    a.cu_q = cu_q, a.B = B, a.T_cap = T_cap, a.width = n->width, a.normed = n->normed != 0;
    a.eps = n->rms_eps, a.gain_add = n->gain_plus_one ? 1.0f : 0.0f;
    a.status = ctx->d_status;
    auto rows16 = [](const void* p, long long ld) { return !p || (!(reinterpret_cast<uintptr_t>(p) & 15) && ld % 8 == 0); };
    const bool in16 = rows16(a.x, a.ldx) && rows16(a.residual, a.ldr) && rows16(a.gain, 0) &&
                      !((reinterpret_cast<uintptr_t>(a.out8) | (uintptr_t)(a.out8 ? a.ld8 : 0)) & 7);
    const Access access = !in16 ? kSingle : rows16(a.h_out, a.ldh) && rows16(a.out, a.ldo) ? kVector : kShifted;
    const int slots = (a.width + 7) / 8;
    // Pieces of a thread, us on the device with 1 / 2 / 4 / 8 of them (norm with every output, and quantising):
    //                 16 rows                   quantising               8191 rows                  quantising
    //   2048 wide     2.2 / 2.5 / 3.4           1.7 / 1.8 / 2.2          28.5 / 26.4 / 27.0         14.9 / 11.9 / 11.3
    //   4096          2.4 / 2.7 / 3.4 / 5.6     1.9 / 1.9 / 2.2 / 3.1    55.0 / 52.8 / 49.9 / 55.3  29.5 / 22.4 / 19.6 / 22.0
    //   6144          - / 2.9 / 3.6 / 5.5       - / 2.0 / 2.3 / 3.1      - / 75.2 / 72.9 / 81.7     - / 33.2 / 28.9 / 33.1
    //   8192          - / 3.0 / 3.7 / 5.5       - / 2.0 / 2.3 / 3.2      - / 105 / 96.3 / 102       - / 44.7 / 39.8 / 40.7
    //   12288         - / - / 4.0 / 5.5         - / - / 2.5 / 3.2        - / - / 143 / 172          - / - / 57.0 / 65.3
    // (none: more than 512 threads).  Few rows want few pieces and many rows more of them; the rule goes by the width and lies between
    // (of the rows it could know T_cap alone, not the packed length).  Above 16384 only 8 pieces hold a row.
    const int per = slots <= 256 ? 1 : slots <= 768 ? 2 : slots <= 2048 ? 4 : 8;
    const int threads = ((slots + per - 1) / per + 31) & ~31;
    cudaError_t e = threads == 32 ? launch<1, false>(a, access, 4, 128, stream)
                    : per == 1    ? launch<1, true>(a, access, 1, threads, stream)
                    : per == 2    ? launch<2, true>(a, access, 1, threads, stream)
                    : per == 4    ? launch<4, true>(a, access, 1, threads, stream)
                                  : launch<8, true>(a, access, 1, threads, stream);
    return dcut_check_cuda(ctx, e, "launch rms_norm_kernel");
}
