// dcut_rope_append: rotates the new tokens' query and key heads and appends keys and values to the paged cache.
//
//   n = x / sqrt(mean(x^2) + eps) * gain                              (per head, optional)
//   y_a = n_a cos - n_b sin,  y_b = n_b cos + n_a sin                 angle = position * inv_freq[e],  e = 0 .. R/2 - 1
//   (a, b) = (e, e + R/2) (rotate-half) or (2e, 2e + 1) (interleaved);  elements from R on are passed on
//   K and V go to page block_table[request][s / 16], slot s % 16,  s = position - prefix length of the request's group
//
// Every byte is read once and written once, so the kernel is bound by HBM when there are thousands of tokens and by its
// chain of dependent loads (token -> request -> page) when there are few.  One CTA per token: the rotation of a token is
// the same for all its heads, so the CTA computes R/2 (cos, sin) pairs once, into shared memory.  A thread's unit is 16
// elements of one head, as the two 16-byte vectors that rotate into each other; its first four units are requested before
// the token's place is known (the loads need only the token's number), so the page look-up and the angles hide behind them.
// 8191 tokens of 64 query and 8 key heads of 128 (335 MB): 63 us, 5.3 TB/s.  Four early units on 64 registers move most:
// with two 72 us, with three 65, with six (110 registers) 77; CTAs that walk several tokens, the next one's place looked
// up ahead, 84-118 us (a barrier per token, and registers for two tokens).
// The angle is formed in 64 bits as a fraction of a turn: at position 131072 an fp32 product is off by up to 0.008 rad.
#include <cuda_bf16.h>

#include "dcut_internal.h"

namespace {

constexpr int kMaxThreads = 512;
constexpr int kEarly = 4;            // units per thread that are loaded before the token's page is known

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ void unpack8(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = bf_lo(w[j]);
        x[2 * j + 1] = bf_hi(w[j]);
    }
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
    return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}

// A unit of a token: head `h` (queries, then keys, then values) and the element offsets of its two vectors.
struct Unit {
    int h, lo, hi, pair;      // pair: index of the first of its 8 (cos, sin) pairs, -1 where nothing rotates
};
template <int DH>
__device__ __forceinline__ Unit unit_of(int u, int n_rotated_heads, int R, int interleaved) {
    constexpr int kPer = DH / 16;
    Unit x;
    x.h = u / kPer;
    const int c = u - x.h * kPer;
    if (x.h < n_rotated_heads && 16 * c < R) {
        x.pair = 8 * c;
        x.lo = interleaved ? 16 * c : 8 * c;
        x.hi = interleaved ? 16 * c + 8 : 8 * c + (R >> 1);
    } else {
        x.pair = -1;
        x.lo = 16 * c;
        x.hi = 16 * c + 8;
    }
    return x;
}

template <int DH>
__global__ void __launch_bounds__(kMaxThreads, 2) rope_append_heads_kernel(DcutRopeArgs a) {
    constexpr int kPer = DH / 16;
    __shared__ float cos_s[DH / 2], sin_s[DH / 2];
    __shared__ int prefix_s, covers_s;
    dcut_pdl_wait();
    dcut_pdl_launch_dependents();
    const int tok = blockIdx.x, tid = threadIdx.x;
    const int req = a.tok_req[tok], pos = a.tok_pos[tok];     // together with cu_q: one trip to memory
    const int T = a.cu_q ? a.cu_q[a.B] : a.T_cap;
    if (T > a.T_cap && tok == 0 && tid == 0) atomicExch(a.status, DCUT_DEV_BAD_ROWS);
    if (tok >= T || req < 0) return;                          // behind the last token, or padding
    const int Hq = a.q ? a.n_q_heads : 0, Hr = Hq + a.n_kv_heads, units = (Hr + a.n_kv_heads) * kPer;

    auto source = [&](const Unit& x) -> const __nv_bfloat16* {
        if (x.h < Hq) return a.q + tok * a.q_token_stride + x.h * a.q_head_stride;
        if (x.h < Hr) return a.k + tok * a.k_token_stride + (x.h - Hq) * a.k_head_stride;
        return a.v + tok * a.v_token_stride + (x.h - Hr) * a.v_head_stride;
    };
    uint4 early[kEarly][2];
#pragma unroll
    for (int i = 0; i < kEarly; ++i) {
        const int u = tid + i * blockDim.x;
        if (u < units) {
            const Unit x = unit_of<DH>(u, Hr, a.rotary_dim, a.interleaved);
            const __nv_bfloat16* src = source(x);
            early[i][0] = *reinterpret_cast<const uint4*>(src + x.lo);
            early[i][1] = *reinterpret_cast<const uint4*>(src + x.hi);
        }
    }
    int prefix = 0;
    if (a.n_groups) {
        if (tid == 0) covers_s = 0;
        __syncthreads();
        for (int g = tid; g < a.n_groups; g += blockDim.x) {  // the request's group: one, where cu_group is as it should be
            const int len = a.prefix_lens[g];
            if (a.cu_group[g] <= req && req < a.cu_group[g + 1]) {
                atomicAdd(&covers_s, 1);
                prefix_s = len;
            }
        }
        __syncthreads();
        prefix = covers_s == 1 ? prefix_s : -1;
    }
    const long long slot = (long long)pos - prefix;
    if (req >= a.B || pos < 0 || prefix < 0 || slot < 0 || slot / 16 >= a.block_table_stride) {
        if (tid == 0) atomicExch(a.status, DCUT_DEV_BAD_APPEND);
        return;
    }
    const int page = a.block_table[(size_t)req * a.block_table_stride + slot / 16];
    for (int e = tid; e < a.rotary_dim >> 1; e += blockDim.x) {
        const double turns = (double)pos * a.inv_freq[e] * 0.15915494309189535;    // 1 / (2 pi)
        sincospif((float)(2.0 * (turns - rint(turns))), &sin_s[e], &cos_s[e]);
    }
    __syncthreads();
    if (page < 0 || page >= a.num_pages) {
        if (tid == 0) atomicExch(a.status, DCUT_DEV_BAD_PAGE);
        return;
    }
    const size_t cache_row = (size_t)page * a.n_kv_heads * 16 + (slot & 15);      // + 16 per head

    auto finish = [&](int u, const uint4& v0, const uint4& v1) {
        // (called by whole warps; lanes past the last unit take part in the shuffles only)
        const bool live = u < units;
        const Unit x = unit_of<DH>(live ? u : units - 1, Hr, a.rotary_dim, a.interleaved);
        __nv_bfloat16* dst = x.h < Hq   ? a.q_out + ((size_t)tok * a.n_q_heads + x.h) * DH
                             : x.h < Hr ? a.k_cache + (cache_row + (size_t)(x.h - Hq) * 16) * DH
                                        : a.v_cache + (cache_row + (size_t)(x.h - Hr) * 16) * DH;
        const __nv_bfloat16* gain = x.h < Hq ? a.q_gain : x.h < Hr ? a.k_gain : nullptr;
        uint4 r0 = v0, r1 = v1;
        float p[8], q[8];
        unpack8(v0, p);
        unpack8(v1, q);
        if (a.q_gain || a.k_gain) {
            float ss = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) ss += p[j] * p[j] + q[j] * q[j];
#pragma unroll
            for (int o = 1; o < kPer; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);   // a head's units are neighbouring lanes
            if (gain) {
                const float inv = 1.0f / sqrtf(ss / (float)DH + a.rms_eps);
                float g0[8], g1[8];
                unpack8(*reinterpret_cast<const uint4*>(gain + x.lo), g0);
                unpack8(*reinterpret_cast<const uint4*>(gain + x.hi), g1);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    p[j] *= inv * g0[j];
                    q[j] *= inv * g1[j];
                }
            }
        }
        if (x.pair >= 0) {
            if (a.interleaved) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float c0 = cos_s[x.pair + j], s0 = sin_s[x.pair + j], c1 = cos_s[x.pair + 4 + j], s1 = sin_s[x.pair + 4 + j];
                    const float p0 = p[2 * j], p1 = p[2 * j + 1], q0 = q[2 * j], q1 = q[2 * j + 1];
                    p[2 * j] = p0 * c0 - p1 * s0;
                    p[2 * j + 1] = p1 * c0 + p0 * s0;
                    q[2 * j] = q0 * c1 - q1 * s1;
                    q[2 * j + 1] = q1 * c1 + q0 * s1;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float c0 = cos_s[x.pair + j], s0 = sin_s[x.pair + j], p0 = p[j], q0 = q[j];
                    p[j] = p0 * c0 - q0 * s0;
                    q[j] = q0 * c0 + p0 * s0;
                }
            }
        }
        if (x.pair >= 0 || gain) {                            // what neither turns nor is scaled keeps its bits (a NaN's too)
            r0 = pack8(p);
            r1 = pack8(q);
        }
        if (live) {
            *reinterpret_cast<uint4*>(dst + x.lo) = r0;
            *reinterpret_cast<uint4*>(dst + x.hi) = r1;
        }
    };
#pragma unroll
    for (int i = 0; i < kEarly; ++i) {
        const int u = tid + i * blockDim.x;
        if (u - (tid & 31) < units) finish(u, early[i][0], early[i][1]);
    }
    for (int u = tid + kEarly * blockDim.x; u - (tid & 31) < units; u += blockDim.x) {
        const Unit x = unit_of<DH>(u < units ? u : units - 1, Hr, a.rotary_dim, a.interleaved);
        const __nv_bfloat16* src = source(x);
        finish(u, *reinterpret_cast<const uint4*>(src + x.lo), *reinterpret_cast<const uint4*>(src + x.hi));
    }
}

}  // namespace

dcut_status dcut_launch_rope_append(dcut_ctx* ctx, const DcutRopeArgs& a, int T_cap, cudaStream_t stream) {
    const int units = ((a.q ? a.n_q_heads : 0) + 2 * a.n_kv_heads) * (ctx->lim.head_dim / 16);
    int threads = ((units + kEarly - 1) / kEarly + 31) & ~31;  // every unit of a token early, where the heads allow it
    if (threads > kMaxThreads) threads = kMaxThreads;
    if (threads < 64) threads = 64;
    auto* kernel = ctx->lim.head_dim == 128 ? rope_append_heads_kernel<128> : rope_append_heads_kernel<64>;
    return dcut_check_cuda(ctx, dcut_launch_pdl(kernel, dim3(T_cap), dim3(threads), 0, stream, a), "launch rope_append_heads_kernel");
}
