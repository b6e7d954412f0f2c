// Head rows between a model's projection and the cache, in one pass: RMS norm of every query and key head,
// position rotation, and -- for keys and values -- the append to the paged pool.
//
// For a query or key row x (128 elements, fp32 arithmetic, one rounding at the end):
//   y = x * rsqrt(mean(x^2) + eps) * w                              (when a norm is set)
//   (z_a, z_b) = A (y_a cos t - y_b sin t, y_b cos t + y_a sin t)   for every pair j = (a, b) that rotates
// with t = position * inv_freq[j]; pair j is elements (j, j + pairs) or (2 j, 2 j + 1).  Value rows are only rounded.
//
// The angle is taken in turns, position * (inv_freq / 2 pi), in fp64: a position of a million loses 16 bits of an
// fp32 angle before the reduction.  What is left after subtracting the nearest whole turn fits fp32, and
// sincospif needs no further reduction.
//
// Bound by HBM (a row is read once and written once, 10 flops an element) or, for a few tokens, by launch
// latency.  A half-warp works on one row, 16 bytes of bf16 per lane; the partner elements of a rotation with
// pairs (j, j + pairs) are read a second time by their lane (an L1 hit) rather than shuffled.  A warp takes rows
// of one kind (queries, keys or values) of one token, so that the angles and the weights are computed once and
// held in registers as two factors per element: z = inv * (x * f + x_partner * g).
#include <cuda_fp16.h>

#include "internal.h"

namespace lzk {

namespace {

constexpr int kRowThreads = 256;
constexpr int kElems = 8;                          // elements of a row per lane

struct RowsParams {
    RowsArgs a;
    double turns[kMaxPairs];                       // inv_freq / (2 pi)
    int groups[3], per_warp[3];                    // per kind (q, k, v): row groups of a token, rows per group
    int tasks_per_token;
    long long tasks;
};

__device__ __forceinline__ void load8(const void* row, int dtype, int c, float (&x)[kElems]) {
    if (dtype == kTypeF32) {
        const float4* p = reinterpret_cast<const float4*>(row) + 2 * c;
        const float4 a = p[0], b = p[1];
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        return;
    }
    const uint4 v = reinterpret_cast<const uint4*>(row)[c];
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (dtype == kTypeBF16) {
            x[2 * i] = bf16_lo_as_float(w[i]);
            x[2 * i + 1] = bf16_hi_as_float(w[i]);
        } else {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
    }
}

__device__ __forceinline__ uint4 pack8_bf16(const float (&y)[kElems]) {
    return make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
}

__device__ __forceinline__ void store8(void* row, int dtype, int c, const float (&y)[kElems]) {
    if (dtype == kTypeF32) {
        float4* p = reinterpret_cast<float4*>(row) + 2 * c;
        p[0] = make_float4(y[0], y[1], y[2], y[3]);
        p[1] = make_float4(y[4], y[5], y[6], y[7]);
    } else if (dtype == kTypeBF16) {
        reinterpret_cast<uint4*>(row)[c] = pack8_bf16(y);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2 h = __floats2half2_rn(y[2 * i], y[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        reinterpret_cast<uint4*>(row)[c] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

__device__ __forceinline__ const uint8_t* row_at(const RowView& v, int l, int b, int i, int head) {
    return reinterpret_cast<const uint8_t*>(v.data) +
           (l * v.stride_layer + b * v.stride_batch + i * v.stride_token + head * v.stride_head) * (v.dtype == kTypeF32 ? 4 : 2);
}

__global__ void __launch_bounds__(kRowThreads) rows_kernel(const __grid_constant__ RowsParams p) {
    const RowsArgs& a = p.a;
    const int lane = threadIdx.x & 31, half = lane >> 4, c = lane & 15;
    const long long task = (long long)blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);
    if (task >= p.tasks) return;
    const long long tk = task / p.tasks_per_token;
    int grp = (int)(task - tk * p.tasks_per_token);
    int kind = 0;                                   // 0: queries, 1: keys, 2: values
    while (grp >= p.groups[kind]) grp -= p.groups[kind++];
    const int heads = kind == 0 ? a.q_heads : a.kv_heads;
    const int i = (int)(tk % a.n_tokens);
    const int lb = (int)(tk / a.n_tokens), l = lb / a.batch, b = lb % a.batch;
    const RowView& in = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
    const int head0 = grp * p.per_warp[kind];
    const int head_end = min(heads, head0 + p.per_warp[kind]);

    // where this lane's elements 8 c .. 8 c + 7 take part in the rotation
    const bool turns = kind < 2 && 8 * c < 2 * a.pairs;
    const int shift = turns && !a.interleaved ? (8 * c < a.pairs ? a.pairs / 8 : -(a.pairs / 8)) : 0;   // chunk of the partners
    float f[kElems], g[kElems];
#pragma unroll
    for (int e = 0; e < kElems; ++e) {
        f[e] = 1.f;
        g[e] = 0.f;
    }
    const float* w = kind == 0 ? a.q_weight : kind == 1 ? a.k_weight : nullptr;
    if (kind < 2 && a.pairs > 0) {
        const double pos = (double)(a.positions ? a.positions[(size_t)b * a.n_tokens + i] : (long long)a.first_position + i);
        // Every angle is needed by several lanes (both halves of the warp; both partners): each computes two.
        float cs[2], sn[2];
        const int j0 = a.interleaved ? 4 * c + 2 * half : 8 * (c % max(a.pairs / 8, 1)) + 4 * half + 2 * (shift < 0);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const double t = pos * p.turns[min(j0 + e, kMaxPairs - 1)];
            sincospif(2.f * (float)(t - rint(t)), &sn[e], &cs[e]);
            sn[e] *= a.amplitude;
            cs[e] *= a.amplitude;
        }
        if (a.interleaved) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float cv = __shfl_sync(0xffffffffu, cs[e & 1], (e >> 1) * 16 + c);
                const float sv = __shfl_sync(0xffffffffu, sn[e & 1], (e >> 1) * 16 + c);
                if (turns) {
                    f[2 * e] = f[2 * e + 1] = cv;
                    g[2 * e] = -sv;
                    g[2 * e + 1] = sv;
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < kElems; ++e) {
                const int k = e >> 1;               // computed by half k / 2, by the lower partner (k even) or the upper one
                const int src = turns ? (k >> 1) * 16 + c % (a.pairs / 8) + (k & 1) * (a.pairs / 8) : lane;
                const float cv = __shfl_sync(0xffffffffu, cs[e & 1], src);
                const float sv = __shfl_sync(0xffffffffu, sn[e & 1], src);
                if (turns) {
                    f[e] = cv;
                    g[e] = shift > 0 ? -sv : sv;
                }
            }
        }
    }
    if (w) {
        w += (size_t)l * kHeadDim;
#pragma unroll
        for (int e = 0; e < kElems; ++e) {
            f[e] *= w[8 * c + e];
            g[e] *= a.interleaved ? w[8 * c + (e ^ 1)] : w[8 * (c + shift) + e];
        }
    }

    for (int head = head0 + half; head < head_end; head += 2) {
        const uint32_t mask = head - half + 1 < head_end ? 0xffffffffu : 0x0000ffffu;     // an odd row at the end
        const uint8_t* row = row_at(in, l, b, i, head);
        float x[kElems], y[kElems];
        load8(row, in.dtype, c, x);
        if (a.interleaved || shift == 0) {
#pragma unroll
            for (int e = 0; e < kElems; ++e) y[e] = turns ? x[e ^ 1] : 0.f;
        } else {
            load8(row, in.dtype, c + shift, y);
        }
        float inv = 1.f;
        if (w) {
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < kElems; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
            for (int s = 1; s < 16; s <<= 1) ss += __shfl_xor_sync(mask, ss, s);
            inv = rsqrtf(ss * (1.f / kHeadDim) + a.eps);
        }
#pragma unroll
        for (int e = 0; e < kElems; ++e) x[e] = inv * fmaf(y[e], g[e], x[e] * f[e]);
        __syncwarp(mask);                           // in place: every lane has read its partner's elements
        if (kind == 0 || a.pool == nullptr) {
            const RowView& out = kind == 0 ? a.q_out : a.k_out;
            store8(const_cast<uint8_t*>(row_at(out, l, b, i, head)), out.dtype, c, x);
        } else {
            const size_t u = (size_t)lb * a.kv_heads + head;
            const int slot = a.slot + i, r = slot % kPageTokens;
            if (!in_bounds(slot >= 0 && slot < a.capacity, a.status)) continue;
            const int32_t pp = a.page_table[u * a.pages_per_unit + slot / kPageTokens];
            if (!in_bounds(pp >= 0 && pp < a.total_pages, a.status)) continue;
            uint8_t* dst = a.pool + (size_t)pp * kPageBytes + (kind == 1 ? 0 : kPageHalfBytes) + r * kRowBytes;
            *reinterpret_cast<uint4*>(dst + swz_chunk(c, r) * 16) = pack8_bf16(x);
            if (kind == 1 && c == 0) {              // a new token: active at its own step, MRI = 0
                const size_t s = u * a.capacity + slot;
                a.tsm[s] = make_int2(a.ts, 0);
                a.pos[s] = a.pos_first + i;
                a.pbar[s] = 0.f;
            }
        }
    }
}

}  // namespace

cudaError_t rows_launch(const RowsArgs& a, const double* inv_freq, int num_sms, cudaStream_t stream) {
    RowsParams p;
    p.a = a;
    for (int j = 0; j < kMaxPairs; ++j) p.turns[j] = j < a.pairs ? inv_freq[j] / 6.283185307179586476925 : 0.0;
    const int heads[3] = {a.q.data ? a.q_heads : 0, a.k.data ? a.kv_heads : 0, a.v.data ? a.kv_heads : 0};
    const long long tokens = (long long)a.layers * a.batch * a.n_tokens;
    p.tasks_per_token = 0;
    for (int k = 0; k < 3; ++k) {
        p.per_warp[k] = 2;
        p.groups[k] = (heads[k] + 1) / 2;
        p.tasks_per_token += p.groups[k];
    }
    p.tasks = tokens * p.tasks_per_token;
    const long long blocks = (p.tasks + kRowThreads / 32 - 1) / (kRowThreads / 32);
    if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
    rows_kernel<<<(unsigned)blocks, kRowThreads, 0, stream>>>(p);
    return cudaGetLastError();
}

}  // namespace lzk
