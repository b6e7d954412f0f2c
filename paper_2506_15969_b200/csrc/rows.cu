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
// latency.  At 256 bytes in and out per row an SM has 22 clocks for a row, so what decides is the number of
// instructions: a half-warp works on one row; each lane holds two groups of four elements chosen so that the partners of
// a rotation sit in the same lane (no exchange, nothing read twice); angles, weights and signs are folded into four
// factors per pair that a warp computes once for all the heads of a kind (queries, keys, values) it takes of a token,
//   z_a = (inv a) f_a + (inv b) g_a,  z_b = (inv b) f_b + (inv a) g_b,
// and the arithmetic runs two elements per instruction.
//
// Measured on B200 (copy bandwidth 6.54 TB/s): 32768 tokens of 40 + 8 bf16 heads 128 us, 6.3 TB/s; 131072 tokens of 8 key and
// 8 value heads into pages 183 us, 5.9 TB/s; one token 3.6 us.  Looking for rows whose squares overflow is 2 us of the 183 (a
// vote per stage; a vote per row 3).
#include <cuda_fp16.h>

#include <type_traits>

#include "internal.h"
#include "tensor.cuh"

namespace lzk {

namespace {

constexpr int kRowThreads = 128;
constexpr int kStages = 3;                         // of a warp's ring of rows in shared memory
constexpr int kStageBytes = 2048;                  // eight rows of 16-bit elements, four of 32-bit ones

struct RowsParams {
    RowsArgs a;
    double turns[kMaxPairs];                       // inv_freq / (2 pi)
    uint32_t groups[3], per_warp[3];               // per kind (q, k, v): row groups of a token, rows per group
    uint32_t joint;                                // one warp takes all rows of a token, kind after kind
    uint32_t tasks_per_token, row_tasks, tasks;    // warps for rows, then (paged) warps for 32 tokens' state words each
};

// Four elements as they come from memory, and as they go back.
template <int kType>
struct Quad {
    uint32_t w[kType == kTypeF32 ? 4 : 2];
    __device__ __forceinline__ void load(uint32_t smem) {
        if constexpr (kType == kTypeF32)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(smem) : "memory");
        else
            asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(smem) : "memory");
    }
    __device__ __forceinline__ void unpack(float (&x)[4]) const {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if constexpr (kType == kTypeF32) {
                x[2 * i] = __uint_as_float(w[2 * i]);
                x[2 * i + 1] = __uint_as_float(w[2 * i + 1]);
            } else if constexpr (kType == kTypeBF16) {
                x[2 * i] = bf16_lo_as_float(w[i]);
                x[2 * i + 1] = bf16_hi_as_float(w[i]);
            } else {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
                x[2 * i] = f.x;
                x[2 * i + 1] = f.y;
            }
        }
    }
};

template <int kType>
__device__ __forceinline__ void store4(uint8_t* p, const float (&x)[4]) {
    if constexpr (kType == kTypeF32) {
        *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    } else if constexpr (kType == kTypeBF16) {
        *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
    } else {
        const __half2 h0 = __floats2half2_rn(x[0], x[1]), h1 = __floats2half2_rn(x[2], x[3]);
        *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&h0), *reinterpret_cast<const uint32_t*>(&h1));
    }
}

// Where a warp's rows come from and go to: heads one after the other, this lane's two groups of four elements.
struct WarpRows {
    int heads;
    int src_a, src_b;                               // bytes of the groups in a row of the input
    uint8_t* dst;                                   // first group of the first head
    long long dst_step;
    int dst_b;                                      // bytes from the first group to the second
    int32_t page;                                   // kPaged: lane h's is head h's; and the byte offsets in a page
    uint32_t page_a, page_b;
};

__device__ __forceinline__ void copy16(uint32_t smem, const uint8_t* src, bool on) {     // zeros where `on` is false
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem), "l"(__cvta_generic_to_global(src)), "r"(on ? 16 : 0) : "memory");
}

struct Factors {
    uint64_t fa[2], ga[2], fb[2], gb[2];           // two fp32 each
};

// The rows of a warp go through a ring of asynchronous copies: what limits a plain loop is the latency of its loads, since a
// warp's factors leave registers for few rows in flight.  A row is copied before it is written (in place).
template <int kIn>
struct RowRing {
    static constexpr int kRowIn = kHeadDim * (kIn == kTypeF32 ? 4 : 2);
    static constexpr int kRows = kStageBytes / kRowIn;                     // per stage
    static constexpr int kChunks = kRowIn / 16;
    uint32_t base, put, get;
    const uint8_t* src;                             // this lane's first 16-byte chunk of the next stage
    long long step;                                 // bytes from one of the lane's chunks to the next
    int to_fetch;                                   // rows of the segment not fetched yet

    __device__ __forceinline__ void init(uint32_t ring) {
        const int lane = threadIdx.x & 31;
        base = ring;
        put = ring + lane * 16;
        get = ring + (lane >> 4) * kRowIn;
        to_fetch = 0;
    }
    // The next rows to fetch: one kind's heads.
    __device__ __forceinline__ void segment(const uint8_t* first, long long row_step, int rows) {
        const int lane = threadIdx.x & 31;
        src = first + (lane % kChunks) * 16 + lane / kChunks * row_step;
        step = 32 / kChunks * row_step;
        to_fetch = rows;
    }
    // One stage of the segment (nothing when it is exhausted).
    __device__ __forceinline__ void fetch() {
        if (to_fetch > 0) {
            const int row = (threadIdx.x & 31) / kChunks;
#pragma unroll
            for (int i = 0; i < kStageBytes / 512; ++i) {
                copy16(put + 512 * i, src, row + i * (32 / kChunks) < to_fetch);
                src += step;
            }
            to_fetch -= kRows;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        put = put + kStageBytes < base + kStages * kStageBytes ? put + kStageBytes : base + (threadIdx.x & 31) * 16;
    }
    __device__ __forceinline__ void wait() {        // the oldest stage has arrived, and the one before it is read
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
        __syncwarp();
    }
    __device__ __forceinline__ void next() {
        get = get + kStageBytes < base + kStages * kStageBytes ? get + kStageBytes : get - (kStages - 1) * kStageBytes;
    }
};

// Over the 16 lanes of a row.
__device__ __forceinline__ float sum_of_squares(const uint64_t (&va)[2], const uint64_t (&vb)[2]) {
    float s0, s1;
    unpack2(add2(fma2(va[0], va[0], mul2(va[1], va[1])), fma2(vb[0], vb[0], mul2(vb[1], vb[1]))), s0, s1);
    float ss = s0 + s1;
#pragma unroll
    for (int s = 1; s < 16; s <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, s);
    return ss;
}

// Queries or keys.  `refill` fetches the stage that follows those in flight.
template <int kIn, int kOut, bool kInterleaved, bool kPaged, class Refill>
__device__ __forceinline__ void turn_rows(const RowsArgs& a, const WarpRows& r, bool norm, bool turns, const Factors& f, RowRing<kIn>& ring,
                                          Refill refill) {
    constexpr int kRowIn = RowRing<kIn>::kRowIn, kRows = RowRing<kIn>::kRows, kBatch = kRows / 2;      // rows per half-warp
    const int half = (threadIdx.x >> 4) & 1;
    uint8_t* dst = kPaged ? nullptr : r.dst + half * r.dst_step;
    const float mean = 1.f / kHeadDim;
    // Row k of this half-warp's in the stage; its sum of squares.  kLarge: squares of elements from 1.6e18 on do not fit fp32, but
    // those of a row times 2^-70 do, and its norm is 2^-70 of the row's.
    auto turn_row = [&](int k, int left, uint8_t* to, auto large) {
        constexpr bool kLarge = decltype(large)::value;
        Quad<kIn> qa, qb;
        qa.load(ring.get + 2 * k * kRowIn + r.src_a);
        qb.load(ring.get + 2 * k * kRowIn + r.src_b);
        const int32_t pp = kPaged ? __shfl_sync(0xffffffffu, r.page, r.heads - left + 2 * k) : 0;
        float xa[4], xb[4];
        qa.unpack(xa);
        qb.unpack(xb);
        uint64_t va[2], vb[2];                      // the pairs' first elements, their second ones
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float* x = i ? xb : xa;
            va[i] = kInterleaved ? pack2(x[0], x[2]) : pack2(xa[2 * i], xa[2 * i + 1]);
            vb[i] = kInterleaved ? pack2(x[1], x[3]) : pack2(xb[2 * i], xb[2 * i + 1]);
        }
        float inv = 1.f, ss = 0.f;
        if (norm) {
            ss = sum_of_squares(va, vb);
            float eps = a.eps;
            if (kLarge) {
                const float scale = ss == INFINITY ? 0x1p-70f : 1.f;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    va[i] = mul2(va[i], pack2(scale, scale));
                    vb[i] = mul2(vb[i], pack2(scale, scale));
                }
                ss = sum_of_squares(va, vb);
                eps = eps * scale * scale;
            }
            inv = rsqrtf(fmaf(ss, mean, eps));
        }
        const uint64_t inv2 = pack2(inv, inv);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint64_t ya = mul2(va[i], inv2), yb = mul2(vb[i], inv2);
            uint64_t ua = mul2(ya, f.fa[i]), ub = mul2(yb, f.fb[i]);
            if (turns) {                            // (elements that stay must not meet others: 0 * inf)
                ua = fma2(yb, f.ga[i], ua);
                ub = fma2(ya, f.gb[i], ub);
            }
            float z0, z1, z2, z3;
            unpack2(ua, z0, z1);
            unpack2(ub, z2, z3);
            if constexpr (kInterleaved) {
                float* x = i ? xb : xa;
                x[0] = z0; x[1] = z2; x[2] = z1; x[3] = z3;
            } else {
                xa[2 * i] = z0; xa[2 * i + 1] = z1;
                xb[2 * i] = z2; xb[2 * i + 1] = z3;
            }
        }
        if (left > 2 * k) {
            if constexpr (!kPaged) {
                store4<kOut>(to, xa);
                store4<kOut>(to + r.dst_b, xb);
            } else if (in_bounds(pp >= 0 && pp < a.total_pages, a.status)) {
                uint8_t* page = a.pool + (size_t)pp * kPageBytes;
                store4<kTypeBF16>(page + r.page_a, xa);
                store4<kTypeBF16>(page + r.page_b, xb);
            }
        }
        return ss;
    };
    for (int left = r.heads - half; left + half > 0; left -= kRows) {
        ring.wait();
        refill();
        float top = 0.f;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            top = fmaxf(top, turn_row(k, left, dst, std::false_type{}));
            if constexpr (!kPaged) dst += 2 * r.dst_step;
        }
        if (norm && __any_sync(0xffffffffu, top == INFINITY)) {      // the stage once more (a branch per row would keep rows from overlapping)
#pragma unroll 1
            for (int k = 0; k < kBatch; ++k) turn_row(k, left, kPaged ? nullptr : dst + 2 * (k - kBatch) * r.dst_step, std::true_type{});
        }
        ring.next();
    }
}

// Values: 16 bytes of bf16 per lane, bits as they are or rounded.  `at`: this lane's byte offset in a page.
template <int kIn, class Refill>
__device__ __forceinline__ void copy_rows(const RowsArgs& a, int heads, int32_t page_of, uint32_t at, RowRing<kIn>& ring, Refill refill) {
    constexpr int kRowIn = RowRing<kIn>::kRowIn, kRows = RowRing<kIn>::kRows, kBatch = kRows / 2;
    const int half = (threadIdx.x >> 4) & 1, c = threadIdx.x & 15;
    for (int left = heads - half; left + half > 0; left -= kRows) {
        ring.wait();
        refill();
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            uint4 v;
            const uint32_t from = ring.get + 2 * k * kRowIn + c * (kRowIn / 16);
            if constexpr (kIn == kTypeBF16) {
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(from) : "memory");
            } else {
                Quad<kIn> q0, q1;
                q0.load(from);
                q1.load(from + kRowIn / 32);
                float x[4], y[4];
                q0.unpack(x);
                q1.unpack(y);
                v = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
            }
            const int32_t pp = __shfl_sync(0xffffffffu, page_of, heads - left + 2 * k);
            if (left > 2 * k && in_bounds(pp >= 0 && pp < a.total_pages, a.status))
                *reinterpret_cast<uint4*>(a.pool + (size_t)pp * kPageBytes + at) = v;
        }
        ring.next();
    }
}

// One input type and one type of the output views per launch; keys and values go to the pages when there is a pool.
template <int kIn, int kOut, bool kInterleaved>
__global__ void __launch_bounds__(kRowThreads, 6) rows_kernel(const __grid_constant__ RowsParams p) {
    __shared__ __align__(16) uint8_t rings[kRowThreads / 32][kStages * kStageBytes];
    const RowsArgs& a = p.a;
    const int lane = threadIdx.x & 31, half = lane >> 4, c = lane & 15;
    // (indexed by the lane, a parameter is read one address at a time)
    __shared__ double turns_s[kMaxPairs];
    if (a.pairs > 0) {
        if (threadIdx.x < kMaxPairs) turns_s[threadIdx.x] = p.turns[threadIdx.x];
        __syncthreads();
    }
    const uint32_t task = blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);
    if (task >= p.tasks) return;
    if (task >= p.row_tasks) {
        // state words of 32 new tokens, unit by unit: active at their own step, MRI = 0 (Section 4)
        const uint32_t at = (task - p.row_tasks) * 32 + lane, u = at / (uint32_t)a.n_tokens;
        const int i = (int)(at - u * a.n_tokens);
        if (u >= (uint32_t)(a.layers * a.batch * a.kv_heads)) return;
        if (!in_bounds(a.slot + i >= 0 && a.slot + i < a.capacity, a.status)) return;
        const size_t s = (size_t)u * a.capacity + a.slot + i;
        a.tsm[s] = make_int2(a.ts, 0);
        a.pos[s] = a.pos_first + i;
        a.pbar[s] = 0.f;
        return;
    }
    const uint32_t tk = task / p.tasks_per_token;
    uint32_t grp = task - tk * p.tasks_per_token;
    int kind = 0;                                   // 0: queries, 1: keys, 2: values
    if (!p.joint)
        while (grp >= p.groups[kind]) grp -= p.groups[kind++];
    int fetch_kind = kind;
    if (p.joint) kind = fetch_kind = a.q.data ? 0 : 1;
    const int last_kind = !p.joint ? kind : a.v.data ? 2 : a.k.data ? 1 : 0;
    const int lb = (int)(tk / (uint32_t)a.n_tokens), i = (int)(tk - (uint32_t)lb * a.n_tokens);
    const int l = lb / a.batch, b = lb - l * a.batch;
    // Groups of four elements: with pairs (j, j + pairs) group c of the first `pairs` elements and its partners, then the
    // groups that do not rotate two by two; with pairs (2 j, 2 j + 1) two neighbouring groups.
    const int low = kInterleaved ? 0 : a.pairs / 4;
    const int qa = c < low ? c : 2 * low + 2 * (c - low), qb = c < low ? c + low : qa + 1;
    const bool turns = kInterleaved ? 4 * c < a.pairs : c < low;

    // The copies of the first rows run while the angles are computed, and go on from kind to kind without a break.
    RowRing<kIn> ring;
    auto heads_of = [&](int k) { return min((k == 0 ? a.q_heads : a.kv_heads) - (int)(grp * p.per_warp[k]), (int)p.per_warp[k]); };
    auto refill = [&]() {
        if (ring.to_fetch <= 0 && fetch_kind <= last_kind) {
            const RowView& in = fetch_kind == 0 ? a.q : fetch_kind == 1 ? a.k : a.v;
            const long long bytes = kIn == kTypeF32 ? 4 : 2;
            ring.segment(reinterpret_cast<const uint8_t*>(in.data) +
                             (l * in.stride_layer + b * in.stride_batch + i * in.stride_token + (int)(grp * p.per_warp[fetch_kind]) * in.stride_head) * bytes,
                         in.stride_head * bytes, heads_of(fetch_kind));
            ++fetch_kind;
        }
        ring.fetch();
    };
    ring.init(smem_u32(rings[threadIdx.x >> 5]));
#pragma unroll 1
    for (int st = 0; st < kStages - 1; ++st) refill();
    // keys and values: where the token's slot is in the pages of its heads (lane h: head h)
    int32_t page = 0;
    uint32_t slot_row = 0;
    if (last_kind > 0 && a.pool != nullptr) {
        const int slot = a.slot + i, head0 = (int)(grp * p.per_warp[last_kind]);
        if (!in_bounds(slot >= 0 && slot < a.capacity, a.status)) return;
        slot_row = slot % kPageTokens;
        if (lane < heads_of(last_kind)) page = a.page_table[((size_t)lb * a.kv_heads + head0 + lane) * a.pages_per_unit + slot / kPageTokens];
    }
    float cv[4] = {1.f, 1.f, 1.f, 1.f}, sv[4] = {};
    if (kind < 2 && a.pairs > 0) {
        // this lane's pairs are 4 c .. 4 c + 3; the two halves of the warp need the same angles and compute two each
        const double pos = (double)(a.positions ? a.positions[(size_t)b * a.n_tokens + i] : (long long)a.first_position + i);
        float cs[2], sn[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const double t = pos * turns_s[4 * c + 2 * half + e];
            const float turn = (float)(t - rint(t));                   // -1/2 .. 1/2
            // For 16-bit results the hardware's sine and cosine will do: 2^-20.5 off at most, 2^-9 of a rounding step.
            if (kOut == kTypeF32)
                sincospif(2.f * turn, &sn[e], &cs[e]);
            else
                __sincosf(6.283185307f * turn, &sn[e], &cs[e]);
            cs[e] *= a.amplitude;
            sn[e] *= a.amplitude;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = __shfl_sync(0xffffffffu, cs[e & 1], (e >> 1) * 16 + c), y = __shfl_sync(0xffffffffu, sn[e & 1], (e >> 1) * 16 + c);
            cv[e] = turns ? x : 1.f;
            sv[e] = turns ? y : 0.f;
        }
    }

    for (; kind <= last_kind; ++kind) {
        if (kind == 2) {
            copy_rows<kIn>(a, heads_of(2), page, kPageHalfBytes + slot_row * kRowBytes + swz_chunk(c, (int)slot_row) * 16, ring, refill);
            break;
        }
        constexpr int kInBytes = kIn == kTypeF32 ? 4 : 2, kOutBytes = kOut == kTypeF32 ? 4 : 2;
        const bool paged = kind > 0 && a.pool != nullptr;
        WarpRows r;
        r.heads = heads_of(kind);
        r.src_a = 4 * qa * kInBytes;
        r.src_b = 4 * qb * kInBytes;
        if (!paged) {
            const RowView& out = kind == 0 ? a.q_out : a.k_out;
            r.dst_step = out.stride_head * kOutBytes;
            r.dst = reinterpret_cast<uint8_t*>(const_cast<void*>(out.data)) +
                    (l * out.stride_layer + b * out.stride_batch + i * out.stride_token + (int)(grp * p.per_warp[kind]) * out.stride_head + 4 * qa) * kOutBytes;
            r.dst_b = 4 * (qb - qa) * kOutBytes;
        } else {
            r.page = page;
            r.page_a = slot_row * kRowBytes + swz_chunk(qa >> 1, (int)slot_row) * 16 + (qa & 1) * 8;
            r.page_b = slot_row * kRowBytes + swz_chunk(qb >> 1, (int)slot_row) * 16 + (qb & 1) * 8;
        }
        float wa[4] = {1.f, 1.f, 1.f, 1.f}, wb[4] = {1.f, 1.f, 1.f, 1.f};
        const float* w = kind == 0 ? a.q_weight : a.k_weight;
        if (w) {
            const float4 va = reinterpret_cast<const float4*>(w + (size_t)l * kHeadDim)[qa];
            const float4 vb = reinterpret_cast<const float4*>(w + (size_t)l * kHeadDim)[qb];
            const float x[8] = {va.x, va.y, va.z, va.w, vb.x, vb.y, vb.z, vb.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                wa[e] = x[kInterleaved ? 2 * e : e];
                wb[e] = x[kInterleaved ? 2 * e + 1 : 4 + e];
            }
        }
        Factors f;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            f.fa[e] = pack2(wa[2 * e] * cv[2 * e], wa[2 * e + 1] * cv[2 * e + 1]);
            f.gb[e] = pack2(wa[2 * e] * sv[2 * e], wa[2 * e + 1] * sv[2 * e + 1]);
            f.fb[e] = pack2(wb[2 * e] * cv[2 * e], wb[2 * e + 1] * cv[2 * e + 1]);
            f.ga[e] = pack2(-wb[2 * e] * sv[2 * e], -wb[2 * e + 1] * sv[2 * e + 1]);
        }
        if (paged)
            turn_rows<kIn, kOut, kInterleaved, true>(a, r, w != nullptr, turns, f, ring, refill);
        else
            turn_rows<kIn, kOut, kInterleaved, false>(a, r, w != nullptr, turns, f, ring, refill);
    }
}

template <int kIn, int kOut>
void launch(const RowsParams& p, uint32_t blocks, cudaStream_t stream) {
    if (p.a.interleaved)
        rows_kernel<kIn, kOut, true><<<blocks, kRowThreads, 0, stream>>>(p);
    else
        rows_kernel<kIn, kOut, false><<<blocks, kRowThreads, 0, stream>>>(p);
}

template <int kIn>
void launch(const RowsParams& p, int out, uint32_t blocks, cudaStream_t stream) {
    if (out == kTypeF32)
        launch<kIn, kTypeF32>(p, blocks, stream);
    else if (out == kTypeF16)
        launch<kIn, kTypeF16>(p, blocks, stream);
    else
        launch<kIn, kTypeBF16>(p, blocks, stream);
}

}  // namespace

cudaError_t rows_launch(const RowsArgs& a, const double* turns, int num_sms, cudaStream_t stream) {
    RowsParams p;
    p.a = a;
    for (int j = 0; j < kMaxPairs; ++j) p.turns[j] = turns[j];
    const int heads[3] = {a.q.data ? a.q_heads : 0, a.k.data ? a.kv_heads : 0, a.v.data ? a.kv_heads : 0};
    const long long tokens = (long long)a.layers * a.batch * a.n_tokens;
    // Rows per warp: all rows of a token, so that its angles and pages are found once (a warp knows the pages of 32 heads); or, as
    // long as that leaves SMs without 8 warps, fewer and fewer heads of a kind, two at least (a warp takes two rows at a
    // time).  Measured at 1536 tokens of 40 + 8 heads, one warp each against six: 10.8 and 14.8 us; at 512 tokens of 28 + 4 heads
    // 7.2 us in one warp each, 5.7 us in three.
    const long long enough = 8ll * num_sms;
    p.joint = a.kv_heads <= 32 && tokens >= enough;
    p.tasks_per_token = 1;
    for (int k = 0; k < 3; ++k) {
        p.per_warp[k] = heads[k];
        p.groups[k] = 0;
    }
    for (int most = 32; !p.joint; most /= 2) {
        p.tasks_per_token = 0;
        for (int k = 0; k < 3; ++k) {
            p.per_warp[k] = most;
            p.groups[k] = (heads[k] + most - 1) / most;
            p.tasks_per_token += p.groups[k];
        }
        if (most == 2 || tokens * p.tasks_per_token >= enough) break;
    }
    const long long row_tasks = tokens * p.tasks_per_token;
    const long long state_tasks = a.pool ? (tokens * a.kv_heads + 31) / 32 : 0;
    if (row_tasks + state_tasks > 0x7fffffffll) return cudaErrorInvalidValue;
    p.row_tasks = (uint32_t)row_tasks;
    p.tasks = (uint32_t)(row_tasks + state_tasks);
    const uint32_t blocks = (p.tasks + kRowThreads / 32 - 1) / (kRowThreads / 32);
    const int in = a.q.data ? a.q.dtype : a.k.dtype, out = a.q_out.data ? a.q_out.dtype : a.k_out.dtype;
    if (in == kTypeF32)
        launch<kTypeF32>(p, out, blocks, stream);
    else if (in == kTypeF16)
        launch<kTypeF16>(p, out, blocks, stream);
    else
        launch<kTypeBF16>(p, out, blocks, stream);
    return cudaGetLastError();
}

}  // namespace lzk
