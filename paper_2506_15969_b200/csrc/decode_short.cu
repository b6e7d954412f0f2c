// Decode attention over short own caches behind a shared prefix: a warp per cache unit.
//
// Same mathematics as decode.cu (Appendix A, Eq. (attn), over the prefix's tokens and the own ones; pbar and Eq. (1) for the own
// ones), for units of at most 384 own tokens -- sequences that have just begun to answer.  Such a unit is a chain of short
// dependent steps: a block of nine warps on it spends its time in barriers and merges (896 units take 33 us whether they hold
// 1 token or 64).  Here every warp walks units of its own: it fetches its tiles of 16 tokens (4 KiB of K, 4 KiB of V) itself
// through a ring, keeps all heads' O^T in registers, adds the prefix's partial sums to it in the same layout, and
// meets no other warp between the start and the end of the launch.  Eight units per SM are in flight.  Queries and partial
// sums come through shared memory as whole rows: 165 registers; read in fragment layout from global memory 231.
//
// Bound by HBM for many units (512 bytes a token); for few by the latency of one unit.  Measured on B200, both launches behind a
// prefix of 64 tokens, 16 query and 4 KV heads, caches in turn that L2 does not hold together; a warp per unit / a block per unit, us:
//   own tokens       64            128           256           384
//    448 units   22.7 / 26.8   25.0 / 27.0
//    608 units   22.7 / 28.9   25.9 / 30.0   32.9 / 35.0   39.7 / 40.9
//   1184 units   24.6 / 39.1   28.8 / 41.1   41.0 / 51.1   53.3 / 59.4
//   1200 units   24.8 / 39.1   29.5 / 41.2   45.2 / 50.7   62.4 / 61.4
//   1500 units   28.8 / 44.4   36.5 / 46.8   54.3 / 57.6   72.2 / 71.9
//   1800 units   28.9 / 49.4   36.9 / 51.6   55.5 / 65.7   74.1 / 81.3
//   2368 units   30.9 / 59.6   41.1 / 62.8   64.2 / 80.1   86.5 / 99.3
//   2400 units   31.3 / 59.8   41.6 / 62.6   68.6 / 80.2   97.7 / 101
//   3584 units   39.1 / 80.0   55.2 / 84.2   90.2 / 110     131 / 139
//   4096 units   43.1 / 88.6   62.6 / 94.3    103 / 124     143 / 156
// The walk is fixed, 1184 warps: just beyond a whole round (1200 to 1500 units, 2400) its last one is nearly empty, and with 384 tokens the
// two are level there.  With 8 KV heads: 448 units 30.9 / 28.9 at 256 tokens and 37.1 / 33.0 at 384, 3584 units 173 / 172 at 512;
// 320 units level at 64 tokens (20.4 / 20.8), the block ahead at 128 (22.9 / 20.8).
// Hence: at most 384 tokens, three units per SM up to 128 tokens and four beyond.
#include "internal.h"

namespace lzk {

namespace {

constexpr int kWarps = 8;
constexpr int kTileTokens = 16;
constexpr int kTileHalf = kTileTokens * kRowBytes;              // K or V of a tile: 4 KiB
constexpr int kTileBytes = 2 * kTileHalf;
constexpr int kRing = 2;
constexpr int kMaxTiles = kShortTokens / kTileTokens;
constexpr int kSets = 2;                                        // partial sums of the prefix fetched while the unit streams
constexpr int kSumRow = kHeadDim * 4 + 16;                      // a partial sum's O: a fragment read meets no bank twice
constexpr int kQRow = kRowBytes + 16;
// of a warp: the ring, the next unit's queries, the unit's first partial sums
constexpr int kOffQ = kRing * kTileBytes, kOffSums = kOffQ + kMaxGroup * kQRow, kWarpBytes = kOffSums + kSets * kMaxGroup * kSumRow;
constexpr int kOffBars = kWarps * kWarpBytes;
constexpr int kSmem = kOffBars + kWarps * kRing * 8 + 64;
constexpr uint32_t kTmemCols = 256;                             // four columns per tile; warps w and w + 4 share lanes
static_assert(2 * 4 * kMaxTiles <= kTmemCols, "");
constexpr float kRaiseMargin = 8.f;

struct ShortParams {
    const uint8_t* pool;
    const int32_t* page_table;
    const __nv_bfloat16* q;
    __nv_bfloat16* out;
    float* pbar;
    int2* tsm;
    int32_t* status;
    int units, group, pages_per_unit, capacity, total_pages;
    int n, t;
    float alpha, scale_log2, inv_group;
    PrefixView prefix;
    unsigned long long wait_limit_ns;
    int stop_after_tiles;                                       // diagnostics: a warp fetches no tile beyond this many (-1: off)
};

// Bounded wait; false (and the status word set) once the limit has passed.
__device__ __forceinline__ bool wait_tile(uint64_t* bar, uint32_t parity, int32_t* status, unsigned long long limit_ns) {
    uint32_t spins = 0;
    uint64_t t_start = 0;
    while (!mbar_try_wait(bar, parity)) {
        if ((++spins & 0xFF) == 0) {
            const uint64_t now = global_timer_ns();
            if (t_start == 0) {
                t_start = now;
            } else if (now - t_start > limit_ns) {
                atomicOr(status, kStatusWaitTimeout);
                return false;
            }
        }
    }
    return true;
}

__device__ __forceinline__ void copy16(uint32_t smem, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(__cvta_generic_to_global(src)) : "memory");
}
// This warp's copies have arrived, for all its lanes.
__device__ __forceinline__ void copies_done() {
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();
}

__global__ void __launch_bounds__(kWarps * 32, 1) decode_short_kernel(const __grid_constant__ ShortParams p) {
    extern __shared__ __align__(1024) uint8_t smem[];
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kOffBars + kWarps * kRing * 8);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t* ring = smem + warp * kWarpBytes;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + kOffBars) + warp * kRing;
    if (lane == 0) {
        for (int i = 0; i < kRing; ++i) mbar_init(&full[i], 1);
        fence_barrier_init();
    }
    if (warp == 0) {                           // tensor memory for the logits
        tmem_alloc(tmem_slot, kTmemCols);
        tmem_relinquish_alloc_permit();
    }
    tmem_fence_before_sync();
    __syncthreads();
    tmem_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    const uint32_t tmem = tmem_base + ((uint32_t)(32 * (warp & 3)) << 16) + (warp >> 2) * 4 * kMaxTiles;

    const int G = p.group, tiles = (p.n + kTileTokens - 1) / kTileTokens;
    const int walker = warp * gridDim.x + blockIdx.x, walkers = gridDim.x * kWarps;      // (few units spread over all SMs)

    // ---- the fetching side of the warp: tiles in walk order, up to kRing ahead of the one in use
    int f_unit = walker, f_tile = 0;
    uint32_t fetched = 0, used = 0;
    auto page_entry = [&](int u) {             // the lanes keep the unit's few page numbers
        const int pages = (p.n + kPageTokens - 1) / kPageTokens;
        return u < p.units && lane < pages ? p.page_table[(size_t)u * p.pages_per_unit + lane] : 0;
    };
    int32_t f_entry = page_entry(f_unit), f_next = page_entry(f_unit + walkers);
    auto fetch = [&]() {
        if (tiles == 0 || f_unit >= p.units) return;
        if (p.stop_after_tiles >= 0 && fetched >= (uint32_t)p.stop_after_tiles) return;
        int32_t pp = __shfl_sync(0xffffffffu, f_entry, f_tile * kTileTokens / kPageTokens);
        if (pp < 0 || pp >= p.total_pages) {
            if (lane == 0) atomicOr(p.status, kStatusBadIndex);
            pp = 0;
        }
        if (lane == 0) {
            const uint32_t st = fetched % kRing;
            const uint8_t* src = p.pool + (size_t)pp * kPageBytes + (f_tile * kTileTokens % kPageTokens) * kRowBytes;
            mbar_arrive_expect_tx(&full[st], kTileBytes);
            bulk_load(ring + st * kTileBytes, src, kTileHalf, &full[st]);
            bulk_load(ring + st * kTileBytes + kTileHalf, src + kPageHalfBytes, kTileHalf, &full[st]);
        }
        ++fetched;
        if (++f_tile == tiles) {
            f_tile = 0;
            f_unit += walkers;
            f_entry = f_next;
            f_next = page_entry(f_unit + walkers);
        }
    };
    for (int i = 0; i < kRing; ++i) fetch();

    // ---- fragment coordinates, as in decode.cu: S^T rows are tokens, O^T rows are head dimensions, columns query heads
    const int g = lane >> 2, qd = lane & 3, h0 = 2 * qd, h1 = h0 + 1;
    const bool h0_on = h0 < G, h1_on = h1 < G;
    const uint32_t lrow = lane & 7;
    const uint32_t k_row = ((lane & 7) + 8 * ((lane >> 3) & 1)) * kRowBytes, v_row = kTileHalf + ((lane & 7) + 8 * (lane >> 4)) * kRowBytes;
    const uint32_t k_term = ((lane >> 4) ^ lrow) << 4, v_term = (((lane >> 3) & 1) ^ lrow) << 4;
    const uint32_t ring_base = smem_u32(ring);

    // Queries and partial sums come as whole rows through shared memory (in fragment layout their loads would touch eight
    // sectors each, 80 of them per unit).
    const uint32_t q_s = ring_base + kOffQ, sums_s = ring_base + kOffSums;
    uint32_t qb[8][2];
    auto copy_q = [&](int u) {
        for (int h = lane >> 4; h < G; h += 2)
            copy16(q_s + h * kQRow + 16 * (lane & 15), p.q + ((size_t)u * G + h) * kHeadDim + 8 * (lane & 15));
    };
    auto read_q = [&]() {                      // Q as the B operand: rows are heads, two 16-dimension steps per instruction
#pragma unroll
        for (int ks = 0; ks < 8; ks += 2)
            ldmatrix_x4(qb[ks][0], qb[ks][1], qb[ks + 1][0], qb[ks + 1][1], q_s + (lane & 7) * kQRow + 32 * ks + 16 * (lane >> 3));
    };
    float2 ml[kSets];                          // lane h: head h's (reference, l) of the sets
    auto copy_sets = [&](int u, int s0) {
#pragma unroll
        for (int k = 0; k < kSets; ++k) {
            ml[k] = make_float2(-INFINITY, 0.f);
            if (s0 + k >= p.prefix.plan.slots) continue;
            const long long row = (s0 + k) * p.prefix.plan.rows + (long long)u * G;
            if (lane < G) ml[k] = p.prefix.ml[row + lane];
            for (int h = 0; h < G; ++h) copy16(sums_s + (k * kMaxGroup + h) * kSumRow + 16 * lane, p.prefix.o + (row + h) * kHeadDim + 4 * lane);
        }
    };
    for (int h = G; h < kMaxGroup; ++h)        // rows of heads that are not there
        if (lane < 16) *reinterpret_cast<uint4*>(ring + kOffQ + h * kQRow + 16 * lane) = make_uint4(0u, 0u, 0u, 0u);
    if (walker < p.units) copy_q(walker);
    copies_done();

    bool first = true, alive = true;
    for (int u = walker; u < p.units && alive; u += walkers) {
        read_q();
        __syncwarp();
        if (u + walkers < p.units) copy_q(u + walkers);
        if (!first) copy_sets(u, 0);
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
        float o[8][4];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;

        for (int j = 0; j < tiles; ++j) {
            const uint32_t st = used % kRing;
            alive = __all_sync(0xffffffffu, wait_tile(&full[st], (used / kRing) & 1u, p.status, p.wait_limit_ns));
            if (!alive) break;
            const uint32_t tile = ring_base + st * kTileBytes;

            // S^T = K Q^T, two accumulator chains over the 8 k-steps
            float sa[4] = {0.f, 0.f, 0.f, 0.f}, sb[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < 8; ks += 2) {
                uint32_t a0, a1, a2, a3;
                ldmatrix_x4(a0, a1, a2, a3, tile + k_row + (k_term ^ ((ks & 3) << 5)) + 128 * (ks >> 2));
                mma_bf16_16816(sa, a0, a1, a2, a3, qb[ks][0], qb[ks][1]);
                ldmatrix_x4(a0, a1, a2, a3, tile + k_row + (k_term ^ (((ks + 1) & 3) << 5)) + 128 * (ks >> 2));
                mma_bf16_16816(sb, a0, a1, a2, a3, qb[ks + 1][0], qb[ks + 1][1]);
            }
            float x00 = (sa[0] + sb[0]) * p.scale_log2;      // token g,     head h0
            float x01 = (sa[1] + sb[1]) * p.scale_log2;      // token g,     head h1
            float x10 = (sa[2] + sb[2]) * p.scale_log2;      // token g + 8, head h0
            float x11 = (sa[3] + sb[3]) * p.scale_log2;      // token g + 8, head h1
            const int left = p.n - j * kTileTokens;
            if (left < kTileTokens) {
                // slots past n: no weight, and V rows of zeros whatever an earlier sequence left in them
                if (g >= left) x00 = x01 = -INFINITY;
                if (g + 8 >= left) x10 = x11 = -INFINITY;
                for (int e = lane; e < (kTileTokens - left) * kChunksPerRow; e += 32)
                    *reinterpret_cast<uint4*>(ring + st * kTileBytes + kTileHalf + left * kRowBytes + e * 16) = make_uint4(0u, 0u, 0u, 0u);
                fence_proxy_async();          // the stage's next tile is written through the async proxy
                __syncwarp();
            }
            tmem_st4(tmem + 4 * j, x00, x01, x10, x11);      // kept for pbar

            // the reference is raised only when some logit is more than 2^8 above it (always on the first tile)
            float t0 = fmaxf(x00, x10), t1 = fmaxf(x01, x11);
            if (__any_sync(0xffffffffu, t0 > m0 + kRaiseMargin || t1 > m1 + kRaiseMargin)) {
#pragma unroll
                for (int s = 4; s < 32; s <<= 1) {
                    t0 = fmaxf(t0, __shfl_xor_sync(0xffffffffu, t0, s));
                    t1 = fmaxf(t1, __shfl_xor_sync(0xffffffffu, t1, s));
                }
                const float n0 = fmaxf(m0, t0), n1 = fmaxf(m1, t1);
                const float c0 = n0 == m0 ? 1.f : fast_exp2(m0 - n0), c1 = n1 == m1 ? 1.f : fast_exp2(m1 - n1);
                m0 = n0;
                m1 = n1;
                l0 *= c0;
                l1 *= c1;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    o[i][0] *= c0;
                    o[i][1] *= c1;
                    o[i][2] *= c0;
                    o[i][3] *= c1;
                }
            }
            const float r0 = m0 == -INFINITY ? 0.f : m0, r1 = m1 == -INFINITY ? 0.f : m1;
            const float p00 = fast_exp2(x00 - r0), p01 = fast_exp2(x01 - r1);
            const float p10 = fast_exp2(x10 - r0), p11 = fast_exp2(x11 - r1);
            l0 += p00 + p10;
            l1 += p01 + p11;

            // O^T += V^T P^T, P as two bf16 terms (hi + lo: 16 mantissa bits), as in decode.cu
            const uint32_t hi0 = pack_bf16(p00, p01), hi1 = pack_bf16(p10, p11);
            const uint32_t lo0 = pack_bf16(p00 - bf16_lo_as_float(hi0), p01 - bf16_hi_as_float(hi0));
            const uint32_t lo1 = pack_bf16(p10 - bf16_lo_as_float(hi1), p11 - bf16_hi_as_float(hi1));
            const uint32_t bh0 = movmatrix_trans(hi0), bh1 = movmatrix_trans(hi1);
            const uint32_t bl0 = movmatrix_trans(lo0), bl1 = movmatrix_trans(lo1);
#pragma unroll
            for (int mt = 0; mt < 8; ++mt) {
                uint32_t a0, a1, a2, a3;
                ldmatrix_x4_trans(a0, a1, a2, a3, tile + v_row + (v_term ^ ((mt & 3) << 5)) + 128 * (mt >> 2));
                mma_bf16_16816(o[mt], a0, a1, a2, a3, bh0, bh1);
                mma_bf16_16816(o[mt], a0, a1, a2, a3, bl0, bl1);
            }
            ++used;
            __syncwarp();                      // the stage is read: fetch the tile after those in flight
            fetch();
        }
        if (!alive) break;

        // ---- the prefix's sums.  The launch may begin beside the end of the prefix launch (own pages and queries come from earlier
        // ones); its sums are waited for here, once.
        if (first) {
            asm volatile("griddepcontrol.wait;" ::: "memory");
            copy_sets(u, 0);
            first = false;
        }
#pragma unroll
        for (int s = 4; s < 32; s <<= 1) {
            l0 += __shfl_xor_sync(0xffffffffu, l0, s);
            l1 += __shfl_xor_sync(0xffffffffu, l1, s);
        }
        for (int s = 0;; s += kSets) {
            copies_done();
#pragma unroll
            for (int k = 0; k < kSets; ++k) {
                const float a0 = __shfl_sync(0xffffffffu, ml[k].x, h0), a1 = __shfl_sync(0xffffffffu, ml[k].x, h1);
                const float b0 = __shfl_sync(0xffffffffu, ml[k].y, h0), b1 = __shfl_sync(0xffffffffu, ml[k].y, h1);
                const bool on0 = a0 > -INFINITY, on1 = a1 > -INFINITY;       // what an absent set's O holds is anything
                const float n0 = fmaxf(m0, a0), n1 = fmaxf(m1, a1);
                const float c0 = m0 == -INFINITY ? 0.f : fast_exp2(m0 - n0), c1 = m1 == -INFINITY ? 0.f : fast_exp2(m1 - n1);
                const float d0 = on0 ? fast_exp2(a0 - n0) : 0.f, d1 = on1 ? fast_exp2(a1 - n1) : 0.f;
                const float* v0 = reinterpret_cast<const float*>(ring + kOffSums + (k * kMaxGroup + h0) * kSumRow) + g;
                const float* v1 = v0 + kSumRow / 4;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    o[i][0] = o[i][0] * c0 + (on0 ? v0[16 * i] * d0 : 0.f);
                    o[i][1] = o[i][1] * c1 + (on1 ? v1[16 * i] * d1 : 0.f);
                    o[i][2] = o[i][2] * c0 + (on0 ? v0[16 * i + 8] * d0 : 0.f);
                    o[i][3] = o[i][3] * c1 + (on1 ? v1[16 * i + 8] * d1 : 0.f);
                }
                l0 = l0 * c0 + b0 * d0;
                l1 = l1 * c1 + b1 * d1;
                m0 = n0;
                m1 = n1;
            }
            __syncwarp();
            if (s + kSets >= p.prefix.plan.slots) break;
            copy_sets(u, s + kSets);
        }

        // ---- output: (dimension, head) fragments turned into rows of two dimensions per lane
        const float inv0 = 1.f / l0, inv1 = 1.f / l1;
        __nv_bfloat16* out = p.out + ((size_t)u * G + g) * kHeadDim + 2 * qd;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t lo = movmatrix_trans(pack_bf16(o[i][0] * inv0, o[i][1] * inv1));
            const uint32_t hi = movmatrix_trans(pack_bf16(o[i][2] * inv0, o[i][3] * inv1));
            if (g < G) {
                *reinterpret_cast<uint32_t*>(out + 16 * i) = lo;
                *reinterpret_cast<uint32_t*>(out + 16 * i + 8) = hi;
            }
        }

        // ---- pbar and Eq. (1) of the own tokens
        const float lse0 = m0 + log2f(l0), lse1 = m1 + log2f(l1);
        const size_t row = (size_t)u * p.capacity;
        if (tiles > 0) tmem_wait_st();
        for (int j = 0; j < tiles; ++j) {
            float x00, x01, x10, x11;
            tmem_ld4(tmem + 4 * j, x00, x01, x10, x11);
            tmem_wait_ld();
            float a0 = h0_on ? fast_exp2(x00 - lse0) : 0.f, a1 = h0_on ? fast_exp2(x10 - lse0) : 0.f;
            if (h1_on) {
                a0 += fast_exp2(x01 - lse1);
                a1 += fast_exp2(x11 - lse1);
            }
#pragma unroll
            for (int s = 1; s < 4; s <<= 1) {
                a0 += __shfl_xor_sync(0xffffffffu, a0, s);
                a1 += __shfl_xor_sync(0xffffffffu, a1, s);
            }
            if (qd < 2) {                      // the lanes 0 and 1 of a quad finish one token each
                const int i = j * kTileTokens + g + 8 * qd;
                if (i < p.n && in_bounds(p.n <= p.capacity, p.status)) {
                    const float pb = (qd == 0 ? a0 : a1) * p.inv_group;
                    p.pbar[row + i] = pb;
                    if (pb >= p.alpha) {       // MRI = max(MRI, t - TS), TS = t
                        const int2 old = p.tsm[row + i];
                        p.tsm[row + i] = make_int2(p.t, max(old.y, p.t - old.x));
                    }
                }
            }
        }
    }
    // A warp that gave up: what it has in flight lands before the block exits, and the launch does not end before the prefix launch
    // does (work queued behind it may write what that one still reads).
    if (!alive) {
        if (first) asm volatile("griddepcontrol.wait;" ::: "memory");
        copies_done();
        if (lane == 0)
            for (uint32_t k = used; k < fetched; ++k) wait_tile(&full[k % kRing], (k / kRing) & 1u, p.status, p.wait_limit_ns);
    }
    tmem_fence_before_sync();
    __syncthreads();
    if (warp == 0) {
        tmem_fence_after_sync();
        tmem_dealloc(tmem_base, kTmemCols);
    }
}

}  // namespace

cudaError_t decode_short_prepare() {
    return cudaFuncSetAttribute(decode_short_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
}

DecodePlan decode_short_plan() {
    DecodePlan plan = {};
    plan.splits = plan.groups = 1;
    plan.stages = kRing;
    plan.smem_bytes = kSmem;
    return plan;
}

int decode_short_blocks(int units, int num_sms) {
    return units < num_sms ? units : num_sms;
}

cudaError_t decode_short_launch(const DecodeConfig& c, const DecodeArgs& a, int num_sms, cudaStream_t stream) {
    ShortParams p;
    p.pool = a.pool;
    p.page_table = a.state.page_table;
    p.q = reinterpret_cast<const __nv_bfloat16*>(a.q);
    p.out = reinterpret_cast<__nv_bfloat16*>(a.out);
    p.pbar = a.state.pbar;
    p.tsm = a.state.tsm;
    p.status = a.state.status;
    p.units = c.units;
    p.group = c.group;
    p.pages_per_unit = c.pages_per_unit;
    p.capacity = c.capacity;
    p.total_pages = c.units * c.pages_per_unit;
    p.n = a.n;
    p.t = a.t;
    p.alpha = c.alpha;
    p.scale_log2 = 1.4426950408889634f / sqrtf((float)kHeadDim);
    p.inv_group = 1.0f / (float)c.group;
    p.prefix = a.prefix;
    p.wait_limit_ns = c.wait_limit_ns;
    p.stop_after_tiles = c.stop_after_pages < 0 ? -1 : c.stop_after_pages * (kPageTokens / kTileTokens);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(decode_short_blocks(c.units, num_sms), 1, 1);
    cfg.blockDim = dim3(kWarps * 32, 1, 1);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.behind_prefix ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, decode_short_kernel, p);
}

}  // namespace lzk
