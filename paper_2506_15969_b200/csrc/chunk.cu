// Attention of a chunk of new tokens over a paged cache: everything before the chunk, and the chunk itself causally.
//
// The last T of a unit's n tokens are the chunk (their keys and values are in the pages).  For token i of the chunk and each of
// the G query heads of its KV head, over the attached prefix and the own tokens j <= n - T + i:
//   x[j] = q . k_j / sqrt(D) * log2 e,   m >= max_j x[j] - 8,   l = sum_j exp2(x[j] - m),   out = sum_j exp2(x[j] - m) v_j / l
// in one pass over the keys, m being raised as it goes (Appendix A, Eq. (attn), for many rows at once).
//
// Structure: that of the kernel over a shared prefix (prefix.cu), with other rows.  A row tile is 128 accumulator rows =
// floor(128 / G) tokens x G heads of one unit, an item is two neighbouring row tiles (or the odd last one), which share the key
// tiles that they read; the walk over (item, key tile of 128 tokens) is cut into equal contiguous parts, one per persistent block,
// so a causal chunk leaves no block idle and a few rows over a long cache are spread over all SMs.  An item that one block has for
// itself is written out directly; the sums of one that several blocks share go through memory, and the last of them
// to arrive joins them, in the order of the keys (no second launch, and the same bits every time).
//
// P is one bf16 term (half a step is 2^-9 of a weight below a power of two's upper end, 2^-8 at worst; errors of different keys
// do not add up in one direction) and l is summed in fp32 before that rounding: a second term, as the kernels for single tokens
// have it, would be another P V product, a third of the tensor core's work where it is what bounds a long chunk.
//
// Masks act on the logits by selection, so keys that a row does not see may hold anything.  Values enter a product, where a zero
// weight times infinity is no zero: value rows that no row of the item sees are zeroed in shared memory before they are used, and a
// row whose logits are finite and whose output is not -- a value inside the chunk, seen by later rows of the same
// item only, or one that the row sees itself -- is computed again over its own keys alone.
//
// Warp roles: warps 0-15 softmax and output, warp 16 TMA producer, warps 17 and 18 MMA issuers, one per stream.  All mbarrier waits are bounded.
#include <string.h>

#include <cuda_fp16.h>

#include "internal.h"
#include "tensor.cuh"

namespace lzk {

namespace {

constexpr int kTile = 128;                         // rows of a row tile, keys of a key tile
constexpr int kBoxBytes = kTile * 128;             // half an operand: 128 rows x 64 bf16
constexpr int kOperandBytes = 2 * kBoxBytes;       // a 128 x 128 bf16 operand (32 KiB)
constexpr int kRing = 5;                           // K and V tiles in flight, in the order they are used
constexpr int kStreamWarps = 8;                    // two warps per 32 accumulator rows, half of the columns each
constexpr int kProducer = 2 * kStreamWarps, kIssuer = kProducer + 1, kThreads = 32 * (kIssuer + 2);      // an issuer per stream
constexpr float kRaiseMargin = 8.f;                // log2 units a logit may exceed the reference by

constexpr int kOffQ = 0;                           // two row tiles
constexpr int kOffRing = kOffQ + 2 * kOperandBytes;
constexpr int kOffMisc = kOffRing + kRing * kOperandBytes;
constexpr int kOffExchange = kOffMisc + 1024;      // [2 streams][128 rows][2]: what the two threads of a row tell each other
constexpr int kSmem = kOffExchange + 2048;

constexpr uint32_t kColS = 0, kColO = 256, kTmemCols = 512;     // per stream: 128 columns of S / P, 128 of O

struct Bars {
    uint64_t q_full[2], q_empty[2];
    uint64_t full[kRing], empty[kRing];
    uint64_t s_full[2], p_full[2][2], o_full[2];   // [stream]; P comes in two halves
    uint64_t drain[2];
};

struct ChunkParams {
    ChunkPlan plan;
    const uint8_t* pages;
    const uint8_t* prefix_pages;
    const int32_t* page_table;
    const int32_t* prefix_table;
    int pages_per_unit, total_pages, prefix_pages_per_unit, prefix_total_pages;
    RowView q, out;
    float* o;
    float2* ml;
    int32_t* counters;
    float* norms;
    int32_t* status;
    float scale_log2;
    unsigned long long wait_limit_ns;
    int stop_after_tiles;
};

__device__ __forceinline__ int part_begin(const ChunkPlan& p, int block) { return block * p.per + min(block, p.extra); }
// Block that works on step x.
__device__ __forceinline__ int block_of(const ChunkPlan& p, int x) {
    const int longer = p.extra * (p.per + 1);
    return x < longer ? x / (p.per + 1) : p.extra + (x - longer) / p.per;
}

// One block's part of an item: key tiles [k0, k1) of kt.
struct Piece {
    int unit, pair, start;                         // the item, and the step it starts at
    int kt, k0, k1;
    bool both;                                     // two row tiles, a stream each; else one, the key tiles in turn
    __device__ __forceinline__ int tiles() const { return k1 - k0; }
    // key tiles of stream s, and the t-th of them
    __device__ __forceinline__ int stream_tiles(int s) const { return both ? k1 - k0 : (k1 - k0 + 1 - s) >> 1; }
    __device__ __forceinline__ int key_tile(int s, int t) const { return both ? k0 + t : k0 + 2 * t + s; }
};

struct Walk {
    int x, end, unit, pair, start;
    __device__ __forceinline__ void begin(const ChunkPlan& pl, int block) {
        x = part_begin(pl, block);
        end = part_begin(pl, block + 1);
        unit = x / pl.unit_steps;
        start = unit * pl.unit_steps;
        pair = 0;
        for (int kt = chunk_key_tiles(pl, 0); x - start >= kt; kt = chunk_key_tiles(pl, ++pair)) start += kt;
    }
    __device__ __forceinline__ bool more() const { return x < end; }
    __device__ __forceinline__ Piece next(const ChunkPlan& pl) {
        Piece pc;
        pc.unit = unit;
        pc.pair = pair;
        pc.start = start;
        pc.kt = chunk_key_tiles(pl, pair);
        pc.k0 = x - start;
        pc.k1 = min(pc.kt, pc.k0 + (end - x));
        pc.both = 2 * pair + 1 < pl.tiles;
        x += pc.tiles();
        if (pc.k1 == pc.kt) {
            start += pc.kt;
            if (++pair == pl.pairs) {
                pair = 0;
                ++unit;
            }
        }
        return pc;
    }
};

// 64 columns of the accumulator times a factor per row.
__device__ __noinline__ void rescale(uint32_t cols, float f) {
#pragma unroll 1
    for (int c = 0; c < 64; c += 16) {
        float o[16];
        tmem_ld16(cols + c, o);
        tmem_wait_ld();
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(o[i] * f);
        tmem_st16(cols + c, w);
    }
    tmem_wait_st();
}

// Layer, sequence and KV head of a unit, and its row of the prefix's page table.
struct UnitAt {
    int layer, seq, head, prefix_unit;
};
__device__ __forceinline__ UnitAt unit_at(const ChunkPlan& pl, int unit) {
    UnitAt a;
    a.head = unit % pl.kv_heads;
    const int ls = unit / pl.kv_heads;
    a.seq = ls % pl.batch;
    a.layer = ls / pl.batch;
    a.prefix_unit = pl.prefix_n > 0 ? ls / pl.prefix_share * pl.kv_heads + a.head : 0;     // (sequences of a layer divide among its prefixes)
    return a;
}

__device__ __forceinline__ long long row_offset(const RowView& v, const UnitAt& at, int tok, int head) {
    return at.layer * v.stride_layer + at.seq * v.stride_batch + tok * v.stride_token + head * v.stride_head;
}

// The page numbers of key tiles in ascending order, the prefix's before the own.
struct KeyPages {
    PageList pages;
    bool own;
    __device__ __forceinline__ void open(const ChunkParams& p, int unit, const UnitAt& at, int kt) {
        const ChunkPlan& pl = p.plan;
        own = kt >= pl.prefix_tiles;
        if (own)
            pages.open(p.page_table + (long long)unit * p.pages_per_unit, (pl.context + pl.tokens - 1) / kPageTokens, 2 * (kt - pl.prefix_tiles));
        else
            pages.open(p.prefix_table + (long long)at.prefix_unit * p.prefix_pages_per_unit, (pl.prefix_n - 1) / kPageTokens, 2 * kt);
        pages.fetch(pages.first);
    }
};

// A row over its own keys alone, from global memory, for a known reference and sum: a whole warp, lane -> columns 4 lane .. + 3.
__device__ __noinline__ float4 redo_row(const ChunkParams& p, int unit, int tok, int g, float m, float l) {
    const ChunkPlan& pl = p.plan;
    const UnitAt at = unit_at(pl, unit);
    const int lane = threadIdx.x & 31;
    const uint4* q = reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(p.q.data) +
                                                    row_offset(p.q, at, tok, at.head * pl.group + g));
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int own = 0; own < 2; ++own) {
        const int keys = own ? pl.context + tok + 1 : pl.prefix_n, total = own ? p.total_pages : p.prefix_total_pages;
        const int32_t* table = own ? p.page_table + (long long)unit * p.pages_per_unit
                                   : p.prefix_table + (long long)at.prefix_unit * p.prefix_pages_per_unit;
        const uint8_t* pool = own ? p.pages : p.prefix_pages;
        auto page_of = [&](int j) {
            const int32_t pp = table[j / kPageTokens];
            return pp >= 0 && pp < total ? pp : 0;
        };
        for (int base = 0; base < keys; base += 32) {
            float w = 0.f;
            if (base + lane < keys) {
                const int j = base + lane, r = j % kPageTokens;
                const uint8_t* row = pool + (size_t)page_of(j) * kPageBytes + r * kRowBytes;
                float x = 0.f;
                for (int c = 0; c < kChunksPerRow; ++c) {
                    const uint4 a = q[c], b = *reinterpret_cast<const uint4*>(row + swz_chunk(c, r) * 16);
                    const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        x = fmaf(bf16_lo_as_float(aw[i]), bf16_lo_as_float(bw[i]), x);
                        x = fmaf(bf16_hi_as_float(aw[i]), bf16_hi_as_float(bw[i]), x);
                    }
                }
                w = fast_exp2(fmaf(x, p.scale_log2, -m));
            }
            const int some = min(32, keys - base);
            for (int i = 0; i < some; ++i) {
                const float wi = __shfl_sync(0xffffffffu, w, i);
                const int j = base + i, r = j % kPageTokens;
                const uint8_t* row = pool + (size_t)page_of(j) * kPageBytes + kPageHalfBytes + r * kRowBytes;
                const uint2 v = *reinterpret_cast<const uint2*>(row + swz_chunk(lane >> 1, r) * 16 + (lane & 1) * 8);
                acc[0] = fmaf(wi, bf16_lo_as_float(v.x), acc[0]);
                acc[1] = fmaf(wi, bf16_hi_as_float(v.x), acc[1]);
                acc[2] = fmaf(wi, bf16_lo_as_float(v.y), acc[2]);
                acc[3] = fmaf(wi, bf16_hi_as_float(v.y), acc[3]);
            }
        }
    }
    const float inv = 1.f / l;
    return make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi, int dtype) { return dtype == kTypeBF16 ? pack_bf16(lo, hi) : pack_f16(lo, hi); }

// Four output elements from column col on (a multiple of 4).
__device__ __forceinline__ void store4(const RowView& out, long long at, int col, const float4& v) {
    if (out.dtype == kTypeF32)
        *reinterpret_cast<float4*>(reinterpret_cast<float*>(const_cast<void*>(out.data)) + at + col) = v;
    else
        *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(const_cast<void*>(out.data)) + at + col) =
            make_uint2(pack_pair(v.x, v.y, out.dtype), pack_pair(v.z, v.w, out.dtype));
}
// Sixteen, from a multiple of 16 on.
__device__ __forceinline__ void store16(const RowView& out, long long at, int col, const float (&v)[16]) {
    if (out.dtype == kTypeF32) {
        float4* dst = reinterpret_cast<float4*>(reinterpret_cast<float*>(const_cast<void*>(out.data)) + at + col);
#pragma unroll
        for (int i = 0; i < 4; ++i) dst[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    } else {
        uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(const_cast<void*>(out.data)) + at + col);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            dst[i] = make_uint4(pack_pair(v[8 * i], v[8 * i + 1], out.dtype), pack_pair(v[8 * i + 2], v[8 * i + 3], out.dtype),
                                pack_pair(v[8 * i + 4], v[8 * i + 5], out.dtype), pack_pair(v[8 * i + 6], v[8 * i + 7], out.dtype));
    }
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }

__global__ void __launch_bounds__(kThreads, 1)
chunk_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_kv, const __grid_constant__ CUtensorMap map_prefix,
             const __grid_constant__ ChunkParams p) {
    extern __shared__ __align__(1024) uint8_t smem[];
    Bars* bars = reinterpret_cast<Bars*>(smem + kOffMisc);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kOffMisc + 512);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    volatile int* last_flag = reinterpret_cast<volatile int*>(tmem_slot + 2);      // [2 streams][4 quarters of a row tile]
    const ChunkPlan& pl = p.plan;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    Walk walk;
    walk.begin(pl, blockIdx.x);

    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bars->q_full[i], 1);
            mbar_init(&bars->q_empty[i], 2);       // (one arrival per stream)
            mbar_init(&bars->s_full[i], 1);
            for (int h = 0; h < 2; ++h) mbar_init(&bars->p_full[i][h], kStreamWarps);
            mbar_init(&bars->o_full[i], 1);
        }
        for (int i = 0; i < kRing; ++i) {
            mbar_init(&bars->full[i], 1);
            mbar_init(&bars->empty[i], 2);
        }
        mbar_init(&bars->drain[0], 1);
        mbar_init(&bars->drain[1], 1);
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == kProducer && lane == 0) {
        prefetch_map(&map_q);
        prefetch_map(&map_kv);
    }
    // rows of a row tile that no query row ever fills (128 is no multiple of G): zeros, like all of Q before the first tile
    for (int i = threadIdx.x; i < 2 * kOperandBytes / 16; i += kThreads)
        reinterpret_cast<uint4*>(smem + kOffQ)[i] = make_uint4(0u, 0u, 0u, 0u);
    fence_proxy_async();
    if (warp == 0) {
        tmem_alloc(tmem_slot, kTmemCols);
        tmem_relinquish_alloc_permit();
    }
    tmem_fence_before_sync();
    __syncthreads();
    tmem_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    const unsigned long long limit = p.wait_limit_ns;

    if (warp == kProducer) {
        // ------------------------------------------------------------------ TMA producer
        // (the whole warp: the lanes keep 32 page numbers, one elected lane issues the copies)
        Ring rr, qr;
        bool ok = true;
        int k_tiles = 0;
        const uint32_t q_bytes = (uint32_t)(pl.tile_tokens * pl.group) * 256u;
        auto wait_on = [&](uint64_t* bar, uint32_t parity) { ok = __all_sync(0xffffffffu, wait_bar(bar, parity, abort_flag, p.status, limit)); };
        while (walk.more() && ok) {
            const Piece pc = walk.next(pl);
            const UnitAt at = unit_at(pl, pc.unit);
            KeyPages k_pages, v_pages;
            k_pages.open(p, pc.unit, at, pc.k0);
            v_pages = k_pages;
            // a K (half = 0) or V (half = 1) tile: 64 rows x 64 elements per box, two pages, both halves of the rows
            auto load_tile = [&](KeyPages& list, int kt, int half) {
                if (!list.own && kt >= pl.prefix_tiles) list.open(p, pc.unit, at, kt);
                const int page = 2 * (list.own ? kt - pl.prefix_tiles : kt), total = list.own ? p.total_pages : p.prefix_total_pages;
                const CUtensorMap* map = list.own ? &map_kv : &map_prefix;
                // (a tile's second page may lie behind the last one: any page will do, its keys are masked)
                int32_t p0 = list.pages.at(page), p1 = list.pages.at(page + 1);
                if (p0 < 0 || p0 >= total || p1 < 0 || p1 >= total) {
                    if (lane == 0) atomicOr(p.status, kStatusBadIndex);
                    p0 = p1 = 0;
                }
                const uint32_t st = rr.stage(kRing);
                wait_on(&bars->empty[st], rr.parity(kRing) ^ 1u);
                if (!ok) return;
                uint8_t* dst = smem + kOffRing + st * kOperandBytes;
                if (elect_one()) {
                    mbar_arrive_expect_tx(&bars->full[st], kOperandBytes);
                    tma_load_3d(dst, map, 0, half * kPageTokens, p0, &bars->full[st]);
                    tma_load_3d(dst + kBoxBytes / 2, map, 0, half * kPageTokens, p1, &bars->full[st]);
                    tma_load_3d(dst + kBoxBytes, map, 64, half * kPageTokens, p0, &bars->full[st]);
                    tma_load_3d(dst + kBoxBytes + kBoxBytes / 2, map, 64, half * kPageTokens, p1, &bars->full[st]);
                }
                __syncwarp();
                ++rr.count;
            };
            for (int s = 0; s < (pc.both ? 2 : 1) && ok; ++s) {
                const uint32_t qs = qr.stage(2);
                wait_on(&bars->q_empty[qs], qr.parity(2) ^ 1u);
                if (!ok) break;
                uint8_t* dst = smem + kOffQ + qs * kOperandBytes;
                const int tok = (2 * pc.pair + s) * pl.tile_tokens;
                if (elect_one()) {
                    mbar_arrive_expect_tx(&bars->q_full[qs], q_bytes);
                    tma_load_5d(dst, &map_q, 0, at.head * pl.group, tok, at.seq, at.layer, &bars->q_full[qs]);
                    tma_load_5d(dst + kBoxBytes, &map_q, 64, at.head * pl.group, tok, at.seq, at.layer, &bars->q_full[qs]);
                }
                __syncwarp();
                ++qr.count;
            }
            const int ahead = pc.both ? 1 : 2, nt = pc.tiles();
            auto load_k = [&](int j) {
                // diagnostics: no copy beyond the first stop_after_tiles K tiles
                if (p.stop_after_tiles >= 0 && k_tiles >= p.stop_after_tiles) ok = false;
                ++k_tiles;
                if (ok) load_tile(k_pages, pc.k0 + j, 0);
            };
            for (int j = 0; j < min(ahead, nt) && ok; ++j) load_k(j);
            for (int j = 0; j < nt && ok; ++j) {
                load_tile(v_pages, pc.k0 + j, 1);
                if (ok && j + ahead < nt) load_k(j + ahead);
            }
        }
        // the copies already issued land before the block exits, whoever gives up and when
        auto drain = [&](uint64_t* full, const Ring& r, uint32_t n) {
            const uint32_t last = r.count < n ? r.count : n;
            for (uint32_t k = r.count - last; k < r.count; ++k)
                wait_bar(&full[k % n], (k / n) & 1u, abort_flag, p.status, limit, false);
        };
        drain(bars->full, rr, kRing);
        drain(bars->q_full, qr, 2);
    } else if (warp >= kIssuer) {
        // ------------------------------------------------------------------ MMA issuers, one warp per stream
        // Who issues when, the turns between the two warps and the uses of the ring that each looks at: as in prefix.cu.
        const int s = warp - kIssuer;
        uint32_t p_uses = 0, uses = 0, q_uses = 0;  // products issued; uses of the K / V ring and of the Q slots by earlier pieces
        bool ok = true;                             // a warp that gave up goes through the same turns without issuing
        bool behind = false;                        // the piece before ended with the other stream's turn (stream 0 looks)
        auto wait_on = [&](uint64_t* bar, uint32_t parity) {
            if (ok) ok = __all_sync(0xffffffffu, wait_bar(bar, parity, abort_flag, p.status, limit));
        };
        uint32_t seen = 0;                          // uses of the ring that this warp has looked at
        auto look_at = [&](uint32_t uses_to, bool reads_last) {
            for (; seen < uses_to; ++seen) {
                const uint32_t st = seen % kRing;
                wait_on(&bars->full[st], (seen / kRing) & 1u);
                if (reads_last && seen + 1 == uses_to) continue;
                if (ok && elect_one()) mbar_arrive(&bars->empty[st]);
                __syncwarp();
            }
        };
        const uint32_t s_col = tmem_base + kColS + s * 128, o_col = tmem_base + kColO + s * 128;
        const uint64_t q_desc = smem_desc(smem_u32(smem + kOffQ), 16, 1024), k_desc = smem_desc(smem_u32(smem + kOffRing), 16, 1024);
        const uint64_t v_desc = smem_desc(smem_u32(smem + kOffRing), kBoxBytes, 1024);
        constexpr uint32_t kStep = kOperandBytes >> 4;              // from operand to operand, in a descriptor's units
        // O += P V for the keys of P's half `part`: the first or the second 32 of every 64
        auto issue_o = [&](uint32_t st, int part, bool first) {
            const uint64_t b = v_desc + st * kStep;
#pragma unroll
            for (int i = 0; i < 4; ++i) {           // 16 keys per instruction
                const int s8 = (i >> 1) * 4 + part * 2 + (i & 1);
                umma_bf16_ts(o_col, s_col + (s8 >> 2) * 64 + (s8 & 3) * 8, b + s8 * (2048 >> 4), instr_desc(true), !first || i > 0);
            }
        };
        while (walk.more()) {
            const Piece pc = walk.next(pl);
            const int nt = pc.tiles(), mine = pc.stream_tiles(s), step = pc.both ? 1 : 2, turns = pc.both ? 2 * nt : nt;
            const uint32_t q_use = q_uses + (pc.both ? s : 0), q_slot = q_use & 1u;
            q_uses += pc.both ? 2 : 1;
            // The ring holds K_0 (one tile ahead; with alternating streams K_0, K_1), then V_j, K_(j + ahead) in turn.
            const int ahead = pc.both ? 1 : 2, lead = min(ahead, nt);
            auto v_use = [&](int j) { return uses + lead + j + min(j, nt - lead); };
            auto k_use = [&](int j) { return j < ahead ? uses + j : v_use(j - ahead) + 1; };
            auto issue_s = [&](uint32_t st, bool last) {               // (by one lane) S = Q K^T
                const uint64_t a = q_desc + q_slot * kStep, b = k_desc + st * kStep;
#pragma unroll
                for (int s8 = 0; s8 < 8; ++s8) {    // 16 head dimensions per instruction: 32 bytes inside a box row
                    const uint32_t off = ((s8 >> 2) * kBoxBytes + (s8 & 3) * 32) >> 4;
                    umma_bf16(s_col, a + off, b + off, instr_desc(false), s8 > 0);
                }
                umma_commit(&bars->s_full[s]);
                umma_commit(&bars->empty[st]);
                if (last) {                         // (Q of two row tiles: each stream reads its own, and answers for the other)
                    if (pc.both) mbar_arrive(&bars->q_empty[q_slot]);
                    umma_commit(&bars->q_empty[q_slot]);
                }
            };
            wait_on(&bars->q_full[q_slot], (q_use >> 1) & 1u);
            int j = pc.both ? 0 : s;
            if (mine > 0) {
                const uint32_t use = k_use(j);
                look_at(use + 1, true);
                tmem_fence_after_sync();
                if (ok && elect_one()) issue_s(use % kRing, mine == 1);
            } else if (ok && elect_one()) {
                mbar_arrive(&bars->q_empty[q_slot]);
            }
            __syncwarp();
            // value rows that no row of the item sees become zeros (both streams write the same ones)
            auto clear_unseen = [&](int kt, uint32_t st) {
                const int to = kt < pl.prefix_tiles
                                   ? pl.prefix_n - kt * kTile
                                   : pl.context + min(pl.tokens, 2 * pl.tile_tokens * (pc.pair + 1)) - (kt - pl.prefix_tiles) * kTile;
                if (to >= kTile) return;
                uint8_t* v = smem + kOffRing + st * kOperandBytes;
                for (int i = max(to, 0) * 8 + lane; i < kTile * 8; i += 32) {
                    reinterpret_cast<uint4*>(v)[i] = make_uint4(0u, 0u, 0u, 0u);
                    reinterpret_cast<uint4*>(v + kBoxBytes)[i] = make_uint4(0u, 0u, 0u, 0u);
                }
                fence_proxy_async();
                __syncwarp();
            };
            for (int t = 0; t < mine; ++t, j += step) {
                const int turn = 2 * t + s;         // the streams take turns: 0, 1, 0, 1 ..
                const bool more = t + 1 < mine;
                const uint32_t vu = v_use(j), vs = vu % kRing, ku = more ? k_use(j + step) : 0u, ks = ku % kRing;
                look_at(vu + 1, true);
                if (ok) clear_unseen(pc.k0 + j, vs);
                if (more) look_at(ku + 1, true);
                wait_on(&bars->p_full[s][0], p_uses & 1u);
                if (turn > 0 || behind) named_barrier_sync(13 + s, 64);
                tmem_fence_after_sync();
                if (ok && elect_one()) issue_o(vs, 0, t == 0);
                __syncwarp();
                wait_on(&bars->p_full[s][1], p_uses & 1u);
                ++p_uses;
                tmem_fence_after_sync();
                if (ok && elect_one()) {
                    issue_o(vs, 1, false);
                    umma_commit(&bars->empty[vs]);
                    if (more)
                        issue_s(ks, t + 2 == mine);
                    else
                        umma_commit(&bars->o_full[s]);
                }
                __syncwarp();
                if (turn + 1 < turns || (s == 1 && walk.more())) asm volatile("bar.arrive %0, %1;" ::"r"(13 + (s ^ 1)), "r"(64) : "memory");
            }
            behind = (turns & 1) == 0;
            uses += 2 * nt;
            look_at(uses, false);                   // (the other stream's last ones)
        }
        // every MMA issued by this warp is complete before tensor memory goes back
        if (elect_one()) umma_commit(&bars->drain[s]);
        __syncwarp();
        wait_bar(&bars->drain[s], 0, abort_flag, p.status, limit, false);
    } else {
        // ------------------------------------------------------------------ softmax and output
        // Accumulator row = TMEM lane; the warps w and w + 4 of a stream share 32 rows and take 64 of the 128 columns each (a
        // row's chain of exponentials is what a stream's turn is made of: two threads halve it).
        const int s = warp / kStreamWarps, hf = (warp >> 2) & 1, quarter = warp & 3, row = 32 * quarter + lane;
        const uint32_t lane_base = tmem_base + ((uint32_t)(32 * quarter) << 16);
        const uint32_t s_cols = lane_base + kColS + s * 128 + hf * 64, o_cols = lane_base + kColO + s * 128 + hf * 64;
        float* mine = reinterpret_cast<float*>(smem + kOffExchange) + (s * kTile + row) * 2 + hf;
        const float* other = reinterpret_cast<const float*>(smem + kOffExchange) + (s * kTile + row) * 2 + (hf ^ 1);
        const int pair_bar = 1 + s * 4 + quarter, quad_bar = 9 + quarter;      // of the two warps of a row; of the four of both streams
        uint32_t s_uses = 0, o_uses = 0;
        // A warp whose wait gives up goes on through the same loops, so that its partner's barriers get all their threads, but waits
        // for nothing any more; what it computes means nothing.
        bool dead = false;
        auto wait_on = [&](uint64_t* bar, uint32_t parity) {
            const bool gave_up = dead || !wait_bar(bar, parity, abort_flag, p.status, limit);
            dead = __any_sync(0xffffffffu, gave_up);
        };
        const int r_tok = row / pl.group, r_head = row - r_tok * pl.group;     // token and head of this row inside its tile
        while (walk.more()) {
            const Piece pc = walk.next(pl);
            const int nt = pc.stream_tiles(s);
            const int tile = 2 * pc.pair + (pc.both ? s : 0), tok0 = tile * pl.tile_tokens;
            const int tok = tok0 + r_tok;
            const bool valid = r_tok < pl.tile_tokens && tok < pl.tokens;
            const bool warp_on = __any_sync(0xffffffffu, valid);       // (the same in both warps of the rows)
            // own keys that this row sees, and that every row of the tile sees
            const int sees = pl.context + (valid ? tok + 1 : pl.tokens), all_see = pl.context + tok0 + 1;
            float m = -INFINITY, l = 0.f;
            for (int t = 0; t < nt; ++t) {
                wait_on(&bars->s_full[s], s_uses & 1u);
                ++s_uses;
                tmem_fence_after_sync();
                if (warp_on) {
                    float v[2][32];
                    tmem_ld32(s_cols, v[0]);
                    tmem_ld32(s_cols + 32, v[1]);
                    tmem_wait_ld();
                    const int kt = pc.key_tile(s, t);
                    const bool own = kt >= pl.prefix_tiles;
                    const int key0 = (own ? kt - pl.prefix_tiles : kt) * kTile + hf * 64;
                    if (key0 + 64 > (own ? all_see : pl.prefix_n)) {
                        const int to = (own ? sees : pl.prefix_n) - key0;
#pragma unroll
                        for (int c = 0; c < 2; ++c)
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[c][i] = 32 * c + i < to ? v[c][i] : -INFINITY;
                    }
                    float mx[4] = {v[0][0], v[0][1], v[1][0], v[1][1]};
#pragma unroll
                    for (int i = 2; i < 32; i += 2) {
                        mx[(i >> 1) & 1] = fmax3(mx[(i >> 1) & 1], v[0][i], v[0][i + 1]);
                        mx[2 + ((i >> 1) & 1)] = fmax3(mx[2 + ((i >> 1) & 1)], v[1][i], v[1][i + 1]);
                    }
                    // the row's maximum over both halves; both threads of the row take the same decisions from here on
                    *mine = fmax3(mx[0], mx[1], fmaxf(mx[2], mx[3]));
                    named_barrier_sync(pair_bar, 64);
                    const float top = fmaxf(*mine, *other) * p.scale_log2;
                    if (__any_sync(0xffffffffu, top > m + kRaiseMargin && valid)) {
                        const float to = fmaxf(m, top);
                        const float f = m == to ? 1.f : fast_exp2(m - to);
                        if (t > 0) rescale(o_cols, f);
                        l *= f;
                        m = to;
                    }
                    const float ref = m == -INFINITY ? 0.f : m;      // every logit -inf: all weights are zero
                    const uint64_t scale2 = pack2(p.scale_log2, p.scale_log2), minus2 = pack2(-ref, -ref);
                    uint64_t sum0 = pack2(0.f, 0.f), sum1 = sum0;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {                      // 16 columns at a time
                        if (c == 2) {                                  // the first half of P is there: its product may begin
                            tmem_wait_st();
                            tmem_fence_before_sync();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&bars->p_full[s][0]);
                        }
                        uint32_t w16[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float x0 = v[c >> 1][16 * (c & 1) + 2 * i], x1 = v[c >> 1][16 * (c & 1) + 2 * i + 1];
                            float e0, e1;
                            unpack2(fma2(pack2(x0, x1), scale2, minus2), e0, e1);
                            e0 = fast_exp2(e0);
                            e1 = fast_exp2(e1);
                            w16[i] = pack_bf16(e0, e1);
                            if (i & 1)
                                sum1 = add2(sum1, pack2(e0, e1));
                            else
                                sum0 = add2(sum0, pack2(e0, e1));
                        }
                        tmem_st8(s_cols + 8 * c, w16);                 // two keys per column
                    }
                    float a0, a1;
                    unpack2(add2(sum0, sum1), a0, a1);
                    l += a0 + a1;
                    tmem_wait_st();
                } else if (lane == 0) {
                    mbar_arrive(&bars->p_full[s][0]);
                }
                tmem_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars->p_full[s][1]);
            }
            // ---- the piece's sums
            if (nt > 0) {
                wait_on(&bars->o_full[s], o_uses & 1u);
                ++o_uses;
            }
            tmem_fence_after_sync();
            const bool speaks = hf == 0 && (pc.both || s == 0);        // one thread per row
            auto put_norm = [&](int row_i, float reference, float inv) {
                float* norm = p.norms + ((long long)pc.unit * pl.tiles + tile) * 2 * kTile + row_i;
                norm[0] = reference;
                norm[kTile] = inv;
            };
            if (warp_on) {
                const UnitAt at = unit_at(pl, pc.unit);
                const bool whole = pc.tiles() == pc.kt;
                const long long out_at = valid ? row_offset(p.out, at, tok, at.head * pl.group + r_head) : 0;
                // where shared sums of this item go: a block has at most two such pieces, one at either end of its part
                auto slot_of = [&](int block, int first_step) { return 2 * block + (first_step == part_begin(pl, block) ? 0 : 1); };
                const int half = pc.both ? s : 0;
                const long long sums_at = ((long long)(2 * blockIdx.x + (pc.start + pc.k0 == part_begin(pl, blockIdx.x) ? 0 : 1)) * 2 + half) * kTile + row;
                *mine = l;
                named_barrier_sync(pair_bar, 64);
                l += *other;
                named_barrier_sync(pair_bar, 64);
                // 16 columns of sums, final or to be joined
                bool sound = true;
                auto put = [&](int col, float (&o)[16], float inv) {
                    if (!valid) return;
                    if (whole) {
                        float odd = 0.f;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            o[i] *= inv;
                            odd = fmaf(o[i], 0.f, odd);                // (not a number as soon as one of them is not finite)
                        }
                        sound = sound && odd == 0.f;
                        store16(p.out, out_at, col, o);
                    } else {
                        float4* dst = reinterpret_cast<float4*>(p.o + sums_at * kHeadDim + col);
#pragma unroll
                        for (int i = 0; i < 4; ++i) dst[i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                    }
                };
                int col0 = 64 * hf, cols = 64;                         // of this thread's row
                if (pc.both) {
                    const float inv = 1.f / l;
#pragma unroll 1
                    for (int c = 0; c < 64; c += 16) {
                        float o[16];
                        tmem_ld16(o_cols + c, o);
                        tmem_wait_ld();
                        put(col0 + c, o, inv);
                    }
                } else {
                    // The two streams' sums into one: four threads per row, 32 columns each.  (Each stream's warps have waited for
                    // their own accumulator; the barrier passes that on.)
                    *mine = hf ? l : m;
                    tmem_fence_before_sync();
                    named_barrier_sync(quad_bar, 128);
                    tmem_fence_after_sync();
                    const float2* ml = reinterpret_cast<const float2*>(smem + kOffExchange) + row;
                    const float2 a0 = ml[0], a1 = ml[kTile];
                    m = fmaxf(a0.x, a1.x);
                    const float f0 = a0.x > -INFINITY ? fast_exp2(a0.x - m) : 1.f, f1 = a1.x > -INFINITY ? fast_exp2(a1.x - m) : 1.f;
                    l = a0.y * f0 + a1.y * f1;                         // (a stream without a tile has m = -inf, l = 0)
                    const float inv = 1.f / l;
                    col0 = 64 * s + 32 * hf;
                    cols = 32;
#pragma unroll 1
                    for (int c = 0; c < 32; c += 16) {
                        float o0[16], o1[16];
                        tmem_ld16(lane_base + kColO + col0 + c, o0);
                        tmem_ld16(lane_base + kColO + 128 + col0 + c, o1);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) o0[i] = o0[i] * f0 + (pc.tiles() > 1 ? o1[i] * f1 : 0.f);
                        put(col0 + c, o0, inv);
                    }
                    tmem_fence_before_sync();
                    named_barrier_sync(quad_bar, 128);                 // all are done with both accumulators and the exchange
                }
                if (whole) {
                    if (p.norms && speaks && valid) put_norm(row, m, 1.f / l);
                    // rows that a value reached which they do not see (or that see one that is not finite)
                    unsigned again = __ballot_sync(0xffffffffu, valid && !sound && finite(l) && finite(m));
                    while (again) {
                        const int i = __ffs(again) - 1;
                        again &= again - 1;
                        const int tok_i = __shfl_sync(0xffffffffu, tok, i), head_i = __shfl_sync(0xffffffffu, r_head, i);
                        const float m_i = __shfl_sync(0xffffffffu, m, i), l_i = __shfl_sync(0xffffffffu, l, i);
                        const float4 o = redo_row(p, pc.unit, tok_i, head_i, m_i, l_i);
                        if (4 * lane >= col0 && 4 * lane < col0 + cols)
                            store4(p.out, row_offset(p.out, at, tok_i, at.head * pl.group + head_i), 4 * lane, o);
                    }
                } else {
                    if (valid && speaks) p.ml[sums_at] = make_float2(m, l);
                    // the last block of the item to come here joins the sums of all
                    const int first_block = block_of(pl, pc.start), blocks = block_of(pl, pc.start + pc.kt - 1) - first_block + 1;
                    const int bar = pc.both ? pair_bar : quad_bar, threads = pc.both ? 64 : 128;
                    __threadfence();
                    named_barrier_sync(bar, threads);
                    if (speaks && lane == 0) {
                        int* counter = p.counters + (first_block * 2 + half) * 4 + quarter;
                        const bool last = atomicAdd(counter, 1) == blocks - 1;
                        if (last) *counter = 0;                        // (for the next launch)
                        last_flag[half * 4 + quarter] = last;
                    }
                    named_barrier_sync(bar, threads);
                    if (last_flag[half * 4 + quarter]) {
                        __threadfence();
                        const int warps = threads / 32, nth = pc.both ? hf : 2 * s + hf;
                        for (int i = nth; i < 32; i += warps) {        // a row per warp, four columns per lane
                            const int row_i = 32 * quarter + i, tok_r = row_i / pl.group, tok_i = tok0 + tok_r;
                            if (tok_r >= pl.tile_tokens || tok_i >= pl.tokens) break;
                            auto sums_of = [&](int b) {
                                const int block = first_block + b;
                                return ((long long)slot_of(block, b == 0 ? pc.start : part_begin(pl, block)) * 2 + half) * kTile + row_i;
                            };
                            float top = -INFINITY;
                            for (int b = lane; b < blocks; b += 32) top = fmaxf(top, __ldcg(&p.ml[sums_of(b)]).x);
#pragma unroll
                            for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                            float sum = 0.f;
                            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
                            for (int b = 0; b < blocks; ++b) {
                                const float2 ml = __ldcg(&p.ml[sums_of(b)]);
                                const float4 part = __ldcg(reinterpret_cast<const float4*>(p.o + sums_of(b) * kHeadDim) + lane);
                                // (no logit above -inf: sums of zero, or not a number, that count as they are)
                                const float f = ml.x > -INFINITY ? fast_exp2(ml.x - top) : 1.f;
                                sum = fmaf(ml.y, f, sum);
                                o.x = fmaf(part.x, f, o.x);
                                o.y = fmaf(part.y, f, o.y);
                                o.z = fmaf(part.z, f, o.z);
                                o.w = fmaf(part.w, f, o.w);
                            }
                            const float inv = 1.f / sum;
                            o = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
                            const int head_i = row_i - tok_r * pl.group;
                            const bool good = finite(o.x) && finite(o.y) && finite(o.z) && finite(o.w);
                            if (!__all_sync(0xffffffffu, good) && finite(sum) && finite(top)) o = redo_row(p, pc.unit, tok_i, head_i, top, sum);
                            store4(p.out, row_offset(p.out, at, tok_i, at.head * pl.group + head_i), 4 * lane, o);
                            if (p.norms && lane == 0) put_norm(row_i, top, inv);
                        }
                    }
                }
            }
            tmem_fence_before_sync();
        }
    }

    tmem_fence_before_sync();
    __syncthreads();
    if (warp == 0) {
        tmem_fence_after_sync();
        tmem_dealloc(tmem_base, kTmemCols);
    }
}

}  // namespace

ChunkPlan chunk_plan(int layers, int batch, int kv_heads, int group, int n, int tokens, int prefix_n, int prefix_share, int num_sms) {
    ChunkPlan pl;
    pl.layers = layers;
    pl.batch = batch;
    pl.kv_heads = kv_heads;
    pl.group = group;
    pl.tokens = tokens;
    pl.context = n - tokens;
    pl.tile_tokens = kTile / group < tokens ? kTile / group : tokens;
    pl.tiles = (tokens + pl.tile_tokens - 1) / pl.tile_tokens;
    pl.pairs = (pl.tiles + 1) / 2;
    pl.prefix_n = prefix_n;
    pl.prefix_tiles = (prefix_n + kTile - 1) / kTile;
    pl.prefix_share = prefix_share;
    long long steps = 0;
    for (int j = 0; j < pl.pairs; ++j) steps += chunk_key_tiles(pl, j);
    const long long work = (long long)layers * batch * kv_heads * steps;
    pl.unit_steps = steps > 0x40000000 ? 0 : (int)steps;
    if (num_sms > kChunkMaxBlocks) num_sms = kChunkMaxBlocks;
    pl.blocks = work > 0x40000000 ? 0 : (int)(work < num_sms ? work : num_sms);
    pl.per = pl.extra = 0;
    if (pl.blocks == 0) return pl;
    pl.per = (int)(work / pl.blocks);
    pl.extra = (int)(work % pl.blocks);
    return pl;
}

size_t chunk_ml_offset(int num_sms) {
    const size_t blocks = num_sms < kChunkMaxBlocks ? num_sms : kChunkMaxBlocks;
    return blocks * 2 * 2 * kTile * kHeadDim * sizeof(float);
}
size_t chunk_sums_bytes(int num_sms) { return chunk_ml_offset(num_sms) / kHeadDim / sizeof(float) * (kHeadDim * sizeof(float) + sizeof(float2)); }

cudaError_t chunk_prepare() { return cudaFuncSetAttribute(chunk_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem); }

bool chunk_query_map(const ChunkPlan& plan, const RowView& q, PrefixPool* out) {
    // q [layers][batch][tokens][heads][128]: box = 64 elements x G heads x a row tile's tokens, 128-byte swizzle; tokens behind the
    // last one read as zero
    static_assert(sizeof(PrefixPool) == sizeof(CUtensorMap), "");
    const cuuint64_t dims[5] = {(cuuint64_t)kHeadDim, (cuuint64_t)plan.group * plan.kv_heads, (cuuint64_t)plan.tokens, (cuuint64_t)plan.batch,
                                (cuuint64_t)plan.layers};
    const long long given[4] = {q.stride_head, q.stride_token, q.stride_batch, q.stride_layer};
    cuuint64_t strides[4];
    for (int i = 0; i < 4; ++i) strides[i] = dims[i + 1] > 1 ? (cuuint64_t)given[i] * 2 : (cuuint64_t)kRowBytes;
    const cuuint32_t box[5] = {64, (cuuint32_t)plan.group, (cuuint32_t)plan.tile_tokens, 1, 1};
    CUtensorMap map;
    if (!make_map(&map, q.data, 5, dims, strides, box)) return false;
    memcpy(out, &map, sizeof(map));
    return true;
}

cudaError_t chunk_launch(const ChunkPlan& plan, const ChunkArgs& a, cudaStream_t stream) {
    CUtensorMap mq, mkv, mpre;
    memcpy(&mq, a.q_map, sizeof(mq));
    memcpy(&mkv, a.pool, sizeof(mkv));
    memcpy(&mpre, a.prefix_pool ? a.prefix_pool : a.pool, sizeof(mpre));
    ChunkParams p;
    p.plan = plan;
    p.pages = a.pages;
    p.prefix_pages = a.prefix_pages;
    p.page_table = a.page_table;
    p.prefix_table = a.prefix_table;
    p.pages_per_unit = a.pages_per_unit;
    p.total_pages = a.total_pages;
    p.prefix_pages_per_unit = a.prefix_pages_per_unit;
    p.prefix_total_pages = a.prefix_total_pages;
    p.q = a.q;
    p.out = a.out;
    p.o = a.o;
    p.ml = a.ml;
    p.counters = a.counters;
    p.norms = a.norms;
    p.status = a.status;
    p.scale_log2 = 1.4426950408889634f / sqrtf((float)kHeadDim);
    p.wait_limit_ns = a.wait_limit_ns;
    p.stop_after_tiles = a.stop_after_tiles;
    chunk_kernel<<<plan.blocks, kThreads, kSmem, stream>>>(mq, mkv, mpre, p);
    return cudaGetLastError();
}

}  // namespace lzk
