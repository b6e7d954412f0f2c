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
// so a causal chunk leaves no block idle and a few rows over a long cache are spread over all SMs; short items stay whole, one per block.
// An item that one block has for itself is written out directly; the sums of one that several blocks share go through memory, and the
// last of them to arrive joins them, or join_kernel where they are many: in the order of the blocks, the same bits every time.
//
// P is one bf16 term (a weight is off by at most 2^-8 of itself, and errors of different keys do not add up in one direction:
// outputs are 0.0023 off in the mean square where their own rounding to bf16 is 0.0017) and l is summed in fp32 before that rounding:
// a second term, as the kernels for single tokens have it, would be another P V product, half as much again for the tensor core, whose
// power is what limits a long chunk.
//
// What bounds it.  Long chunks: power, and behind it a stream's chain of logits, weights and products.  40 heads, 4096 tokens behind
// 28671: 1960 us in short runs (1.31 PFLOP/s), 2270 to 2290 over and over (1.13), the SM clock then near 1.5 GHz of 1.965; of the pair of
// streams' turn of 3240 clocks the tensor core works 2050 (62 % under a profiler), 1830 are the softmax of one stream, the rest
// its hand-overs; key tiles take 512 clocks of shared memory besides the products' own reads, which alone fill it.  Few tokens: HBM,
// 4 tokens of 32 sequences, 8196 keys: 330 to 363 us for 2.16 GB.  Between them beginnings and ends of items: 4 sequences, 511
// tokens behind 1000: 3 us besides 2 us a step for a whole item, 11 for the last one that is joined.
// Tried and not kept: half key tiles with logits ahead (N = 64 takes 48 clocks of shared memory per product where N = 128 takes 64: long
// document 2390 -> 2590); polynomials for a part of the exponentials (1 %); weights against the running reference with the maximum
// beside them (8 % slower); polling instead of sleeping on barriers (none); two threads per row (2 to 8 % slower).
//
// Masks act on the logits by selection, so keys that a row does not see may hold anything.  Values enter a product, where a zero
// weight times infinity is no zero: value rows that no row of the item sees are zeroed in shared memory before they are used, and a
// row whose logits are finite and whose output is not -- a value inside the chunk, seen by later rows of the same
// item only, or one that the row sees itself -- is computed again over its own keys alone.
//
// Warp roles: warps 0-7 softmax and output, warp 8 TMA producer, warps 9 and 10 MMA issuers, one per stream.  All mbarrier waits are bounded.
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
constexpr int kStreamWarps = 4;                    // a thread per accumulator row
constexpr int kProducer = 2 * kStreamWarps, kIssuer = kProducer + 1, kThreads = 32 * (kIssuer + 3);      // an issuer per stream; a whole number of warpgroups
constexpr int kLeastSteps = 4;                     // of a block's part
constexpr int kJoinSteps = 10;                     // that a join costs: items whose parts would not be shorter by more stay whole
constexpr int kJoinFrom = 2, kJoinFromMany = 6;    // blocks that share an item: more are joined by a launch of their own (of many blocks itself)
constexpr long long kInStepBytes = 64ll << 20;     // of keys and values: more do not stay in L2 by themselves (2000 tokens alone, 8 MB: 54.6 us, in step 58.5)
constexpr float kRaiseMargin = 8.f;                // log2 units a logit may exceed the reference by

constexpr int kOffQ = 0;                           // two row tiles
constexpr int kOffRing = kOffQ + 2 * kOperandBytes;
constexpr int kOffMisc = kOffRing + kRing * kOperandBytes;
constexpr int kOffExchange = kOffMisc + 1024;      // [2 streams][128 rows] (m, l): what the streams' threads of a row tell each other
constexpr int kOffAside = kOffMisc + 576, kAsideInts = 14;      // per softmax warp
static_assert(kOffAside + 2 * kStreamWarps * kAsideInts * 4 <= kOffExchange, "");
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
    int beside;                                    // the next launch begins beside the end of this one
    int weighed;                                   // ... and the weights' launch beside the end of join_kernel
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

// The pieces of a block's part.  An item that the block before has begun comes last: so all blocks begin at an item's first key tile,
// and as whole items of a head are nearly of one length, the blocks of that head read the same key tiles at about the same time
// (4096 tokens behind 28671, over and over: 2430 us in the items' order, 2290 like this).
struct Walk {
    int x, end, unit, pair, start;
    int last_unit, last_pair, last_start;          // the item that comes last; a unit below 0: none (any more)
    __device__ __forceinline__ void item_done(const ChunkPlan& pl) {
        start += chunk_item_steps(pl, pair);
        x = start;
        if (++pair == pl.pairs) {
            pair = 0;
            ++unit;
        }
    }
    __device__ __forceinline__ void begin(const ChunkPlan& pl, int block) {
        last_unit = -1;
        if (pl.whole) {                            // an item per block
            unit = block / pl.pairs;
            pair = block - unit * pl.pairs;
            start = unit * pl.unit_steps;
            for (int j = 0; j < pair; ++j) start += chunk_item_steps(pl, j);
            x = start;
            end = start + chunk_key_tiles(pl, pair);
            return;
        }
        x = part_begin(pl, block);
        end = part_begin(pl, block + 1);
        unit = x / pl.unit_steps;
        start = unit * pl.unit_steps;
        pair = 0;
        for (int n = chunk_item_steps(pl, 0); x - start >= n; n = chunk_item_steps(pl, ++pair)) start += n;
        if (x - start >= chunk_key_tiles(pl, pair)) item_done(pl);     // (behind the item's key tiles)
        if (pl.in_step && x > start && start + chunk_item_steps(pl, pair) < end) {
            last_unit = unit, last_pair = pair, last_start = start;
            item_done(pl);
        }
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
        if (pc.k1 == pc.kt) item_done(pl);
        if (x >= end && last_unit >= 0) {
            x = part_begin(pl, blockIdx.x), unit = last_unit, pair = last_pair, start = last_start;
            end = start + chunk_key_tiles(pl, pair);
            last_unit = -1;
        }
        return pc;
    }
};

// The accumulator's 128 columns times a factor per row.  (Few registers at a time: the caller's are full of logits.)
__device__ __forceinline__ void rescale(uint32_t cols, float f) {
#pragma unroll 1
    for (int c = 0; c < kHeadDim; c += 8) {
        float o[8];
        tmem_ld4(cols + c, o[0], o[1], o[2], o[3]);
        tmem_ld4(cols + c + 4, o[4], o[5], o[6], o[7]);
        tmem_wait_ld();
        tmem_st4(cols + c, o[0] * f, o[1] * f, o[2] * f, o[3] * f);
        tmem_st4(cols + c + 4, o[4] * f, o[5] * f, o[6] * f, o[7] * f);
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
// x[c] of lane q is 16-byte chunk c of the q-th row of its quad of lanes; afterwards x[j] of lane q is chunk q of row j.
__device__ __forceinline__ void turn_quads(uint32_t (&x)[4][4], int lane) {
#pragma unroll
    for (int bit = 1; bit < 4; bit <<= 1) {
        const bool up = lane & bit;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            if (c & bit) continue;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? x[c][w] : x[c | bit][w], bit);
                (up ? x[c][w] : x[c | bit][w]) = got;
            }
        }
    }
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }

// The last of the own keys [from, to) with a value that is not finite, or -1: a whole warp.
__device__ __noinline__ int last_bad_value(const ChunkParams& p, int unit, int from, int to) {
    const int lane = threadIdx.x & 31;
    for (int j = to - 1; j >= from; --j) {
        int32_t pp = p.page_table[(long long)unit * p.pages_per_unit + j / kPageTokens];
        if (pp < 0 || pp >= p.total_pages) pp = 0;
        const uint2 v = *reinterpret_cast<const uint2*>(p.pages + (size_t)pp * kPageBytes + kPageHalfBytes + (j % kPageTokens) * kRowBytes + lane * 8);
        const bool odd = !finite(bf16_lo_as_float(v.x)) || !finite(bf16_hi_as_float(v.x)) || !finite(bf16_lo_as_float(v.y)) || !finite(bf16_hi_as_float(v.y));
        if (__any_sync(0xffffffffu, odd)) return j;
    }
    return -1;
}

// Rows that are computed again side by side: a key or value that is fetched serves all of them.  65536 keys, 32 rows in each of eight warps:
// 690 ms one at a time, 283 two.  Few instructions count as well, also where none is ever run: three rows and longer unrolled loops, 166 ms,
// made calls without any such row slower by what no longer fits beside the rest of the kernels (64 tokens behind 30000: 44 -> 50 us).
constexpr int kRedoRows = 2;
constexpr unsigned long long kRedoNs = 20000;      // that a warp's rows take per key, at most: 4.3 us as above, with room

// Rows (lanes of `again`) that a value reached which they do not see, or see: the first kind again, over their own keys alone, for the
// references and sums that are known, from global memory.  A whole warp: a key per lane, then columns 4 lane .. + 3 of the outputs.
// The block's other warps wait meanwhile: chunk_launch() adds to their limit what it may take.
__device__ __noinline__ void redo_rows(const ChunkParams& p, int unit, int pair, int tile, int row, unsigned again, float m, float l, int col0, int cols) {
    const ChunkPlan& pl = p.plan;
    const int lane = threadIdx.x & 31;
    const int r_tok = row / pl.group, r_head = row - r_tok * pl.group, tok = tile * pl.tile_tokens + r_tok;
    const UnitAt at = unit_at(pl, unit);
    const int to = pl.context + min(pl.tokens, 2 * pl.tile_tokens * (pair + 1));       // (behind them there are zeros)
    const int bad = last_bad_value(p, unit, pl.context + tile * pl.tile_tokens + 1, to);
    __syncwarp();                                          // other lanes have stored parts of the rows that are stored again here
    again &= __ballot_sync(0xffffffffu, bad > pl.context + tok);
    const float inv = 1.f / l;
    while (again) {
        int who[kRedoRows], sees[kRedoRows];               // (where fewer are left, the last one several times)
        const uint4* q[kRedoRows];
        float ref[kRedoRows], acc[kRedoRows][4];
        int most = 0;
#pragma unroll
        for (int r = 0; r < kRedoRows; ++r) {
            who[r] = again ? __ffs(again) - 1 : who[r > 0 ? r - 1 : 0];
            again &= again - 1;                            // (0 stays 0)
            const int tok_r = __shfl_sync(0xffffffffu, tok, who[r]), head_r = __shfl_sync(0xffffffffu, r_head, who[r]);
            q[r] = reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(p.q.data) + row_offset(p.q, at, tok_r, at.head * pl.group + head_r));
            ref[r] = __shfl_sync(0xffffffffu, m, who[r]);
            sees[r] = pl.context + tok_r + 1;
            most = max(most, sees[r]);
            acc[r][0] = acc[r][1] = acc[r][2] = acc[r][3] = 0.f;
        }
#pragma unroll 1
        for (int own = 0; own < 2; ++own) {
            const int keys = own ? most : pl.prefix_n, total = own ? p.total_pages : p.prefix_total_pages;
            const int32_t* table = own ? p.page_table + (long long)unit * p.pages_per_unit
                                       : p.prefix_table + (long long)at.prefix_unit * p.prefix_pages_per_unit;
            const uint8_t* pool = own ? p.pages : p.prefix_pages;
#pragma unroll 1
            for (int base = 0; base < keys; base += 32) {  // (half a page: rows behind the last key are there, whatever they hold)
                const int32_t pp = table[base / kPageTokens];
                const uint8_t* page = pool + (size_t)(pp >= 0 && pp < total ? pp : 0) * kPageBytes;
                const int first = base % kPageTokens, kr = first + lane;
                float w[kRedoRows];
#pragma unroll
                for (int r = 0; r < kRedoRows; ++r) w[r] = 0.f;
#pragma unroll 1
                for (int c = 0; c < kChunksPerRow; ++c) {
                    const uint4 b = *reinterpret_cast<const uint4*>(page + kr * kRowBytes + swz_chunk(c, kr) * 16);
                    const uint32_t bw[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                    for (int r = 0; r < kRedoRows; ++r) {
                        const uint4 a = q[r][c];
                        const uint32_t aw[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            w[r] = fmaf(bf16_lo_as_float(aw[i]), bf16_lo_as_float(bw[i]), w[r]);
                            w[r] = fmaf(bf16_hi_as_float(aw[i]), bf16_hi_as_float(bw[i]), w[r]);
                        }
                    }
                }
#pragma unroll
                for (int r = 0; r < kRedoRows; ++r)        // (below zero: not seen)
                    w[r] = base + lane < (own ? sees[r] : keys) ? fast_exp2(fmaf(w[r], p.scale_log2, -ref[r])) : -1.f;
#pragma unroll 1
                for (int i0 = 0; i0 < 32; i0 += 4) {
                    uint2 v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int vr = first + i0 + i;
                        v[i] = *reinterpret_cast<const uint2*>(page + kPageHalfBytes + vr * kRowBytes + swz_chunk(lane >> 1, vr) * 16 + (lane & 1) * 8);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int r = 0; r < kRedoRows; ++r) {
                            const float wi = __shfl_sync(0xffffffffu, w[r], i0 + i);
                            if (wi < 0.f) continue;
                            acc[r][0] = fmaf(wi, bf16_lo_as_float(v[i].x), acc[r][0]);
                            acc[r][1] = fmaf(wi, bf16_hi_as_float(v[i].x), acc[r][1]);
                            acc[r][2] = fmaf(wi, bf16_lo_as_float(v[i].y), acc[r][2]);
                            acc[r][3] = fmaf(wi, bf16_hi_as_float(v[i].y), acc[r][3]);
                        }
                }
            }
        }
#pragma unroll
        for (int r = 0; r < kRedoRows; ++r) {
            const float inv_r = __shfl_sync(0xffffffffu, inv, who[r]);
            const int tok_r = __shfl_sync(0xffffffffu, tok, who[r]), head_r = __shfl_sync(0xffffffffu, r_head, who[r]);
            if (4 * lane >= col0 && 4 * lane < col0 + cols)
                store4(p.out, row_offset(p.out, at, tok_r, at.head * pl.group + head_r), 4 * lane,
                       make_float4(acc[r][0] * inv_r, acc[r][1] * inv_r, acc[r][2] * inv_r, acc[r][3] * inv_r));
        }
    }
}

// What finish_piece() is told: by value, so that nothing of it is fetched from the parameters there.
struct Finish {
    uint8_t* out;                                  // of this thread's row; null: no such row
    float4* o;                                     // shared sums, slot 0
    float2* ml;
    int* counter;                                  // of this tile's quarter; null: join_kernel joins
    float* norm;                                   // of this thread's row, or null
    int dtype;
    int blocks, first_block, slot0;                // that share the item (1: whole), and the first one's slot
    int own_slot;
    int unit, pair;
    bool both, two;                                // two row tiles, a stream each; else one, and do both streams have a key tile of it?
};

// A piece's sums, for the warps of rows that exist: the output of an item that is the block's own, else its share in memory, and from
// the last block of the item to come here the output of all.  (Not inlined: the loop over the keys needs the registers.)
__device__ __noinline__ void finish_piece(const ChunkParams* p, uint8_t* smem, uint32_t tmem_base, const Finish f, float m, float l) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int s = warp / kStreamWarps, quarter = warp & 3, row = 32 * quarter + lane;
    const uint32_t lane_base = tmem_base + ((uint32_t)(32 * quarter) << 16);
    const int both_bar = 1 + quarter;                      // of the two streams' warps of 32 rows
    const bool whole = f.blocks == 1, speaks = f.both || s == 0;       // one thread per row
    const int half = f.both ? s : 0;
    // the columns of this thread's row that are its own from here on: all, or, of a single row tile, half of them
    int col0 = 0, cols = kHeadDim;
    float f0 = 1.f, f1 = 0.f;                              // factors of the two streams' accumulators
    if (!f.both) {
        // (Each stream's warps have waited for their own accumulator; the barrier passes that on.)
        float2* ml = reinterpret_cast<float2*>(smem + kOffExchange) + row;
        ml[s * kTile] = make_float2(m, l);
        tmem_fence_before_sync();
        named_barrier_sync(both_bar, 64);
        tmem_fence_after_sync();
        const float2 a0 = ml[0], a1 = ml[kTile];
        m = fmaxf(a0.x, a1.x);
        f0 = a0.x > -INFINITY ? fast_exp2(a0.x - m) : 1.f;
        f1 = a1.x > -INFINITY ? fast_exp2(a1.x - m) : 1.f;
        l = a0.y * f0 + a1.y * f1;                         // (a stream without a tile has m = -inf, l = 0)
        col0 = 64 * s;
        cols = 64;
    }
    auto own_sums = [&](int c, float (&o)[32]) {           // columns c .. c + 31 of the accumulator
        if (f.both) {
            tmem_ld32(lane_base + kColO + s * 128 + c, o);
            tmem_wait_ld();
        } else {
            float o1[32];
            tmem_ld32(lane_base + kColO + c, o);
            tmem_ld32(lane_base + kColO + 128 + c, o1);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = o[i] * f0 + (f.two ? o1[i] * f1 : 0.f);
        }
    };
    // Sums in memory, 16 bytes of a row at a time, the rows of a tile side by side: a block has at most two pieces of shared
    // items, one at either end of its part.
    auto tile_of = [&](int slot) { return (slot * 2 + half) * kTile; };
    auto slot_of = [&](int b) { return b == 0 ? f.slot0 : 2 * (f.first_block + b); };
    bool emits = whole;
    if (!whole) {
        if (f.out && speaks) f.ml[tile_of(f.own_slot) + row] = make_float2(m, l);
        float4* dst = f.o + (long long)tile_of(f.own_slot) * (kHeadDim / 4) + row;
#pragma unroll 1
        for (int c = col0; c < col0 + cols; c += 32) {
            float o[32];
            own_sums(c, o);
            if (!f.out) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) dst[(c / 4 + i) * kTile] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
        }
        if (f.counter) {
            // the last block of the item to come here joins the sums of all
            volatile int* last_flag = reinterpret_cast<volatile int*>(smem + kOffMisc + 512 + 8) + half * 4 + quarter;
            auto all_here = [&] {
                if (f.both)
                    __syncwarp();
                else
                    named_barrier_sync(both_bar, 64);
            };
            __threadfence();
            all_here();
            if (speaks && lane == 0) {
                const bool last = atomicAdd(f.counter, 1) == f.blocks - 1;
                if (last) *f.counter = 0;                      // (for the next launch)
                *last_flag = last;
            }
            all_here();
            emits = *last_flag != 0;
            if (emits) {
                __threadfence();
                m = -INFINITY;
                l = 0.f;
                if (f.out) {
#pragma unroll 4
                    for (int b = 0; b < f.blocks; ++b) {
                        const float2 ml = __ldcg(&f.ml[tile_of(slot_of(b)) + row]);
                        const float top = fmaxf(m, ml.x);
                        if (m > -INFINITY) l *= fast_exp2(m - top);
                        m = top;
                        l = fmaf(ml.y, ml.x > -INFINITY ? fast_exp2(ml.x - m) : 1.f, l);
                    }
                }
            }
        }
    }
    if (emits) {
        // quads of lanes hand each other's rows round, so that a row's 64 bytes are stored by neighbours
        uint8_t* out_of[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) out_of[j] = reinterpret_cast<uint8_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(f.out), (lane & ~3) + j));
        const float inv = 1.f / l;
        const uint64_t inv2 = pack2(inv, inv), zero2 = pack2(0.f, 0.f);
        uint64_t odd = zero2;                              // (not a number as soon as an output is not finite)
        const bool wide = f.dtype == kTypeF32;
        auto put_quads = [&](uint32_t (&x)[4][4], int byte) {
            turn_quads(x, lane);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (out_of[j]) *reinterpret_cast<uint4*>(out_of[j] + byte + 16 * (lane & 3)) = make_uint4(x[j][0], x[j][1], x[j][2], x[j][3]);
        };
#pragma unroll 1
        for (int c = col0; c < col0 + cols; c += 32) {
            float o[32];
            if (whole) {
                own_sums(c, o);
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = 0.f;
#pragma unroll 2
                for (int b = 0; b < f.blocks && f.out; ++b) {      // (512 bytes of a row in flight)
                    const int from = tile_of(slot_of(b));
                    const float top = __ldcg(&f.ml[from + row].x);
                    const float4* src = f.o + (long long)from * (kHeadDim / 4) + row;
                    float4 v4[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) v4[i] = __ldcg(&src[(c / 4 + i) * kTile]);
                    // (no logit above -inf: sums of zero, or not a number, that count as they are)
                    const float w = top > -INFINITY ? fast_exp2(top - m) : 1.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        o[4 * i] = fmaf(v4[i].x, w, o[4 * i]);
                        o[4 * i + 1] = fmaf(v4[i].y, w, o[4 * i + 1]);
                        o[4 * i + 2] = fmaf(v4[i].z, w, o[4 * i + 2]);
                        o[4 * i + 3] = fmaf(v4[i].w, w, o[4 * i + 3]);
                    }
                }
            }
            uint32_t x[4][4];
            if (wide) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint64_t v = mul2(pack2(o[16 * h + 2 * i], o[16 * h + 2 * i + 1]), inv2);
                        odd = fma2(v, zero2, odd);
                        float v0, v1;
                        unpack2(v, v0, v1);
                        x[i >> 1][2 * (i & 1)] = __float_as_uint(v0);
                        x[i >> 1][2 * (i & 1) + 1] = __float_as_uint(v1);
                    }
                    put_quads(x, 4 * (c + 16 * h));
                }
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint64_t v = mul2(pack2(o[2 * i], o[2 * i + 1]), inv2);
                    odd = fma2(v, zero2, odd);
                    float v0, v1;
                    unpack2(v, v0, v1);
                    x[i >> 2][i & 3] = pack_pair(v0, v1, f.dtype);
                }
                put_quads(x, 2 * c);
            }
        }
        float odd0, odd1;
        unpack2(odd, odd0, odd1);
        const bool sound = odd0 + odd1 == 0.f;
        if (f.norm && speaks) {
            f.norm[0] = -m;
            f.norm[kTile] = inv;
        }
        const unsigned again = __ballot_sync(0xffffffffu, f.out && !sound && finite(l) && finite(m));
        if (again) redo_rows(*p, f.unit, f.pair, 2 * f.pair + half, row, again, m, l, col0, cols);
    }
    if (!f.both) {
        tmem_fence_before_sync();
        named_barrier_sync(both_bar, 64);                  // both are done with both accumulators and the exchange
    }
}

// The sums of items that several blocks share, where many share one.  A block of threads per 32 rows of a row tile and 32 columns: a
// thread has a row, eight columns and every fourth of the item's blocks, kJoinBatch of them in flight, and the four parts are added up
// in order.  Latency bounds it: in the chunk kernel the last block to come has all of an item's sums to fetch by itself (1 token behind
// 30000, 2 KV heads: 67 us, like this 18.4; 4 tokens behind 131071, 8 KV heads: 108 and 89, of which 82 are the bytes).
constexpr int kJoinColumns = 8, kJoinGroups = 4, kJoinParts = 4, kJoinBatch = 8;
constexpr int kJoinThreads = 32 * kJoinGroups * kJoinParts;       // (and registers that an SM holds one block of)
// Shared memory that it asks for and does not use: without it 32 tokens behind 16000 take 25.7 us
// instead of 24.8, 16 behind 65535 54.3 instead of 53.5, others the same.
constexpr int kJoinSmem = 100 * 1024;

__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ ChunkParams p) {
    __shared__ float2 part_ml[kJoinParts][32];
    __shared__ float part_o[kJoinParts][kJoinGroups * kJoinColumns][32];
    const ChunkPlan& pl = p.plan;
    if (p.weighed) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31, group = (threadIdx.x >> 5) % kJoinGroups, part = (threadIdx.x >> 5) / kJoinGroups;
    constexpr int kAcross = kHeadDim / (kJoinGroups * kJoinColumns);
    const int col0 = (blockIdx.z % kAcross * kJoinGroups + group) * kJoinColumns;
    const int unit = blockIdx.x / pl.pairs, pair = blockIdx.x - unit * pl.pairs, half = blockIdx.y, tile = 2 * pair + half;
    const int row = 32 * (blockIdx.z / kAcross) + lane, r_tok = row / pl.group, tok = tile * pl.tile_tokens + r_tok;
    const bool valid = r_tok < pl.tile_tokens && tok < pl.tokens;
    int start = unit * pl.unit_steps;
    for (int j = 0; j < pair; ++j) start += chunk_item_steps(pl, j);
    const int first_block = block_of(pl, start), blocks = block_of(pl, start + chunk_key_tiles(pl, pair) - 1) - first_block + 1;
    const int slot0 = 2 * first_block + (start == part_begin(pl, first_block) ? 0 : 1);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (blocks == 1 || tile >= pl.tiles) return;           // (whole: the output is there)
    const int some = valid ? blocks : 0;
    float m = -INFINITY, l = 0.f, o[kJoinColumns] = {};
    for (int b0 = part; b0 < some; b0 += kJoinParts * kJoinBatch) {
        float2 ml[kJoinBatch];
        float4 v[kJoinBatch][kJoinColumns / 4];
#pragma unroll
        for (int i = 0; i < kJoinBatch; ++i) {
            const int b = b0 + kJoinParts * i;
            ml[i] = make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int c = 0; c < kJoinColumns / 4; ++c) v[i][c] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (b >= some) continue;
            const int from = ((b == 0 ? slot0 : 2 * (first_block + b)) * 2 + half) * kTile;
            ml[i] = __ldcg(&p.ml[from + row]);
            const float4* src = reinterpret_cast<const float4*>(p.o) + (long long)from * (kHeadDim / 4) + row;
#pragma unroll
            for (int c = 0; c < kJoinColumns / 4; ++c) v[i][c] = __ldcg(&src[(col0 / 4 + c) * kTile]);
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < kJoinBatch; ++i) top = fmaxf(top, ml[i].x);
        // (no logit above -inf: sums of zero, or not a number, that count as they are)
        auto factor = [&](float x) { return x > -INFINITY ? fast_exp2(x - top) : 1.f; };
        const float f = factor(m);
        m = top;
        l *= f;
#pragma unroll
        for (int k = 0; k < kJoinColumns; ++k) o[k] *= f;
#pragma unroll
        for (int i = 0; i < kJoinBatch; ++i) {
            const float w = factor(ml[i].x);
            l = fmaf(ml[i].y, w, l);
#pragma unroll
            for (int c = 0; c < kJoinColumns / 4; ++c) {
                o[4 * c] = fmaf(v[i][c].x, w, o[4 * c]);
                o[4 * c + 1] = fmaf(v[i][c].y, w, o[4 * c + 1]);
                o[4 * c + 2] = fmaf(v[i][c].z, w, o[4 * c + 2]);
                o[4 * c + 3] = fmaf(v[i][c].w, w, o[4 * c + 3]);
            }
        }
    }
    if (group == 0) part_ml[part][lane] = make_float2(m, l);
#pragma unroll
    for (int k = 0; k < kJoinColumns; ++k) part_o[part][group * kJoinColumns + k][lane] = o[k];
    __syncthreads();
    if (part > 0) return;
    float2 ml[kJoinParts];
    m = -INFINITY;
#pragma unroll
    for (int i = 0; i < kJoinParts; ++i) {
        ml[i] = part_ml[i][lane];
        m = fmaxf(m, ml[i].x);
    }
    l = 0.f;
#pragma unroll
    for (int k = 0; k < kJoinColumns; ++k) o[k] = 0.f;
#pragma unroll
    for (int i = 0; i < kJoinParts; ++i) {
        const float w = ml[i].x > -INFINITY ? fast_exp2(ml[i].x - m) : 1.f;
        l = fmaf(ml[i].y, w, l);
#pragma unroll
        for (int k = 0; k < kJoinColumns; ++k) o[k] = fmaf(part_o[i][group * kJoinColumns + k][lane], w, o[k]);
    }
    const float inv = 1.f / l;
    const UnitAt at = unit_at(pl, unit);
    const long long to = row_offset(p.out, at, tok, at.head * pl.group + row - r_tok * pl.group);
    float odd = 0.f;                                       // (not a number as soon as an output is not finite)
#pragma unroll
    for (int i = 0; i < kJoinColumns; i += 4) {
        const float4 v = make_float4(o[i] * inv, o[i + 1] * inv, o[i + 2] * inv, o[i + 3] * inv);
        odd = fmaf(v.x, 0.f, fmaf(v.y, 0.f, fmaf(v.z, 0.f, fmaf(v.w, 0.f, odd))));
        if (valid) store4(p.out, to, col0 + i, v);
    }
    if (p.norms && col0 == 0 && valid) {
        float* norm = p.norms + ((long long)unit * pl.tiles + tile) * 2 * kTile + row;
        norm[0] = -m;
        norm[kTile] = inv;
    }
    const unsigned again = __ballot_sync(0xffffffffu, valid && !(odd == 0.f) && finite(l) && finite(m));
    if (again) redo_rows(p, unit, pair, tile, row, again, m, l, col0, kJoinColumns);
}

__global__ void __launch_bounds__(kThreads, 1)
chunk_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_kv, const __grid_constant__ CUtensorMap map_prefix,
             const __grid_constant__ ChunkParams p) {
    extern __shared__ __align__(1024) uint8_t smem[];
    Bars* bars = reinterpret_cast<Bars*>(smem + kOffMisc);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kOffMisc + 512);      // then the abort flag, and [2 streams][4 quarters] of finish_piece()
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const ChunkPlan& pl = p.plan;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (p.beside) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
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
    // the producer's first page numbers, asked for before everything else
    KeyPages first_pages;
    if (warp == kProducer) {
        if (lane == 0) {
            prefetch_map(&map_q);
            prefetch_map(&map_kv);
        }
        if (walk.more()) first_pages.open(p, walk.unit, unit_at(pl, walk.unit), walk.x - walk.start);
    }
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
            KeyPages k_pages = first_pages, v_pages;
            if (rr.count > 0) k_pages.open(p, pc.unit, at, pc.k0);
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
            const int ahead = pc.both ? 1 : 2, nt = pc.tiles();
            auto load_k = [&](int j) {
                // diagnostics: no copy beyond the first stop_after_tiles K tiles
                if (p.stop_after_tiles >= 0 && k_tiles >= p.stop_after_tiles) ok = false;
                ++k_tiles;
                if (ok) load_tile(k_pages, pc.k0 + j, 0);
            };
            auto load_q = [&](int s) {
                const uint32_t qs = qr.stage(2);
                wait_on(&bars->q_empty[qs], qr.parity(2) ^ 1u);
                if (!ok) return;
                uint8_t* dst = smem + kOffQ + qs * kOperandBytes;
                const int tok = (2 * pc.pair + s) * pl.tile_tokens;
                if (elect_one()) {
                    mbar_arrive_expect_tx(&bars->q_full[qs], q_bytes);
                    tma_load_5d(dst, &map_q, 0, at.head * pl.group, tok, at.seq, at.layer, &bars->q_full[qs]);
                    tma_load_5d(dst + kBoxBytes, &map_q, 64, at.head * pl.group, tok, at.seq, at.layer, &bars->q_full[qs]);
                }
                __syncwarp();
                ++qr.count;
            };
            // The first keys come before the queries, whose slots are free only when the last logits of the piece before are done; at
            // the start the queries need no page number.
            const bool early = rr.count == 0;
            for (int i = 0; i < 2; ++i) {
                if ((i == 0) == early)
                    for (int s = 0; s < (pc.both ? 2 : 1) && ok; ++s) load_q(s);
                else
                    for (int j = 0; j < min(ahead, nt) && ok; ++j) load_k(j);
            }
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
    } else if (warp >= kIssuer && warp < kIssuer + 2) {
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
        // O += P V for the first or the second 64 keys
        auto issue_o = [&](uint32_t st, int part, bool first) {
            const uint64_t b = v_desc + st * kStep;
#pragma unroll
            for (int i = 0; i < 4; ++i) {           // 16 keys per instruction
                const int s8 = 4 * part + i;
                umma_bf16_ts(o_col, s_col + s8 * 8, b + s8 * (2048 >> 4), instr_desc(true), !first || i > 0);
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
    } else if (warp < kProducer) {
        // ------------------------------------------------------------------ softmax and output
        // Accumulator row = TMEM lane = thread: a row's logits are all in one thread's registers, so nothing is exchanged between the
        // maximum and the weights (two threads per row halve the exponentials' chain, but not their time on the special function
        // units, and wait for each other).
        const int s = warp / kStreamWarps, quarter = warp & 3, row = 32 * quarter + lane;
        const uint32_t s_cols = tmem_base + ((uint32_t)(32 * quarter) << 16) + kColS + s * 128;                // (O is kColO - kColS further)
        uint32_t s_uses = 0, o_uses = 0;
        // A warp whose wait gives up goes on through the same loops, so that its partner's barriers get all their threads, but waits
        // for nothing any more; what it computes means nothing.
        bool dead = false;
        auto wait_on = [&](uint64_t* bar, uint32_t parity) {
            const bool gave_up = dead || !wait_bar(bar, parity, abort_flag, p.status, limit);
            dead = __any_sync(0xffffffffu, gave_up);
        };
        const int r_tok = row / pl.group;                              // token of this row inside its tile
        // Where the walk is waits in shared memory: the loop over the keys needs the registers.
        volatile int* aside = reinterpret_cast<volatile int*>(smem + kOffAside) + warp * kAsideInts;
        auto put_aside = [&](const Walk& w) {
            aside[0] = w.x, aside[1] = w.end, aside[2] = w.unit, aside[3] = w.pair, aside[4] = w.start;    // (all lanes the same)
            aside[11] = w.last_unit, aside[12] = w.last_pair, aside[13] = w.last_start;
            __syncwarp();
        };
        put_aside(walk);
        while (aside[0] < aside[1]) {
            float m = -INFINITY, l = 0.f;
            bool warp_on;
            int nt;
            {
                Walk here{aside[0], aside[1], aside[2], aside[3], aside[4], aside[11], aside[12], aside[13]};
                const Piece pc = here.next(pl);
                __syncwarp();
                aside[5] = pc.unit, aside[6] = pc.pair, aside[7] = pc.start, aside[8] = pc.kt, aside[9] = pc.k0, aside[10] = pc.k1;
                put_aside(here);
                nt = pc.stream_tiles(s);
                const int tok0 = (2 * pc.pair + (pc.both ? s : 0)) * pl.tile_tokens, tok = tok0 + r_tok;
                const bool valid = r_tok < pl.tile_tokens && tok < pl.tokens;
                warp_on = __any_sync(0xffffffffu, valid);
                const float margin = valid ? kRaiseMargin : INFINITY;  // (a row that does not exist raises nothing)
                // keys before the first one of a tile, and own keys that this row sees, and that every row of the tile sees; of
                // the prefix's tiles all rows see the same
                int key0 = pc.key_tile(s, 0) * kTile - pl.prefix_tiles * kTile;
                const int sees = pl.context + (valid ? tok + 1 : pl.tokens), all_see = pl.context + tok0 + 1, step = pc.both ? kTile : 2 * kTile;
#pragma unroll 1
                for (int t = 0; t < nt; ++t, key0 += step) {
                    wait_on(&bars->s_full[s], s_uses & 1u);
                    ++s_uses;
                    tmem_fence_after_sync();
                    if (warp_on) {
                        float v[4][32];
#pragma unroll
                        for (int c = 0; c < 4; ++c) tmem_ld32(s_cols + 32 * c, v[c]);
                        tmem_wait_ld();
                        const int all_to = key0 < 0 ? pl.prefix_n - pl.prefix_tiles * kTile - key0 : all_see - key0;
                        if (all_to < kTile) {                          // this row sees the first `to` of the keys
                            const int to = key0 < 0 ? all_to : sees - key0;
#pragma unroll
                            for (int c = 0; c < 4; ++c)
#pragma unroll
                                for (int i = 0; i < 32; ++i) v[c][i] = 32 * c + i < to ? v[c][i] : -INFINITY;
                        }
                        float mx[4];
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            mx[c] = fmaxf(v[c][0], v[c][1]);
#pragma unroll
                            for (int i = 2; i < 32; i += 2) mx[c] = fmax3(mx[c], v[c][i], v[c][i + 1]);
                        }
                        const float top = fmax3(mx[0], mx[1], fmaxf(mx[2], mx[3])) * p.scale_log2;
                        if (__any_sync(0xffffffffu, top > m + margin)) {
                            const float next = fmaxf(m, top);
                            const float f = m == next ? 1.f : fast_exp2(m - next);
                            if (t > 0) rescale(s_cols + kColO - kColS, f);
                            l *= f;
                            m = next;
                        }
                        const float ref = m == -INFINITY ? 0.f : m;      // every logit -inf: all weights are zero
                        const uint64_t scale2 = pack2(p.scale_log2, p.scale_log2), minus2 = pack2(-ref, -ref);
                        uint64_t sum0 = pack2(0.f, 0.f), sum1 = sum0;
#pragma unroll
                        for (int c = 0; c < 8; ++c) {                      // 16 columns at a time
                            if (c == 4) {                                  // the first half of P is there: its product may begin
                                tmem_wait_st();
                                tmem_fence_before_sync();
                                __syncwarp();
                                if (lane == 0) mbar_arrive(&bars->p_full[s][0]);
                            }
                            uint32_t w16[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                float e0, e1;
                                unpack2(fma2(pack2(v[c >> 1][16 * (c & 1) + 2 * i], v[c >> 1][16 * (c & 1) + 2 * i + 1]), scale2, minus2), e0, e1);
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
            }
            // ---- the piece's sums
            if (nt > 0) {
                wait_on(&bars->o_full[s], o_uses & 1u);
                ++o_uses;
            }
            tmem_fence_after_sync();
            if (warp_on) {
                const Piece pc{aside[5], aside[6], aside[7], aside[8], aside[9], aside[10], 2 * aside[6] + 1 < pl.tiles};
                const UnitAt at = unit_at(pl, pc.unit);
                const int tile = 2 * pc.pair + (pc.both ? s : 0), tok = tile * pl.tile_tokens + r_tok, half = pc.both ? s : 0;
                const bool valid = r_tok < pl.tile_tokens && tok < pl.tokens;
                Finish f;
                f.dtype = p.out.dtype;
                f.out = valid ? reinterpret_cast<uint8_t*>(const_cast<void*>(p.out.data)) +
                                    row_offset(p.out, at, tok, at.head * pl.group + row - r_tok * pl.group) * (f.dtype == kTypeF32 ? 4 : 2)
                              : nullptr;
                f.norm = valid && p.norms ? p.norms + ((long long)pc.unit * pl.tiles + tile) * 2 * kTile + row : nullptr;
                f.o = reinterpret_cast<float4*>(p.o);
                f.ml = p.ml;
                f.unit = pc.unit;
                f.pair = pc.pair;
                f.both = pc.both;
                f.two = pc.tiles() > 1;
                f.blocks = 1;
                f.first_block = f.slot0 = f.own_slot = 0;
                f.counter = nullptr;
                if (pc.tiles() != pc.kt) {
                    f.first_block = block_of(pl, pc.start);
                    f.blocks = block_of(pl, pc.start + pc.kt - 1) - f.first_block + 1;
                    f.slot0 = 2 * f.first_block + (pc.start == part_begin(pl, f.first_block) ? 0 : 1);
                    f.own_slot = 2 * (int)blockIdx.x + (pc.start + pc.k0 == part_begin(pl, blockIdx.x) ? 0 : 1);
                    if (!pl.joins) f.counter = p.counters + (f.first_block * 2 + half) * 4 + quarter;
                }
                finish_piece(&p, smem, tmem_base, f, m, l);
            }
            tmem_fence_before_sync();
        }
    } else {
        // ------------------------------------------------------------------ the last warp
        // Rows of a row tile that no query row ever fills (a chunk of few tokens; 128 is no multiple of G) become zeros.  An accumulator
        // row depends on its own row only and nobody looks at these, so it does not matter when; but products of zeros take less power, and
        // power limits the clock (4 tokens of 32 sequences, over and over: 366 -> 356 us).
        const int filled = pl.tile_tokens * pl.group, each = (kTile - filled) * 8;     // 16-byte parts of half a slot
        for (int part = 0; part < 4; ++part)                                           // 2 slots x 2 halves of the rows
            for (int i = lane; i < each; i += 32) reinterpret_cast<uint4*>(smem + kOffQ + part * kBoxBytes + filled * 128)[i] = make_uint4(0u, 0u, 0u, 0u);
        fence_proxy_async();
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
    for (int j = 0; j < pl.pairs; ++j) steps += chunk_item_steps(pl, j);
    const long long work = (long long)layers * batch * kv_heads * steps;
    pl.unit_steps = steps > 0x40000000 ? 0 : (int)steps;
    if (num_sms > kChunkMaxBlocks) num_sms = kChunkMaxBlocks;
    const long long items = (long long)layers * batch * kv_heads * pl.pairs;
    const long long parts = (work + kLeastSteps - 1) / kLeastSteps;
    pl.blocks = work > 0x40000000 ? 0 : (int)(parts < num_sms ? parts : num_sms);
    pl.per = pl.extra = 0;
    pl.whole = pl.joins = pl.in_step = false;
    if (pl.blocks == 0) return pl;
    // Items that several blocks share cost a join, so items whose parts would not be much shorter stay whole, one per block, however
    // unequal they are (8 KV heads, 32 heads: 200 tokens alone 12.7 us whole, 22.7 in equal parts; 500 behind 500 24.6 and 27.9; 500 behind
    // 2500, 27 steps against 12: 50.8 whole, 40.4 in parts).
    pl.whole = items <= num_sms && chunk_item_steps(pl, pl.pairs - 1) <= work / pl.blocks + kJoinSteps;
    if (pl.whole) {
        pl.blocks = (int)items;
        return pl;
    }
    pl.per = (int)(work / pl.blocks);
    pl.extra = (int)(work % pl.blocks);
    pl.in_step = pl.pairs > 1 && (long long)layers * batch * kv_heads * chunk_key_tiles(pl, pl.pairs - 1) * 2 * kOperandBytes > kInStepBytes;
    const long long join_blocks = items * (pl.tiles > 1 ? 2 : 1) * ((pl.tile_tokens * group + 31) / 32) * (kHeadDim / (kJoinGroups * kJoinColumns));
    // The last block of an item to come joins it in the chunk kernel at the price of a launch for two or three; beyond that, or where the
    // join's own blocks, of which an SM holds one at a time, take more than two turns, beyond six, join_kernel does (64 tokens behind
    // 3000: 31.9 and 22.6 us; 200 behind 4000, 1024 blocks for the join, 4 to an item: 35.8 and 41.1; 100 behind 12000, 9 to an item: 57.2 and 41.0).
    if (chunk_key_tiles(pl, pl.pairs - 1) > (long long)(join_blocks <= 2 * num_sms ? kJoinFrom : kJoinFromMany) * pl.per) pl.joins = true;
    return pl;
}

size_t chunk_ml_offset(int num_sms) {
    const size_t blocks = num_sms < kChunkMaxBlocks ? num_sms : kChunkMaxBlocks;
    return blocks * 2 * 2 * kTile * kHeadDim * sizeof(float);
}
size_t chunk_sums_bytes(int num_sms) { return chunk_ml_offset(num_sms) / kHeadDim / sizeof(float) * (kHeadDim * sizeof(float) + sizeof(float2)); }

cudaError_t chunk_prepare() {
    const cudaError_t e = cudaFuncSetAttribute(join_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kJoinSmem);
    return e == cudaSuccess ? cudaFuncSetAttribute(chunk_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) : e;
}

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
    p.wait_limit_ns = a.wait_limit_ns + kRedoNs * (unsigned long long)(plan.prefix_n + plan.context + plan.tokens);
    p.stop_after_tiles = a.stop_after_tiles;
    p.beside = plan.joins || a.weighed;
    p.weighed = a.weighed;
    chunk_kernel<<<plan.blocks, kThreads, kSmem, stream>>>(mq, mkv, mpre, p);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || !plan.joins) return e;
    cudaLaunchAttribute beside = {};
    beside.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    beside.val.programmaticStreamSerializationAllowed = 1;
    const int rows = plan.tile_tokens * plan.group;
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(plan.layers * plan.batch * plan.kv_heads * plan.pairs, plan.tiles > 1 ? 2 : 1, (rows + 31) / 32 * (kHeadDim / (kJoinGroups * kJoinColumns)));
    c.blockDim = dim3(kJoinThreads);
    c.dynamicSmemBytes = kJoinSmem;
    c.stream = stream;
    c.attrs = &beside;
    c.numAttrs = 1;
    return cudaLaunchKernelEx(&c, join_kernel, p);
}

}  // namespace lzk
