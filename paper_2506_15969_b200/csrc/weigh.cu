// The weight that every cached token receives from a chunk of query rows, and the running sum of a decode step's.
//
// For own token j of a unit, over the T tokens of the chunk and the G heads of its KV head:
//   weight[j] (+)= 1 / G sum over rows r that see j of exp2(x_r[j] - m_r) / l_r
// with the logits x and the rows' references m and sums l as in chunk.cu, which leaves the last two in memory.  A row's sum is
// known only after all its keys, hence a second pass over the logits, but no second product: keys are the accumulator rows here
// (S = K Q^T), so a key's sum over the query rows stays in four threads' registers, in fp32 throughout, and is written once.
//
// An item is a pair of 128-key tiles of a unit with the row tiles of the chunk that see it; the walk over (item, row
// tile) is cut into equal contiguous parts, one per persistent block, as in chunk.cu; sums of an item that several blocks share go
// through memory and the last of them to arrive adds them up in order.  Three key tiles and the row tiles of three steps are in
// shared memory, and two pairs of logit tiles in tensor memory, so that the tensor core runs ahead of the exponentials.
//
// Bound by the exponentials, one per row and key (the tensor core needs half their time): 16 units, 4096 rows of 4096 tokens each, 160 to
// 187 us, special function units 70 % busy under a profiler (a quarter of them as polynomials of degree 5 on the fma pipe changed
// nothing; the next columns fetched while these are summed was slower); few rows: HBM,
// the keys once.
//
// Warp roles: warps 0-15 exponentials, warp 16 TMA producer, warp 17 MMA issuer.  All mbarrier waits are bounded.
#include <string.h>

#include "internal.h"
#include "tensor.cuh"

namespace lzk {

namespace {

constexpr int kTile = 128;                         // keys of a key tile, rows of a row tile
constexpr int kBoxBytes = kTile * 128;             // half an operand: 128 rows x 64 bf16
constexpr int kOperandBytes = 2 * kBoxBytes;
constexpr int kRing = 3;                           // row tiles in flight
constexpr int kExpWarps = 16;                      // four warps per 32 keys of both tiles, a quarter of the rows each
constexpr int kProducer = kExpWarps, kIssuer = kProducer + 1, kThreads = 32 * (kIssuer + 1);

constexpr int kKeys = 3;                           // key tiles in flight
constexpr int kOffK = 0;
constexpr int kOffRing = kOffK + kKeys * kOperandBytes;
constexpr int kOffNorms = kOffRing + kRing * kOperandBytes;     // [kRing][2][128]
constexpr int kNormBytes = 2 * kTile * 4;
constexpr int kOffParts = kOffNorms + kRing * kNormBytes;       // [3 quarters of the rows][2 key tiles][128]
constexpr int kSmem = kOffParts + 3 * 2 * kTile * 4;
constexpr uint32_t kTmemCols = 512;                // [2 buffers][2 key tiles][128]

struct Bars {
    uint64_t k_full[kKeys], k_empty[kKeys];
    uint64_t full[kRing], empty[kRing];
    uint64_t s_full[2], s_empty[2];                // [buffer]
    uint64_t drain;
};

struct WeighParams {
    WeighPlan plan;
    ChunkPlan chunk;
    const int32_t* page_table;
    const float* norms;                            // minus the reference, then 1 / l
    float* weights;
    float* sums;                                   // [2 blocks][2 key tiles][128]
    int32_t* counters;
    int32_t* status;
    int pages_per_unit, total_pages, capacity, add;
    float scale_log2, inv_group;
    unsigned long long wait_limit_ns;
    int stop_after_tiles;
};

__device__ __forceinline__ int part_begin(const WeighPlan& p, int block) { return block * p.per + min(block, p.extra); }
__device__ __forceinline__ int block_of(const WeighPlan& p, int x) {
    const int longer = p.extra * (p.per + 1);
    return x < longer ? x / (p.per + 1) : p.extra + (x - longer) / p.per;
}

// One block's part of an item: row tiles [q0, q1) of first .. tiles.
struct Piece {
    int unit, pair, start;                         // the item, and the step it starts at
    int first, q0, q1, tiles;
};

struct Walk {
    int x, end, unit, pair, start;
    __device__ __forceinline__ int steps(const WeighParams& p) const { return p.chunk.tiles - weigh_first_tile(p.chunk, pair); }
    __device__ __forceinline__ void begin(const WeighParams& p, int block) {
        const WeighPlan& pl = p.plan;
        x = part_begin(pl, block);
        end = part_begin(pl, block + 1);
        unit = x / pl.unit_steps;
        start = unit * pl.unit_steps;
        // items before the chunk's first token all take every row tile
        pair = min((x - start) / p.chunk.tiles, min(p.chunk.context / (2 * kTile), pl.pairs - 1));
        start += pair * p.chunk.tiles;
        for (int n = steps(p); x - start >= n; n = steps(p)) {
            start += n;
            ++pair;
        }
    }
    __device__ __forceinline__ bool more() const { return x < end; }
    __device__ __forceinline__ Piece next(const WeighParams& p) {
        Piece pc;
        pc.unit = unit;
        pc.pair = pair;
        pc.start = start;
        pc.tiles = p.chunk.tiles;
        pc.first = weigh_first_tile(p.chunk, pair);
        pc.q0 = pc.first + (x - start);
        pc.q1 = min(pc.tiles, pc.q0 + (end - x));
        x += pc.q1 - pc.q0;
        if (pc.q1 == pc.tiles) {
            start += pc.tiles - pc.first;
            if (++pair == p.plan.pairs) {
                pair = 0;
                ++unit;
            }
        }
        return pc;
    }
};

__device__ __forceinline__ uint64_t exp2_pair(uint64_t x) {
    float x0, x1;
    unpack2(x, x0, x1);
    return pack2(fast_exp2(x0), fast_exp2(x1));
}

__global__ void __launch_bounds__(kThreads, 1)
weigh_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_kv, const __grid_constant__ WeighParams p) {
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ Bars bars;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_word, last_flag[4];
    volatile int* abort_flag = &abort_word;
    const ChunkPlan& ch = p.chunk;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    Walk walk;
    walk.begin(p, blockIdx.x);

    if (threadIdx.x == 0) {
        for (int i = 0; i < kKeys; ++i) {
            mbar_init(&bars.k_full[i], 1);
            mbar_init(&bars.k_empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bars.s_full[i], 1);
            mbar_init(&bars.s_empty[i], kExpWarps);
        }
        for (int i = 0; i < kRing; ++i) {
            mbar_init(&bars.full[i], 1);
            mbar_init(&bars.empty[i], 1 + kExpWarps);       // the products, and everyone who reads the norms
        }
        mbar_init(&bars.drain, 1);
        abort_word = 0;
        fence_barrier_init();
    }
    if (warp == kProducer && lane == 0) {
        prefetch_map(&map_q);
        prefetch_map(&map_kv);
    }
    // (rows of a row tile that no query row fills hold whatever they hold: their columns are left out)
    if (warp == 0) {
        tmem_alloc(&tmem_slot, kTmemCols);
        tmem_relinquish_alloc_permit();
    }
    tmem_fence_before_sync();
    __syncthreads();
    tmem_fence_after_sync();
    const uint32_t tmem_base = tmem_slot;
    asm volatile("griddepcontrol.wait;" ::: "memory");     // (the chunk launch's norms)
    const unsigned long long limit = p.wait_limit_ns;

    if (warp == kProducer) {
        // ------------------------------------------------------------------ TMA producer
        Ring rr, kr;
        bool ok = true;
        int k_tiles = 0;
        const uint32_t q_bytes = (uint32_t)(ch.tile_tokens * ch.group) * 256u;
        auto wait_on = [&](uint64_t* bar, uint32_t parity) { ok = __all_sync(0xffffffffu, wait_bar(bar, parity, abort_flag, p.status, limit)); };
        while (walk.more() && ok) {
            const Piece pc = walk.next(p);
            const int head = pc.unit % ch.kv_heads, ls = pc.unit / ch.kv_heads;
            // diagnostics: no copy beyond the first stop_after_tiles K tiles
            if (p.stop_after_tiles >= 0 && k_tiles + 2 > p.stop_after_tiles) break;
            k_tiles += 2;
            const int last_page = (ch.context + ch.tokens - 1) / kPageTokens;
            int32_t page = p.page_table[(long long)pc.unit * p.pages_per_unit + min(4 * pc.pair + (lane & 3), last_page)];
            if (page < 0 || page >= p.total_pages) {
                atomicOr(p.status, kStatusBadIndex);
                page = 0;
            }
            for (int s = 0; s < 2 && ok; ++s) {            // a stream's tile: two pages, both halves of the rows
                const uint32_t ks = kr.stage(kKeys);
                const int32_t p0 = __shfl_sync(0xffffffffu, page, 2 * s), p1 = __shfl_sync(0xffffffffu, page, 2 * s + 1);
                wait_on(&bars.k_empty[ks], kr.parity(kKeys) ^ 1u);
                if (!ok) break;
                uint8_t* dst = smem + kOffK + ks * kOperandBytes;
                if (elect_one()) {
                    mbar_arrive_expect_tx(&bars.k_full[ks], kOperandBytes);
                    tma_load_3d(dst, &map_kv, 0, 0, p0, &bars.k_full[ks]);
                    tma_load_3d(dst + kBoxBytes / 2, &map_kv, 0, 0, p1, &bars.k_full[ks]);
                    tma_load_3d(dst + kBoxBytes, &map_kv, 64, 0, p0, &bars.k_full[ks]);
                    tma_load_3d(dst + kBoxBytes + kBoxBytes / 2, &map_kv, 64, 0, p1, &bars.k_full[ks]);
                }
                __syncwarp();
                ++kr.count;
            }
            for (int t = pc.q0; t < pc.q1 && ok; ++t) {
                const uint32_t st = rr.stage(kRing);
                wait_on(&bars.empty[st], rr.parity(kRing) ^ 1u);
                if (!ok) break;
                if (elect_one()) {
                    uint8_t* dst = smem + kOffRing + st * kOperandBytes;
                    mbar_arrive_expect_tx(&bars.full[st], q_bytes + kNormBytes);
                    tma_load_5d(dst, &map_q, 0, head * ch.group, t * ch.tile_tokens, ls % ch.batch, ls / ch.batch, &bars.full[st]);
                    tma_load_5d(dst + kBoxBytes, &map_q, 64, head * ch.group, t * ch.tile_tokens, ls % ch.batch, ls / ch.batch, &bars.full[st]);
                    bulk_load(smem + kOffNorms + st * kNormBytes, p.norms + ((long long)pc.unit * ch.tiles + t) * 2 * kTile, kNormBytes, &bars.full[st]);
                }
                __syncwarp();
                ++rr.count;
            }
        }
        // the copies already issued land before the block exits, whoever gives up and when
        auto drain = [&](uint64_t* full, const Ring& r, uint32_t n) {
            const uint32_t last = r.count < n ? r.count : n;
            for (uint32_t k = r.count - last; k < r.count; ++k)
                wait_bar(&full[k % n], (k / n) & 1u, abort_flag, p.status, limit, false);
        };
        drain(bars.full, rr, kRing);
        drain(bars.k_full, kr, kKeys);
    } else if (warp == kIssuer) {
        // ------------------------------------------------------------------ MMA issuer
        bool ok = true;
        auto wait_on = [&](uint64_t* bar, uint32_t parity) {
            if (ok) ok = __all_sync(0xffffffffu, wait_bar(bar, parity, abort_flag, p.status, limit));
        };
        Ring rr, kr, sr;
        const uint64_t k_desc = smem_desc(smem_u32(smem + kOffK), 16, 1024), q_desc = smem_desc(smem_u32(smem + kOffRing), 16, 1024);
        constexpr uint32_t kStep = kOperandBytes >> 4;
        while (walk.more() && ok) {
            const Piece pc = walk.next(p);
            uint32_t ks[2];
            for (int s = 0; s < 2; ++s, ++kr.count) {
                ks[s] = kr.stage(kKeys);
                wait_on(&bars.k_full[ks[s]], kr.parity(kKeys));
            }
            for (int t = pc.q0; t < pc.q1 && ok; ++t) {
                const uint32_t st = rr.stage(kRing), buf = sr.stage(2);
                wait_on(&bars.full[st], rr.parity(kRing));
                wait_on(&bars.s_empty[buf], sr.parity(2) ^ 1u);
                tmem_fence_after_sync();
                if (ok && elect_one()) {
                    for (int s = 0; s < 2; ++s) {
                        const uint64_t a = k_desc + ks[s] * kStep, b = q_desc + st * kStep;
#pragma unroll
                        for (int s8 = 0; s8 < 8; ++s8) {
                            const uint32_t off = ((s8 >> 2) * kBoxBytes + (s8 & 3) * 32) >> 4;
                            umma_bf16(tmem_base + (buf * 2 + s) * 128, a + off, b + off, instr_desc(false), s8 > 0);
                        }
                        if (t + 1 == pc.q1) umma_commit(&bars.k_empty[ks[s]]);
                    }
                    umma_commit(&bars.s_full[buf]);
                    umma_commit(&bars.empty[st]);
                }
                __syncwarp();
                ++rr.count;
                ++sr.count;
            }
        }
        // every MMA issued is complete before tensor memory goes back
        if (elect_one()) umma_commit(&bars.drain);
        __syncwarp();
        wait_bar(&bars.drain, 0, abort_flag, p.status, limit, false);
    } else {
        // ------------------------------------------------------------------ exponentials
        // Accumulator row = TMEM lane = key; a thread takes key `row` of both tiles and 32 of the 128 rows of the chunk, so that what it
        // fetches of the rows serves two exponentials.
        const int cq = warp >> 2, quarter = warp & 3, row = 32 * quarter + lane;
        const uint32_t lane_base = tmem_base + ((uint32_t)(32 * quarter) << 16) + 32 * cq;
        const int quad_bar = 1 + quarter;
        bool dead = false;
        auto wait_on = [&](uint64_t* bar, uint32_t parity) {
            const bool gave_up = dead || !wait_bar(bar, parity, abort_flag, p.status, limit);
            dead = __any_sync(0xffffffffu, gave_up);
        };
        Ring rr, sr;
        const uint64_t scale2 = pack2(p.scale_log2, p.scale_log2);
        const int n = ch.context + ch.tokens;
        float* parts = reinterpret_cast<float*>(smem + kOffParts) + row;       // [cq - 1][tile][128]
        while (walk.more()) {
            const Piece pc = walk.next(p);
            const int key0 = 2 * pc.pair * kTile + 32 * quarter;               // of this warp, in the first tile; kTile further in the second
            float sum[2] = {0.f, 0.f};
            for (int t = pc.q0; t < pc.q1; ++t) {
                const uint32_t st = rr.stage(kRing), buf = sr.stage(2);
                wait_on(&bars.full[st], rr.parity(kRing));                      // (the norms)
                wait_on(&bars.s_full[buf], sr.parity(2));
                tmem_fence_after_sync();
                const float* norm = reinterpret_cast<const float*>(smem + kOffNorms + st * kNormBytes) + 32 * cq;
                const int tok0 = t * ch.tile_tokens, rows = min(ch.tile_tokens, ch.tokens - tok0) * ch.group - 32 * cq;
                // Columns [0, rows) are rows of the chunk.  All of them see all keys of the warp in a tile that ends before them; none sees
                // keys behind the last token.
                if (rows > 0) {
                    float v[2][32];
                    tmem_ld32(lane_base + buf * 256, v[0]);
                    tmem_ld32(lane_base + buf * 256 + 128, v[1]);
                    tmem_wait_ld();
                    if (key0 + kTile + 31 <= ch.context + tok0 && rows >= 32) {
                        uint64_t c0[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)}, c1[2] = {c0[0], c0[0]};       // (sums of 32 rows first: short chains)
#pragma unroll
                        for (int i = 0; i < 32; i += 4) {
                            const float4 m = *reinterpret_cast<const float4*>(norm + i), f = *reinterpret_cast<const float4*>(norm + kTile + i);
#pragma unroll
                            for (int s = 0; s < 2; ++s) {
                                const uint64_t x0 = fma2(pack2(v[s][i], v[s][i + 1]), scale2, pack2(m.x, m.y));
                                const uint64_t x1 = fma2(pack2(v[s][i + 2], v[s][i + 3]), scale2, pack2(m.z, m.w));
                                c0[s] = fma2(exp2_pair(x0), pack2(f.x, f.y), c0[s]);
                                c1[s] = fma2(exp2_pair(x1), pack2(f.z, f.w), c1[s]);
                            }
                        }
#pragma unroll
                        for (int s = 0; s < 2; ++s) {
                            float a0, a1;
                            unpack2(add2(c0[s], c1[s]), a0, a1);
                            sum[s] += a0 + a1;
                        }
                    } else {
#pragma unroll
                        for (int s = 0; s < 2; ++s) {
                            const int key = key0 + s * kTile;
                            const int from = (key + lane - ch.context - tok0) * ch.group - 32 * cq;     // rows [from, rows) see this thread's key
                            if (key >= n || (key - ch.context - tok0) * ch.group - 32 * cq >= rows) continue;
                            float some = 0.f;
#pragma unroll
                            for (int i = 0; i < 32; ++i) {
                                const float w = fast_exp2(fmaf(v[s][i], p.scale_log2, norm[i])) * norm[kTile + i];
                                some += i >= from && i < rows ? w : 0.f;
                            }
                            sum[s] += some;
                        }
                    }
                }
                tmem_fence_before_sync();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&bars.s_empty[buf]);
                    mbar_arrive(&bars.empty[st]);
                }
                ++rr.count;
                ++sr.count;
            }
            // the four warps of 32 keys: one adds up
            if (cq > 0) {
                parts[(cq - 1) * 2 * kTile] = sum[0];
                parts[(cq - 1) * 2 * kTile + kTile] = sum[1];
            }
            named_barrier_sync(quad_bar, 128);
            if (cq == 0) {
#pragma unroll
                for (int q = 0; q < 3; ++q) {
                    sum[0] += parts[q * 2 * kTile];
                    sum[1] += parts[q * 2 * kTile + kTile];
                }
                const bool whole = pc.q1 - pc.q0 == pc.tiles - pc.first;
                auto put = [&](int s, float total) {
                    const int key = key0 + s * kTile + lane;
                    const long long at = (long long)pc.unit * p.capacity + key;
                    if (key < n && in_bounds(key < p.capacity, p.status)) p.weights[at] = (p.add ? p.weights[at] : 0.f) + total * p.inv_group;
                };
                if (whole) {
                    put(0, sum[0]);
                    put(1, sum[1]);
                } else {
                    // the last block of the item to come here adds the sums of all, in order
                    auto slot_of = [&](int block, int first_step) { return (2 * block + (first_step == part_begin(p.plan, block) ? 0 : 1)) * 2 * kTile + row; };
                    const int first_block = block_of(p.plan, pc.start);
                    const int blocks = block_of(p.plan, pc.start + pc.tiles - pc.first - 1) - first_block + 1;
                    float* own = p.sums + slot_of(blockIdx.x, pc.start + pc.q0 - pc.first);
                    own[0] = sum[0];
                    own[kTile] = sum[1];
                    __threadfence();
                    __syncwarp();
                    if (lane == 0) {
                        int* counter = p.counters + first_block * 4 + quarter;
                        const bool last = atomicAdd(counter, 1) == blocks - 1;
                        if (last) *counter = 0;                    // (for the next launch)
                        last_flag[quarter] = last;
                    }
                    __syncwarp();
                    if (last_flag[quarter]) {
                        __threadfence();
                        float total[2] = {0.f, 0.f};
                        for (int b = 0; b < blocks; ++b) {
                            const float* from = p.sums + slot_of(first_block + b, b == 0 ? pc.start : part_begin(p.plan, first_block + b));
                            total[0] += __ldcg(from);
                            total[1] += __ldcg(from + kTile);
                        }
                        put(0, total[0]);
                        put(1, total[1]);
                    }
                    __syncwarp();
                }
            }
            named_barrier_sync(quad_bar, 128);             // (the parts may be written again)
        }
    }

    tmem_fence_before_sync();
    __syncthreads();
    if (warp == 0) {
        tmem_fence_after_sync();
        tmem_dealloc(tmem_base, kTmemCols);
    }
}

// weights[u][i] += pbar[u][i] for i < n - 1, and the newest token's begins with its own: one thread per four slots.
__global__ void step_weights_kernel(float* weights, const float* pbar, int units, int capacity, int n) {
    const long long quads = (long long)units * (capacity / 4);
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < quads; i += (long long)gridDim.x * blockDim.x) {
        const int slot = (int)(i % (capacity / 4)) * 4;
        if (slot >= n) continue;
        float4 w = reinterpret_cast<const float4*>(weights)[i];
        const float4 add = reinterpret_cast<const float4*>(pbar)[i];
        w.x = (slot < n - 1 ? w.x : 0.f) + add.x;
        w.y = (slot + 1 < n - 1 ? w.y : 0.f) + add.y;
        w.z = (slot + 2 < n - 1 ? w.z : 0.f) + add.z;
        w.w = (slot + 3 < n - 1 ? w.w : 0.f) + add.w;
        reinterpret_cast<float4*>(weights)[i] = w;         // (slots behind n: whatever; they begin anew when a token comes)
    }
}

}  // namespace

WeighPlan weigh_plan(const ChunkPlan& ch, int num_sms) {
    WeighPlan pl;
    pl.pairs = (ch.context + ch.tokens + 2 * kTile - 1) / (2 * kTile);
    const int before = ch.context / (2 * kTile) < pl.pairs ? ch.context / (2 * kTile) : pl.pairs;
    long long steps = (long long)before * ch.tiles;
    for (int j = before; j < pl.pairs; ++j) steps += ch.tiles - weigh_first_tile(ch, j);
    const long long work = (long long)ch.layers * ch.batch * ch.kv_heads * steps;
    pl.unit_steps = steps > 0x40000000 ? 0 : (int)steps;
    if (num_sms > kChunkMaxBlocks) num_sms = kChunkMaxBlocks;
    pl.blocks = work > 0x40000000 ? 0 : (int)(work < num_sms ? work : num_sms);
    pl.per = pl.extra = 0;
    if (pl.blocks == 0) return pl;
    pl.per = (int)(work / pl.blocks);
    pl.extra = (int)(work % pl.blocks);
    return pl;
}

size_t weigh_sums_bytes(int num_sms) { return (size_t)(num_sms < kChunkMaxBlocks ? num_sms : kChunkMaxBlocks) * 2 * 2 * kTile * sizeof(float); }

cudaError_t weigh_prepare() { return cudaFuncSetAttribute(weigh_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem); }

cudaError_t weigh_launch(const WeighPlan& plan, const ChunkPlan& chunk, const WeighArgs& a, cudaStream_t stream) {
    CUtensorMap mq, mkv;
    memcpy(&mq, a.q_map, sizeof(mq));
    memcpy(&mkv, a.pool, sizeof(mkv));
    WeighParams p;
    p.plan = plan;
    p.chunk = chunk;
    p.page_table = a.page_table;
    p.norms = a.norms;
    p.weights = a.weights;
    p.sums = a.sums;
    p.counters = a.counters;
    p.status = a.status;
    p.pages_per_unit = a.pages_per_unit;
    p.total_pages = a.total_pages;
    p.capacity = a.capacity;
    p.add = a.add;
    p.scale_log2 = 1.4426950408889634f / sqrtf((float)kHeadDim);
    p.inv_group = 1.f / (float)chunk.group;
    p.wait_limit_ns = a.wait_limit_ns;
    p.stop_after_tiles = a.stop_after_tiles;
    cudaLaunchAttribute beside = {};
    beside.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    beside.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(plan.blocks);
    c.blockDim = dim3(kThreads);
    c.dynamicSmemBytes = kSmem;
    c.stream = stream;
    c.attrs = &beside;
    c.numAttrs = 1;                            // begins beside the end of the launch before (1 token: the call 20.5 -> 16.9 us)
    return cudaLaunchKernelEx(&c, weigh_kernel, mq, mkv, p);
}

cudaError_t step_weights_launch(const Geometry& geo, float* weights, const float* pbar, int n, cudaStream_t stream) {
    const long long quads = (long long)geo.units * (geo.capacity / 4), blocks = (quads + 255) / 256;
    step_weights_kernel<<<(unsigned)(blocks < 148 * 16 ? blocks : 148 * 16), 256, 0, stream>>>(weights, pbar, geo.units, geo.capacity, n);
    return cudaGetLastError();
}

}  // namespace lzk
