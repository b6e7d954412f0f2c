// Attention of a batch over a prefix that its sequences share, computed once for all of them.
//
// The prefix is another handle's cache: its units are (layer, prefix sequence, KV head), and `share` sequences of the
// decoding handle attend to each.  For the share * G query rows of a prefix unit and the prefix's tokens i
// (Appendix A, Eq. (attn), restricted to the prefix):
//   x[i] = q . k_i / sqrt(D) * log2 e,   m >= max_i x[i] - 8,   l = sum_i exp2(x[i] - m),   o = sum_i exp2(x[i] - m) v_i
// (m, l, o) are written as partial sums; the decode kernel starts a unit's softmax over its own tokens from them, so
// the probabilities it emits are those of the joint softmax.
//
// K / V of the prefix are read once per pair of row tiles, 512 bytes per token, where every sequence would read them by
// itself.  Few rows: HBM, behind a part that does not grow with the prefix; many rows: the tensor core
// (S, and P V twice) and the softmax between its products.  Measured on B200, this kernel under a profiler: 8 KV heads,
// 65521 tokens, 64 rows, 269 MB read, 54.8 us, tensor pipe 47 % busy; 4 layers x 8 KV heads, 8192 tokens, 640 rows, 127 us,
// tensor pipe 64 %, issue slots 43 %.  Of the second case's tensor work a sixth is on empty rows: a tile holds whole sequences, 25 of
// 5 heads, and 128 of them fill five tiles and 3 sequences of a sixth.  P as one bf16 term took the second case (whole call, then 187 us) to 174 us; it leaves P 8
// mantissa bits where the framework's other attention kernels keep 16, and is not used.
//
// Structure: persistent blocks, one per SM.  A row tile is 128 accumulator rows = floor(128 / G) sequences x G heads, an
// item is a prefix unit with two of its row tiles (or its single, or odd last one), and the walk over (item, key tile
// of 128 tokens) is cut into equal contiguous parts, one per block, so no wave is left half full (a step of a single row tile counts
// like one of a pair, though it costs the tensor core half: with an odd number of tiles the blocks on pairs end last); a row gets
// one set of partial sums per block that worked on its item.
//
// Two streams of eight softmax warps (two threads per accumulator row) alternate on the tensor core: with two row tiles a
// stream has a tile and every key tile; with one, the streams take the key tiles in turn and join their sums at the end.
//   S = Q K^T (tcgen05.mma, operands in shared memory, accumulator in tensor memory), softmax against a reference that
//   is raised -- and O rescaled in tensor memory -- only when a logit exceeds it by more than 2^8, P written over S
//   as two bf16 terms (hi + lo: 16 mantissa bits, as in the other attention kernels here), O += P V with P as the
//   tensor-memory operand.
// MMAs of one thread complete in order, and S of a stream's next tile is issued after O += P V of the tile before (they share
// tensor-memory columns): once S has arrived the warps may rescale O without any further wait.
//
// Pages keep 16-byte chunk c of row r at c ^ (r & 7) of every 128-byte half row.  A plain (unswizzled) TMA box of 64 rows x
// 128 bytes therefore lands as a 128-byte-swizzled operand; a key tile is four boxes from two pages.
//
// Warp roles: warps 0-15 softmax and output, warp 16 TMA producer, warps 17 and 18 MMA issuers, one per stream.  All mbarrier waits are bounded.
#include <string.h>

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

struct PrefixParams {
    PrefixPlan plan;
    const int32_t* page_table;
    float* o;
    float2* ml;
    int32_t* status;
    int n, pages_per_unit, total_pages;
    float scale_log2;
    unsigned long long wait_limit_ns;
    int stop_after_tiles;
};

// One block's part of an item: key tiles [k0, k1).
struct Piece {
    int item, k0, k1;
    bool both;                                     // two row tiles, a stream each; else one, the key tiles in turn
    __device__ __forceinline__ int tiles() const { return k1 - k0; }
    // key tiles of stream s, and the t-th of them
    __device__ __forceinline__ int stream_tiles(int s) const { return both ? k1 - k0 : (k1 - k0 + 1 - s) >> 1; }
    __device__ __forceinline__ int key_tile(int s, int t) const { return both ? k0 + t : k0 + 2 * t + s; }
};

__device__ __forceinline__ Piece piece_at(const PrefixPlan& pl, int x, int end) {
    Piece pc;
    pc.item = x / pl.key_tiles;
    pc.k0 = x - pc.item * pl.key_tiles;
    pc.k1 = min(pl.key_tiles, pc.k0 + (end - x));
    pc.both = 2 * (pc.item % pl.pairs) + 1 < pl.tiles;
    return pc;
}

__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&v)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(v[0]), "r"(v[1]),
                 "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}

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

__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
}

// A unit's page numbers, 32 at a time in the lanes of a warp.
struct PageList {
    const int32_t* table;
    int last, first;                               // last page of the unit; first page of those in the lanes
    int32_t entry;
    __device__ __forceinline__ void open(const int32_t* t, int last_page, int page) {
        table = t;
        last = last_page;
        first = page;
    }
    __device__ __forceinline__ void fetch(int page) {
        first = page;
        entry = table[min(page + (int)(threadIdx.x & 31), last)];
    }
    __device__ __forceinline__ int32_t at(int page) {      // pages are asked for in ascending order
        if (page >= first + 32) fetch(page);
        return __shfl_sync(0xffffffffu, entry, page - first);
    }
};

__global__ void __launch_bounds__(kThreads, 1)
prefix_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_kv, const __grid_constant__ PrefixParams p) {
    extern __shared__ __align__(1024) uint8_t smem[];
    Bars* bars = reinterpret_cast<Bars*>(smem + kOffMisc);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kOffMisc + 512);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const PrefixPlan& pl = p.plan;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int begin = prefix_begin(pl, blockIdx.x), end = prefix_begin(pl, blockIdx.x + 1);

    // the producer's first page numbers, asked for before everything else
    PageList k_pages, v_pages;
    if (warp == kProducer) {
        if (lane == 0) {
            prefetch_map(&map_q);
            prefetch_map(&map_kv);
        }
        const Piece pc = piece_at(pl, begin, end);
        k_pages.open(p.page_table + (long long)(pc.item / pl.pairs) * p.pages_per_unit, (p.n - 1) / kPageTokens, 2 * pc.k0);
        k_pages.fetch(2 * pc.k0);
        v_pages = k_pages;
    }
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
    // every block is resident: the decode launch may take the SMs that this one leaves (it waits for the sums itself)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const unsigned long long limit = p.wait_limit_ns;

    if (warp == kProducer) {
        // ------------------------------------------------------------------ TMA producer
        // (the whole warp: the lanes keep 32 page numbers, one elected lane issues the copies)
        Ring rr, qr;
        bool ok = true;
        int k_tiles = 0;
        const uint32_t q_bytes = (uint32_t)(pl.tile_seqs * pl.group) * 256u;
        auto wait_on = [&](uint64_t* bar, uint32_t parity) { ok = __all_sync(0xffffffffu, wait_bar(bar, parity, abort_flag, p.status, limit)); };
        // a K (half = 0) or V (half = 1) tile: 64 rows x 64 elements per box, two pages, both halves of the rows
        auto load_tile = [&](PageList& pages, int kt, int half) {
            // (a tile's second page may lie behind the last one: any page will do, its keys are masked)
            int32_t p0 = pages.at(2 * kt), p1 = pages.at(2 * kt + 1);
            if (p0 < 0 || p0 >= p.total_pages || p1 < 0 || p1 >= p.total_pages) {
                if (lane == 0) atomicOr(p.status, kStatusBadIndex);
                p0 = p1 = 0;
            }
            const uint32_t st = rr.stage(kRing);
            wait_on(&bars->empty[st], rr.parity(kRing) ^ 1u);
            if (!ok) return;
            uint8_t* dst = smem + kOffRing + st * kOperandBytes;
            if (elect_one()) {
                mbar_arrive_expect_tx(&bars->full[st], kOperandBytes);
                tma_load_3d(dst, &map_kv, 0, half * kPageTokens, p0, &bars->full[st]);
                tma_load_3d(dst + kBoxBytes / 2, &map_kv, 0, half * kPageTokens, p1, &bars->full[st]);
                tma_load_3d(dst + kBoxBytes, &map_kv, 64, half * kPageTokens, p0, &bars->full[st]);
                tma_load_3d(dst + kBoxBytes + kBoxBytes / 2, &map_kv, 64, half * kPageTokens, p1, &bars->full[st]);
            }
            __syncwarp();
            ++rr.count;
        };
        for (int x = begin; x < end && ok;) {
            const Piece pc = piece_at(pl, x, end);
            const int unit = pc.item / pl.pairs;                       // (layer, prefix sequence, head)
            const int head = unit % pl.kv_heads, seq0 = unit / pl.kv_heads * pl.share;
            const int tile0 = 2 * (pc.item % pl.pairs);
            if (x != begin) {
                k_pages.open(p.page_table + (long long)unit * p.pages_per_unit, (p.n - 1) / kPageTokens, 2 * pc.k0);
                k_pages.fetch(2 * pc.k0);
                v_pages = k_pages;
            }
            x += pc.tiles();
            for (int s = 0; s < (pc.both ? 2 : 1) && ok; ++s) {
                const uint32_t qs = qr.stage(2);
                wait_on(&bars->q_empty[qs], qr.parity(2) ^ 1u);
                if (!ok) break;
                uint8_t* dst = smem + kOffQ + qs * kOperandBytes;
                const int seq = seq0 + (tile0 + s) * pl.tile_seqs;
                if (elect_one()) {
                    mbar_arrive_expect_tx(&bars->q_full[qs], q_bytes);
                    tma_load_4d(dst, &map_q, 0, 0, head, seq, &bars->q_full[qs]);
                    tma_load_4d(dst + kBoxBytes, &map_q, 64, 0, head, seq, &bars->q_full[qs]);
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
        // A warp walks its loop as a whole (so that descriptors and addresses stay in uniform registers) and one elected lane, the
        // same every time, issues.  The tensor core queues few instructions and a ready barrier costs 150 clocks to look at, so
        // with one issuer it idled a third of the time between two streams' turns; two issuers left to themselves
        // let the streams fall into step (both in the softmax, then both at the tensor core).  So each does its waiting
        // beforehand and they hand the tensor core to each other turn by turn, which keeps the streams half a step apart.  The turns
        // go on from piece to piece: stream 0 takes a piece's first turn behind the last one of the piece before, whoever had
        // that.  So neither warp is ever more than one turn ahead, and no barrier sees the same warp arrive twice in a phase -- the
        // barriers have no time limit, and what ends every wait on them is that both warps walk all their turns.
        const int s = warp - kIssuer;
        uint32_t p_uses = 0, uses = 0, q_uses = 0;  // products issued; uses of the K / V ring and of the Q slots by earlier pieces
        bool ok = true;                             // a warp that gave up goes through the same turns without issuing
        bool behind = false;                        // the piece before ended with the other stream's turn (stream 0 looks)
        auto wait_on = [&](uint64_t* bar, uint32_t parity) {
            if (ok) ok = __all_sync(0xffffffffu, wait_bar(bar, parity, abort_flag, p.status, limit));
        };
        // Every buffer expects both streams: it is handed back by a commit, once the MMAs issued so far are done, or at once by a
        // stream that does not read it.  A wait for a phase of a barrier means something only to a warp that saw the phase before:
        // a page may come in long after the pages asked for behind it, and a warp that only looked at its own uses of the ring
        // took a stage for full that still waited for an earlier use's load.  So each warp looks at all uses, in order, and hands
        // back those of the other stream; the producer cannot lap a warp that has yet to look.
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
            for (int i = 0; i < 4; ++i) {           // 16 keys per instruction; P = hi + lo, two products
                const int s8 = (i >> 1) * 4 + part * 2 + (i & 1);
                const uint32_t a_col = s_col + (s8 >> 1) * 32 + (s8 & 1) * 8;
                umma_bf16_ts(o_col, a_col, b + s8 * (2048 >> 4), instr_desc(true), !first || i > 0);
                umma_bf16_ts(o_col, a_col + 16, b + s8 * (2048 >> 4), instr_desc(true), 1u);
            }
        };
        for (int x = begin; x < end;) {
            const Piece pc = piece_at(pl, x, end);
            const int nt = pc.tiles(), mine = pc.stream_tiles(s), step = pc.both ? 1 : 2, turns = pc.both ? 2 * nt : nt;
            x += nt;
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
            for (int t = 0; t < mine; ++t, j += step) {
                const int turn = 2 * t + s;         // the streams take turns: 0, 1, 0, 1 ..
                const bool more = t + 1 < mine;
                const uint32_t vu = v_use(j), vs = vu % kRing, ku = more ? k_use(j + step) : 0u, ks = ku % kRing;
                look_at(vu + 1, true);
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
                if (turn + 1 < turns || (s == 1 && x < end)) asm volatile("bar.arrive %0, %1;" ::"r"(13 + (s ^ 1)), "r"(64) : "memory");
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
        const int s = warp / kStreamWarps, hf = (warp >> 2) & 1, row = 32 * (warp & 3) + lane;
        const uint32_t lane_base = tmem_base + ((uint32_t)(32 * (warp & 3)) << 16);
        const uint32_t s_cols = lane_base + kColS + s * 128 + hf * 64, o_cols = lane_base + kColO + s * 128 + hf * 64;
        float* mine = reinterpret_cast<float*>(smem + kOffExchange) + (s * kTile + row) * 2 + hf;
        const float* other = reinterpret_cast<const float*>(smem + kOffExchange) + (s * kTile + row) * 2 + (hf ^ 1);
        const int pair_bar = 1 + s * 4 + (warp & 3);                   // of the two warps
        uint32_t s_uses = 0, o_uses = 0;
        // A warp whose wait gives up goes on through the same loops, so that its partner's barriers get all their threads, but waits
        // for nothing any more; what it computes means nothing.
        bool dead = false;
        auto wait_on = [&](uint64_t* bar, uint32_t parity) {
            const bool gave_up = dead || !wait_bar(bar, parity, abort_flag, p.status, limit);
            dead = __any_sync(0xffffffffu, gave_up);
        };
        for (int x = begin; x < end;) {
            const Piece pc = piece_at(pl, x, end);
            x += pc.tiles();
            const int nt = pc.stream_tiles(s);
            const int tile = 2 * (pc.item % pl.pairs) + (pc.both ? s : 0);
            const int r = row / pl.group;                              // sequence inside the row tile
            const int seq = tile * pl.tile_seqs + r;
            const bool valid = r < pl.tile_seqs && seq < pl.share;
            const bool warp_on = __any_sync(0xffffffffu, valid);       // (the same in both warps of the rows)
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
                    const int key0 = pc.key_tile(s, t) * kTile + hf * 64;
                    if (key0 + 64 > p.n) {
#pragma unroll
                        for (int c = 0; c < 2; ++c)
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[c][i] = key0 + 32 * c + i < p.n ? v[c][i] : -INFINITY;
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
                        uint32_t hi[8], lo[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float x0 = v[c >> 1][16 * (c & 1) + 2 * i], x1 = v[c >> 1][16 * (c & 1) + 2 * i + 1];
                            float e0, e1, d0, d1;
                            unpack2(fma2(pack2(x0, x1), scale2, minus2), e0, e1);
                            e0 = fast_exp2(e0);
                            e1 = fast_exp2(e1);
                            const uint64_t w = pack2(e0, e1);
                            hi[i] = pack_bf16(e0, e1);
                            unpack2(sub2(w, pack2(bf16_lo_as_float(hi[i]), bf16_hi_as_float(hi[i]))), d0, d1);
                            lo[i] = pack_bf16(d0, d1);
                            if (i & 1)
                                sum1 = add2(sum1, w);
                            else
                                sum0 = add2(sum0, w);
                        }
                        // a chunk of 32 keys: 16 columns of hi terms, then 16 of lo terms
                        tmem_st8(s_cols + 32 * (c >> 1) + 8 * (c & 1), hi);
                        tmem_st8(s_cols + 32 * (c >> 1) + 16 + 8 * (c & 1), lo);
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
            // ---- the piece's partial sums
            const int nth = (int)blockIdx.x - prefix_block_of(pl, pc.item * pl.key_tiles), unit = pc.item / pl.pairs;
            const int u = (unit / pl.kv_heads * pl.share + seq) * pl.kv_heads + unit % pl.kv_heads;     // of the decoding handle
            const long long at = nth * pl.rows + (long long)u * pl.group + (row - r * pl.group);
            const bool writes = valid && in_bounds(nth >= 0 && nth < pl.slots && at >= 0 && at < pl.slots * pl.rows, p.status);
            if (nt > 0) {
                wait_on(&bars->o_full[s], o_uses & 1u);
                ++o_uses;
            }
            tmem_fence_after_sync();
            if (warp_on) {
                *mine = l;
                named_barrier_sync(pair_bar, 64);
                l += *other;
                named_barrier_sync(pair_bar, 64);
                float4* dst = reinterpret_cast<float4*>(p.o + at * kHeadDim);
                if (pc.both) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float o[32];
                        tmem_ld32(o_cols + 32 * c, o);
                        tmem_wait_ld();
                        if (writes) {
#pragma unroll
                            for (int i = 0; i < 8; ++i) dst[16 * hf + 8 * c + i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                        }
                    }
                } else {
                    // The two streams' sums into one: four threads per row, 32 columns each.  (Each stream's warps have waited for
                    // their own accumulator; the barrier passes that on.)
                    *mine = hf ? l : m;
                    tmem_fence_before_sync();
                    named_barrier_sync(9 + (warp & 3), 128);
                    tmem_fence_after_sync();
                    const float2* ml = reinterpret_cast<const float2*>(smem + kOffExchange) + row;
                    const float2 a0 = ml[0], a1 = ml[kTile];
                    m = fmaxf(a0.x, a1.x);
                    const float f0 = a0.x > -INFINITY ? fast_exp2(a0.x - m) : 0.f, f1 = a1.x > -INFINITY ? fast_exp2(a1.x - m) : 0.f;
                    l = a0.y * f0 + a1.y * f1;
                    const int col = 64 * s + 32 * hf;
#pragma unroll
                    for (int c = 0; c < 32; c += 16) {
                        float o0[16], o1[16];
                        tmem_ld16(lane_base + kColO + col + c, o0);
                        tmem_ld16(lane_base + kColO + 128 + col + c, o1);
                        tmem_wait_ld();
                        if (writes) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) o0[i] = o0[i] * f0 + (pc.tiles() > 1 ? o1[i] * f1 : 0.f);
#pragma unroll
                            for (int i = 0; i < 4; ++i) dst[(col + c) / 4 + i] = make_float4(o0[4 * i], o0[4 * i + 1], o0[4 * i + 2], o0[4 * i + 3]);
                        }
                    }
                    tmem_fence_before_sync();
                    named_barrier_sync(9 + (warp & 3), 128);           // all are done with both accumulators and the exchange
                }
            }
            tmem_fence_before_sync();
            if (writes && hf == 0 && (pc.both || s == 0)) p.ml[at] = make_float2(m, l);
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

PrefixPlan prefix_plan(int layers, int batch, int prefixes, int kv_heads, int group, int n, int num_sms) {
    PrefixPlan pl;
    pl.kv_heads = kv_heads;
    pl.batch = batch;
    pl.share = batch / prefixes;
    pl.group = group;
    pl.tile_seqs = kTile / group < pl.share ? kTile / group : pl.share;
    pl.tiles = (pl.share + pl.tile_seqs - 1) / pl.tile_seqs;
    pl.pairs = (pl.tiles + 1) / 2;
    pl.key_tiles = (n + kTile - 1) / kTile;
    pl.rows = (long long)layers * batch * kv_heads * group;
    pl.slots = 0;
    const long long items = (long long)layers * prefixes * kv_heads * pl.pairs, work = items * pl.key_tiles;
    pl.blocks = work > 0x40000000 ? 0 : (int)(work < num_sms ? work : num_sms);
    if (pl.blocks == 0) return pl;
    pl.per = (int)(work / pl.blocks);
    pl.extra = (int)(work % pl.blocks);
    // most blocks that touch one item
    const int pieces = (pl.key_tiles + pl.per - 1) / pl.per + 1;
    pl.slots = pieces < pl.blocks ? pieces : pl.blocks;
    return pl;
}

int prefix_most_slots(int layers, int batch, int prefixes, int kv_heads, int group, int capacity, int num_sms) {
    int most = 0;
    for (int n = kTile; n < capacity + kTile; n += kTile) {
        const int slots = prefix_plan(layers, batch, prefixes, kv_heads, group, n < capacity ? n : capacity, num_sms).slots;
        if (slots > most) most = slots;
    }
    return most;
}

namespace {

__global__ void clear_sums_kernel(float2* ml, long long count) {
    const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (i < count) ml[i] = make_float2(-INFINITY, 0.f);
}

}  // namespace

cudaError_t prefix_clear_launch(const PrefixPlan& plan, float2* ml, cudaStream_t stream) {
    const long long count = plan.slots * plan.rows;
    clear_sums_kernel<<<(unsigned)((count + 255) / 256), 256, 0, stream>>>(ml, count);
    return cudaGetLastError();
}

cudaError_t prefix_prepare(const uint8_t* pool, int total_pages, PrefixPool* out) {
    // [pages][64 K rows, then 64 V rows][128]; the rows are stored swizzled already
    static_assert(sizeof(PrefixPool) == sizeof(CUtensorMap), "");
    const cuuint64_t dims[3] = {(cuuint64_t)kHeadDim, (cuuint64_t)2 * kPageTokens, (cuuint64_t)total_pages};
    const cuuint64_t strides[2] = {(cuuint64_t)kRowBytes, (cuuint64_t)kPageBytes};
    const cuuint32_t box[3] = {64, (cuuint32_t)kPageTokens, 1};
    CUtensorMap map;
    if (!make_map(&map, pool, 3, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_NONE)) return cudaErrorInvalidValue;
    memcpy(out, &map, sizeof(map));
    return cudaFuncSetAttribute(prefix_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
}

cudaError_t prefix_launch(const PrefixPlan& plan, const PrefixArgs& a, cudaStream_t stream) {
    CUtensorMap mq, mkv;
    {
        // q [layers * batch][kv_heads][G][128]: box = 64 elements x G heads x 1 KV head x tile_seqs sequences, 128-byte swizzle;
        // sequences behind the last one read as zero, those of the next prefix are rows that nobody looks at
        const cuuint64_t dims[4] = {(cuuint64_t)kHeadDim, (cuuint64_t)plan.group, (cuuint64_t)plan.kv_heads,
                                    (cuuint64_t)a.layers * plan.batch};
        const cuuint64_t strides[3] = {(cuuint64_t)kRowBytes, (cuuint64_t)plan.group * kRowBytes,
                                       (cuuint64_t)plan.kv_heads * plan.group * kRowBytes};
        const cuuint32_t box[4] = {64, (cuuint32_t)plan.group, 1, (cuuint32_t)plan.tile_seqs};
        if (!make_map(&mq, a.q, 4, dims, strides, box)) return cudaErrorInvalidValue;
    }
    memcpy(&mkv, a.pool, sizeof(mkv));
    PrefixParams p;
    p.plan = plan;
    p.page_table = a.page_table;
    p.o = a.o;
    p.ml = a.ml;
    p.status = a.status;
    p.n = a.n;
    p.pages_per_unit = a.pages_per_unit;
    p.total_pages = a.total_pages;
    p.scale_log2 = 1.4426950408889634f / sqrtf((float)kHeadDim);
    p.wait_limit_ns = a.wait_limit_ns;
    p.stop_after_tiles = a.stop_after_tiles;
    prefix_kernel<<<plan.blocks, kThreads, kSmem, stream>>>(mq, mkv, p);
    return cudaGetLastError();
}

}  // namespace lzk
