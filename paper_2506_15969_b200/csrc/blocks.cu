// Attention over the blocks of a cache that a cheap score selects, for a decode step's queries.
//
// A block is a page, 64 tokens.  For every block b before the newest its keys' bounds are kept, per dimension d:
//   high_b[d] = max_i k_i[d],   low_b[d] = min_i k_i[d]
// and a unit's G query heads give it the score
//   s_b = sum_g sum_d max(q_g[d] high_b[d], q_g[d] low_b[d]) = sum_d (P[d] high_b[d] + N[d] low_b[d]),
//   P[d] = sum_g max(q_g[d], 0),  N[d] = sum_g min(q_g[d], 0)
// (a side that no head is on counts nothing, whatever its bound; a zero q times an infinite bound is no number):
// no key between the bounds has larger logits summed over the heads.  Which blocks are read does not depend on fp32 rounding: blocks near
// the cut are compared by scores in fp64, where the products are exact (all of them in fp64 is four times slower than their bytes:
// 128 units of 2047 blocks, 77 us instead of 20, most of it conversions).
// The newest block (the only one that may be partly filled) and the blocks - 1 best others, of equals the older, become a
// page table of their own, in order, which the decode kernel reads like any other: K and V of blocks * 64 tokens instead of n.
//
//   bounds_kernel -- the bounds, once per block (keys behind the newest block do not change any more); HBM: 256 units of 16384 tokens,
//                    1.07 GB, 166 us, 6.5 TB/s
//   pick_kernel   -- one block of threads per unit: scores, radix select over them, page table, list.  512 bytes per block, a
//                    warp per block, lanes 0-15 the high row, 16-31 the low one: 128 units of 2047 blocks 40 us, 3.4 TB/s, half of it
//                    the select and the beginning
//   score_kernel  -- the scores by many blocks of threads, for long caches of few units
#include "internal.h"
#include "select.cuh"

namespace lzk {

namespace {

__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b) {
    const __nv_bfloat162 r = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t min_pair(uint32_t a, uint32_t b) {
    const __nv_bfloat162 r = __hmin2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}

// A warp per block: lane -> logical chunk lane & 15 of the rows with the parity of lane >> 4.
__global__ void __launch_bounds__(256) bounds_kernel(BlocksArgs a, int first, int count) {
    const int lane = threadIdx.x & 31, c = lane & 15;
    const long long total = (long long)a.geo.units * count;
    const int total_pages = a.geo.units * a.geo.pages_per_unit;
    for (long long w = ((long long)blockIdx.x * blockDim.x + threadIdx.x) >> 5; w < total; w += ((long long)gridDim.x * blockDim.x) >> 5) {
        const int u = (int)(w / count), b = first + (int)(w % count);
        const int32_t pp = a.page_table[(size_t)u * a.geo.pages_per_unit + b];
        if (pp < 0 || pp >= total_pages) {
            if (lane == 0) atomicOr(a.status, kStatusBadIndex);
            continue;
        }
        const uint8_t* page = a.pool + (size_t)pp * kPageBytes;
        uint4 hi, lo;
        hi = lo = *reinterpret_cast<const uint4*>(page + (lane >> 4) * kRowBytes + swz_chunk(c, lane >> 4) * 16);
#pragma unroll 8
        for (int r = 2 + (lane >> 4); r < kPageTokens; r += 2) {
            const uint4 x = *reinterpret_cast<const uint4*>(page + r * kRowBytes + swz_chunk(c, r) * 16);
            hi = make_uint4(max_pair(hi.x, x.x), max_pair(hi.y, x.y), max_pair(hi.z, x.z), max_pair(hi.w, x.w));
            lo = make_uint4(min_pair(lo.x, x.x), min_pair(lo.y, x.y), min_pair(lo.z, x.z), min_pair(lo.w, x.w));
        }
        auto across = [](uint32_t v) { return __shfl_xor_sync(0xffffffffu, v, 16); };
        hi = make_uint4(max_pair(hi.x, across(hi.x)), max_pair(hi.y, across(hi.y)), max_pair(hi.z, across(hi.z)), max_pair(hi.w, across(hi.w)));
        lo = make_uint4(min_pair(lo.x, across(lo.x)), min_pair(lo.y, across(lo.y)), min_pair(lo.z, across(lo.z)), min_pair(lo.w, across(lo.w)));
        uint4* out = reinterpret_cast<uint4*>(a.bounds) + ((size_t)u * a.geo.pages_per_unit + b) * 2 * kChunksPerRow;
        out[lane] = lane < 16 ? hi : lo;
    }
}

// Larger scores have larger keys; what is no number comes first of all.
__device__ __forceinline__ unsigned long long exact_key(double s) {
    if (s != s) return ~0ull;
    const long long b = __double_as_longlong(s == 0.0 ? 0.0 : s);
    return b < 0 ? ~(unsigned long long)b : (unsigned long long)b | 0x8000000000000000ull;
}
__device__ __forceinline__ uint32_t rough_key(float s) {
    if (s != s) return ~0u;
    const uint32_t b = __float_as_uint(s == 0.f ? 0.f : s);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float rough_score(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key); }

// A lane's part of P (lanes 0-15) or N for its eight dimensions; which of these have a head on that side; which have one whose q is zero.
struct Sides {
    double part[8];
    unsigned on, zero;
};
__device__ __forceinline__ Sides sides_of(const BlocksArgs& a, int u) {
    const int lane = threadIdx.x & 31, c = lane & 15, G = a.geo.group;
    Sides s = {{0, 0, 0, 0, 0, 0, 0, 0}, 0u, 0u};
    const uint4* q = reinterpret_cast<const uint4*>(a.q) + (size_t)u * G * kChunksPerRow + c;
    uint4 x[kMaxGroup];                    // (all of them asked for at once)
#pragma unroll
    for (int g = 0; g < kMaxGroup; ++g) x[g] = g < G ? q[g * kChunksPerRow] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int g = 0; g < kMaxGroup; ++g) {
        if (g >= G) break;
        const uint32_t w[4] = {x[g].x, x[g].y, x[g].z, x[g].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float e0 = bf16_lo_as_float(w[i]), e1 = bf16_hi_as_float(w[i]);
            // (what is no number goes into both sums)
            const bool on0 = e0 != e0 || (lane < 16 ? e0 > 0.f : e0 < 0.f), on1 = e1 != e1 || (lane < 16 ? e1 > 0.f : e1 < 0.f);
            s.part[2 * i] += on0 ? (double)e0 : 0.0;
            s.part[2 * i + 1] += on1 ? (double)e1 : 0.0;
            s.on |= ((on0 ? 1u : 0u) | (on1 ? 2u : 0u)) << (2 * i);
            s.zero |= ((e0 == 0.f ? 1u : 0u) | (e1 == 0.f ? 2u : 0u)) << (2 * i);
        }
    }
    return s;
}

__device__ __forceinline__ const uint4* bound_rows(const BlocksArgs& a, int u) {
    return reinterpret_cast<const uint4*>(a.bounds) + (size_t)u * a.geo.pages_per_unit * 2 * kChunksPerRow;
}

// Is either of two bf16 values infinite or no number?
__device__ __forceinline__ bool pair_not_finite(uint32_t w) { return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u; }

// A side's factor with a bound of any value: nothing where no head is on that side, no number where a head's zero meets an infinity.
__device__ __forceinline__ double side_term(const Sides& s, int i, float bound) {
    if (fabsf(bound) < INFINITY) return s.part[i] * (double)bound;
    if (s.zero >> i & 1u) return (double)NAN;
    return s.on >> i & 1u ? s.part[i] * (double)bound : 0.0;
}

// The score of one block in fp64, in every lane.
__device__ __forceinline__ double exact_score(const uint4* rows, const Sides& s, int b) {
    const uint4 x = __ldg(rows + (size_t)b * 2 * kChunksPerRow + (threadIdx.x & 31));
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    double v = 0.0;
    if (pair_not_finite(w[0]) || pair_not_finite(w[1]) || pair_not_finite(w[2]) || pair_not_finite(w[3])) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v += side_term(s, 2 * j, bf16_lo_as_float(w[j])) + side_term(s, 2 * j + 1, bf16_hi_as_float(w[j]));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v = fma(s.part[2 * j], (double)bf16_lo_as_float(w[j]), v);
            v = fma(s.part[2 * j + 1], (double)bf16_hi_as_float(w[j]), v);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

constexpr int kBatch = 8;                  // blocks that a warp sums at once; as many are under way
// An fp32 score is off by less than this of the sum of its terms' magnitudes: P rounded, eight products and five sums, 14 roundings
// of 2^-24, with room; and, where products leave the range of normal numbers, by a step of 2^-150 each (256 of them, and as many that the
// sum of magnitudes lacks), with room.
constexpr float kRoughError = 1.f / (1 << 19), kRoughFloor = 0x1p-140f;

// Rough scores of kBatch blocks, that of the i-th in the i-th kBatch-th of the lanes.  The sums over the lanes are folded into
// each other: half of them go to the other half of the lanes at every step, nine exchanges instead of forty.  `size` grows to the
// largest sum of magnitudes that this lane's dimensions had.
__device__ __forceinline__ void load_batch(const uint4* rows, int b0, int count, uint4 (&x)[kBatch]) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
        x[i] = b0 + i < count ? __ldg(rows + (size_t)(b0 + i) * 2 * kChunksPerRow + (threadIdx.x & 31)) : make_uint4(0u, 0u, 0u, 0u);
}
__device__ __forceinline__ float rough_batch(const uint4 (&x)[kBatch], const float (&side)[8], float& size) {
    const int lane = threadIdx.x & 31;
    float v[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
        float sum = 0.f, all = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float lo = bf16_lo_as_float(w[j]), hi = bf16_hi_as_float(w[j]);
            sum = fmaf(side[2 * j], lo, sum);
            sum = fmaf(side[2 * j + 1], hi, sum);
            all = fmaf(fabsf(side[2 * j]), fabsf(lo), all);
            all = fmaf(fabsf(side[2 * j + 1]), fabsf(hi), all);
        }
        v[i] = sum;
        size = all > size || all != all ? all : size;
    }
#pragma unroll
    for (int half = kBatch / 2, bit = 16; half > 0; half >>= 1, bit >>= 1) {
        const bool up = lane & bit;
#pragma unroll
        for (int i = 0; i < half; ++i) {
            const float give = up ? v[i] : v[i + half], own = up ? v[i + half] : v[i];
            v[i] = own + __shfl_xor_sync(0xffffffffu, give, bit);
        }
    }
#pragma unroll
    for (int bit = 16 / kBatch; bit > 0; bit >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], bit);
    return v[0];
}

// Scores the blocks that a warp takes (from b0 on, `step` apart) into `put`; returns the largest sum of magnitudes, or more.
template <typename Put>
__device__ __forceinline__ float rough_scores(const BlocksArgs& a, int u, int count, int b0, int step, const Put& put) {
    const int lane = threadIdx.x & 31;
    const Sides s = sides_of(a, u);
    float side[8], size = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) side[i] = (float)s.part[i];
    const uint4* rows = bound_rows(a, u);
    uint4 x[2][kBatch];
    load_batch(rows, b0, count, x[0]);
    auto batch = [&](int i) {                              // (the next one is under way while one is summed)
        load_batch(rows, b0 + step, count, x[i ^ 1]);
        const float score = rough_batch(x[i], side, size);
        const int b = b0 + lane / (32 / kBatch);
        if (lane % (32 / kBatch) == 0 && b < count) put(b, rough_key(score));
        b0 += step;
    };
    while (b0 < count) {
        batch(0);
        if (b0 < count) batch(1);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) size += __shfl_xor_sync(0xffffffffu, size, o);
    return size;
}

constexpr int kCachedKeys = 16384;         // of a unit in shared memory; of longer caches they stay in L2
constexpr int kScoreWarps = 8;
// Up to here, and where there are units for half of the SMs, a unit's own block of threads scores its blocks; else many score first.
// (256 units of 1024 blocks, whole call: 50 us alone, 64 with a launch of its own; 2 units of 1024: 28.7 and 22.6; 128 of 255: 20.9, 22.5.)
constexpr int kScoreAlone = 256;

// a.rough: per unit pages_per_unit rough keys, and behind them one sum of magnitudes per warp of this launch.
__global__ void __launch_bounds__(32 * kScoreWarps) score_kernel(BlocksArgs a, int count) {
    const int u = blockIdx.y, warp = blockIdx.x * kScoreWarps + (threadIdx.x >> 5);
    uint32_t* keys = a.rough + (size_t)u * 2 * a.geo.pages_per_unit;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const float size = rough_scores(a, u, count, warp * kBatch, gridDim.x * kScoreWarps * kBatch, [&](int b, uint32_t key) { keys[b] = key; });
    if ((threadIdx.x & 31) == 0) reinterpret_cast<float*>(keys)[a.geo.pages_per_unit + warp] = size;
}

// Candidates are blocks 0 .. count - 1, `picked` of them (may be 0, or all) are taken; then the newest block.  The cut comes from
// rough scores in fp32: with E the most that one is off, a block more than 2 E above the rough cut is above the exact one and a
// block more than 2 E below it below, and only those between are scored in fp64 -- a handful, or, where scores are no numbers or
// alike, up to all.  score_warps = 0: the scores are made here.
template <int kThreads>
__global__ void __launch_bounds__(kThreads) pick_kernel(BlocksArgs a, int count, int picked, int asked, int score_warps) {
    constexpr int kWarps = kThreads / 32;
    extern __shared__ uint32_t cached[];
    __shared__ TopShared<unsigned long long> wide;
    TopShared<uint32_t>& sh = *reinterpret_cast<TopShared<uint32_t>*>(&wide);      // (one select after the other)
    __shared__ uint32_t least[kWarps], most[kWarps];
    __shared__ float sizes[kWarps];
    __shared__ int between[kSurvivors];
    __shared__ unsigned long long exact[kSurvivors];
    const int u = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint32_t* stored = a.rough + (size_t)u * 2 * a.geo.pages_per_unit;
    const int32_t* table = a.page_table + (size_t)u * a.geo.pages_per_unit;
    int32_t* to = a.table + (size_t)u * a.geo.pages_per_unit;
    int32_t* list = a.selected ? a.selected + (size_t)u * asked : nullptr;
    uint32_t* keys = count <= kCachedKeys ? cached : stored;
    const bool chosen = picked > 0 && picked < count;
    const int32_t own_page = tid <= count ? table[tid] : 0, last_page = table[count];      // (asked for before they are needed)
    auto put = [&](int j, int block) {
        to[j] = block == tid ? own_page : block == count ? last_page : table[block];
        if (list) list[j] = block;
    };
    float size = 0.f;
    if (chosen && score_warps == 0) {
        size = rough_scores(a, u, count, warp * kBatch, kWarps * kBatch, [&](int b, uint32_t key) { keys[b] = key; });
    } else {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        if (chosen) {
            if (keys == cached)
                for (int i = tid; i < count; i += kThreads) cached[i] = __ldcg(stored + i);
            for (int i = tid; i < score_warps; i += kThreads) {
                const float s = __ldcg(reinterpret_cast<const float*>(stored) + a.geo.pages_per_unit + i);
                size = s > size || s != s ? s : size;
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                const float s = __shfl_xor_sync(0xffffffffu, size, o);
                size = s > size || s != s ? s : size;
            }
        }
    }
    if (picked == count) {                                  // all of them
        for (int b = tid; b < count; b += kThreads) put(b, b);
    } else if (chosen) {
        if (lane == 0) sizes[warp] = size;
        __syncthreads();
        for (int w = 0; w < kWarps; ++w) size = sizes[w] > size || sizes[w] != sizes[w] ? sizes[w] : size;
        uint32_t kth;
        if (count <= kThreads) {                            // few: ranked one against the other
            int above = 0, equal = 0;
            const uint32_t mine = tid < count ? keys[tid] : 0u;
            for (int j = 0; j < count; ++j) {
                above += keys[j] > mine;
                equal += keys[j] == mine;
            }
            if (tid < count && above < picked && picked <= above + equal) least[0] = mine;
            __syncthreads();
            kth = least[0];
        } else {
            // Scores of a unit are mostly of one magnitude: counted from the least one, the leading digits of their keys differ.
            uint32_t lo = ~0u, hi = 0u;
            for (int i = tid; i < count; i += kThreads) {
                lo = min(lo, keys[i]);
                hi = max(hi, keys[i]);
            }
            lo = __reduce_min_sync(0xffffffffu, lo);
            hi = __reduce_max_sync(0xffffffffu, hi);
            if (lane == 0) {
                least[warp] = lo;
                most[warp] = hi;
            }
            __syncthreads();
            for (int w = 0; w < kWarps; ++w) {
                lo = min(lo, least[w]);
                hi = max(hi, most[w]);
            }
            const Cut<uint32_t> cut = top_cut<kThreads, uint32_t>(count, picked, 32 - __clz(hi - lo), sh, [&](int i) { return keys[i] - lo; });
            // (the cut may lie between two keys: the k-th is the least one above it)
            kth = cut.kth + lo;
            if (cut.ties == 0) {
                uint32_t next = ~0u;
                for (int i = tid; i < count; i += kThreads)
                    if (keys[i] > kth) next = min(next, keys[i]);
                next = __reduce_min_sync(0xffffffffu, next);
                __syncthreads();
                if (lane == 0) least[warp] = next;
                __syncthreads();
                for (int w = 0; w < kWarps; ++w) next = min(next, least[w]);
                kth = next;
            }
        }
        const float t = rough_score(kth), reach = 2.f * (kRoughError * size + kRoughFloor);
        // 1: above whatever the exact scores are, 0: below, 2: between (all of them where something is no number or infinite)
        const bool sane = fabsf(t) < INFINITY && reach < INFINITY;
        auto side_of = [&](uint32_t key) {
            if (!sane || key == ~0u) return 2;
            const float s = rough_score(key);
            return s > t + reach ? 1 : s < t - reach ? 0 : 2;
        };
        int sure = 0, open = 0;
        for (int i = tid; i < count; i += kThreads) {
            const int side = side_of(keys[i]);
            sure += side == 1;
            open += side == 2;
        }
        int all_sure, all_open;
        block_rank<kThreads>(sure, sh.warp_sums, &all_sure);
        const int open_before = block_rank<kThreads>(open, sh.warp_sums, &all_open);
        const int need = picked - all_sure;
        // afterwards a key is ~0 for a block that is taken and 0 for one that is not
        if (all_open == need) {
            for (int i = tid; i < count; i += kThreads) keys[i] = side_of(keys[i]) != 0 ? ~0u : 0u;
        } else if (all_open <= kSurvivors) {
            int at = open_before;
            for (int i = tid; i < count; i += kThreads) {
                const int side = side_of(keys[i]);
                if (side == 2 && at < kSurvivors) between[at++] = i;
                keys[i] = side == 1 ? ~0u : 0u;
            }
            __syncthreads();
            const Sides s = sides_of(a, u);
            for (int i = warp; i < all_open; i += kWarps) {
                const unsigned long long key = exact_key(exact_score(bound_rows(a, u), s, between[i]));
                if (lane == 0) exact[i] = key;
            }
            __syncthreads();
            if (tid < all_open) {                           // of equals the older
                int before = 0;
                for (int j = 0; j < all_open; ++j) before += exact[j] > exact[tid] || (exact[j] == exact[tid] && between[j] < between[tid]);
                if (before < need) keys[between[tid]] = ~0u;
            }
        } else {
            // many: all their exact keys, and a select over those (0 is no exact key)
            const Sides s = sides_of(a, u);
            unsigned long long* exacts = a.exact + (size_t)u * a.geo.pages_per_unit;
            for (int i = warp; i < count; i += kWarps) {
                const unsigned long long key = side_of(keys[i]) == 2 ? exact_key(exact_score(bound_rows(a, u), s, i)) : 0ull;
                if (lane == 0) exacts[i] = key;
            }
            __syncthreads();
            const Cut<unsigned long long> last = top_cut<kThreads, unsigned long long>(count, need, 64, wide, [&](int i) { return exacts[i]; });
            const int per = (count + kThreads - 1) / kThreads, from = min(count, tid * per), till = min(count, from + per);
            int ties = 0;
            for (int i = from; i < till; ++i) ties += exacts[i] == last.kth;
            int total, tie = block_rank<kThreads>(ties, sh.warp_sums, &total);
            for (int i = from; i < till; ++i) {             // of equals the older
                const bool take = side_of(keys[i]) == 1 || exacts[i] > last.kth || (exacts[i] == last.kth && tie < last.ties);
                tie += exacts[i] == last.kth;
                keys[i] = take ? ~0u : 0u;
            }
        }
        __syncthreads();
        const int seg = ((count + kWarps - 1) / kWarps + 31) / 32 * 32;
        const int seg_b = min(count, warp * seg), seg_e = min(count, seg_b + seg);
        int kept = 0, all;
        for (int i0 = seg_b; i0 < seg_e; i0 += 32) kept += __popc(__ballot_sync(0xffffffffu, i0 + lane < seg_e && keys[min(i0 + lane, count - 1)] != 0u));
        int dst = __shfl_sync(0xffffffffu, block_rank<kThreads>(lane == 0 ? kept : 0, sh.warp_sums, &all), 0);
        for (int i0 = seg_b; i0 < seg_e; i0 += 32) {
            const bool keep = i0 + lane < seg_e && keys[min(i0 + lane, count - 1)] != 0u;
            const unsigned keep_mask = __ballot_sync(0xffffffffu, keep);
            const int j = dst + __popc(keep_mask & ((1u << lane) - 1u));
            if (keep && j < picked) put(j, i0 + lane);
            dst += __popc(keep_mask);
        }
        if (tid == 0 && all != picked) atomicOr(a.status, kStatusBadIndex);
    }
    if (tid == 0) put(picked, count);
    if (list)
        for (int j = picked + 1 + tid; j < asked; j += kThreads) list[j] = -1;
}

}  // namespace

cudaError_t bounds_launch(const BlocksArgs& a, int first, int count, int num_sms, cudaStream_t stream) {
    if (count <= 0) return cudaSuccess;
    const long long blocks = ((long long)a.geo.units * count + 7) / 8;
    bounds_kernel<<<(unsigned)(blocks < num_sms * 8LL ? blocks : num_sms * 8LL), 256, 0, stream>>>(a, first, count);
    return cudaGetLastError();
}

cudaError_t blocks_prepare() {
    return cudaFuncSetAttribute(pick_kernel<512>, cudaFuncAttributeMaxDynamicSharedMemorySize, kCachedKeys * (int)sizeof(uint32_t));
}

cudaError_t pick_launch(const BlocksArgs& a, int count, int picked, int asked, int num_sms, int* launches, cudaStream_t stream) {
    *launches = 1;
    const bool chosen = picked > 0 && picked < count;
    int score_warps = 0;
    if (chosen && count > kScoreAlone && a.geo.units < num_sms / 2) {
        // Too few units to fill the GPU with a block of threads each: many score, then one each picks.  (Far from the limit of a grid's second dimension; the warps' sums fit behind the keys)
        const int per = kScoreWarps * kBatch, most = (4 * num_sms + a.geo.units - 1) / a.geo.units, parts = (count + per - 1) / per;
        const dim3 grid(parts < most ? parts : most, a.geo.units);
        score_warps = (int)grid.x * kScoreWarps;
        score_kernel<<<grid, 32 * kScoreWarps, 0, stream>>>(a, count);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
        *launches = 2;
    }
    cudaLaunchAttribute beside = {};
    beside.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    beside.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(a.geo.units);
    const int threads = count <= 128 ? 128 : count <= 256 ? 256 : 512;     // (a key each, where they are few)
    c.blockDim = dim3(threads);
    c.dynamicSmemBytes = chosen && count <= kCachedKeys ? (size_t)count * sizeof(uint32_t) : 0;
    c.stream = stream;
    c.attrs = &beside;
    c.numAttrs = score_warps > 0 ? 1 : 0;      // begins beside the end of the scores
    return cudaLaunchKernelEx(&c, threads == 128 ? pick_kernel<128> : threads == 256 ? pick_kernel<256> : pick_kernel<512>, a, count, picked, asked, score_warps);
}

}  // namespace lzk
