// Attention over the blocks of a cache that a cheap score selects, for a decode step's queries.
//
// A block is a page, 64 tokens.  For every block b before the newest its keys' bounds are kept, per dimension d:
//   high_b[d] = max_i k_i[d],   low_b[d] = min_i k_i[d]
// and a unit's G query heads give it the score
//   s_b = sum_g sum_d max(q_g[d] high_b[d], q_g[d] low_b[d]) = sum_d (P[d] high_b[d] + N[d] low_b[d]),
//   P[d] = sum_g max(q_g[d], 0),  N[d] = sum_g min(q_g[d], 0):
// no key between the bounds has larger logits summed over the heads.  The products are exact, and the sums are taken in fp64, where
// orders of magnitude and of summation do not move a score past its neighbour: which blocks are read does not depend on rounding.
// The newest block (the only one that may be partly filled) and the blocks - 1 best others, of equals the older, become a
// page table of their own, in order, which the decode kernel reads like any other: K and V of blocks * 64 tokens instead of n.
//
//   bounds_kernel -- the bounds, once per block (keys behind the newest block do not change any more)
//   score_kernel  -- 512 bytes per block and 256 fp64 fmas: a warp per block, lanes 0-15 the high row, 16-31 the low one
//   pick_kernel   -- one block of threads per unit: radix select over the scores, page table, list
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

// Larger scores have larger keys; what is no number comes first of all.  (The select starts at 1: 0 is no score's.)
__device__ __forceinline__ unsigned long long score_key(double s) {
    if (s != s) return ~0ull;
    const long long b = __double_as_longlong(s == 0.0 ? 0.0 : s);
    return b < 0 ? ~(unsigned long long)b : (unsigned long long)b | 0x8000000000000000ull;
}

constexpr int kScoreThreads = 256, kBlocksPerWarp = 8;

__global__ void __launch_bounds__(kScoreThreads) score_kernel(BlocksArgs a, int count) {
    const int u = blockIdx.y, lane = threadIdx.x & 31, c = lane & 15, G = a.geo.group;
    // this lane's eight dimensions of P (lanes 0-15) or N
    double part[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    const uint4* q = reinterpret_cast<const uint4*>(a.q) + (size_t)u * G * kChunksPerRow + c;
    for (int g = 0; g < G; ++g) {
        const uint4 x = q[g * kChunksPerRow];
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float e0 = bf16_lo_as_float(w[i]), e1 = bf16_hi_as_float(w[i]);
            // (what is no number goes into both sums)
            part[2 * i] += e0 != e0 || (lane < 16 ? e0 > 0.f : e0 < 0.f) ? (double)e0 : 0.0;
            part[2 * i + 1] += e1 != e1 || (lane < 16 ? e1 > 0.f : e1 < 0.f) ? (double)e1 : 0.0;
        }
    }
    const int warp = (blockIdx.x * kScoreThreads + threadIdx.x) >> 5, b0 = warp * kBlocksPerWarp;
    const uint4* rows = reinterpret_cast<const uint4*>(a.bounds) + (size_t)u * a.geo.pages_per_unit * 2 * kChunksPerRow + lane;
    uint4 x[kBlocksPerWarp];
#pragma unroll
    for (int i = 0; i < kBlocksPerWarp; ++i)
        x[i] = b0 + i < count ? rows[(size_t)(b0 + i) * 2 * kChunksPerRow] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int i = 0; i < kBlocksPerWarp; ++i) {
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
        double s = 0.0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            s = fma(part[2 * j], (double)bf16_lo_as_float(w[j]), s);
            s = fma(part[2 * j + 1], (double)bf16_hi_as_float(w[j]), s);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0 && b0 + i < count) a.keys[(size_t)u * a.geo.pages_per_unit + b0 + i] = score_key(s);
    }
}

constexpr int kPickThreads = 512, kPickWarps = kPickThreads / 32;

// Candidates are blocks 0 .. count - 1, `picked` of them (may be 0, or all) are taken; then the newest block.
__global__ void __launch_bounds__(kPickThreads) pick_kernel(BlocksArgs a, int count, int picked, int asked) {
    __shared__ TopShared<unsigned long long> sh;
    const int u = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const unsigned long long* keys = a.keys + (size_t)u * a.geo.pages_per_unit;
    const int32_t* table = a.page_table + (size_t)u * a.geo.pages_per_unit;
    int32_t* to = a.table + (size_t)u * a.geo.pages_per_unit;
    int32_t* list = a.selected ? a.selected + (size_t)u * asked : nullptr;
    auto put = [&](int j, int block) {
        to[j] = table[block];
        if (list) list[j] = block;
    };
    if (picked == count) {                                  // all of them
        for (int b = tid; b < count; b += kPickThreads) put(b, b);
    } else if (picked > 0) {
        const Cut<unsigned long long> cut = top_cut<kPickThreads, unsigned long long>(count, picked, sh, [&](int i) { return keys[i]; });
        const int seg = ((count + kPickWarps - 1) / kPickWarps + 31) / 32 * 32;
        const int seg_b = min(count, warp * seg), seg_e = min(count, seg_b + seg);
        const unsigned lt = (1u << lane) - 1u;
        int above = 0, ties = 0;
        for (int i0 = seg_b; i0 < seg_e; i0 += 32) {
            const bool in = i0 + lane < seg_e;
            const unsigned long long x = in ? keys[i0 + lane] : 0ull;
            above += __popc(__ballot_sync(0xffffffffu, in && x > cut.kth));
            ties += __popc(__ballot_sync(0xffffffffu, in && x == cut.kth));
        }
        int all;
        const int ties_before = __shfl_sync(0xffffffffu, block_rank<kPickThreads>(lane == 0 ? ties : 0, sh.warp_sums, &all), 0);
        const int kept = above + max(0, min(ties, cut.ties - ties_before));
        const int before = __shfl_sync(0xffffffffu, block_rank<kPickThreads>(lane == 0 ? kept : 0, sh.warp_sums, &all), 0);
        int dst = before, tie = ties_before;
        for (int i0 = seg_b; i0 < seg_e; i0 += 32) {
            const bool in = i0 + lane < seg_e;
            const unsigned long long x = in ? keys[i0 + lane] : 0ull;
            const bool equal = in && x == cut.kth;
            const unsigned tie_mask = __ballot_sync(0xffffffffu, equal);
            const bool keep = in && (x > cut.kth || (equal && tie + __popc(tie_mask & lt) < cut.ties));
            const unsigned keep_mask = __ballot_sync(0xffffffffu, keep);
            const int j = dst + __popc(keep_mask & lt);
            if (keep && j < picked) put(j, i0 + lane);
            dst += __popc(keep_mask);
            tie += __popc(tie_mask);
        }
        if (tid == 0 && all != picked) atomicOr(a.status, kStatusBadIndex);
    }
    if (tid == 0) put(picked, count);
    if (list)
        for (int j = picked + 1 + tid; j < asked; j += kPickThreads) list[j] = -1;
}

}  // namespace

cudaError_t bounds_launch(const BlocksArgs& a, int first, int count, int num_sms, cudaStream_t stream) {
    if (count <= 0) return cudaSuccess;
    const long long blocks = ((long long)a.geo.units * count + 7) / 8;
    bounds_kernel<<<(unsigned)(blocks < num_sms * 8LL ? blocks : num_sms * 8LL), 256, 0, stream>>>(a, first, count);
    return cudaGetLastError();
}

cudaError_t pick_launch(const BlocksArgs& a, int count, int picked, int asked, cudaStream_t stream) {
    if (picked > 0 && picked < count) {
        const int per = kScoreThreads / 32 * kBlocksPerWarp;
        for (int u0 = 0; u0 < a.geo.units; u0 += 65535) {  // (a grid's second dimension ends at 65535)
            BlocksArgs part = a;
            part.q = reinterpret_cast<const uint4*>(a.q) + (size_t)u0 * a.geo.group * kChunksPerRow;
            part.bounds = reinterpret_cast<uint8_t*>(a.bounds) + (size_t)u0 * a.geo.pages_per_unit * 2 * kRowBytes;
            part.keys += (size_t)u0 * a.geo.pages_per_unit;
            const int some = a.geo.units - u0 < 65535 ? a.geo.units - u0 : 65535;
            score_kernel<<<dim3((count + per - 1) / per, some), kScoreThreads, 0, stream>>>(part, count);
        }
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    pick_kernel<<<a.geo.units, kPickThreads, 0, stream>>>(a, count, picked, asked);
    return cudaGetLastError();
}

}  // namespace lzk
