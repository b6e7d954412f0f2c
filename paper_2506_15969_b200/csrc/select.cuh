// The k largest of a block's keys: radix select with 11-bit digits, most significant first.
#pragma once

#include "common.cuh"

namespace lzk {

constexpr int kDigitBits = 11, kBins = 1 << kDigitBits;
constexpr int kSurvivors = 256;            // few enough to be ranked one against the other

template <typename Key>
struct TopShared {
    unsigned hist[kBins];
    Key surv[kSurvivors];
    int warp_sums[32];
    Key prefix;
    int rem, count, n_surv;
};

// What stays of `count` keys: those above `kth`, and `ties` of those equal to it.
template <typename Key>
struct Cut {
    Key kth;
    int ties;
};

// Sum over the lower threads (and, in `total`, over all) of one int each.  Every thread of a block of kThreads calls it.
template <int kThreads>
__device__ __forceinline__ int block_rank(int v, int* warp_sums, int* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += up;
    }
    __syncthreads();                       // (the sums may still be read from a call before)
    if (lane == 31) warp_sums[warp] = incl;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        before += w < warp ? warp_sums[w] : 0;
        all += warp_sums[w];
    }
    *total = all;
    return before + incl - v;
}

// The cut of the k largest (1 <= k <= count) of key(0) .. key(count - 1), all below 2^width.  One pass over the keys per digit, until
// the k-th key's bin is wanted whole or holds few keys, which are ranked directly.
template <int kThreads, typename Key, typename Load>
__device__ Cut<Key> top_cut(int count, int k, int width, TopShared<Key>& sh, const Load& key) {
    static_assert(kBins % kThreads == 0, "");
    constexpr int kPer = kBins / kThreads;
    const int tid = threadIdx.x;
    Key prefix = 0, mask = 0;
    int rem = k;
    for (int left = width; left > 0;) {
        const int bits = left < kDigitBits ? left : kDigitBits, shift = left - bits;
        for (int i = tid; i < kBins; i += kThreads) sh.hist[i] = 0;
        __syncthreads();
        for (int i0 = 0; i0 < count; i0 += kThreads) {
            const int i = i0 + tid;
            const Key x = i < count ? key(i) : Key(0);
            const bool on = i < count && (x & mask) == prefix;
            const unsigned digit = on ? (unsigned)(x >> shift) & (unsigned)(kBins - 1) & ((1u << bits) - 1u) : kBins;
            // equal keys are common (weights that are all zero): one addition for a warp that agrees
            int same;
            __match_all_sync(0xffffffffu, digit, &same);
            if (same) {
                if (on && (tid & 31) == 0) atomicAdd(&sh.hist[digit], 32u);
            } else if (on) {
                atomicAdd(&sh.hist[digit], 1u);
            }
        }
        __syncthreads();
        // bins from the top: thread t takes bins kBins - 1 - kPer t and below
        int own = 0;
#pragma unroll
        for (int b = 0; b < kPer; ++b) own += (int)sh.hist[kBins - 1 - kPer * tid - b];
        int total;
        int above = block_rank<kThreads>(own, sh.warp_sums, &total);
        if (above < rem && rem <= above + own) {
#pragma unroll 1
            for (int b = 0; b < kPer; ++b) {
                const int bin = kBins - 1 - kPer * tid - b, here = (int)sh.hist[bin];
                if (rem <= above + here) {
                    sh.prefix = prefix | ((Key)bin << shift);
                    sh.rem = rem - above;
                    sh.count = here;
                    break;
                }
                above += here;
            }
        }
        __syncthreads();
        prefix = sh.prefix;
        rem = sh.rem;
        mask |= (Key)((1u << bits) - 1u) << shift;
        left = shift;
        const int here = sh.count;
        if (here == rem) {                 // the whole bin stays: everything from the prefix on
            if (left == 0 || prefix == 0) return Cut<Key>{prefix, rem};
            return Cut<Key>{(Key)(prefix - 1), 0};
        }
        if (left > 0 && here <= kSurvivors && here <= kThreads) {
            if (tid == 0) sh.n_surv = 0;
            __syncthreads();
            for (int i = tid; i < count; i += kThreads) {
                const Key x = key(i);
                if ((x & mask) == prefix) sh.surv[atomicAdd(&sh.n_surv, 1)] = x;
            }
            __syncthreads();
            if (tid < here) {
                const Key mine = sh.surv[tid];
                int greater = 0, equal = 0;
                for (int j = 0; j < here; ++j) {
                    greater += sh.surv[j] > mine;
                    equal += sh.surv[j] == mine;
                }
                if (greater < rem && rem <= greater + equal) {     // equal keys all write the same two values
                    sh.prefix = mine;
                    sh.rem = rem - greater;
                }
            }
            __syncthreads();
            return Cut<Key>{sh.prefix, sh.rem};
        }
        __syncthreads();
    }
    return Cut<Key>{prefix, rem};       // (of no width at all: every key is zero, and k of them stay)
}

}  // namespace lzk
