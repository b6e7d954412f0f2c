// Selection by the weight that tokens have received, and a cache cut down into another one.
//   weigh_select_kernel -- the budget - R - S heaviest of the unprotected slots, of equals the more recent (the tie rule of evict.cu),
//                          as the list "slot src[j] moves to slot j"
//   keep_kernel         -- gather of the listed rows and their state into another handle's pages
//   compact_weights_kernel -- the weights of an eviction in place
#include "internal.h"
#include "select.cuh"

namespace lzk {

namespace {

constexpr int kCachedKeys = 40 * 1024;     // keys of a unit kept in shared memory; longer caches read theirs from L2 in every pass

// Orders like the weights; what is no number counts as heavier than any.
__device__ __forceinline__ uint32_t weight_key(float w) {
    const uint32_t b = __float_as_uint(w);
    if ((b & 0x7FFFFFFFu) > 0x7F800000u) return 0xFFFFFFFFu;
    if (b == 0x80000000u) return 0x80000000u;              // (minus zero equals zero)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// One block per unit.  Three passes over 4 bytes per candidate find the cut (fewer when keys are few), two more write the list; the
// bytes are read from HBM once, and instructions bound it: 1024 units of 8192 tokens 57 us (1024 threads per unit 77), 4 us of bytes.
template <int kThreads, bool kCached>
__global__ void __launch_bounds__(kThreads) weigh_select_kernel(Geometry geo, StateView st, const float* weights, EvictArgs a) {
    constexpr int kWarps = kThreads / 32;
    extern __shared__ uint32_t cached[];
    __shared__ TopShared<uint32_t> sh;
    const int u = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int S = a.n_initial, R = a.n_recent, count = a.n - R - S, k = a.budget - R - S;
    int32_t* src = a.src + (size_t)u * a.budget;
    if (!in_bounds(S >= 0 && R >= 0 && k > 0 && k <= count && a.n <= geo.capacity && a.budget <= a.n, st.status)) return;
    const float* w = weights + (size_t)u * geo.capacity + S;
    if (kCached) {
        for (int i = tid; i < count; i += kThreads) cached[i] = weight_key(w[i]);
        __syncthreads();
    }
    auto key = [&](int i) -> uint32_t { return kCached ? cached[i] : weight_key(__ldg(w + i)); };
    const Cut<uint32_t> cut = top_cut<kThreads, uint32_t>(count, k, 32, sh, key);

    // Each warp owns a contiguous segment and walks it 32 at a time: ranks in slot order come from ballots.
    const int seg = ((count + kWarps - 1) / kWarps + 31) / 32 * 32;
    const int seg_b = min(count, warp * seg), seg_e = min(count, seg_b + seg);
    const unsigned lt = (1u << lane) - 1u;
    int above = 0, ties = 0;
    for (int i0 = seg_b; i0 < seg_e; i0 += 32) {
        const uint32_t x = i0 + lane < seg_e ? key(i0 + lane) : 0u;
        const bool in = i0 + lane < seg_e;
        above += __popc(__ballot_sync(0xffffffffu, in && x > cut.kth));
        ties += __popc(__ballot_sync(0xffffffffu, in && x == cut.kth));
    }
    int all_ties, all_kept;
    // (a warp's sums count once: lane 0 brings them, and every lane gets those of the warps before)
    const int ties_before = __shfl_sync(0xffffffffu, block_rank<kThreads>(lane == 0 ? ties : 0, sh.warp_sums, &all_ties), 0);
    const int first_tie = all_ties - cut.ties;             // of equals the more recent stay
    const int kept = above + max(0, min(ties, ties_before + ties - first_tie));
    const int kept_before = __shfl_sync(0xffffffffu, block_rank<kThreads>(lane == 0 ? kept : 0, sh.warp_sums, &all_kept), 0);
    int dst = S + kept_before, tie = ties_before, gone_first = count;
    for (int i0 = seg_b; i0 < seg_e; i0 += 32) {
        const bool in = i0 + lane < seg_e;
        const uint32_t x = in ? key(i0 + lane) : 0u;
        const bool equal = in && x == cut.kth;
        const unsigned tie_mask = __ballot_sync(0xffffffffu, equal);
        const bool keep = in && (x > cut.kth || (equal && tie + __popc(tie_mask & lt) >= first_tie));
        const unsigned keep_mask = __ballot_sync(0xffffffffu, keep), gone = __ballot_sync(0xffffffffu, in && !keep);
        const int to = dst + __popc(keep_mask & lt);
        if (keep && to < a.budget - R) src[to] = S + i0 + lane;
        if (gone != 0u && gone_first == count) gone_first = i0 + __ffs(gone) - 1;
        dst += __popc(keep_mask);
        tie += __popc(tie_mask);
    }
    for (int j = tid; j < S; j += kThreads) src[j] = j;
    for (int r = tid; r < R; r += kThreads) src[a.budget - R + r] = a.n - R + r;
    if (tid == 0) sh.count = count;
    __syncthreads();
    if (lane == 0 && gone_first < count) atomicMin(&sh.count, gone_first);
    __syncthreads();
    if (tid == 0) {
        a.first_moved[u] = S + sh.count;
        if (all_kept != k) atomicOr(st.status, kStatusBadIndex);
    }
}

constexpr int kKeepThreads = 512, kRowsPerWarp = kPageTokens / (kKeepThreads / 32);

// One block per destination page: the rows of 64 tokens in flight at once, K in the lower half of each warp, V in the upper.
// Bound by HBM, rows of 256 bytes scattered over the pages: 528 bytes per kept token read and written, and its weight.  1024 units, 2048
// of 8192 tokens: 385 us, 5.7 TB/s (four rows per warp; eight 420, two 550).  A begin beside the end of the selection: nothing for few
// units, 447 -> 462 us for the whole call of these.
__global__ void __launch_bounds__(kKeepThreads) keep_kernel(KeepArgs a) {
    const int u = blockIdx.y, d0 = blockIdx.x * kPageTokens, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int half = lane < 16 ? 0 : kPageHalfBytes, cp = lane & 15;
    const int32_t* src = a.src ? a.src + (size_t)u * a.keep : nullptr;
    const int32_t dpage = a.to.page_table[(size_t)u * a.to_geo.pages_per_unit + blockIdx.x];
    if (dpage < 0 || dpage >= a.to_geo.units * a.to_geo.pages_per_unit) {
        if (threadIdx.x == 0) atomicOr(a.to.status, kStatusBadIndex);
        return;
    }
    uint4 val[kRowsPerWarp];
    int from[kRowsPerWarp];
#pragma unroll
    for (int i = 0; i < kRowsPerWarp; ++i) {
        const int d = d0 + warp + kKeepThreads / 32 * i;
        from[i] = d >= a.keep ? -1 : src ? src[d] : d;
        if (from[i] >= a.n) from[i] = -1;
    }
#pragma unroll
    for (int i = 0; i < kRowsPerWarp; ++i) {
        if (from[i] < 0) continue;
        const int32_t pp = a.from.page_table[(size_t)u * a.from_geo.pages_per_unit + from[i] / kPageTokens];
        if (pp < 0 || pp >= a.from_geo.units * a.from_geo.pages_per_unit) {
            atomicOr(a.to.status, kStatusBadIndex);
            from[i] = -1;
            continue;
        }
        val[i] = __ldcs(reinterpret_cast<const uint4*>(a.from_pool + (size_t)pp * kPageBytes + half + (from[i] % kPageTokens) * kRowBytes + cp * 16));
    }
    uint8_t* page = a.to_pool + (size_t)dpage * kPageBytes + half;
#pragma unroll
    for (int i = 0; i < kRowsPerWarp; ++i) {
        if (from[i] < 0) continue;
        const int dr = warp + kKeepThreads / 32 * i;
        *reinterpret_cast<uint4*>(page + dr * kRowBytes + swz_chunk(cp ^ (from[i] & 7), dr) * 16) = val[i];
    }
    const int d = d0 + threadIdx.x;
    if (threadIdx.x < kPageTokens && d < a.keep) {
        const int s = src ? src[d] : d;
        if (s < 0 || s >= a.n) return;
        const size_t f = (size_t)u * a.from_geo.capacity + s, t = (size_t)u * a.to_geo.capacity + d;
        a.to.tsm[t] = a.from.tsm[f];
        a.to.pos[t] = a.from.pos[f];
        if (a.to_weights) a.to_weights[t] = a.from_weights ? a.from_weights[f] : 0.f;
    }
}

// One block per unit, destinations front to back: sources lie at or behind their destinations and ascend (as in compact_kernel).
constexpr int kCompactThreads = 1024;

__global__ void __launch_bounds__(kCompactThreads) compact_weights_kernel(Geometry geo, float* weights, EvictArgs a) {
    const int32_t* src = a.src + (size_t)blockIdx.x * a.budget;
    float* w = weights + (size_t)blockIdx.x * geo.capacity;
    const int first = a.first_moved[blockIdx.x];
    if (first < 0) return;
    for (int d0 = first; d0 < a.budget; d0 += kCompactThreads) {
        const int d = d0 + threadIdx.x, s = d < a.budget ? src[d] : -1;
        const float v = s >= 0 && s < a.n ? w[s] : 0.f;
        __syncthreads();
        if (s >= 0 && s < a.n) w[d] = v;
        __syncthreads();
    }
}

__global__ void weights_score_kernel(Geometry geo, const float* weights, int unit_begin, int unit_count, int n, double* out) {
    const size_t total = (size_t)unit_count * geo.capacity;
    for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (size_t)gridDim.x * blockDim.x)
        out[i] = (int)(i % geo.capacity) < n ? (double)weights[(size_t)unit_begin * geo.capacity + i] : 0.0;
}

}  // namespace

cudaError_t keep_prepare() {
    return cudaFuncSetAttribute(weigh_select_kernel<1024, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kCachedKeys * (int)sizeof(uint32_t));
}

cudaError_t weigh_select_launch(const Geometry& geo, StateView st, const float* weights, const EvictArgs& a, cudaStream_t stream) {
    const int count = a.n - a.n_recent - a.n_initial;
    const size_t smem = (size_t)count * sizeof(uint32_t);
    if (count <= 2048)
        weigh_select_kernel<256, true><<<geo.units, 256, smem, stream>>>(geo, st, weights, a);
    else if (count <= 8192)
        weigh_select_kernel<512, true><<<geo.units, 512, smem, stream>>>(geo, st, weights, a);
    else if (count <= kCachedKeys)
        weigh_select_kernel<1024, true><<<geo.units, 1024, smem, stream>>>(geo, st, weights, a);
    else
        weigh_select_kernel<1024, false><<<geo.units, 1024, 0, stream>>>(geo, st, weights, a);
    return cudaGetLastError();
}

cudaError_t keep_launch(const KeepArgs& a, cudaStream_t stream) {
    const int units = a.to_geo.units, pages = (a.keep + kPageTokens - 1) / kPageTokens;
    // (a grid's second dimension ends at 65535)
    for (int u0 = 0; u0 < units; u0 += 65535) {
        KeepArgs part = a;
        const int count = units - u0 < 65535 ? units - u0 : 65535;
        part.from.page_table += (size_t)u0 * a.from_geo.pages_per_unit;
        part.to.page_table += (size_t)u0 * a.to_geo.pages_per_unit;
        part.from.tsm += (size_t)u0 * a.from_geo.capacity;
        part.from.pos += (size_t)u0 * a.from_geo.capacity;
        part.to.tsm += (size_t)u0 * a.to_geo.capacity;
        part.to.pos += (size_t)u0 * a.to_geo.capacity;
        if (a.src) part.src += (size_t)u0 * a.keep;
        if (a.from_weights) part.from_weights += (size_t)u0 * a.from_geo.capacity;
        if (a.to_weights) part.to_weights += (size_t)u0 * a.to_geo.capacity;
        keep_kernel<<<dim3(pages, count), kKeepThreads, 0, stream>>>(part);
    }
    return cudaGetLastError();
}

cudaError_t compact_weights_launch(const Geometry& geo, float* weights, const EvictArgs& a, cudaStream_t stream) {
    compact_weights_kernel<<<geo.units, kCompactThreads, 0, stream>>>(geo, weights, a);
    return cudaGetLastError();
}

cudaError_t weights_score_launch(const Geometry& geo, const float* weights, int unit_begin, int unit_count, int n, double* out, cudaStream_t stream) {
    const size_t total = (size_t)unit_count * geo.capacity;
    const int blocks = (int)((total + 255) / 256 < 148 * 8 ? (total + 255) / 256 : 148 * 8);
    weights_score_kernel<<<blocks, 256, 0, stream>>>(geo, weights, unit_begin, unit_count, n, out);
    return cudaGetLastError();
}

}  // namespace lzk
