// C-ABI layer: host-side handle, argument validation, step / eviction schedule, launches.
#include <limits.h>
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <atomic>
#include <map>
#include <utility>
#include <vector>

#include "../../include/lazyev.h"
#include "internal.h"

using namespace lzk;

// Units per SM from which own caches of n tokens behind a prefix get a warp each (measured pairs: decode_short.cu).
constexpr int short_units_per_sm(int n) { return n <= 128 ? 3 : 4; }
constexpr int kHostChunks = 3;            // unit ranges the host-buffer entry point pipelines copies over

struct lazyev {
    // configuration
    int layers = 0, batch = 1, q_heads = 0, kv_heads = 0, head_dim = 0;
    int budget = 0, budget_now = 0, window = 0, n_recent = 0, n_initial = 0, max_prefill = 0;
    float alpha = 0.f;
    int auto_evict = 1, score_mode = LAZYEV_SCORE_H1_PLUS_H2, force_splits = 0, force_stages = 0, force_groups = 0;
    int prompt_mode = LAZYEV_PROMPT_TILED;
    float* prompt_dump = nullptr;          // optional per-row probabilities of the prompt pass (caller's device memory)
    int prompt_dump_begin = 0, prompt_dump_count = 0;
    unsigned long long wait_limit_ns = 2000000000ull;   // bounded waits in the kernels give up after this long
    int stop_after_pages = -1;             // diagnostics: starve the decode kernel's page ring (-1: off)
    int fuse_append = 1;                   // small problems: the append runs inside the decode launch
    // derived at bind
    bool bound = false, prefilled = false;
    int units = 0, group = 0, capacity = 0, pages_per_unit = 0;
    int device = -1, num_sms = 0, max_smem = 0;
    cudaStream_t stream = nullptr;
    uint8_t* pool = nullptr;
    StateView st = {};
    int32_t* src = nullptr;
    int32_t* first_moved = nullptr;
    int32_t* radix_list = nullptr;         // [units] + the counter behind it
    // staging of the host-buffer entry points: two slots, so that the copies of one step run beside
    // the kernels of the step before it
    uint8_t* stage_q[2] = {nullptr, nullptr};
    uint8_t* stage_k[2] = {nullptr, nullptr};
    uint8_t* stage_v[2] = {nullptr, nullptr};
    uint8_t* stage_out[2] = {nullptr, nullptr};
    double* stage_score = nullptr;
    unsigned long long* stage_hist = nullptr;
    uint8_t* stage_rows = nullptr;         // queries of lazyev_decode_step_rows(), normalised and rotated
    // the weights that tokens receive (lazyev_set_weights), and what the calls on a whole cache keep
    int weights_on = 0;
    float* weights = nullptr;              // [units][capacity], behind the status word in the state region
    int32_t* counters = nullptr;           // scratch of the chunk kernels, zero between launches: [2][kChunkCounters]
    bool counted = false;                  // such a kernel has been launched, or captured
    PrefixPool own_pool = {};              // the own pool as the chunk kernels address it
    uint8_t* block_space = nullptr;        // lazyev_set_block_workspace()
    int indexed = 0;                       // blocks, from the first on, whose bounds are in it
    double* h2_table = nullptr;            // H2 term per MRI value (scratch), valid for h2_table_mode
    int h2_table_mode = -1;
    // host-buffer entry point: copy streams and events, created at its first call
    cudaStream_t copy_in = nullptr, copy_out = nullptr;
    // second launch of a step (the partly filled last round) runs beside the end of the main launch
    cudaStream_t tail_stream = nullptr;
    cudaEvent_t ev_fork = nullptr, ev_join = nullptr;
    cudaEvent_t ev_in[kHostChunks + 1] = {}, ev_done[kHostChunks + 1] = {}, ev_ready = nullptr;
    // asynchronous host-buffer steps: completion event per staging slot, steps queued so far, and
    // whether the slot's last step may still be in flight
    cudaEvent_t ev_step_done[2] = {nullptr, nullptr};
    long long host_seq = 0;
    bool slot_busy[2] = {false, false};
    int last_host_ranges = 0;
    // what the calls that take projected rows do to queries and keys
    double turns[kMaxPairs] = {0};         // per position: inv_freq / (2 pi)
    int pairs = 0, interleaved = 0;
    float amplitude = 1.f, norm_eps = 0.f;
    const float* q_weight = nullptr;
    const float* k_weight = nullptr;
    // a prefix shared by this handle's sequences (another handle), and how many handles share this one
    lazyev* shared = nullptr;
    PrefixPlan prefix_plan = {};
    PrefixPool prefix_pool = {};           // the prefix's pool as the kernel addresses it
    float* prefix_o = nullptr;
    float2* prefix_ml = nullptr;
    std::atomic<int> users{0};             // (its users may live on threads of their own)
    // progress
    int t = 0, n = 0, prefill = 0;
    int pos_base = 0;                      // position of the first own token: the prefix's next one
    long long launches = 0, evictions = 0;
    DecodePlan last_plan = {};
    int last_grid = 0, last_tail_units = 0, last_tail_splits = 0;
    struct Shape {
        int splits = 1, clusters = 1, tail_splits = 0, tail_units = 0, forced_splits = 0, forced_stages = 0, forced_groups = 0;
    };
    std::map<int, Shape> plan_cache;                       // pages in use -> launch shape
    // optional per-kernel timing with CUDA events
    struct Span {
        cudaEvent_t start, stop;
        int kind;
        double bytes;
    };
    bool profiling = false;
    std::vector<Span> pending;
    std::vector<cudaEvent_t> free_events;
    lazyev_profile_t prof = {};
    char err[256] = {0};
};

namespace {

constexpr int kScoreStageUnits = 32;      // units whose scores one dump pass evaluates
constexpr int kMaxHistBins = 1 << 16;     // bins of lazyev_mri_histogram()

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

int fail(lazyev_t* h, int code, const char* fmt, ...) {
    if (h) {
        va_list ap;
        va_start(ap, fmt);
        vsnprintf(h->err, sizeof(h->err), fmt, ap);
        va_end(ap);
    }
    return code;
}

int cuda_fail(lazyev_t* h, cudaError_t e, const char* what) {
    return fail(h, LAZYEV_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}

void derive(lazyev_t* h) {
    h->units = h->layers * h->batch * h->kv_heads;
    h->group = h->q_heads / h->kv_heads;
    const int cap = (h->budget > h->max_prefill ? h->budget : h->max_prefill) + h->window;
    h->pages_per_unit = (cap + kPageTokens - 1) / kPageTokens;
    h->capacity = h->pages_per_unit * kPageTokens;
}

struct Sizes {
    size_t kv, state, scratch;
    size_t off_tsm, off_pos, off_pbar, off_status, off_weights;                     // inside state
    size_t off_first, off_rlist, off_q, off_k, off_v, off_out, off_score, off_hist, off_h2, off_rows, off_counters;    // inside scratch
};

Sizes sizes_of(const lazyev_t* h) {
    Sizes s;
    const size_t slots = (size_t)h->units * h->capacity;
    s.kv = (size_t)h->units * h->pages_per_unit * kPageBytes;
    size_t off = align_up((size_t)h->units * h->pages_per_unit * sizeof(int32_t), 256);
    s.off_tsm = off;                       // (TS, MRI) pairs
    off += align_up(slots * 8, 256);
    s.off_pos = off;
    off += align_up(slots * 4, 256);
    s.off_pbar = off;
    off += align_up(slots * 4, 256);
    s.off_status = off;
    off += 256;
    s.off_weights = off;
    if (h->weights_on) off += align_up(slots * 4, 256);
    s.state = off;
    off = align_up((size_t)h->units * h->budget * sizeof(int32_t), 256);
    s.off_first = off;
    off += align_up((size_t)h->units * sizeof(int32_t), 256);
    s.off_rlist = off;
    off += align_up(((size_t)h->units + 1) * sizeof(int32_t), 256);
    const size_t qbytes = (size_t)h->layers * h->batch * h->q_heads * kRowBytes;
    const size_t kbytes = (size_t)h->layers * h->batch * h->kv_heads * kRowBytes;
    s.off_q = off;                          // each staging area holds two slots
    off += 2 * align_up(qbytes, 256);
    s.off_k = off;
    off += 2 * align_up(kbytes, 256);
    s.off_v = off;
    off += 2 * align_up(kbytes, 256);
    s.off_out = off;
    off += 2 * align_up(qbytes, 256);
    s.off_score = off;
    off += align_up((size_t)kScoreStageUnits * h->capacity * sizeof(double), 256);
    s.off_hist = off;
    off += align_up((size_t)kMaxHistBins * sizeof(unsigned long long), 256);
    s.off_h2 = off;
    off += align_up((size_t)kH2TableEntries * sizeof(double), 256);
    s.off_rows = off;
    off += align_up(qbytes, 256);
    s.off_counters = off;
    off += 2 * kChunkCounters * sizeof(int32_t);
    s.scratch = off;
    return s;
}

Geometry geometry(const lazyev_t* h) { return Geometry{h->units, h->group, h->pages_per_unit, h->capacity}; }

int check_device_status(lazyev_t* h) {
    int32_t status = 0;
    cudaError_t e = cudaMemcpyAsync(&status, h->st.status, sizeof(status), cudaMemcpyDeviceToHost, h->stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(h->stream);
    if (e != cudaSuccess) return cuda_fail(h, e, "reading the device status word");
    if (status != 0) return fail(h, LAZYEV_EDEVICE, "device status word = %d (1: wait timed out, 2: bad index)", status);
    return LAZYEV_OK;
}

enum { kSpanAppend = 0, kSpanDecode = 1, kSpanSelect = 2, kSpanCompact = 3 };

cudaEvent_t take_event(lazyev_t* h) {
    if (!h->free_events.empty()) {
        cudaEvent_t e = h->free_events.back();
        h->free_events.pop_back();
        return e;
    }
    cudaEvent_t e = nullptr;
    cudaEventCreate(&e);
    return e;
}

// Brackets one kernel launch with events when profiling is on.
struct SpanGuard {
    lazyev_t* h;
    lazyev::Span span;
    bool on;
    SpanGuard(lazyev_t* h_, int kind, double bytes, bool counted = true) : h(h_), on(h_->profiling && counted) {
        if (!on) return;
        span.start = take_event(h);
        span.stop = take_event(h);
        span.kind = kind;
        span.bytes = bytes;
        cudaEventRecord(span.start, h->stream);
    }
    ~SpanGuard() {
        if (!on) return;
        cudaEventRecord(span.stop, h->stream);
        h->pending.push_back(span);
    }
};

int collect_profile(lazyev_t* h) {
    if (h->pending.empty()) return LAZYEV_OK;
    cudaError_t e = cudaStreamSynchronize(h->stream);
    if (e != cudaSuccess) return cuda_fail(h, e, "stream synchronisation");
    for (const lazyev::Span& sp : h->pending) {
        float ms = 0.f;
        cudaEventElapsedTime(&ms, sp.start, sp.stop);
        switch (sp.kind) {
            case kSpanAppend: h->prof.append_ms += ms; h->prof.append_launches++; break;
            case kSpanDecode: h->prof.decode_ms += ms; h->prof.decode_launches++; h->prof.decode_bytes += sp.bytes; break;
            case kSpanSelect: h->prof.select_ms += ms; h->prof.select_launches++; h->prof.select_bytes += sp.bytes; break;
            default: h->prof.compact_ms += ms; h->prof.compact_launches++; break;
        }
        h->free_events.push_back(sp.start);
        h->free_events.push_back(sp.stop);
    }
    h->pending.clear();
    return LAZYEV_OK;
}

// Candidates of an eviction over n cached tokens, or -1 when the select kernel cannot hold them.
int candidates_of(const lazyev_t* h, int n) {
    const int ncand = n - h->n_recent - h->n_initial;
    if (ncand <= 0 || (h->score_mode != LAZYEV_SCORE_WEIGHT && select_smem_bytes(ncand) > 200 * 1024)) return -1;
    return ncand;
}

bool evict_due_at(const lazyev_t* h, int t, int n) { return t != 0 && t % h->window == 0 && n > h->budget_now; }

// Which tokens stay when every unit is cut to `keep` of its h->n tokens: the select launches, into the work lists `src` and
// `first_moved`, the bound scratch region's or the library's own.  `counted`: the profile's sums take them in.
int run_select(lazyev_t* h, int keep, int32_t* src, int32_t* first_moved, int32_t* radix_list, bool counted, EvictArgs* args) {
    const int ncand = candidates_of(h, h->n);
    if (ncand < 0)
        return fail(h, LAZYEV_EINVAL, "eviction over %d candidates is not supported", h->n - h->n_recent - h->n_initial);
    cudaError_t e;
    const bool by_weight = h->score_mode == LAZYEV_SCORE_WEIGHT;
    if (!by_weight && h->h2_table_mode != h->score_mode) {      // the H2 term per MRI value, in the variant the mode selects
        e = h2_table_launch(h->score_mode, kH2TableEntries, h->h2_table, h->stream);
        if (e != cudaSuccess) return cuda_fail(h, e, "H2 table launch");
        h->h2_table_mode = h->score_mode;
        h->launches += 1;
    }
    EvictArgs& a = *args;
    a.n = h->n;
    a.budget = keep;
    a.n_recent = h->n_recent;
    a.n_initial = h->n_initial;
    a.t = h->t;
    a.score_mode = h->score_mode;
    a.src = src;
    a.first_moved = first_moved;
    a.h2_table = h->h2_table;
    a.h2_entries = kH2TableEntries;
    a.radix_list = radix_list;
    a.radix_count = radix_list + h->units;
    const Geometry geo = geometry(h);
    {
        // algorithmic bytes: TS and MRI (the weight) of every candidate read, the source list written
        SpanGuard g(h, kSpanSelect, (double)h->units * ((by_weight ? 4.0 : 8.0) * ncand + 4.0 * a.budget), counted);
        e = by_weight ? weigh_select_launch(geo, h->st, h->weights, a, h->stream) : select_launch(geo, h->st, a, h->num_sms, h->stream);
    }
    if (e != cudaSuccess) return cuda_fail(h, e, "select kernel launch");
    h->launches += by_weight ? 1 : 2;        // (the selection by score is two launches)
    return LAZYEV_OK;
}

// Cuts every unit to its `keep` < h->n best tokens, in place.
int run_cut(lazyev_t* h, int keep, int* evicted, int32_t* src, int32_t* first_moved, int32_t* radix_list) {
    EvictArgs a;
    const int rc = run_select(h, keep, src, first_moved, radix_list, true, &a);
    if (rc != LAZYEV_OK) return rc;
    const Geometry geo = geometry(h);
    cudaError_t e;
    {
        SpanGuard g(h, kSpanCompact, 0.0);
        e = compact_launch(geo, h->pool, h->st, a, h->stream);
    }
    if (e != cudaSuccess) return cuda_fail(h, e, "compact kernel launch");
    h->launches += 1;
    if (h->weights) {
        e = compact_weights_launch(geo, h->weights, a, h->stream);
        if (e != cudaSuccess) return cuda_fail(h, e, "weight compaction launch");
        h->launches += 1;
    }
    h->indexed = 0;                          // (the blocks hold other tokens now)
    h->evictions += 1;
    if (evicted) *evicted = h->n - keep;
    h->n = keep;
    if (h->profiling) {
        // rows that actually moved: every destination from the first evicted slot on
        std::vector<int32_t> first(h->units);
        e = cudaMemcpyAsync(first.data(), first_moved, first.size() * 4, cudaMemcpyDeviceToHost, h->stream);
        if (e == cudaSuccess) e = cudaStreamSynchronize(h->stream);
        if (e != cudaSuccess) return cuda_fail(h, e, "first_moved download");
        double rows = 0;
        for (int32_t f : first) rows += a.budget - f;
        // per moved row: K and V rows and three state words read and written, one source index read
        h->prof.compact_bytes += rows * (2.0 * (2 * kRowBytes + 12) + 4.0);
        h->prof.compact_rows += rows;
    }
    return LAZYEV_OK;
}

// The lagged eviction of Section 4 at the current step, if one is due.
int run_evict(lazyev_t* h, int* evicted, int32_t* src, int32_t* first_moved, int32_t* radix_list) {
    if (evicted) *evicted = 0;
    if (!evict_due_at(h, h->t, h->n)) return LAZYEV_OK;
    return run_cut(h, h->budget_now, evicted, src, first_moved, radix_list);
}

// A new sequence's tokens [slot, slot + count) have received nothing yet.
cudaError_t clear_weights(lazyev_t* h, int slot, int count) {
    if (!h->weights || count <= 0) return cudaSuccess;
    return cudaMemset2DAsync(h->weights + slot, (size_t)h->capacity * sizeof(float), 0, (size_t)count * sizeof(float), h->units, h->stream);
}

// Host side of a pipelined step: queries come from and outputs go to host memory in unit ranges, on
// two copy streams, while the decode launches of the other ranges run.
struct HostPipe {
    const uint8_t* q_host;
    uint8_t* out_host;
};

// The new token of a step (S1), when the step has one.
struct NewToken {
    const void* k;
    const void* v;
    int position;
};

// The prefix launch of a step (a handle with a shared prefix): partial sums of every query row over the prefix, which
// the decode launches start from.
cudaError_t run_prefix(lazyev_t* h, const void* q) {
    const lazyev_t* src = h->shared;
    PrefixArgs a;
    a.pool = &h->prefix_pool;
    a.page_table = src->st.page_table;
    a.n = src->n;
    a.pages_per_unit = src->pages_per_unit;
    a.total_pages = src->units * src->pages_per_unit;
    a.layers = h->layers;
    a.q = q;
    a.o = h->prefix_o;
    a.ml = h->prefix_ml;
    a.status = h->st.status;
    a.wait_limit_ns = h->wait_limit_ns;
    a.stop_after_tiles = h->stop_after_pages;
    h->launches += 1;
    return prefix_launch(h->prefix_plan, a, h->stream);
}

// How a step's attention over n own tokens is launched.
struct DecodeLaunch {
    DecodeConfig config;
    lazyev::Shape shape;
    DecodePlan plan, tail_plan;
    bool brief;                            // a warp per unit
};

// Chooses it, or refuses the call; queues nothing.
int choose_decode(lazyev_t* h, const void* q, const void* out, int n, bool track, DecodeLaunch* launch) {
    // (the kernels load pairs of elements of q, or tiles of it over a prefix, and store single elements of out)
    if (h->shared && ((uintptr_t)q & 15)) return fail(h, LAZYEV_EINVAL, "q must be 16-byte aligned while a prefix is attached");
    if (((uintptr_t)q & 3) || ((uintptr_t)out & 1)) return fail(h, LAZYEV_EINVAL, "q must be 4-byte aligned, out 2-byte aligned");
    cudaError_t e = cudaSuccess;
    const DecodeConfig c{h->units, h->group, h->pages_per_unit, h->capacity, track ? h->alpha : INFINITY, h->force_splits, h->force_stages, h->force_groups,
                         h->wait_limit_ns, h->stop_after_pages, h->shared != nullptr};
    // Launch shape, chosen per number of pages in use and cached.  For every cluster size whose logits
    // fit, a small time model gives the time of the rounds of the round-robin walk; the main launch is
    // the size with the least total.  A partly filled last round goes to a second launch with larger
    // clusters when that is faster, so that more SMs share its units.
    const int np = (n + kPageTokens - 1) / kPageTokens;
    // Short own caches behind a prefix: one launch with a warp per unit, where there are enough units for it.  It stores two
    // elements of `out` at a time, the block-per-unit kernel single ones: an `out` at an odd element goes there.
    const bool brief = h->shared && n <= kShortTokens && h->units >= short_units_per_sm(n) * h->num_sms && h->force_splits == 0 &&
                       h->force_stages == 0 && h->force_groups == 0 && ((uintptr_t)out & 3) == 0;
    auto cached = h->plan_cache.find(np);
    const bool planned = cached != h->plan_cache.end() && cached->second.forced_splits == h->force_splits &&
                         cached->second.forced_stages == h->force_stages && cached->second.forced_groups == h->force_groups;
    if (!planned && !brief) {
        lazyev::Shape best;
        best.forced_splits = h->force_splits;
        best.forced_stages = h->force_stages;
        best.forced_groups = h->force_groups;
        // Time model, in units of the time one block needs for one page when it is not limited by HBM
        // (fitted on B200 at 8 k tokens per unit): a round of `m` units on clusters of s blocks takes
        //   max(pages per block + kFixedPages, kHbmPageTime * m * np / SMs) / ring weight
        // -- a fixed cost per unit (merge, pipeline refill), and the HBM floor once many SMs stream; a second
        // launch costs kSecondLaunchPages on top of its round.
        static const double kRingWeight[7] = {0, 0, 0.70, 0.90, 0.96, 0.99, 1.0};
        constexpr double kFixedPages = 8.0, kHbmPageTime = 1.12, kSecondLaunchPages = 10.0;
        int max_clusters[9] = {0}, stages_of[9] = {0};
        for (int s = 1; s <= 8; ++s) {
            if (h->force_splits == 0 && s > 1 && (np < 2 * s)) continue;       // at least two pages per block
            DecodePlan plan;
            if (decode_plan(c, n + kPageTokens, h->max_smem, s, &plan) != 0) continue;   // room for the page count to grow by one
            int clusters = 0;
            e = decode_max_clusters(plan, &clusters);
            if (e != cudaSuccess) {
                cudaGetLastError();
                continue;
            }
            max_clusters[s] = clusters;
            stages_of[s] = plan.stages;
        }
        auto round_time = [&](int s, int m) {
            const double own = (double)((np + s - 1) / s) + kFixedPages;
            const double hbm = kHbmPageTime * (double)m * np / h->num_sms;
            return (own > hbm ? own : hbm) / kRingWeight[stages_of[s]];
        };
        double best_time = -1.0;
        for (int s = 1; s <= 8; ++s) {
            if (max_clusters[s] < 1 || (h->force_splits > 0 && s != h->force_splits)) continue;
            const int used = max_clusters[s] < h->units ? max_clusters[s] : h->units;
            const int full = h->units / used, rem = h->units % used;
            double time = full * round_time(s, used);
            int ts = 0;
            if (rem > 0) {
                // the partly filled last round: as it is, or in a second launch with larger clusters
                double tail = round_time(s, rem);
                if (full > 0 && h->force_splits == 0)
                    for (int k = s + 1; k <= 8; ++k)
                        if (max_clusters[k] >= rem && rem * k <= h->num_sms &&
                            round_time(k, rem) + kSecondLaunchPages < tail) {
                            tail = round_time(k, rem) + kSecondLaunchPages;
                            ts = k;
                        }
                time += tail;
            }
            if (best_time < 0 || time < 0.98 * best_time) {      // larger clusters only for a clear gain
                best_time = time;
                best.splits = s;
                best.clusters = used;
                best.tail_splits = ts;
                best.tail_units = ts > 0 ? rem : 0;
            }
        }
        if (best_time < 0) return fail(h, LAZYEV_EINVAL, "no decode launch shape fits %d tokens per unit in shared memory", n);
        cached = h->plan_cache.insert_or_assign(np, best).first;
    }
    launch->config = c;
    launch->brief = brief;
    launch->shape = lazyev::Shape();
    launch->shape.clusters = h->units;      // (brief: one walk over all units)
    if (!brief) launch->shape = cached->second;
    launch->plan = {};
    if (brief)
        launch->plan = decode_short_plan();
    else if (decode_plan(c, n, h->max_smem, launch->shape.splits, &launch->plan) != 0)
        return fail(h, LAZYEV_EINVAL, "no decode launch shape fits %d tokens per unit in shared memory", n);
    launch->tail_plan = {};
    if (launch->shape.tail_units > 0 && decode_plan(c, n, h->max_smem, launch->shape.tail_splits, &launch->tail_plan) != 0)
        return fail(h, LAZYEV_EINVAL, "no decode launch shape fits %d tokens per unit in shared memory", n);
    return LAZYEV_OK;
}

// The decode launches of one step: attention of q over the shared prefix, if there is one, and the first n cached tokens of
// every unit with tracking (unless `track` is false) at time t.  `tok` (may be null) is the token to append at slot n - 1 first: as
// a launch of its own, or -- when every block of the decode launch takes exactly one unit, the launch-latency-sized
// problems -- inside the decode launch.
// `view` (may be null) stands for the handle's own state: other pages, another place for the probabilities.
int run_decode(lazyev_t* h, const void* q, void* out, int n, int t, const HostPipe* pipe, const NewToken* tok = nullptr,
               bool track = true, const StateView* view = nullptr) {
    DecodeLaunch launch;
    const int rc = choose_decode(h, q, out, n, track, &launch);
    if (rc != LAZYEV_OK) return rc;
    const DecodeConfig& c = launch.config;
    const lazyev::Shape& shape = launch.shape;
    const DecodePlan &plan = launch.plan, &tail_plan = launch.tail_plan;
    const bool brief = launch.brief;
    cudaError_t e = cudaSuccess;
    const int main_units = h->units - shape.tail_units;
    const int clusters = shape.clusters < main_units ? shape.clusters : main_units;
    const bool fuse_append = tok && h->fuse_append && !brief && shape.tail_units == 0 && main_units <= clusters;
    PrefixView prefix = {};
    if (h->shared) {
        prefix.plan = h->prefix_plan;
        prefix.o = h->prefix_o;
        prefix.ml = h->prefix_ml;
    }
    if (tok && !fuse_append) {
        SpanGuard g(h, kSpanAppend, 0.0);
        e = append_launch(geometry(h), h->pool, h->st, tok->k, tok->v, n - 1, t, tok->position, h->stream);
        if (e != cudaSuccess) return cuda_fail(h, e, "append kernel launch");
        h->launches += 1;
    }
    if (h->shared && !pipe && (e = run_prefix(h, q)) != cudaSuccess) return cuda_fail(h, e, "prefix kernel launch");
    {
        // algorithmic bytes: every cached K and V row read once, one probability written per token,
        // the queries read and the outputs written
        SpanGuard g(h, kSpanDecode, (double)h->units * ((double)n * (2 * kRowBytes + 4) + 2.0 * h->group * kRowBytes));
        // Unit ranges: the main launch as one range, or (host buffers) as up to kHostChunks ranges of whole
        // rounds so that copies of one range overlap the kernel of another; then the last round's units.
        int begin[kHostChunks + 1], count[kHostChunks + 1], ranges = 0;
        const int rounds = (main_units + clusters - 1) / clusters;
        // (short first and last ranges: the first query copy and the last output copy are not overlapped)
        static const int kShare[kHostChunks + 1] = {0, 1, 11, 12};       // cumulative twelfths of the rounds
        const bool split = pipe && rounds >= 12;
        const int parts = split ? kHostChunks : 1;
        for (int r = 0; r < parts; ++r) {
            const int b = split ? rounds * kShare[r] / 12 * clusters : 0;
            int e2 = split ? rounds * kShare[r + 1] / 12 * clusters : main_units;
            if (e2 > main_units) e2 = main_units;
            if (e2 <= b) continue;
            begin[ranges] = b;
            count[ranges++] = e2 - b;
        }
        if (shape.tail_units > 0) {
            begin[ranges] = main_units;
            count[ranges++] = shape.tail_units;
        }
        const size_t unit_bytes = (size_t)h->group * kRowBytes;
        if (pipe) h->last_host_ranges = ranges;
        if (pipe) {
            for (int r = 0; r < ranges && e == cudaSuccess; ++r) {
                e = cudaMemcpyAsync((uint8_t*)const_cast<void*>(q) + begin[r] * unit_bytes, pipe->q_host + begin[r] * unit_bytes,
                                    count[r] * unit_bytes, cudaMemcpyHostToDevice, h->copy_in);
                if (e == cudaSuccess) e = cudaEventRecord(h->ev_in[r], h->copy_in);
            }
            if (h->shared) {       // the prefix launch takes all queries at once
                if (e == cudaSuccess) e = cudaStreamWaitEvent(h->stream, h->ev_in[ranges - 1], 0);
                if (e == cudaSuccess) e = run_prefix(h, q);
            }
        }
        // The last round's units do not depend on the main launch: on a lower-priority stream of their own,
        // forked here (after the append), their blocks take the SMs that the main launch's blocks leave as
        // they finish; the bound stream joins afterwards.
        const bool fork = shape.tail_units > 0 && !pipe && ranges > 1;
        if (fork) {
            if (!h->tail_stream) {
                int lo = 0, hi = 0;
                e = cudaDeviceGetStreamPriorityRange(&lo, &hi);
                if (e == cudaSuccess) e = cudaStreamCreateWithPriority(&h->tail_stream, cudaStreamNonBlocking, lo);
                if (e == cudaSuccess) e = cudaEventCreateWithFlags(&h->ev_fork, cudaEventDisableTiming);
                if (e == cudaSuccess) e = cudaEventCreateWithFlags(&h->ev_join, cudaEventDisableTiming);
            }
            if (e == cudaSuccess) e = cudaEventRecord(h->ev_fork, h->stream);
            if (e == cudaSuccess) e = cudaStreamWaitEvent(h->tail_stream, h->ev_fork, 0);
        }
        for (int r = 0; r < ranges && e == cudaSuccess; ++r) {
            const bool is_tail = shape.tail_units > 0 && r == ranges - 1;
            if (pipe) e = cudaStreamWaitEvent(h->stream, h->ev_in[r], 0);
            if (e != cudaSuccess) break;
            // a range of the main walk continues it; the last round's units are a walk of their own
            DecodeArgs a{h->pool, view ? *view : h->st, q, out, n, t, begin[r], count[r], is_tail ? 0 : begin[r] / clusters,
                         fuse_append ? tok->k : nullptr, fuse_append ? tok->v : nullptr, fuse_append ? tok->position : 0, prefix,
                         h->shared && !pipe && !fork && r == 0 && !h->profiling};
            const bool beside = is_tail && fork;
            if (e != cudaSuccess) break;
            if (brief)
                e = decode_short_launch(c, a, h->num_sms, h->stream);
            else
                e = decode_launch(c, is_tail ? tail_plan : plan, is_tail ? count[r] : (clusters < count[r] ? clusters : count[r]), a,
                              beside ? h->tail_stream : h->stream);
            h->launches += 1;
            if (beside && e == cudaSuccess) {
                e = cudaEventRecord(h->ev_join, h->tail_stream);
                if (e == cudaSuccess) e = cudaStreamWaitEvent(h->stream, h->ev_join, 0);
            }
            if (pipe && e == cudaSuccess) {
                e = cudaEventRecord(h->ev_done[r], h->stream);
                if (e == cudaSuccess) e = cudaStreamWaitEvent(h->copy_out, h->ev_done[r], 0);
                if (e == cudaSuccess)
                    e = cudaMemcpyAsync(pipe->out_host + begin[r] * unit_bytes, (uint8_t*)out + begin[r] * unit_bytes,
                                        count[r] * unit_bytes, cudaMemcpyDeviceToHost, h->copy_out);
            }
        }
    }
    if (e != cudaSuccess) return cuda_fail(h, e, "decode kernel launch");
    h->last_plan = plan;
    h->last_tail_units = shape.tail_units;
    h->last_tail_splits = shape.tail_splits;
    h->last_grid = brief ? decode_short_blocks(h->units, h->num_sms) : clusters * plan.splits;
    return LAZYEV_OK;
}

// Refuses a decode step before anything is queued.
int check_step(lazyev_t* h) {
    if (!h->prefilled && !h->shared) return fail(h, LAZYEV_ESTATE, "decode_step before prefill");
    if (h->users > 0) return fail(h, LAZYEV_ESTATE, "decode_step on a handle that others share as their prefix");
    if (h->n + 1 > h->capacity) return fail(h, LAZYEV_ECAPACITY, "cache full (%d slots per unit)", h->capacity);
    const int t = h->t + 1, n = h->n + 1;
    // A step whose automatic eviction could not run is refused before anything is queued.
    if (h->auto_evict && evict_due_at(h, t, n) && candidates_of(h, n) < 0)
        return fail(h, LAZYEV_EINVAL,
                    "step %d would evict over %d candidates, more than the selection supports; nothing was done", t,
                    n - h->n_recent - h->n_initial);
    return LAZYEV_OK;
}

// The step after its token is in the cache.
int finish_step(lazyev_t* h) {
    h->t += 1;
    h->n += 1;
    h->prefilled = true;                    // (a handle with a prefix may start with no own token)
    if (h->weights) {
        const cudaError_t e = step_weights_launch(geometry(h), h->weights, h->st.pbar, h->n, h->stream);
        if (e != cudaSuccess) return cuda_fail(h, e, "weight kernel launch");
        h->launches += 1;
    }
    if (h->auto_evict) return run_evict(h, nullptr, h->src, h->first_moved, h->radix_list);
    return LAZYEV_OK;
}

int run_step(lazyev_t* h, const void* q, const void* k_new, const void* v_new, void* out, const HostPipe* pipe = nullptr) {
    int rc = check_step(h);
    if (rc != LAZYEV_OK) return rc;
    if (((uintptr_t)k_new | (uintptr_t)v_new) & 15) return fail(h, LAZYEV_EINVAL, "k_new and v_new must be 16-byte aligned");
    const NewToken tok{k_new, v_new, h->pos_base + h->prefill + h->t};
    rc = run_decode(h, q, out, h->n + 1, h->t + 1, pipe, &tok);
    return rc != LAZYEV_OK ? rc : finish_step(h);
}

// ---- projected rows ------------------------------------------------------------------------------------
// The handle is bound and its device is the current one.
int check_device(lazyev_t* h, const char* call) {
    if (!h->bound) return fail(h, LAZYEV_ESTATE, "%s before bind", call);
    int dev = -1;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_fail(h, e, "cudaGetDevice");
    if (dev != h->device) return fail(h, LAZYEV_ESTATE, "%s needs device %d (the one bound to this handle) to be current, not %d", call, h->device, dev);
    return LAZYEV_OK;
}

// Do two different rows of an output view share elements?  Rows overlap when their distance, a sum of (difference of indices) x
// stride over the dimensions, is below a row's length.  Dimensions come by falling stride, and of each only the differences
// are looked at that the later ones can still bring near zero: one, in a view whose dimensions nest.
bool rows_meet(const long long* stride, const long long* extent, int dims, long long at, bool apart) {
    if (dims == 0) return apart && at < kHeadDim && at > -kHeadDim;
    long long reach = kHeadDim - 1;
    for (int i = 1; i < dims; ++i) reach += (extent[i] - 1) * stride[i];
    // d with |at + d * stride| <= reach
    if (stride[0] == 0) return true;
    long long first = (-reach - at) / stride[0] - 1, last = (reach - at) / stride[0] + 1;
    if (first < 1 - extent[0]) first = 1 - extent[0];
    if (last > extent[0] - 1) last = extent[0] - 1;
    for (long long d = first; d <= last; ++d) {
        const long long to = at + d * stride[0];
        if (to <= reach && to >= -reach && rows_meet(stride + 1, extent + 1, dims - 1, to, apart || d != 0)) return true;
    }
    return false;
}

bool output_overlaps(const long long* stride, const int* extent) {
    long long by[4], n[4];
    int dims = 0;
    for (int i = 0; i < 4; ++i) {
        if (extent[i] <= 1) continue;
        const long long s = stride[i] < 0 ? -stride[i] : stride[i];     // (differences have both signs)
        int at = dims++;
        for (; at > 0 && by[at - 1] < s; --at) {
            by[at] = by[at - 1];
            n[at] = n[at - 1];
        }
        by[at] = s;
        n[at] = extent[i];
    }
    return dims > 0 && rows_meet(by, n, dims, 0, false);
}

// The kernels' view of a caller's rows, or EINVAL.
int rows_view(lazyev_t* h, const char* name, const lazyev_rows_t* r, int heads, int n_tokens, bool output, RowView* out) {
    if (!r || !r->data) return fail(h, LAZYEV_EINVAL, "%s: null pointer", name);
    if (r->dtype != LAZYEV_BF16 && r->dtype != LAZYEV_FP16 && r->dtype != LAZYEV_FP32)
        return fail(h, LAZYEV_EINVAL, "%s: unknown type %d", name, r->dtype);
    if ((uintptr_t)r->data & 15) return fail(h, LAZYEV_EINVAL, "%s must be 16-byte aligned", name);
    const long long given[4] = {r->stride_layer, r->stride_batch, r->stride_token, r->stride_head};
    const int extent[4] = {h->layers, h->batch, n_tokens, heads};
    const int elems = r->dtype == LAZYEV_FP32 ? 4 : 8;             // of 16 bytes
    long long stride[4];
    for (int i = 0; i < 4; ++i) {
        stride[i] = extent[i] > 1 ? given[i] : 0;
        if (stride[i] % elems != 0) return fail(h, LAZYEV_EINVAL, "%s: strides must be multiples of 16 bytes", name);
    }
    if (output && output_overlaps(stride, extent)) return fail(h, LAZYEV_EINVAL, "%s: output rows overlap", name);
    *out = RowView{r->data, stride[0], stride[1], stride[2], stride[3], r->dtype};
    return LAZYEV_OK;
}

// One launch reads one type and writes one.
int same_type(lazyev_t* h, const RowView& x, const RowView& y) {
    if (x.data && y.data && x.dtype != y.dtype) return fail(h, LAZYEV_EINVAL, "the rows of a call must be of one type (outputs too)");
    return LAZYEV_OK;
}

RowsArgs rows_args(const lazyev_t* h, int n_tokens, const int32_t* positions, int first_position) {
    RowsArgs a = {};
    a.layers = h->layers;
    a.batch = h->batch;
    a.q_heads = h->q_heads;
    a.kv_heads = h->kv_heads;
    a.n_tokens = n_tokens;
    a.pairs = h->pairs;
    a.interleaved = h->interleaved;
    a.amplitude = h->amplitude;
    a.eps = h->norm_eps;
    a.q_weight = h->q_weight;
    a.k_weight = h->k_weight;
    a.positions = positions;
    a.first_position = first_position;
    a.status = h->st.status;
    return a;
}

// Keys and values go into the pages of the next n_tokens slots, as tokens of time ts.
void rows_to_pages(const lazyev_t* h, int ts, RowsArgs* a) {
    a->pool = h->pool;
    a->page_table = h->st.page_table;
    a->tsm = h->st.tsm;
    a->pos = h->st.pos;
    a->pbar = h->st.pbar;
    a->pages_per_unit = h->pages_per_unit;
    a->capacity = h->capacity;
    a->total_pages = h->units * h->pages_per_unit;
    a->slot = h->n;
    a->ts = ts;
    a->pos_first = h->pos_base + h->prefill + h->t;
}

}  // namespace

extern "C" {

const char* lazyev_strerror(int code) {
    switch (code) {
        case LAZYEV_OK: return "ok";
        case LAZYEV_EINVAL: return "invalid argument";
        case LAZYEV_ESTATE: return "call made in the wrong state";
        case LAZYEV_ECAPACITY: return "cache capacity exceeded";
        case LAZYEV_EDEVICE: return "device-side failure flagged";
        case LAZYEV_ECUDA: return "CUDA runtime error";
        default: return "unknown error code";
    }
}

const char* lazyev_last_error(const lazyev_t* h) { return h ? h->err : "null handle"; }

int lazyev_build_flags(void) { return kBuildFlags; }

int lazyev_create(lazyev_t** handle, int layers, int q_heads, int kv_heads, int head_dim, int budget, int window,
                  float threshold) {
    if (!handle) return LAZYEV_EINVAL;
    *handle = nullptr;
    if (layers <= 0 || q_heads <= 0 || kv_heads <= 0 || budget <= 0 || window <= 0) return LAZYEV_EINVAL;
    if (head_dim != kHeadDim) return LAZYEV_EINVAL;
    if (q_heads % kv_heads != 0 || q_heads / kv_heads > kMaxGroup) return LAZYEV_EINVAL;
    if (budget <= window) return LAZYEV_EINVAL;
    if (!(threshold >= 0.f)) return LAZYEV_EINVAL;
    lazyev_t* h = new (std::nothrow) lazyev();
    if (!h) return LAZYEV_EINVAL;
    h->layers = layers;
    h->q_heads = q_heads;
    h->kv_heads = kv_heads;
    h->head_dim = head_dim;
    h->budget = h->budget_now = h->max_prefill = budget;
    h->window = window;
    h->n_recent = window;
    h->alpha = threshold;
    derive(h);
    *handle = h;
    return LAZYEV_OK;
}

int lazyev_set_batch(lazyev_t* h, int batch) {
    if (!h) return LAZYEV_EINVAL;
    if (h->bound) return fail(h, LAZYEV_ESTATE, "set_batch after bind");
    if (batch <= 0) return fail(h, LAZYEV_EINVAL, "batch must be positive");
    h->batch = batch;
    derive(h);
    return LAZYEV_OK;
}

int lazyev_set_protect(lazyev_t* h, int n_recent, int n_initial) {
    if (!h) return LAZYEV_EINVAL;
    if (h->bound) return fail(h, LAZYEV_ESTATE, "set_protect after bind");
    if (n_recent < 1 || n_initial < 0 || h->budget <= n_recent + n_initial)
        return fail(h, LAZYEV_EINVAL, "need n_recent >= 1, n_initial >= 0 and budget > n_recent + n_initial");
    h->n_recent = n_recent;
    h->n_initial = n_initial;
    return LAZYEV_OK;
}

int lazyev_set_max_prefill(lazyev_t* h, int n_tokens) {
    if (!h) return LAZYEV_EINVAL;
    if (h->bound) return fail(h, LAZYEV_ESTATE, "set_max_prefill after bind");
    if (n_tokens <= 0) return fail(h, LAZYEV_EINVAL, "max_prefill must be positive");
    h->max_prefill = n_tokens;
    derive(h);
    return LAZYEV_OK;
}

int lazyev_set_budget(lazyev_t* h, int budget_now) {
    if (!h) return LAZYEV_EINVAL;
    if (budget_now <= h->n_recent + h->n_initial || budget_now > h->budget)
        return fail(h, LAZYEV_EINVAL, "budget_now must be in (n_recent + n_initial, budget]");
    h->budget_now = budget_now;
    return LAZYEV_OK;
}

int lazyev_set_auto_evict(lazyev_t* h, int on) {
    if (!h) return LAZYEV_EINVAL;
    h->auto_evict = on != 0;
    return LAZYEV_OK;
}

int lazyev_set_score_mode(lazyev_t* h, int mode) {
    if (!h) return LAZYEV_EINVAL;
    if (mode < 0 || mode > LAZYEV_SCORE_WEIGHT) return fail(h, LAZYEV_EINVAL, "unknown score mode %d", mode);
    if (mode == LAZYEV_SCORE_WEIGHT && !h->weights_on) return fail(h, LAZYEV_EINVAL, "selection by weight needs lazyev_set_weights()");
    h->score_mode = mode;
    return LAZYEV_OK;
}

int lazyev_set_weights(lazyev_t* h, int on) {
    if (!h) return LAZYEV_EINVAL;
    if (h->bound) return fail(h, LAZYEV_ESTATE, "set_weights after bind");
    if (!on && h->score_mode == LAZYEV_SCORE_WEIGHT) return fail(h, LAZYEV_EINVAL, "selection by weight needs the weights");
    h->weights_on = on != 0;
    return LAZYEV_OK;
}

int lazyev_set_splits(lazyev_t* h, int splits) {
    if (!h) return LAZYEV_EINVAL;
    if (splits < 0 || splits > 8) return fail(h, LAZYEV_EINVAL, "splits must be 0 (automatic) or 1..8");
    h->force_splits = splits;
    return LAZYEV_OK;
}

int lazyev_set_stages(lazyev_t* h, int stages) {
    if (!h) return LAZYEV_EINVAL;
    if (stages != 0 && (stages < 2 || stages > 6)) return fail(h, LAZYEV_EINVAL, "stages must be 0 or 2..6");
    h->force_stages = stages;
    return LAZYEV_OK;
}

int lazyev_set_groups(lazyev_t* h, int groups) {
    if (!h) return LAZYEV_EINVAL;
    if (groups < 0 || groups > 2) return fail(h, LAZYEV_EINVAL, "groups must be 0 (automatic), 1 or 2");
    h->force_groups = groups;
    return LAZYEV_OK;
}

int lazyev_query_sizes(const lazyev_t* h, size_t* kv_bytes, size_t* state_bytes, size_t* scratch_bytes) {
    if (!h) return LAZYEV_EINVAL;
    const Sizes s = sizes_of(h);
    if (kv_bytes) *kv_bytes = s.kv;
    if (state_bytes) *state_bytes = s.state;
    if (scratch_bytes) *scratch_bytes = s.scratch;
    return LAZYEV_OK;
}

int lazyev_bind(lazyev_t* h, void* kv_pool, void* state, void* scratch, void* cuda_stream) {
    if (!h) return LAZYEV_EINVAL;
    if (h->bound) return fail(h, LAZYEV_ESTATE, "already bound");
    if (!kv_pool || !state || !scratch) return fail(h, LAZYEV_EINVAL, "null device pointer");
    if (((uintptr_t)kv_pool | (uintptr_t)state | (uintptr_t)scratch) & 255)
        return fail(h, LAZYEV_EINVAL, "device regions must be 256-byte aligned");
    cudaError_t e = cudaGetDevice(&h->device);
    if (e != cudaSuccess) return cuda_fail(h, e, "cudaGetDevice");
    int major = 0, minor = 0;              // (single attributes: the whole property record takes milliseconds to fill)
    e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, h->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, h->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&h->num_sms, cudaDevAttrMultiProcessorCount, h->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&h->max_smem, cudaDevAttrMaxSharedMemoryPerBlockOptin, h->device);
    if (e != cudaSuccess) return cuda_fail(h, e, "cudaDeviceGetAttribute");
    if (major != 10) return fail(h, LAZYEV_ECUDA, "this library is built for sm_100a only (device is sm_%d%d)", major, minor);
    if ((e = decode_prepare()) != cudaSuccess) return cuda_fail(h, e, "decode kernel set-up");
    if ((e = decode_short_prepare()) != cudaSuccess) return cuda_fail(h, e, "decode kernel set-up");
    if ((e = select_prepare()) != cudaSuccess) return cuda_fail(h, e, "select kernel set-up");
    if ((e = chunk_prepare()) != cudaSuccess) return cuda_fail(h, e, "chunk kernel set-up");
    if ((e = weigh_prepare()) != cudaSuccess) return cuda_fail(h, e, "weight kernel set-up");
    if ((e = keep_prepare()) != cudaSuccess) return cuda_fail(h, e, "select kernel set-up");
    if ((e = blocks_prepare()) != cudaSuccess) return cuda_fail(h, e, "block selection set-up");

    const Sizes s = sizes_of(h);
    h->stream = (cudaStream_t)cuda_stream;
    h->pool = (uint8_t*)kv_pool;
    uint8_t* sp = (uint8_t*)state;
    h->st.page_table = (int32_t*)sp;
    h->st.tsm = (int2*)(sp + s.off_tsm);
    h->st.pos = (int32_t*)(sp + s.off_pos);
    h->st.pbar = (float*)(sp + s.off_pbar);
    h->st.status = (int32_t*)(sp + s.off_status);
    uint8_t* cp = (uint8_t*)scratch;
    h->src = (int32_t*)cp;
    h->first_moved = (int32_t*)(cp + s.off_first);
    h->radix_list = (int32_t*)(cp + s.off_rlist);
    {
        const size_t qslot = align_up((size_t)h->layers * h->batch * h->q_heads * kRowBytes, 256);
        const size_t kslot = align_up((size_t)h->layers * h->batch * h->kv_heads * kRowBytes, 256);
        for (int i = 0; i < 2; ++i) {
            h->stage_q[i] = cp + s.off_q + i * qslot;
            h->stage_k[i] = cp + s.off_k + i * kslot;
            h->stage_v[i] = cp + s.off_v + i * kslot;
            h->stage_out[i] = cp + s.off_out + i * qslot;
        }
    }
    h->stage_score = (double*)(cp + s.off_score);
    h->stage_hist = (unsigned long long*)(cp + s.off_hist);
    h->h2_table = (double*)(cp + s.off_h2);
    h->h2_table_mode = -1;
    h->stage_rows = cp + s.off_rows;
    h->counters = (int32_t*)(cp + s.off_counters);
    if (h->weights_on) h->weights = (float*)(sp + s.off_weights);
    if ((e = prefix_prepare(h->pool, h->units * h->pages_per_unit, &h->own_pool)) != cudaSuccess) return cuda_fail(h, e, "tensor map of the pool");

    // Slots past n are read (and masked) by the decode kernel's last page: they must hold finite values.
    e = cudaMemsetAsync(h->pool, 0, s.kv, h->stream);
    if (e == cudaSuccess) e = cudaMemsetAsync(h->counters, 0, 2 * kChunkCounters * sizeof(int32_t), h->stream);
    if (e == cudaSuccess && h->weights) e = cudaMemsetAsync(h->weights, 0, s.state - s.off_weights, h->stream);
    if (e != cudaSuccess) return cuda_fail(h, e, "clearing the KV pool");
    e = init_state_launch(geometry(h), h->st, h->stream);
    if (e != cudaSuccess) return cuda_fail(h, e, "state initialisation launch");
    h->launches += 1;
    h->bound = true;
    return LAZYEV_OK;
}

int lazyev_set_page_table(lazyev_t* h, const int32_t* host_table) {
    if (!h) return LAZYEV_EINVAL;
    if (!h->bound || h->prefilled) return fail(h, LAZYEV_ESTATE, "set_page_table is only valid between bind and prefill");
    if (!host_table) return fail(h, LAZYEV_EINVAL, "null page table");
    const size_t total = (size_t)h->units * h->pages_per_unit;
    std::vector<char> seen(total, 0);
    for (size_t i = 0; i < total; ++i) {
        const int32_t p = host_table[i];
        if (p < 0 || (size_t)p >= total || seen[p]) return fail(h, LAZYEV_EINVAL, "page table is not a permutation");
        seen[p] = 1;
    }
    cudaError_t e = cudaMemcpyAsync(h->st.page_table, host_table, total * sizeof(int32_t), cudaMemcpyHostToDevice, h->stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(h->stream);
    if (e != cudaSuccess) return cuda_fail(h, e, "page table upload");
    return LAZYEV_OK;
}

int lazyev_prefill(lazyev_t* h, const void* k, const void* v, int n_tokens) {
    if (!h) return LAZYEV_EINVAL;
    if (!h->bound) return fail(h, LAZYEV_ESTATE, "prefill before bind");
    if (h->prefilled) return fail(h, LAZYEV_ESTATE, "prefill called twice");
    if (!k || !v || n_tokens <= 0) return fail(h, LAZYEV_EINVAL, "null pointer or non-positive token count");
    if (n_tokens > h->max_prefill) return fail(h, LAZYEV_ECAPACITY, "prompt of %d tokens exceeds max_prefill = %d", n_tokens, h->max_prefill);
    if (((uintptr_t)k | (uintptr_t)v) & 15) return fail(h, LAZYEV_EINVAL, "k and v must be 16-byte aligned");
    cudaError_t e = prefill_launch(geometry(h), h->pool, h->st, k, v, n_tokens, INT_MIN, h->pos_base, h->stream);
    if (e == cudaSuccess) e = clear_weights(h, 0, n_tokens);
    if (e != cudaSuccess) return cuda_fail(h, e, "prefill kernel launch");
    h->launches += 1;
    h->prefilled = true;
    h->prefill = n_tokens;
    h->n = n_tokens;
    h->t = 0;
    return LAZYEV_OK;
}

namespace {
int host_wait(lazyev_t* h, int allowed);
int detach(lazyev_t* h);
}

int lazyev_reset(lazyev_t* h) {
    if (!h) return LAZYEV_EINVAL;
    if (!h->bound) return fail(h, LAZYEV_ESTATE, "reset before bind");
    if (h->users > 0) return fail(h, LAZYEV_ESTATE, "reset of a handle that others share as their prefix");
    if (h->copy_in) {                       // steps queued through the asynchronous host entry point finish first
        const int rc = host_wait(h, 0);
        if (rc != LAZYEV_OK) return rc;
    }
    const int rc = detach(h);
    if (rc != LAZYEV_OK) return rc;
    // Old rows stay in the pool: slots past n are masked, they only have to be finite.  The state arrays
    // are rewritten by the next prompt load and by every append; the device status word is cleared.
    cudaError_t e = cudaMemsetAsync(h->st.status, 0, 64, h->stream);
    // (a launch that gave up may have left counts behind, a replayed one too)
    if (e == cudaSuccess && h->counted) e = cudaMemsetAsync(h->counters, 0, 2 * kChunkCounters * sizeof(int32_t), h->stream);
    if (e != cudaSuccess) return cuda_fail(h, e, "clearing the device status word");
    h->indexed = 0;
    h->prefilled = false;
    h->t = h->n = h->prefill = h->pos_base = 0;
    h->budget_now = h->budget;
    return LAZYEV_OK;
}

int lazyev_prefill_observed(lazyev_t* h, const void* q, const void* k, const void* v, int n_tokens, void* out) {
    if (!h) return LAZYEV_EINVAL;
    if (!h->bound) return fail(h, LAZYEV_ESTATE, "prefill before bind");
    if (h->prefilled) return fail(h, LAZYEV_ESTATE, "prefill called twice");
    if (h->shared) return fail(h, LAZYEV_ESTATE, "prefill_observed does not run over an attached prefix");
    if (!q || !k || !v || !out || n_tokens <= 0) return fail(h, LAZYEV_EINVAL, "null pointer or non-positive token count");
    if (n_tokens > h->max_prefill) return fail(h, LAZYEV_ECAPACITY, "prompt of %d tokens exceeds max_prefill = %d", n_tokens, h->max_prefill);
    if (h->prompt_mode == LAZYEV_PROMPT_TILED && (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)out) & 15))
        return fail(h, LAZYEV_EINVAL, "q, k, v and out must be 16-byte aligned");
    if ((((uintptr_t)k | (uintptr_t)v) & 15) || ((uintptr_t)q & 3) || ((uintptr_t)out & 1))
        return fail(h, LAZYEV_EINVAL, "k and v must be 16-byte aligned, q 4-byte and out 2-byte aligned");
    // rows are loaded with TS = their own time j - (P - 1) <= 0 and MRI = 0
    cudaError_t e = prefill_launch(geometry(h), h->pool, h->st, k, v, n_tokens, 1 - n_tokens, 0, h->stream);
    if (e == cudaSuccess) e = clear_weights(h, 0, n_tokens);
    if (e != cudaSuccess) return cuda_fail(h, e, "prefill kernel launch");
    h->launches += 1;
    if (h->prompt_mode == LAZYEV_PROMPT_TILED) {
        // one launch: tiled causal attention on the tensor cores, K / V read once per query tile
        PromptArgs a;
        a.q = q;
        a.k = k;
        a.v = v;
        a.out = out;
        a.n_tokens = n_tokens;
        a.alpha = h->alpha;
        a.dump = h->prompt_dump;
        a.dump_begin = h->prompt_dump_begin;
        a.dump_count = h->prompt_dump_count;
        a.wait_limit_ns = h->wait_limit_ns;
        a.stop_after_tiles = h->stop_after_pages;
        e = prompt_launch(geometry(h), h->st, a, h->num_sms, h->stream);
        if (e != cudaSuccess) return cuda_fail(h, e, "prompt kernel launch");
        h->launches += 1;
    } else {
        // the prompt replayed through the decode kernel, one row per launch
        const size_t row_bytes = (size_t)h->layers * h->batch * h->q_heads * kRowBytes;
        for (int j = 0; j < n_tokens; ++j) {
            const int rc = run_decode(h, (const uint8_t*)q + j * row_bytes, (uint8_t*)out + j * row_bytes, j + 1,
                                      j - (n_tokens - 1), nullptr);
            if (rc != LAZYEV_OK) return rc;
            if (h->prompt_dump) {    // row j of the per-row probabilities: tokens 0 .. j of the dumped units
                e = cudaMemcpy2DAsync(h->prompt_dump + (size_t)j * n_tokens, (size_t)n_tokens * n_tokens * sizeof(float),
                                      h->st.pbar + (size_t)h->prompt_dump_begin * h->capacity, (size_t)h->capacity * sizeof(float),
                                      (size_t)(j + 1) * sizeof(float), h->prompt_dump_count, cudaMemcpyDeviceToDevice, h->stream);
                if (e != cudaSuccess) return cuda_fail(h, e, "prompt probability dump");
            }
        }
    }
    h->prefilled = true;
    h->prefill = n_tokens;
    h->n = n_tokens;
    h->t = 0;
    return LAZYEV_OK;
}

int lazyev_set_prompt_mode(lazyev_t* h, int mode) {
    if (!h) return LAZYEV_EINVAL;
    if (mode != LAZYEV_PROMPT_TILED && mode != LAZYEV_PROMPT_REPLAY) return fail(h, LAZYEV_EINVAL, "unknown prompt mode %d", mode);
    h->prompt_mode = mode;
    return LAZYEV_OK;
}

int lazyev_set_prompt_dump(lazyev_t* h, float* device_rows, int unit_begin, int unit_count) {
    if (!h) return LAZYEV_EINVAL;
    if (device_rows && (unit_begin < 0 || unit_count <= 0 || unit_begin + unit_count > h->units))
        return fail(h, LAZYEV_EINVAL, "unit range out of bounds");
    h->prompt_dump = device_rows;
    h->prompt_dump_begin = device_rows ? unit_begin : 0;
    h->prompt_dump_count = device_rows ? unit_count : 0;
    return LAZYEV_OK;
}

int lazyev_set_fused_append(lazyev_t* h, int on) {
    if (!h) return LAZYEV_EINVAL;
    h->fuse_append = on != 0;
    return LAZYEV_OK;
}

int lazyev_debug_starve_page_ring(lazyev_t* h, int pages) {
    if (!h) return LAZYEV_EINVAL;
    if (pages < -1) return fail(h, LAZYEV_EINVAL, "pages must be -1 (off) or >= 0");
    h->stop_after_pages = pages;
    return LAZYEV_OK;
}

int lazyev_set_wait_limit(lazyev_t* h, double seconds) {
    if (!h) return LAZYEV_EINVAL;
    if (!(seconds >= 1e-4 && seconds <= 60.0)) return fail(h, LAZYEV_EINVAL, "wait limit must be between 0.1 ms and 60 s");
    h->wait_limit_ns = (unsigned long long)(seconds * 1e9);
    return LAZYEV_OK;
}

int lazyev_decode_step(lazyev_t* h, const void* q, const void* k_new, const void* v_new, void* out) {
    if (!h) return LAZYEV_EINVAL;
    if (!q || !k_new || !v_new || !out) return fail(h, LAZYEV_EINVAL, "null pointer");
    return run_step(h, q, k_new, v_new, out);
}

namespace {

int host_streams(lazyev_t* h) {      // first host-buffer call: the two copy streams and their events
    if (h->copy_in) return LAZYEV_OK;
    cudaError_t e = cudaStreamCreateWithFlags(&h->copy_in, cudaStreamNonBlocking);
    if (e == cudaSuccess) e = cudaStreamCreateWithFlags(&h->copy_out, cudaStreamNonBlocking);
    for (int i = 0; i <= kHostChunks && e == cudaSuccess; ++i) {
        e = cudaEventCreateWithFlags(&h->ev_in[i], cudaEventDisableTiming);
        if (e == cudaSuccess) e = cudaEventCreateWithFlags(&h->ev_done[i], cudaEventDisableTiming);
    }
    if (e == cudaSuccess) e = cudaEventCreateWithFlags(&h->ev_ready, cudaEventDisableTiming);
    for (int i = 0; i < 2 && e == cudaSuccess; ++i)
        e = cudaEventCreateWithFlags(&h->ev_step_done[i], cudaEventDisableTiming | cudaEventBlockingSync);
    if (e != cudaSuccess) return cuda_fail(h, e, "creating the copy streams");
    return LAZYEV_OK;
}

// Blocks until at most `allowed` (0 or 1) asynchronous host-buffer steps are still in flight.
int host_wait(lazyev_t* h, int allowed) {
    cudaError_t e = cudaSuccess;
    const int newest = (int)((h->host_seq + 1) & 1);       // slot of the step queued last
    for (int k = 0; k < 2; ++k) {
        const int slot = k == 0 ? newest ^ 1 : newest;      // older step first
        if (!h->slot_busy[slot] || (allowed >= 1 && slot == newest)) continue;
        const cudaError_t e1 = cudaEventSynchronize(h->ev_step_done[slot]);
        if (e == cudaSuccess) e = e1;
        h->slot_busy[slot] = false;
    }
    if (e != cudaSuccess) return cuda_fail(h, e, "waiting for a host-buffer step");
    return LAZYEV_OK;
}

}  // namespace

int lazyev_decode_step_host(lazyev_t* h, const void* q, const void* k_new, const void* v_new, void* out) {
    if (!h) return LAZYEV_EINVAL;
    if (!q || !k_new || !v_new || !out) return fail(h, LAZYEV_EINVAL, "null pointer");
    int rc = check_step(h);                 // (before any copy is queued)
    if (rc == LAZYEV_OK) rc = host_streams(h);
    if (rc == LAZYEV_OK) rc = host_wait(h, 0);
    if (rc != LAZYEV_OK) return rc;
    // The copy streams start after everything queued on the bound stream so far (an earlier step's
    // kernels may still read the staging buffers).
    cudaError_t e = cudaEventRecord(h->ev_ready, h->stream);
    if (e == cudaSuccess) e = cudaStreamWaitEvent(h->copy_in, h->ev_ready, 0);
    if (e == cudaSuccess) e = cudaStreamWaitEvent(h->copy_out, h->ev_ready, 0);
    const size_t kbytes = (size_t)h->layers * h->batch * h->kv_heads * kRowBytes;
    if (e == cudaSuccess) e = cudaMemcpyAsync(h->stage_k[0], k_new, kbytes, cudaMemcpyHostToDevice, h->stream);
    if (e == cudaSuccess) e = cudaMemcpyAsync(h->stage_v[0], v_new, kbytes, cudaMemcpyHostToDevice, h->stream);
    if (e != cudaSuccess) return cuda_fail(h, e, "host-to-device copy");
    const HostPipe pipe{(const uint8_t*)q, (uint8_t*)out};
    rc = run_step(h, h->stage_q[0], h->stage_k[0], h->stage_v[0], h->stage_out[0], &pipe);
    // both streams are drained even after an error, so that no copy is left in flight on the caller's buffers
    cudaError_t e1 = cudaStreamSynchronize(h->copy_in), e2 = cudaStreamSynchronize(h->copy_out);
    e = cudaStreamSynchronize(h->stream);
    if (rc != LAZYEV_OK) return rc;
    if (e1 != cudaSuccess || e2 != cudaSuccess || e != cudaSuccess)
        return cuda_fail(h, e1 != cudaSuccess ? e1 : (e2 != cudaSuccess ? e2 : e), "copies of the host-buffer step");
    return LAZYEV_OK;
}

int lazyev_decode_step_host_async(lazyev_t* h, const void* q, const void* k_new, const void* v_new, void* out) {
    if (!h) return LAZYEV_EINVAL;
    if (!q || !k_new || !v_new || !out) return fail(h, LAZYEV_EINVAL, "null pointer");
    int rc = check_step(h);                 // (before any copy is queued)
    if (rc == LAZYEV_OK) rc = host_streams(h);
    if (rc != LAZYEV_OK) return rc;
    const int slot = (int)(h->host_seq & 1);
    // The slot's previous step (two steps back) must be complete before its staging buffers are
    // reused; the step before this one may still be running, and this step's uploads run beside it.
    if (h->slot_busy[slot]) {
        const cudaError_t e0 = cudaEventSynchronize(h->ev_step_done[slot]);
        h->slot_busy[slot] = false;
        if (e0 != cudaSuccess) return cuda_fail(h, e0, "waiting for a host-buffer step");
    }
    const size_t qbytes = (size_t)h->layers * h->batch * h->q_heads * kRowBytes;
    const size_t kbytes = (size_t)h->layers * h->batch * h->kv_heads * kRowBytes;
    cudaError_t e = cudaSuccess;
    if (h->host_seq == 0 || !h->slot_busy[slot ^ 1]) {
        // nothing of ours in flight: order the copy streams after whatever else the bound stream holds
        e = cudaEventRecord(h->ev_ready, h->stream);
        if (e == cudaSuccess) e = cudaStreamWaitEvent(h->copy_in, h->ev_ready, 0);
    }
    if (e == cudaSuccess) e = cudaMemcpyAsync(h->stage_k[slot], k_new, kbytes, cudaMemcpyHostToDevice, h->copy_in);
    if (e == cudaSuccess) e = cudaMemcpyAsync(h->stage_v[slot], v_new, kbytes, cudaMemcpyHostToDevice, h->copy_in);
    if (e == cudaSuccess) e = cudaMemcpyAsync(h->stage_q[slot], q, qbytes, cudaMemcpyHostToDevice, h->copy_in);
    if (e == cudaSuccess) e = cudaEventRecord(h->ev_in[0], h->copy_in);
    if (e == cudaSuccess) e = cudaStreamWaitEvent(h->stream, h->ev_in[0], 0);
    if (e != cudaSuccess) return cuda_fail(h, e, "host-to-device copy");
    rc = run_step(h, h->stage_q[slot], h->stage_k[slot], h->stage_v[slot], h->stage_out[slot]);
    if (rc != LAZYEV_OK) {                  // (no copy is left in flight on the caller's buffers)
        cudaStreamSynchronize(h->copy_in);
        return rc;
    }
    e = cudaEventRecord(h->ev_done[0], h->stream);
    if (e == cudaSuccess) e = cudaStreamWaitEvent(h->copy_out, h->ev_done[0], 0);
    if (e == cudaSuccess) e = cudaMemcpyAsync(out, h->stage_out[slot], qbytes, cudaMemcpyDeviceToHost, h->copy_out);
    if (e == cudaSuccess) e = cudaEventRecord(h->ev_step_done[slot], h->copy_out);
    if (e != cudaSuccess) return cuda_fail(h, e, "device-to-host copy");
    h->slot_busy[slot] = true;
    h->host_seq += 1;
    return LAZYEV_OK;
}

int lazyev_host_wait(lazyev_t* h, int in_flight_allowed) {
    if (!h) return LAZYEV_EINVAL;
    if (in_flight_allowed < 0 || in_flight_allowed > 1) return fail(h, LAZYEV_EINVAL, "in_flight_allowed must be 0 or 1");
    if (!h->copy_in) return LAZYEV_OK;
    return host_wait(h, in_flight_allowed);
}

int lazyev_copy_state(lazyev_t* dst, lazyev_t* src) {
    if (!dst || !src || dst == src) return LAZYEV_EINVAL;
    if (!dst->bound || !src->bound) return fail(dst, LAZYEV_ESTATE, "copy_state needs two bound handles");
    if (!src->prefilled) return fail(dst, LAZYEV_ESTATE, "copy_state from a handle that holds no cache");
    if (dst->prefilled) return fail(dst, LAZYEV_ESTATE, "copy_state into a handle that already holds a cache (reset it first)");
    if (dst->shared != src->shared) return fail(dst, LAZYEV_ESTATE, "copy_state needs the same prefix attached to both handles, or to neither");
    if (dst->device != src->device || dst->layers != src->layers || dst->batch != src->batch || dst->q_heads != src->q_heads ||
        dst->kv_heads != src->kv_heads || dst->capacity != src->capacity || dst->budget != src->budget ||
        dst->window != src->window || dst->n_recent != src->n_recent || dst->n_initial != src->n_initial || dst->weights_on != src->weights_on)
        return fail(dst, LAZYEV_EINVAL, "copy_state needs two handles of the same configuration on the same device");
    const Sizes sz = sizes_of(src);
    cudaEvent_t ready = nullptr;
    cudaError_t e = cudaEventCreateWithFlags(&ready, cudaEventDisableTiming);
    if (e == cudaSuccess) e = cudaEventRecord(ready, src->stream);
    if (e == cudaSuccess) e = cudaStreamWaitEvent(dst->stream, ready, 0);
    // the state region starts with the page table, so the physical pages line up with the copied pool
    if (e == cudaSuccess) e = cudaMemcpyAsync(dst->pool, src->pool, sz.kv, cudaMemcpyDeviceToDevice, dst->stream);
    if (e == cudaSuccess) e = cudaMemcpyAsync(dst->st.page_table, src->st.page_table, sz.state, cudaMemcpyDeviceToDevice, dst->stream);
    // and src's later steps must not overwrite what is still being read
    if (e == cudaSuccess) e = cudaEventRecord(ready, dst->stream);
    if (e == cudaSuccess) e = cudaStreamWaitEvent(src->stream, ready, 0);
    if (ready) cudaEventDestroy(ready);
    if (e != cudaSuccess) return cuda_fail(dst, e, "copy_state");
    dst->prefilled = true;
    dst->t = src->t;
    dst->n = src->n;
    dst->prefill = src->prefill;
    dst->pos_base = src->pos_base;
    dst->budget_now = src->budget_now;
    dst->indexed = 0;
    return LAZYEV_OK;
}

int lazyev_set_rope(lazyev_t* h, const double* inv_freq, int pairs, int interleaved, float amplitude) {
    if (!h) return LAZYEV_EINVAL;
    if (pairs < 0 || pairs > kMaxPairs || pairs % 8 != 0) return fail(h, LAZYEV_EINVAL, "pairs must be a multiple of 8 up to %d", kMaxPairs);
    if (pairs > 0 && !inv_freq) return fail(h, LAZYEV_EINVAL, "null inv_freq");
    if (!isfinite(amplitude)) return fail(h, LAZYEV_EINVAL, "the amplitude must be finite");
    for (int j = 0; j < pairs; ++j)
        if (!isfinite(inv_freq[j])) return fail(h, LAZYEV_EINVAL, "inv_freq[%d] is not finite", j);
    for (int j = 0; j < kMaxPairs; ++j) h->turns[j] = j < pairs ? inv_freq[j] / 6.283185307179586476925 : 0.0;
    h->pairs = pairs;
    h->interleaved = interleaved != 0;
    h->amplitude = amplitude;
    return LAZYEV_OK;
}

int lazyev_set_head_norm(lazyev_t* h, const float* q_weight, const float* k_weight, float eps) {
    if (!h) return LAZYEV_EINVAL;
    if (((uintptr_t)q_weight | (uintptr_t)k_weight) & 15) return fail(h, LAZYEV_EINVAL, "norm weights must be 16-byte aligned");
    if ((q_weight || k_weight) && !(eps > 0.f && isfinite(eps))) return fail(h, LAZYEV_EINVAL, "eps must be positive and finite");
    h->q_weight = q_weight;
    h->k_weight = k_weight;
    h->norm_eps = eps;
    return LAZYEV_OK;
}

int lazyev_norm_rope(lazyev_t* h, const lazyev_rows_t* q, const lazyev_rows_t* k, int n_tokens, const int32_t* positions,
                     int first_position, const lazyev_rows_t* q_out, const lazyev_rows_t* k_out) {
    if (!h) return LAZYEV_EINVAL;
    int rc = check_device(h, "norm_rope");
    if (rc != LAZYEV_OK) return rc;
    if (n_tokens <= 0 || (!q && !k)) return fail(h, LAZYEV_EINVAL, "no rows");
    RowsArgs a = rows_args(h, n_tokens, positions, first_position);
    if (q && (rc = rows_view(h, "q", q, h->q_heads, n_tokens, false, &a.q)) != LAZYEV_OK) return rc;
    if (q && (rc = rows_view(h, "q_out", q_out, h->q_heads, n_tokens, true, &a.q_out)) != LAZYEV_OK) return rc;
    if (k && (rc = rows_view(h, "k", k, h->kv_heads, n_tokens, false, &a.k)) != LAZYEV_OK) return rc;
    if (k && (rc = rows_view(h, "k_out", k_out, h->kv_heads, n_tokens, true, &a.k_out)) != LAZYEV_OK) return rc;
    if ((rc = same_type(h, a.q, a.k)) != LAZYEV_OK || (rc = same_type(h, a.q_out, a.k_out)) != LAZYEV_OK) return rc;
    const cudaError_t e = rows_launch(a, h->turns, h->num_sms, h->stream);
    if (e != cudaSuccess) return cuda_fail(h, e, "norm_rope kernel launch");
    h->launches += 1;
    return LAZYEV_OK;
}

int lazyev_append(lazyev_t* h, const lazyev_rows_t* k, const lazyev_rows_t* v, int n_tokens, const int32_t* positions) {
    if (!h) return LAZYEV_EINVAL;
    int rc = check_device(h, "append");
    if (rc != LAZYEV_OK) return rc;
    if (h->users > 0) return fail(h, LAZYEV_ESTATE, "append to a handle that others share as their prefix");
    if (n_tokens <= 0) return fail(h, LAZYEV_EINVAL, "non-positive token count");
    RowsArgs a = rows_args(h, n_tokens, positions, h->pos_base + h->prefill + h->t);
    if ((rc = rows_view(h, "k", k, h->kv_heads, n_tokens, false, &a.k)) != LAZYEV_OK) return rc;
    if ((rc = rows_view(h, "v", v, h->kv_heads, n_tokens, false, &a.v)) != LAZYEV_OK) return rc;
    if ((rc = same_type(h, a.k, a.v)) != LAZYEV_OK) return rc;
    if (n_tokens > h->capacity - h->n)
        return fail(h, LAZYEV_ECAPACITY, "%d tokens after %d exceed the capacity of %d slots per unit", n_tokens, h->n, h->capacity);
    rows_to_pages(h, h->t, &a);
    cudaError_t e = rows_launch(a, h->turns, h->num_sms, h->stream);
    if (e == cudaSuccess) e = clear_weights(h, h->n, n_tokens);
    if (e != cudaSuccess) return cuda_fail(h, e, "append kernel launch");
    h->launches += 1;
    h->prefilled = true;
    h->prefill += n_tokens;
    h->n += n_tokens;
    return LAZYEV_OK;
}

int lazyev_decode_step_rows(lazyev_t* h, const lazyev_rows_t* q, const lazyev_rows_t* k, const lazyev_rows_t* v,
                            const int32_t* positions, void* out) {
    if (!h) return LAZYEV_EINVAL;
    int rc = check_device(h, "decode_step_rows");
    if (rc != LAZYEV_OK) return rc;
    if (!out) return fail(h, LAZYEV_EINVAL, "null pointer");
    if ((uintptr_t)out & 1) return fail(h, LAZYEV_EINVAL, "out must be 2-byte aligned");
    RowsArgs a = rows_args(h, 1, positions, h->pos_base + h->prefill + h->t);
    if ((rc = rows_view(h, "q", q, h->q_heads, 1, false, &a.q)) != LAZYEV_OK) return rc;
    if ((rc = rows_view(h, "k", k, h->kv_heads, 1, false, &a.k)) != LAZYEV_OK) return rc;
    if ((rc = rows_view(h, "v", v, h->kv_heads, 1, false, &a.v)) != LAZYEV_OK) return rc;
    if ((rc = same_type(h, a.q, a.k)) != LAZYEV_OK || (rc = same_type(h, a.q, a.v)) != LAZYEV_OK) return rc;
    if ((rc = check_step(h)) != LAZYEV_OK) return rc;
    const long long row = kHeadDim, seq = (long long)h->q_heads * row;
    a.q_out = RowView{h->stage_rows, h->batch * seq, seq, 0, row, kTypeBF16};
    rows_to_pages(h, h->t + 1, &a);
    const cudaError_t e = rows_launch(a, h->turns, h->num_sms, h->stream);
    if (e != cudaSuccess) return cuda_fail(h, e, "row kernel launch");
    h->launches += 1;
    rc = run_decode(h, h->stage_rows, out, h->n + 1, h->t + 1, nullptr);
    return rc != LAZYEV_OK ? rc : finish_step(h);
}

// ---- shared prefix ---------------------------------------------------------------------------------
namespace {

// Fits the two handles together; the plan of the shared work on success.
int plan_prefix(lazyev_t* h, const lazyev_t* prefix, PrefixPlan* plan) {
    if (!h->bound || !prefix->bound) return fail(h, LAZYEV_ESTATE, "a shared prefix needs two bound handles");
    if (!prefix->prefilled || prefix->n == 0) return fail(h, LAZYEV_ESTATE, "the prefix handle holds no tokens");
    if (prefix->device != h->device || prefix->layers != h->layers || prefix->q_heads != h->q_heads || prefix->kv_heads != h->kv_heads)
        return fail(h, LAZYEV_EINVAL, "the prefix needs the same layers, heads and device");
    if (h->batch % prefix->batch != 0)
        return fail(h, LAZYEV_EINVAL, "%d sequences do not divide among %d prefixes", h->batch, prefix->batch);
    *plan = prefix_plan(h->layers, h->batch, prefix->batch, h->kv_heads, h->group, prefix->n, h->num_sms);
    if (plan->blocks == 0) return fail(h, LAZYEV_EINVAL, "the shared work of %d prefixes of %d tokens is not supported", prefix->batch, prefix->n);
    return LAZYEV_OK;
}

size_t prefix_o_bytes(const PrefixPlan& p) { return align_up((size_t)p.slots * p.rows * kHeadDim * sizeof(float), 256); }

int detach(lazyev_t* h) {
    lazyev_t* prefix = h->shared;
    if (!prefix) return LAZYEV_OK;
    // what changes the prefix later waits for what reads it now (an event belongs to the device that is current)
    int dev = -1;
    cudaEvent_t done = nullptr;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && dev != h->device) e = cudaSetDevice(h->device);
    if (e == cudaSuccess) e = cudaEventCreateWithFlags(&done, cudaEventDisableTiming);
    if (e == cudaSuccess) e = cudaEventRecord(done, h->stream);
    if (e == cudaSuccess) e = cudaStreamWaitEvent(prefix->stream, done, 0);
    if (done) cudaEventDestroy(done);
    if (dev >= 0 && dev != h->device) cudaSetDevice(dev);
    prefix->users -= 1;
    h->shared = nullptr;
    if (!h->prefilled) h->pos_base = 0;    // no token has a position after the prefix's: an empty handle again
    h->plan_cache.clear();                 // launch shapes differ with and without a prefix
    if (e != cudaSuccess) return cuda_fail(h, e, "detach_prefix");
    return LAZYEV_OK;
}

}  // namespace

int lazyev_query_prefix_workspace(const lazyev_t* h, const lazyev_t* prefix, size_t* bytes) {
    if (!h || !prefix || !bytes) return LAZYEV_EINVAL;
    PrefixPlan plan;
    const int rc = plan_prefix(const_cast<lazyev_t*>(h), prefix, &plan);
    if (rc != LAZYEV_OK) return rc;
    // enough whatever the prefix comes to hold: a caller may ask once and attach later
    plan.slots = prefix_most_slots(h->layers, h->batch, prefix->batch, h->kv_heads, h->group, prefix->capacity, h->num_sms);
    *bytes = prefix_o_bytes(plan) + (size_t)plan.slots * plan.rows * sizeof(float2);
    return LAZYEV_OK;
}

int lazyev_attach_prefix(lazyev_t* h, lazyev_t* prefix, void* workspace) {
    if (!h) return LAZYEV_EINVAL;
    if (!prefix || prefix == h) return fail(h, LAZYEV_EINVAL, "the prefix must be another handle");
    int rc = check_device(h, "attach_prefix");
    if (rc != LAZYEV_OK) return rc;
    if (h->shared) return fail(h, LAZYEV_ESTATE, "a prefix is attached already");
    if (h->users > 0 || prefix->shared) return fail(h, LAZYEV_ESTATE, "a prefix cannot have a prefix of its own");
    PrefixPlan plan;
    if ((rc = plan_prefix(h, prefix, &plan)) != LAZYEV_OK) return rc;
    if (!workspace || ((uintptr_t)workspace & 255)) return fail(h, LAZYEV_EINVAL, "the workspace must be 256-byte aligned");
    cudaError_t e = prefix_prepare(prefix->pool, prefix->units * prefix->pages_per_unit, &h->prefix_pool);
    cudaEvent_t ready = nullptr;
    // (handles that share it already have seen it cleared)
    if (e == cudaSuccess && prefix->users == 0) e = clear_tail_launch(geometry(prefix), prefix->pool, prefix->st, prefix->n, prefix->stream);
    if (e == cudaSuccess) e = cudaEventCreateWithFlags(&ready, cudaEventDisableTiming);
    if (e == cudaSuccess) e = cudaEventRecord(ready, prefix->stream);
    if (e == cudaSuccess) e = cudaStreamWaitEvent(h->stream, ready, 0);
    if (ready) cudaEventDestroy(ready);
    float2* ml = (float2*)((uint8_t*)workspace + prefix_o_bytes(plan));
    if (e == cudaSuccess) e = prefix_clear_launch(plan, ml, h->stream);
    if (e != cudaSuccess) return cuda_fail(h, e, "attach_prefix");
    h->plan_cache.clear();
    h->shared = prefix;
    h->prefix_plan = plan;
    h->prefix_o = (float*)workspace;
    h->prefix_ml = ml;
    h->pos_base = prefix->pos_base + prefix->prefill + prefix->t;
    prefix->users += 1;
    return LAZYEV_OK;
}

int lazyev_detach_prefix(lazyev_t* h) {
    if (!h) return LAZYEV_EINVAL;
    return detach(h);
}

int lazyev_attend(lazyev_t* h, const void* q, void* out) {
    if (!h) return LAZYEV_EINVAL;
    const int rc = check_device(h, "attend");
    if (rc != LAZYEV_OK) return rc;
    if (!q || !out) return fail(h, LAZYEV_EINVAL, "null pointer");
    if (!h->prefilled && !h->shared) return fail(h, LAZYEV_ESTATE, "attend before prefill");
    return run_decode(h, q, out, h->n, h->t, nullptr, nullptr, false);
}

int lazyev_query_state_layout(const lazyev_t* h, size_t* page_table, size_t* ts_mri, size_t* pos, size_t* pbar) {
    if (!h) return LAZYEV_EINVAL;
    const Sizes s = sizes_of(h);
    if (page_table) *page_table = 0;
    if (ts_mri) *ts_mri = s.off_tsm;
    if (pos) *pos = s.off_pos;
    if (pbar) *pbar = s.off_pbar;
    return LAZYEV_OK;
}

int lazyev_query_weights_layout(const lazyev_t* h, size_t* weights) {
    if (!h || !weights) return LAZYEV_EINVAL;
    if (!h->weights_on) return LAZYEV_ESTATE;
    *weights = sizes_of(h).off_weights;
    return LAZYEV_OK;
}

// ---- a chunk of tokens ---------------------------------------------------------------------------------
namespace {

struct ChunkSpace {
    size_t ml, sums, norms, bytes;         // offsets inside the workspace (the shared items' sums come first)
};

ChunkSpace chunk_space(const lazyev_t* h, int n_tokens, int weights) {
    ChunkSpace s;
    s.ml = chunk_ml_offset(h->num_sms);
    s.sums = align_up(chunk_sums_bytes(h->num_sms), 256);
    s.norms = s.sums;
    if (weights != LAZYEV_WEIGHTS_OFF) s.norms += align_up(weigh_sums_bytes(h->num_sms), 256);
    s.bytes = s.norms;
    if (weights != LAZYEV_WEIGHTS_OFF) {
        const ChunkPlan plan = chunk_plan(h->layers, h->batch, h->kv_heads, h->group, n_tokens, n_tokens, 0, 1, h->num_sms);
        s.bytes += (size_t)h->units * plan.tiles * 2 * 128 * sizeof(float);
    }
    return s;
}

ChunkPlan plan_of(const lazyev_t* h, int n, int n_tokens) {
    const lazyev_t* pre = h->shared;
    return chunk_plan(h->layers, h->batch, h->kv_heads, h->group, n, n_tokens, pre ? pre->n : 0, pre ? h->batch / pre->batch : 1, h->num_sms);
}

}  // namespace

int lazyev_debug_chunk_plan(const lazyev_t* h, int n, int n_tokens, int plan[5]) {
    if (!h || !plan) return LAZYEV_EINVAL;
    lazyev_t* w = const_cast<lazyev_t*>(h);
    if (!h->bound) return fail(w, LAZYEV_ESTATE, "debug_chunk_plan before bind");
    if (n_tokens <= 0 || n_tokens > n || n > h->capacity)
        return fail(w, LAZYEV_EINVAL, "a chunk is the last 1 to %d of up to %d cached tokens, not %d", n, h->capacity, n_tokens);
    const ChunkPlan p = plan_of(h, n, n_tokens);
    plan[0] = p.blocks;
    plan[1] = p.blocks > 0 ? weigh_plan(p, h->num_sms).blocks : 0;
    plan[2] = p.whole;
    plan[3] = p.in_step;
    plan[4] = p.joins;
    return LAZYEV_OK;
}

int lazyev_query_chunk_workspace(const lazyev_t* h, int n_tokens, int weights, size_t* bytes) {
    if (!h || !bytes) return LAZYEV_EINVAL;
    lazyev_t* w = const_cast<lazyev_t*>(h);
    if (!h->bound) return fail(w, LAZYEV_ESTATE, "query_chunk_workspace before bind");
    if (n_tokens <= 0 || n_tokens > h->capacity) return fail(w, LAZYEV_EINVAL, "a chunk has 1 to %d tokens", h->capacity);
    if (weights < LAZYEV_WEIGHTS_OFF || weights > LAZYEV_WEIGHTS_ADD) return fail(w, LAZYEV_EINVAL, "unknown use of the weights %d", weights);
    *bytes = chunk_space(h, n_tokens, weights).bytes;
    return LAZYEV_OK;
}

int lazyev_attend_chunk(lazyev_t* h, const lazyev_rows_t* q, int n_tokens, const lazyev_rows_t* out, int weights, void* workspace) {
    if (!h) return LAZYEV_EINVAL;
    int rc = check_device(h, "attend_chunk");
    if (rc != LAZYEV_OK) return rc;
    if (weights < LAZYEV_WEIGHTS_OFF || weights > LAZYEV_WEIGHTS_ADD) return fail(h, LAZYEV_EINVAL, "unknown use of the weights %d", weights);
    if (weights != LAZYEV_WEIGHTS_OFF && !h->weights) return fail(h, LAZYEV_ESTATE, "this handle keeps no weights (lazyev_set_weights)");
    if (n_tokens <= 0 || n_tokens > h->n) return fail(h, LAZYEV_EINVAL, "a chunk is the last 1 to %d cached tokens, not %d", h->n, n_tokens);
    ChunkArgs a = {};
    if ((rc = rows_view(h, "q", q, h->q_heads, n_tokens, false, &a.q)) != LAZYEV_OK) return rc;
    if ((rc = rows_view(h, "out", out, h->q_heads, n_tokens, true, &a.out)) != LAZYEV_OK) return rc;
    if (a.q.dtype != kTypeBF16) return fail(h, LAZYEV_EINVAL, "q must be bfloat16");
    const long long strides[4] = {a.q.stride_layer, a.q.stride_batch, a.q.stride_token, a.q.stride_head};
    const int extent[4] = {h->layers, h->batch, n_tokens, h->q_heads};
    for (int i = 0; i < 4; ++i)
        if (extent[i] > 1 && (strides[i] <= 0 || strides[i] >= (1ll << 38))) return fail(h, LAZYEV_EINVAL, "q: strides must be positive and below 2^38");
    if (!workspace || ((uintptr_t)workspace & 255)) return fail(h, LAZYEV_EINVAL, "the workspace must be 256-byte aligned");
    const lazyev_t* pre = h->shared;
    const ChunkPlan plan = plan_of(h, h->n, n_tokens);
    const WeighPlan wplan = weigh_plan(plan, h->num_sms);
    if (plan.blocks == 0 || wplan.blocks == 0) return fail(h, LAZYEV_EINVAL, "a chunk of %d tokens over %d is not supported", n_tokens, h->n);
    PrefixPool q_map;
    if (!chunk_query_map(plan, a.q, &q_map)) return fail(h, LAZYEV_EINVAL, "q: no tensor map has these strides");
    const ChunkSpace space = chunk_space(h, n_tokens, weights);
    uint8_t* ws = (uint8_t*)workspace;
    a.pool = &h->own_pool;
    a.prefix_pool = pre ? &h->prefix_pool : nullptr;
    a.pages = h->pool;
    a.prefix_pages = pre ? pre->pool : nullptr;
    a.page_table = h->st.page_table;
    a.prefix_table = pre ? pre->st.page_table : nullptr;
    a.pages_per_unit = h->pages_per_unit;
    a.total_pages = h->units * h->pages_per_unit;
    a.prefix_pages_per_unit = pre ? pre->pages_per_unit : 0;
    a.prefix_total_pages = pre ? pre->units * pre->pages_per_unit : 0;
    a.q_map = &q_map;
    a.o = (float*)ws;
    a.ml = (float2*)(ws + space.ml);
    a.counters = h->counters;
    a.norms = weights != LAZYEV_WEIGHTS_OFF ? (float*)(ws + space.norms) : nullptr;
    a.status = h->st.status;
    a.wait_limit_ns = h->wait_limit_ns;
    a.stop_after_tiles = h->stop_after_pages;
    a.weighed = weights != LAZYEV_WEIGHTS_OFF;
    h->counted = true;
    cudaError_t e = chunk_launch(plan, a, h->stream);
    if (e != cudaSuccess) return cuda_fail(h, e, "chunk kernel launch");
    h->launches += plan.joins ? 2 : 1;
    if (weights == LAZYEV_WEIGHTS_OFF) return LAZYEV_OK;
    WeighArgs w = {};
    w.pool = &h->own_pool;
    w.q_map = &q_map;
    w.page_table = h->st.page_table;
    w.pages_per_unit = h->pages_per_unit;
    w.total_pages = a.total_pages;
    w.capacity = h->capacity;
    w.norms = a.norms;
    w.weights = h->weights;
    w.add = weights == LAZYEV_WEIGHTS_ADD;
    w.sums = (float*)(ws + space.sums);
    w.counters = h->counters + kChunkCounters;
    w.status = h->st.status;
    w.wait_limit_ns = h->wait_limit_ns;
    w.stop_after_tiles = h->stop_after_pages;
    e = weigh_launch(wplan, plan, w, h->stream);
    if (e != cudaSuccess) return cuda_fail(h, e, "weight kernel launch");
    h->launches += 1;
    return LAZYEV_OK;
}

// ---- selected blocks -----------------------------------------------------------------------------------
namespace {

struct BlockSpace {
    size_t rough, exact, table, pbar, bytes;       // offsets (the bounds come first)
};

BlockSpace block_space(const lazyev_t* h) {
    const size_t pages = (size_t)h->units * h->pages_per_unit;
    BlockSpace s;
    s.rough = align_up(pages * 2 * kRowBytes, 256);
    s.exact = s.rough + align_up(pages * 2 * sizeof(uint32_t), 256);
    s.table = s.exact + align_up(pages * sizeof(unsigned long long), 256);
    s.pbar = s.table + align_up(pages * sizeof(int32_t), 256);
    s.bytes = s.pbar + align_up((size_t)h->units * h->capacity * sizeof(float), 256);
    return s;
}

BlocksArgs blocks_args(const lazyev_t* h) {
    const BlockSpace s = block_space(h);
    BlocksArgs a = {};
    a.geo = geometry(h);
    a.pool = h->pool;
    a.page_table = h->st.page_table;
    a.bounds = h->block_space;
    a.rough = (uint32_t*)(h->block_space + s.rough);
    a.exact = (unsigned long long*)(h->block_space + s.exact);
    a.table = (int32_t*)(h->block_space + s.table);
    a.status = h->st.status;
    return a;
}

// Bounds of the blocks from `first` on, as far as they are not there yet.
int run_index(lazyev_t* h, int first) {
    const int last = h->n > 0 ? (h->n - 1) / kPageTokens : 0;      // the newest block has none
    if (first > h->indexed) first = h->indexed;
    if (first >= last) return LAZYEV_OK;
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    cudaError_t e = cudaStreamIsCapturing(h->stream, &capture);
    if (e == cudaSuccess) e = bounds_launch(blocks_args(h), first, last - first, h->num_sms, h->stream);
    if (e != cudaSuccess) return cuda_fail(h, e, "bounds kernel launch");
    h->launches += 1;
    if (capture == cudaStreamCaptureStatusNone) h->indexed = last;  // (a graph makes them whenever it is replayed)
    return LAZYEV_OK;
}

}  // namespace

int lazyev_query_block_workspace(const lazyev_t* h, size_t* bytes, size_t* bounds) {
    if (!h || !bytes) return LAZYEV_EINVAL;
    *bytes = block_space(h).bytes;
    if (bounds) *bounds = 0;
    return LAZYEV_OK;
}

int lazyev_set_block_workspace(lazyev_t* h, void* workspace) {
    if (!h) return LAZYEV_EINVAL;
    if (!h->bound) return fail(h, LAZYEV_ESTATE, "set_block_workspace before bind");
    if ((uintptr_t)workspace & 255) return fail(h, LAZYEV_EINVAL, "the workspace must be 256-byte aligned");
    h->block_space = (uint8_t*)workspace;
    h->indexed = 0;
    return LAZYEV_OK;
}

int lazyev_index_blocks(lazyev_t* h, int first_block) {
    if (!h) return LAZYEV_EINVAL;
    const int rc = check_device(h, "index_blocks");
    if (rc != LAZYEV_OK) return rc;
    if (!h->block_space) return fail(h, LAZYEV_ESTATE, "no block workspace (lazyev_set_block_workspace)");
    if (first_block < 0) return fail(h, LAZYEV_EINVAL, "blocks are counted from 0");
    return run_index(h, first_block);
}

int lazyev_attend_sparse(lazyev_t* h, const void* q, int blocks, void* out, int32_t* selected) {
    if (!h) return LAZYEV_EINVAL;
    int rc = check_device(h, "attend_sparse");
    if (rc != LAZYEV_OK) return rc;
    if (!q || !out || blocks <= 0) return fail(h, LAZYEV_EINVAL, "null pointer or non-positive number of blocks");
    if (((uintptr_t)q & 15) || ((uintptr_t)out & 1) || ((uintptr_t)selected & 3))
        return fail(h, LAZYEV_EINVAL, "q must be 16-byte aligned, out 2-byte and selected 4-byte aligned");
    if (!h->block_space) return fail(h, LAZYEV_ESTATE, "no block workspace (lazyev_set_block_workspace)");
    if (!h->prefilled || h->n == 0) return fail(h, LAZYEV_ESTATE, "attend_sparse with no own token cached");
    const int last = (h->n - 1) / kPageTokens, picked = blocks - 1 < last ? blocks - 1 : last;
    const int tokens = picked * kPageTokens + h->n - last * kPageTokens;       // that are read
    DecodeLaunch launch;                     // (refuses before anything is queued)
    if ((rc = choose_decode(h, q, out, tokens, false, &launch)) != LAZYEV_OK) return rc;
    if ((rc = run_index(h, h->indexed)) != LAZYEV_OK) return rc;
    BlocksArgs a = blocks_args(h);
    a.q = q;
    a.selected = selected;
    int launches = 0;
    const cudaError_t e = pick_launch(a, last, picked, blocks, h->num_sms, &launches, h->stream);
    if (e != cudaSuccess) return cuda_fail(h, e, "block selection launch");
    h->launches += launches;
    StateView view = h->st;
    view.page_table = a.table;
    view.pbar = (float*)(h->block_space + block_space(h).pbar);
    return run_decode(h, q, out, tokens, h->t, nullptr, nullptr, false, &view);
}

int lazyev_evict_to(lazyev_t* h, int keep, lazyev_t* dst, int* evicted) {
    if (!h) return LAZYEV_EINVAL;
    if (evicted) *evicted = 0;
    int rc = check_device(h, "evict_to");
    if (rc != LAZYEV_OK) return rc;
    if (!h->prefilled || h->n == 0) return fail(h, LAZYEV_ESTATE, "evict_to before prefill");
    if (keep <= h->n_recent + h->n_initial || keep > h->budget)
        return fail(h, LAZYEV_EINVAL, "keep must be in (n_recent + n_initial, budget]");
    const bool all = h->n <= keep;
    if (!all && candidates_of(h, h->n) < 0)
        return fail(h, LAZYEV_EINVAL, "eviction over %d candidates is not supported", h->n - h->n_recent - h->n_initial);
    if (!dst || dst == h) {
        if (h->users > 0) return fail(h, LAZYEV_ESTATE, "evict_to on a handle that others share as their prefix");
        return all ? LAZYEV_OK : run_cut(h, keep, evicted, h->src, h->first_moved, h->radix_list);
    }
    const int kept = all ? h->n : keep;
    if (!dst->bound) return fail(h, LAZYEV_ESTATE, "evict_to into a handle that is not bound");
    if (dst->device != h->device || dst->layers != h->layers || dst->batch != h->batch || dst->q_heads != h->q_heads || dst->kv_heads != h->kv_heads)
        return fail(h, LAZYEV_EINVAL, "evict_to needs a handle of the same layers, batch, heads and device");
    if (dst->prefilled) return fail(h, LAZYEV_ESTATE, "evict_to into a handle that already holds a cache (reset it first)");
    if (dst->shared != h->shared) return fail(h, LAZYEV_ESTATE, "evict_to needs the same prefix attached to both handles, or to neither");
    if (kept > dst->capacity) return fail(h, LAZYEV_ECAPACITY, "%d tokens exceed the capacity of %d slots per unit", kept, dst->capacity);
    EvictArgs sel = {};
    if (!all && (rc = run_select(h, keep, h->src, h->first_moved, h->radix_list, false, &sel)) != LAZYEV_OK) return rc;
    KeepArgs a = {};
    a.from_geo = geometry(h);
    a.to_geo = geometry(dst);
    a.from = h->st;
    a.to = dst->st;
    a.from_pool = h->pool;
    a.to_pool = dst->pool;
    a.from_weights = h->weights;
    a.to_weights = dst->weights;
    a.src = all ? nullptr : h->src;
    a.keep = kept;
    a.n = h->n;
    cudaEvent_t ready = nullptr;
    cudaError_t e = cudaSuccess;
    if (dst->stream != h->stream) {          // (as in copy_state: the rows move on dst's stream, and h's later work waits for that)
        e = cudaEventCreateWithFlags(&ready, cudaEventDisableTiming);
        if (e == cudaSuccess) e = cudaEventRecord(ready, h->stream);
        if (e == cudaSuccess) e = cudaStreamWaitEvent(dst->stream, ready, 0);
    }
    if (e == cudaSuccess) e = keep_launch(a, dst->stream);
    if (dst->stream != h->stream) {
        if (e == cudaSuccess) e = cudaEventRecord(ready, dst->stream);
        if (e == cudaSuccess) e = cudaStreamWaitEvent(h->stream, ready, 0);
        if (ready) cudaEventDestroy(ready);
    }
    if (e != cudaSuccess) return cuda_fail(h, e, "evict_to");
    dst->launches += 1;
    dst->prefilled = true;
    dst->t = h->t;
    dst->n = kept;
    dst->prefill = h->prefill;
    dst->pos_base = h->pos_base;
    dst->indexed = 0;
    if (evicted) *evicted = h->n - kept;
    return LAZYEV_OK;
}

int lazyev_evict(lazyev_t* h, int* evicted) {
    if (!h) return LAZYEV_EINVAL;
    if (!h->prefilled) return fail(h, LAZYEV_ESTATE, "evict before prefill");
    if (h->users > 0) return fail(h, LAZYEV_ESTATE, "evict on a handle that others share as their prefix");
    return run_evict(h, evicted, h->src, h->first_moved, h->radix_list);
}

// ---- eviction without caller-provided scratch ------------------------------------------------
// Source lists and first-moved indices of lazyev_evict_static(): one array per GPU that loads the
// library, held until the process exits.  4 MiB + 32 KiB: source lists, first-moved indices, and the list
// of units that take the selection's general route.
constexpr size_t kStaticSrcEntries = (size_t)1 << 20;      // units * budget_now must not exceed this
constexpr int kStaticMaxUnits = 4096;
constexpr int kStaticMaxDevices = 64;
static __device__ __align__(256) int32_t g_static_evict_scratch[kStaticSrcEntries + 2 * kStaticMaxUnits + 64];
// Device addresses of the array above, one per device ordinal.  The symbol itself is only a
// host-side stand-in: kernels must be given the address cudaGetSymbolAddress() returns.
static std::atomic<int32_t*> g_static_evict_ptr[kStaticMaxDevices];

int lazyev_evict_static(lazyev_t* h, int* evicted) {
    if (!h) return LAZYEV_EINVAL;
    if (evicted) *evicted = 0;
    if (!h->prefilled) return fail(h, LAZYEV_ESTATE, "evict_static before prefill");
    if (h->users > 0) return fail(h, LAZYEV_ESTATE, "evict_static on a handle that others share as their prefix");
    if (h->units > kStaticMaxUnits || (size_t)h->units * (size_t)h->budget_now > kStaticSrcEntries)
        return fail(h, LAZYEV_ECAPACITY,
                    "evict_static holds %zu source indices for at most %d units; this handle needs %zu for %d units "
                    "(use lazyev_evict with the bound scratch region)",
                    kStaticSrcEntries, kStaticMaxUnits, (size_t)h->units * (size_t)h->budget_now, h->units);
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_fail(h, e, "cudaGetDevice");
    if (dev != h->device || dev < 0 || dev >= kStaticMaxDevices)
        return fail(h, LAZYEV_ESTATE, "evict_static needs device %d (the one bound to this handle) to be current, not %d",
                    h->device, dev);
    int32_t* base = g_static_evict_ptr[dev].load(std::memory_order_acquire);
    if (!base) {    // first call on this device: resolve the array's device address (threads may race; same value)
        e = cudaGetSymbolAddress((void**)&base, g_static_evict_scratch);
        if (e != cudaSuccess || !base) return cuda_fail(h, e, "cudaGetSymbolAddress(static eviction scratch)");
        g_static_evict_ptr[dev].store(base, std::memory_order_release);
    }
    // Same trigger test, kernels, timing spans and accounting as lazyev_evict(); only the work lists
    // live elsewhere.  Every entry below budget is rewritten by the select kernel before the compact
    // kernel reads it, so nothing in the array has to be cleared.
    return run_evict(h, evicted, base, base + kStaticSrcEntries, base + kStaticSrcEntries + kStaticMaxUnits);
}

int lazyev_get_counters(lazyev_t* h, lazyev_counters_t* out) {
    if (!h || !out) return LAZYEV_EINVAL;
    if (!h->bound) return fail(h, LAZYEV_ESTATE, "get_counters before bind");
    int32_t words[16] = {0};
    cudaError_t e = cudaMemcpyAsync(words, h->st.status, sizeof(words), cudaMemcpyDeviceToHost, h->stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(h->stream);
    if (e != cudaSuccess) return cuda_fail(h, e, "reading the device counters");
    out->device_status = words[0];
    out->select_radix_units = words[kCounterRadixUnits];
    out->select_zero_cut_units = words[kCounterZeroCutUnits];
    return LAZYEV_OK;
}

int lazyev_get_info(const lazyev_t* h, lazyev_info_t* out) {
    if (!h || !out) return LAZYEV_EINVAL;
    out->layers = h->layers;
    out->batch = h->batch;
    out->q_heads = h->q_heads;
    out->kv_heads = h->kv_heads;
    out->head_dim = h->head_dim;
    out->units = h->units;
    out->budget = h->budget;
    out->budget_now = h->budget_now;
    out->window = h->window;
    out->n_recent = h->n_recent;
    out->n_initial = h->n_initial;
    out->capacity = h->capacity;
    out->pages_per_unit = h->pages_per_unit;
    out->t = h->t;
    out->n = h->n;
    out->prefill = h->prefill;
    out->splits = h->last_plan.splits;
    out->stages = h->last_plan.stages;
    out->groups = h->last_plan.groups;
    out->tail_units = h->last_tail_units;
    out->tail_splits = h->last_tail_splits;
    out->grid = h->last_grid;
    out->smem_bytes = h->last_plan.smem_bytes;
    out->launches = h->launches;
    out->evictions = h->evictions;
    out->host_ranges = h->last_host_ranges;
    out->prefix_tokens = h->shared ? h->shared->n : 0;
    out->prefix_blocks = h->shared ? h->prefix_plan.blocks : 0;
    out->next_position = h->pos_base + h->prefill + h->t;
    return LAZYEV_OK;
}

int lazyev_dump_state(lazyev_t* h, lazyev_dump_t* d) {
    if (!h || !d) return LAZYEV_EINVAL;
    if (!h->bound) return fail(h, LAZYEV_ESTATE, "dump before bind");
    if (d->unit_begin < 0 || d->unit_count < 0 || d->unit_begin + d->unit_count > h->units)
        return fail(h, LAZYEV_EINVAL, "unit range out of bounds");
    d->t = h->t;
    d->n = h->n;
    d->capacity = h->capacity;
    const size_t cap = h->capacity, first = (size_t)d->unit_begin * cap, count = (size_t)d->unit_count * cap;
    cudaError_t e = cudaSuccess;
    int32_t status = 0;
    e = cudaMemcpyAsync(&status, h->st.status, sizeof(status), cudaMemcpyDeviceToHost, h->stream);
    if (e == cudaSuccess && d->pos) e = cudaMemcpyAsync(d->pos, h->st.pos + first, count * 4, cudaMemcpyDeviceToHost, h->stream);
    std::vector<int2> pairs;               // TS and MRI sit interleaved on the device
    if (e == cudaSuccess && (d->ts || d->mri)) {
        pairs.resize(count);
        e = cudaMemcpyAsync(pairs.data(), h->st.tsm + first, count * sizeof(int2), cudaMemcpyDeviceToHost, h->stream);
    }
    if (e == cudaSuccess && d->pbar) e = cudaMemcpyAsync(d->pbar, h->st.pbar + first, count * 4, cudaMemcpyDeviceToHost, h->stream);
    if (e == cudaSuccess && !pairs.empty()) e = cudaStreamSynchronize(h->stream);
    if (e != cudaSuccess) return cuda_fail(h, e, "state download");
    for (size_t i = 0; i < pairs.size(); ++i) {
        if (d->ts) d->ts[i] = pairs[i].x;
        if (d->mri) d->mri[i] = pairs[i].y;
    }
    if (d->score) {
        const Geometry geo = geometry(h);
        for (int u0 = 0; u0 < d->unit_count; u0 += kScoreStageUnits) {
            const int cnt = d->unit_count - u0 < kScoreStageUnits ? d->unit_count - u0 : kScoreStageUnits;
            e = h->score_mode == LAZYEV_SCORE_WEIGHT
                    ? weights_score_launch(geo, h->weights, d->unit_begin + u0, cnt, h->n, h->stage_score, h->stream)
                    : score_launch(geo, h->st, d->unit_begin + u0, cnt, h->n, h->t, h->score_mode, h->stage_score, h->stream);
            if (e == cudaSuccess)
                e = cudaMemcpyAsync(d->score + (size_t)u0 * cap, h->stage_score, (size_t)cnt * cap * sizeof(double), cudaMemcpyDeviceToHost, h->stream);
            if (e == cudaSuccess) e = cudaStreamSynchronize(h->stream);
            if (e != cudaSuccess) return cuda_fail(h, e, "score download");
            h->launches += 1;
        }
    }
    if (d->k || d->v) {
        // Pages come back raw and are un-swizzled here on the host.
        const int np = (h->n + kPageTokens - 1) / kPageTokens;
        std::vector<int32_t> table((size_t)d->unit_count * h->pages_per_unit);
        e = cudaMemcpyAsync(table.data(), h->st.page_table + (size_t)d->unit_begin * h->pages_per_unit, table.size() * 4, cudaMemcpyDeviceToHost, h->stream);
        if (e == cudaSuccess) e = cudaStreamSynchronize(h->stream);
        if (e != cudaSuccess) return cuda_fail(h, e, "page table download");
        std::vector<uint8_t> page(kPageBytes);
        for (int u = 0; u < d->unit_count; ++u) {
            for (int pg = 0; pg < np; ++pg) {
                const int32_t pp = table[(size_t)u * h->pages_per_unit + pg];
                e = cudaMemcpyAsync(page.data(), h->pool + (size_t)pp * kPageBytes, kPageBytes, cudaMemcpyDeviceToHost, h->stream);
                if (e == cudaSuccess) e = cudaStreamSynchronize(h->stream);
                if (e != cudaSuccess) return cuda_fail(h, e, "page download");
                for (int r = 0; r < kPageTokens; ++r) {
                    const size_t slot = (size_t)u * cap + (size_t)pg * kPageTokens + r;
                    for (int c = 0; c < kChunksPerRow; ++c) {
                        const uint8_t* ks = page.data() + r * kRowBytes + swz_chunk(c, r) * 16;
                        if (d->k) memcpy((uint8_t*)d->k + slot * kRowBytes + c * 16, ks, 16);
                        if (d->v) memcpy((uint8_t*)d->v + slot * kRowBytes + c * 16, ks + kPageHalfBytes, 16);
                    }
                }
            }
        }
    }
    e = cudaStreamSynchronize(h->stream);
    if (e != cudaSuccess) return cuda_fail(h, e, "stream synchronisation");
    d->device_status = status;
    if (status != 0) return fail(h, LAZYEV_EDEVICE, "device status word = %d (1: wait timed out, 2: bad index)", status);
    return LAZYEV_OK;
}

int lazyev_load_state(lazyev_t* h, const lazyev_dump_t* d, int prefill) {
    if (!h || !d) return LAZYEV_EINVAL;
    if (!h->bound) return fail(h, LAZYEV_ESTATE, "load_state before bind");
    if (h->prefilled) return fail(h, LAZYEV_ESTATE, "load_state on a handle that already holds a cache");
    if (d->unit_begin != 0 || d->unit_count != h->units) return fail(h, LAZYEV_EINVAL, "the snapshot must cover all %d units", h->units);
    if (!d->pos || !d->ts || !d->mri || !d->k || !d->v) return fail(h, LAZYEV_EINVAL, "pos, ts, mri, k and v are required");
    // (sequences behind a shared prefix may have begun with no prompt of their own)
    if (d->n <= 0 || d->n > h->capacity || d->capacity < d->n || d->t < 0 || prefill < 0 || (prefill == 0 && !h->shared))
        return fail(h, LAZYEV_EINVAL, "snapshot sizes out of range (n = %d, capacity here = %d)", d->n, h->capacity);
    const size_t scap = (size_t)d->capacity, width = (size_t)d->n * 4;
    cudaError_t e = cudaMemcpy2DAsync(h->st.pos, (size_t)h->capacity * 4, d->pos, scap * 4, width, h->units, cudaMemcpyHostToDevice, h->stream);
    std::vector<int2> pairs((size_t)h->units * d->n);      // interleaved (TS, MRI), rows of n
    for (int u = 0; u < h->units; ++u)
        for (int i = 0; i < d->n; ++i)
            pairs[(size_t)u * d->n + i] = make_int2(d->ts[(size_t)u * scap + i], d->mri[(size_t)u * scap + i]);
    if (e == cudaSuccess)
        e = cudaMemcpy2DAsync(h->st.tsm, (size_t)h->capacity * 8, pairs.data(), (size_t)d->n * 8, (size_t)d->n * 8, h->units,
                              cudaMemcpyHostToDevice, h->stream);
    if (e == cudaSuccess && d->pbar) e = cudaMemcpy2DAsync(h->st.pbar, (size_t)h->capacity * 4, d->pbar, scap * 4, width, h->units, cudaMemcpyHostToDevice, h->stream);
    std::vector<float> weights;
    if (h->weights && h->score_mode == LAZYEV_SCORE_WEIGHT && d->score) {
        weights.resize((size_t)h->units * d->n);
        for (int u = 0; u < h->units; ++u)
            for (int i = 0; i < d->n; ++i) weights[(size_t)u * d->n + i] = (float)d->score[(size_t)u * scap + i];
        if (e == cudaSuccess)
            e = cudaMemcpy2DAsync(h->weights, (size_t)h->capacity * 4, weights.data(), width, width, h->units, cudaMemcpyHostToDevice, h->stream);
    } else if (e == cudaSuccess) {
        e = clear_weights(h, 0, d->n);
    }
    if (e != cudaSuccess) return cuda_fail(h, e, "state upload");
    // K / V rows: swizzled into pages on the host, one page per copy
    const int np = (d->n + kPageTokens - 1) / kPageTokens;
    std::vector<int32_t> table((size_t)h->units * h->pages_per_unit);
    e = cudaMemcpyAsync(table.data(), h->st.page_table, table.size() * 4, cudaMemcpyDeviceToHost, h->stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(h->stream);
    if (e != cudaSuccess) return cuda_fail(h, e, "page table download");
    std::vector<uint8_t> page(kPageBytes);
    for (int u = 0; u < h->units; ++u) {
        for (int pg = 0; pg < np; ++pg) {
            memset(page.data(), 0, kPageBytes);
            for (int r = 0; r < kPageTokens && pg * kPageTokens + r < d->n; ++r) {
                const size_t slot = (size_t)u * scap + (size_t)pg * kPageTokens + r;
                for (int c = 0; c < kChunksPerRow; ++c) {
                    uint8_t* kd = page.data() + r * kRowBytes + swz_chunk(c, r) * 16;
                    memcpy(kd, (const uint8_t*)d->k + slot * kRowBytes + c * 16, 16);
                    memcpy(kd + kPageHalfBytes, (const uint8_t*)d->v + slot * kRowBytes + c * 16, 16);
                }
            }
            const int32_t pp = table[(size_t)u * h->pages_per_unit + pg];
            e = cudaMemcpyAsync(h->pool + (size_t)pp * kPageBytes, page.data(), kPageBytes, cudaMemcpyHostToDevice, h->stream);
            if (e == cudaSuccess) e = cudaStreamSynchronize(h->stream);      // the staging page is reused
            if (e != cudaSuccess) return cuda_fail(h, e, "page upload");
        }
    }
    h->prefilled = true;
    h->prefill = prefill;
    h->n = d->n;
    h->t = d->t;
    h->indexed = 0;
    return LAZYEV_OK;
}

int lazyev_mri_histogram(lazyev_t* h, int unit_begin, int unit_count, long long* host_hist, int bins) {
    if (!h || !host_hist) return LAZYEV_EINVAL;
    if (!h->prefilled) return fail(h, LAZYEV_ESTATE, "mri_histogram before prefill");
    if (unit_begin < 0 || unit_count <= 0 || unit_begin + unit_count > h->units)
        return fail(h, LAZYEV_EINVAL, "unit range out of bounds");
    if (bins < 2 || bins > kMaxHistBins) return fail(h, LAZYEV_EINVAL, "bins must be in [2, %d]", kMaxHistBins);
    cudaError_t e = mri_histogram_launch(geometry(h), h->st, unit_begin, unit_count, h->n, bins, h->stage_hist, h->stream);
    if (e == cudaSuccess)
        e = cudaMemcpyAsync(host_hist, h->stage_hist, (size_t)bins * sizeof(long long), cudaMemcpyDeviceToHost, h->stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(h->stream);
    if (e != cudaSuccess) return cuda_fail(h, e, "MRI histogram");
    h->launches += 1;
    return LAZYEV_OK;
}

int lazyev_mri_quantile(lazyev_t* h, int unit_begin, int unit_count, double fraction, int* value, long long* recurring) {
    if (!h || !value) return LAZYEV_EINVAL;
    if (!(fraction > 0.0 && fraction <= 1.0)) return fail(h, LAZYEV_EINVAL, "fraction must be in (0, 1]");
    std::vector<long long> hist(kMaxHistBins);
    const int rc = lazyev_mri_histogram(h, unit_begin, unit_count, hist.data(), kMaxHistBins);
    if (rc != LAZYEV_OK) return rc;
    long long total = 0;
    for (int b = 1; b < kMaxHistBins; ++b) total += hist[b];
    if (recurring) *recurring = total;
    *value = 0;
    if (total == 0) return LAZYEV_OK;
    // smallest v such that at least fraction * total of the re-activated tokens have MRI <= v
    long long cum = 0;
    for (int b = 1; b < kMaxHistBins; ++b) {
        cum += hist[b];
        if ((double)cum >= fraction * (double)total) {
            *value = b;
            break;
        }
    }
    return LAZYEV_OK;
}

int lazyev_set_profiling(lazyev_t* h, int on) {
    if (!h) return LAZYEV_EINVAL;
    if (!h->bound) return fail(h, LAZYEV_ESTATE, "set_profiling before bind");
    const int rc = collect_profile(h);
    h->profiling = on != 0;
    return rc;
}

int lazyev_get_profile(lazyev_t* h, lazyev_profile_t* out, int reset) {
    if (!h || !out) return LAZYEV_EINVAL;
    const int rc = collect_profile(h);
    if (rc != LAZYEV_OK) return rc;
    *out = h->prof;
    if (reset) h->prof = lazyev_profile_t{};
    return LAZYEV_OK;
}

int lazyev_synchronize(lazyev_t* h) {
    if (!h) return LAZYEV_EINVAL;
    if (!h->bound) return fail(h, LAZYEV_ESTATE, "synchronize before bind");
    if (h->copy_in) {
        const int rc = host_wait(h, 0);
        if (rc != LAZYEV_OK) return rc;
    }
    return check_device_status(h);
}

int lazyev_destroy(lazyev_t* h) {
    if (!h) return LAZYEV_EINVAL;
    if (h->users > 0) return fail(h, LAZYEV_ESTATE, "destroy of a handle that others share as their prefix");
    detach(h);
    if (h->copy_in) host_wait(h, 0);        // no copy of ours may still be writing the caller's host buffers
    for (const lazyev::Span& sp : h->pending) {
        cudaEventDestroy(sp.start);
        cudaEventDestroy(sp.stop);
    }
    for (cudaEvent_t e : h->free_events) cudaEventDestroy(e);
    if (h->tail_stream) cudaStreamDestroy(h->tail_stream);
    if (h->ev_fork) cudaEventDestroy(h->ev_fork);
    if (h->ev_join) cudaEventDestroy(h->ev_join);
    if (h->copy_in) cudaStreamDestroy(h->copy_in);
    if (h->copy_out) cudaStreamDestroy(h->copy_out);
    for (int i = 0; i <= kHostChunks; ++i) {
        if (h->ev_in[i]) cudaEventDestroy(h->ev_in[i]);
        if (h->ev_done[i]) cudaEventDestroy(h->ev_done[i]);
    }
    if (h->ev_ready) cudaEventDestroy(h->ev_ready);
    for (int i = 0; i < 2; ++i)
        if (h->ev_step_done[i]) cudaEventDestroy(h->ev_step_done[i]);
    delete h;
    return LAZYEV_OK;
}

}  // extern "C"
