// Host-side interfaces between the C-ABI layer and the kernel launchers.
#pragma once

#include "common.cuh"

namespace lzk {

// ---- attention over a shared prefix ------------------------------------------------------------------
// How the prefix kernel's work is laid out.
struct PrefixPlan {
    int kv_heads, batch;                // of the handle that decodes
    int share, group;                   // sequences per prefix sequence, query heads per KV head
    int tile_seqs, tiles, pairs;        // sequences per row tile, row tiles per prefix unit, items (pairs of tiles) per unit
    int key_tiles;                      // 128-key tiles of the prefix
    int blocks;                         // the walk over (item, key tile) is cut into `blocks` contiguous parts:
    int per, extra;                     // the first `extra` of per + 1 steps, the others of per
    int slots;                          // most partial sums of a row
    long long rows;                     // query rows = partial sums per slot
};

__host__ __device__ __forceinline__ int prefix_begin(const PrefixPlan& p, int block) {
    return block * p.per + (block < p.extra ? block : p.extra);
}
// Block that works on step x.
__host__ __device__ __forceinline__ int prefix_block_of(const PrefixPlan& p, int x) {
    const int longer = p.extra * (p.per + 1);
    return x < longer ? x / (p.per + 1) : p.extra + (x - longer) / p.per;
}

struct PrefixView {        // what the decode kernel adds to every unit: ml = null for none
    PrefixPlan plan;
    const float* o;        // [slots][rows][128], relative to m
    const float2* ml;      // [slots][rows]: reference (log2 domain, -inf: no such partial sum), sum of exp2(x - reference)
};

struct PrefixPool {
    unsigned long long map[16];         // a tensor map
};

struct PrefixArgs {
    const PrefixPool* pool;
    const int32_t* page_table;
    int n, pages_per_unit, total_pages; // of the prefix handle
    int layers;
    const void* q;
    float* o;
    float2* ml;
    int32_t* status;
    unsigned long long wait_limit_ns;
    int stop_after_tiles;
};
// blocks = 0: more steps than an int counts.
PrefixPlan prefix_plan(int layers, int batch, int prefixes, int kv_heads, int group, int n, int num_sms);
// The most slots of a plan for up to `capacity` tokens (they do not grow with n alone: a longer prefix may have fewer).
int prefix_most_slots(int layers, int batch, int prefixes, int kv_heads, int group, int capacity, int num_sms);
cudaError_t prefix_prepare(const uint8_t* pool, int total_pages, PrefixPool* out);
// Marks every partial sum as absent: a row has up to `slots` of them, and no launch writes those it has not.
cudaError_t prefix_clear_launch(const PrefixPlan& plan, float2* ml, cudaStream_t stream);
cudaError_t prefix_launch(const PrefixPlan& plan, const PrefixArgs& a, cudaStream_t stream);
// Zeroes the slots behind the last token in every unit's last page.
cudaError_t clear_tail_launch(const Geometry& geo, uint8_t* pool, StateView st, int n, cudaStream_t stream);

// ---- decode ------------------------------------------------------------------
struct DecodeConfig {
    int units, group, pages_per_unit, capacity;
    float alpha;
    int force_splits;      // 0 = automatic
    int force_stages;      // 0 = automatic
    int force_groups;      // 0 = automatic; groups of four consumer warps per block (1 or 2)
    unsigned long long wait_limit_ns;   // bounded waits give up after this long
    int stop_after_pages;  // diagnostics: -1 = off
    bool prefix;           // the launches add the partial sums of a shared prefix
};

struct DecodePlan {
    int splits, stages, groups, pages_per_cta, logit_stride, tmem_pages, tmem_cols;
    int off_logits, off_xchg, off_wml, off_slots, off_misc, off_prefix, off_bars, smem_bytes;
};

struct DecodeArgs {
    const uint8_t* pool;
    StateView state;
    const void* q;
    void* out;
    int n;                 // cached tokens per unit, the new one included
    int t;                 // this decode step
    int unit_begin, unit_count;   // the units this launch covers
    int rounds_before;            // whole rounds of the same walk done by earlier launches (0 for a walk of its own)
    const void* k_new;            // non-null: the launch also appends the new token (slot n - 1, TS = t, MRI = 0)
    const void* v_new;
    int append_position;
    PrefixView prefix;            // prefix.ml = null: none
    bool behind_prefix;           // the prefix launch is right before: begin beside its end
};

// Deepest ring and the shared-memory layout for n cached tokens and a cluster of `splits` blocks;
// -1 if nothing fits.
int decode_plan(const DecodeConfig& c, int n, int max_smem, int splits, DecodePlan* plan);
cudaError_t decode_prepare();
cudaError_t decode_max_clusters(const DecodePlan& plan, int* clusters);
cudaError_t decode_launch(const DecodeConfig& c, const DecodePlan& plan, int clusters, const DecodeArgs& a,
                          cudaStream_t stream);

// Short units behind a shared prefix: a warp per unit (a.prefix set, a.n <= kShortTokens, no append inside).
constexpr int kShortTokens = 384;
cudaError_t decode_short_prepare();
DecodePlan decode_short_plan();        // what lazyev_get_info() reports of such a launch
int decode_short_blocks(int units, int num_sms);
cudaError_t decode_short_launch(const DecodeConfig& c, const DecodeArgs& a, int num_sms, cudaStream_t stream);

// ---- cache maintenance ---------------------------------------------------------
cudaError_t init_state_launch(const Geometry& geo, StateView st, cudaStream_t stream);
// ts_first = INT_MIN: every prompt token starts at TS = 0; otherwise token i starts at TS = ts_first + i.
// Token i is recorded at position pos_first + i.
cudaError_t prefill_launch(const Geometry& geo, uint8_t* pool, StateView st, const void* k, const void* v,
                           int n_tokens, int ts_first, int pos_first, cudaStream_t stream);
cudaError_t append_launch(const Geometry& geo, uint8_t* pool, StateView st, const void* k_new, const void* v_new,
                          int slot, int t, int position, cudaStream_t stream);

// ---- head rows: norm, rotation, paged append -------------------------------------------------------
constexpr int kTypeBF16 = 0, kTypeF16 = 1, kTypeF32 = 2;      // LAZYEV_BF16 ...
constexpr int kMaxPairs = kHeadDim / 2;

struct RowView {           // head rows of 128 contiguous elements; strides in elements
    const void* data;      // null: no rows of this kind
    long long stride_layer, stride_batch, stride_token, stride_head;
    int dtype;
};

struct RowsArgs {
    RowView q, k, v, q_out, k_out;      // k_out without a pool, v with one; q, k, v of one type, q_out and k_out too
    int layers, batch, q_heads, kv_heads, n_tokens;
    int pairs, interleaved;             // 0 pairs: no rotation
    float amplitude, eps;
    const float* q_weight;              // [layers][128]; null: no norm
    const float* k_weight;
    const int32_t* positions;           // [batch][n_tokens]; null: first_position + i
    int first_position;
    // keys and values into the pages of token slots slot .. slot + n_tokens - 1 (pool = null: keys go to k_out)
    uint8_t* pool;
    const int32_t* page_table;
    int2* tsm;
    int32_t* pos;
    float* pbar;
    int32_t* status;
    int pages_per_unit, capacity, total_pages, slot, ts, pos_first;
};
// turns: rotation per position of every pair, in whole turns
cudaError_t rows_launch(const RowsArgs& a, const double* turns, int num_sms, cudaStream_t stream);

// ---- prompt pass (causal attention over the prompt with tracking) -----------------------------------
struct PromptArgs {
    const void* q;         // [P][units][group][128] bf16
    const void* k;         // [units][P][128] bf16
    const void* v;
    void* out;             // like q
    int n_tokens;          // P
    float alpha;
    float* dump;           // optional [dump_count][P][P] probabilities per prompt row
    int dump_begin, dump_count;
    unsigned long long wait_limit_ns;
    int stop_after_tiles;  // diagnostics: starve the K-tile ring (-1: off)
};
// TS / MRI of the prompt tokens must already hold their starting values (TS = own time, MRI = 0).
cudaError_t prompt_launch(const Geometry& geo, StateView st, const PromptArgs& a, int num_sms, cudaStream_t stream);

// ---- eviction --------------------------------------------------------------------
struct EvictArgs {
    int n;                 // cached tokens before the eviction
    int budget;            // tokens to keep (B_t)
    int n_recent, n_initial;
    int t;
    int score_mode;
    int32_t* src;          // [units][budget]: slot that moves to slot j
    int32_t* first_moved;  // [units]: first j with src[j] != j (budget if none)
    const double* h2_table;   // H2 term of the score per MRI value, for the mode in score_mode
    int h2_entries;
    int32_t* radix_list;   // [units]: units whose k-th score is not zero (filled by the first select stage)
    int32_t* radix_count;  // [1]
};

constexpr int kH2TableEntries = 1 << 15;    // MRI values covered by the table; larger ones are evaluated directly
// Fills table[m], m < entries, with the H2 term of Eq. (2) in the variant `score_mode` selects.
cudaError_t h2_table_launch(int score_mode, int entries, double* table, cudaStream_t stream);

size_t select_smem_bytes(int n_candidates);
cudaError_t select_prepare();
cudaError_t select_launch(const Geometry& geo, StateView st, const EvictArgs& a, int num_sms, cudaStream_t stream);
cudaError_t compact_launch(const Geometry& geo, uint8_t* pool, StateView st, const EvictArgs& a,
                           cudaStream_t stream);
// Eq. (2) for every slot < n of units [unit_begin, unit_begin + unit_count) into out[unit][capacity].
cudaError_t score_launch(const Geometry& geo, StateView st, int unit_begin, int unit_count, int n, int t,
                         int score_mode, double* out, cudaStream_t stream);

// hist[b] (b < bins - 1) = cached tokens of the unit range with MRI = b; hist[bins - 1] = the rest.
cudaError_t mri_histogram_launch(const Geometry& geo, StateView st, int unit_begin, int unit_count, int n, int bins,
                                 unsigned long long* hist, cudaStream_t stream);

}  // namespace lzk
