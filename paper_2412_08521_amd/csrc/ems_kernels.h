// Internal interface between the host-side C ABI (ems_api.hip) and the kernel files.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ems {

struct ScoreArgs {
    const void* q;
    const void* k;
    float* s_glo;       // [B*Hkv, N]
    float* s_loc;       // [B*Hkv, N]
    float* lse_opt;     // [B*Hq, N] natural log, nullable
    float* lse2;        // [B*Hq, n_pad] base-2 log-sum-exp of c*S, +inf past N (workspace)
    const float* lse_in_nat;  // caller's natural-log row log-sum-exp for pass 2, or null
    float* part_glo;    // [B*Hkv, n_chunks, N] (workspace, n_chunks > 1 only), or of an even deal
    float* part_loc;    // [B*Hkv, n_chunks - loc_chunk0, N]    [B*Hkv, p2_waves + key tiles, keys per tile] each
    int batch, q_heads, kv_heads, head_dim, seq_len, window;
    int n_pad;          // seq_len rounded up to a multiple of 64
    int n_chunks;       // row chunks of pass 2
    int chunk_rows;     // rows per chunk (multiple of 64)
    int loc_chunk0;     // first chunk that holds a last-window row
    float scale_log2e;  // softmax scale * log2(e)
    int p1_groups, p1_per_group;  // pass-1 work grouping per XCD (set by the launcher)
    // Even deals (score_deal): waves per head and stages per wave; 0 waves = the pass takes whole items.
    int p1_waves, p1_len, p2_waves, p2_len;
    int p1_by_block;    // the first pass gives every block one item, by its index
    float* part_m;      // [B*Hq, p1_waves + row tiles, rows per tile] partial running maxima (workspace)
    float* part_l;      // partial sums relative to them
    // Work queues (set by the launchers): a wave takes its work items from the queue of its XCD; once
    // that is empty, the first pass goes on with another XCD's queue, the second pass with a pool that
    // every XCD draws from.
    int* queue;         // [2][kXcds + 1] cursors: second pass, first pass (workspace; cleared before a pass)
    int p1_local;       // first pass: items per XCD queue
    int queue_clear;    // the cursors are known to be clear (the pass follows the first pass's launch)
    int q_dynamic;      // 1: waves stay and take items from the cursors; 0: one item per block, by block index
    int q_share;        // (batch * kv_heads) / 8 heads per XCD queue; 0 = no queues
    int p2_split;       // row chunks below this index are in the pool
    int p2_local, p2_pool;   // items per XCD queue, items in the pool
};

struct SelectArgs {
    const float* s_glo;
    const float* s_loc;
    float* s_gl_opt;    // nullable
    float* pooled;      // [B*Hkv, N] workspace (pooled score = ranking keys; short sequences: Eq. 2 vector)
    // long sequences only (workspace):
    uint32_t* cand_key; // [B*Hkv, N] candidates' keys in integer order form, position order
    int32_t* cand_pos;  // [B*Hkv, N] their positions
    int* coarse_hist;   // [B*Hkv, select_coarse_bins()] keys per leading-bit bin
    float* chunk_sums;  // [B*Hkv, chunks, 2] sums of s_glo / s_loc per chunk
    int* chunk_count;   // [B*Hkv, chunks, 2] where a chunk's candidates start in the list, how many
    int* head_info;     // [B*Hkv] list cursor (ends as the length of the candidate list)
    int n_chunks;       // select_chunks(seq_len)
    int32_t* imp_idx;
    int32_t* tbm_idx;
    int bkv, seq_len, window, n_imp, n_tbm, pool_kernel;
};

struct MergeArgs {
    const void* k;
    const void* v;
    const int32_t* imp_idx;
    const int32_t* tbm_idx;
    void* k_out;
    void* v_out;
    int32_t* kept_pos;
    int32_t* tbm_dest;
    float* tbm_sim;
    float* k_norm;      // [B*Hkv, n_imp + n_tbm] (caller's k_norm_opt or workspace)
    int32_t* slot_count;
    int bkv, head_dim, seq_len, window, budget, n_imp, n_tbm;
    float tau;
    const float* weight;  // [B*Hkv, seq_len] per-token merge weight, or null = plain mean
    int similarity;       // 0 key cosine, 1 value cosine, 2 their product
    // centre slices of the destination search: how many the workspace has room for (dest_max_slices), then, set by the
    // launcher, how many there are and their rows; with one slice the partials are unused
    int slice_rows, n_slices;
    float* part_best;     // [B*Hkv, n_slices, n_tbm] best similarity within the slice
    int32_t* part_arg;    // [B*Hkv, n_slices, n_tbm] its centre
    // set by the launcher: output rows per wave; merge blocks per head, of which the first share the zero
    // class; where their sums go and how many floats a head has there
    int rows_per_wave, merge_blocks, zero_blocks;
    float* zero_part;
    size_t zero_stride;
};

struct ExpandArgs {
    const void* k_cache;
    const void* v_cache;
    const int32_t* kept_pos;
    const int32_t* tbm_idx;
    const int32_t* tbm_dest;
    const float* k_norm;
    void* k_exp;
    void* v_exp;
    int32_t* pos_exp;
    int bkv, head_dim, window, budget, n_imp, n_tbm;
};

// Decode-time state of the compressed cache: one row per (batch, kv-head) in every array.
struct DecodeState {
    void* k_cache;          // [bkv, budget + 1, D]
    void* v_cache;
    float* row_norm;        // [bkv, budget]
    int32_t* entry_count;   // [bkv, n_imp]
    int32_t* entry_tok;     // [bkv, n_imp]
    int32_t* tok_pos;       // [bkv, T]   T = n_imp + n_tbm + window
    int32_t* tok_row;       // [bkv, T]   cache row, -1 = free element
    float* tok_norm;
    float* tok_glo;
    float* tok_past;
    float* tok_cur;
    int32_t* step_count;    // [1]
};

struct DecodeInitArgs {
    DecodeState st;
    const float* s_glo;     // [bkv, seq_len]
    const float* s_loc;
    const int32_t* kept_pos;
    const int32_t* tbm_idx;
    const int32_t* tbm_dest;
    const float* k_norm;
    const int32_t* slot_count;
    int bkv, head_dim, seq_len, window, budget, n_imp, n_tbm;
};

struct DecodeStepArgs {
    DecodeState st;
    const void* q_new;      // [bkv * group, D]
    const void* k_new;      // [bkv, D]
    const void* v_new;
    float* attn_opt;        // [bkv * group, T + 1] or null
    int32_t* decision_opt;  // [bkv, 2] or null
    float* sim_opt;         // [bkv] or null
    float* ws;              // [bkv, (group + 1) * budget] staging when it does not fit in LDS or between launches; or logits [bkv, group, T]
    size_t centre_at;       // behind the logits, in floats: what they leave of the centres' own elements
    float* hand;            // [bkv, kDecodeHandFloats] hand-over record of the sliced step, else null
    int slice_rows, n_slices;   // slices of the rows in the sliced step (decode_split); 0, 1 = one launch
    int tok_slice, n_tok_slices;    // slices of the token table; 0 = it is not cut
    int lds_floats;         // (group + 1) * budget when staged in LDS, else 0
    int lds_centres;        // n_imp when the entries' centre tokens fit behind them, else 0
    int bkv, group, head_dim, seq_len, window, budget, n_imp, n_tbm;
    int step;               // >= 0, or -1: read st.step_count
    float tau, scale_log2e;
};

struct StatsArgs {
    const float* s_glo;     // [bkv, seq_len]   (sparsity)
    const float* s_loc;
    float* p_out;           // [bkv]
    int32_t* n_k_opt;       // [bkv] or null
    const void* k;          // [bkv, seq_len, D] (redundancy)
    const void* v;
    float* r_out;           // [bkv]
    float* best;            // [bkv, seq_len]
    int bkv, head_dim, seq_len;
    int red_waves, red_len; // 16-bit redundancy: waves per head, stages per wave (set by the launcher; else 0)
    float zeta, tau;
};

// Strides (batch, head, token) in elements; *_wide: rows start at multiples of 16 bytes.
struct AppendArgs {
    const void* k;
    const void* v;
    const void* q;              // null: no queries
    void* q_out;
    long long k_sb, k_sh, k_sn, v_sb, v_sh, v_sn, q_sb, q_sh, q_sn, qo_sb, qo_sh, qo_sn, pos_sb, pos_sh, pos_sn;
    const int32_t* start;       // [batch]
    const int32_t* new_len;     // [batch] or null: all n_new
    const int32_t* positions;   // null: the slot
    const float* inv_freq;      // [rot / 2]
    int32_t* len_out;           // [batch] or null
    void* k_pages;              // [num_pages, kv_heads, page_size, D]
    void* v_pages;
    int32_t* pos_pages;         // [num_pages, kv_heads, page_size] or null
    uint8_t* k_scale;           // the same, of pages in 8 bits, or null
    uint8_t* v_scale;
    const int32_t* page_table;  // [batch, max_pages]
    int batch, n_new, kv_heads, group, page_size, num_pages, max_pages, rot;
    int tokens, heads;          // tokens and kv-heads of a block (set by the launcher)
    bool interleaved, k_wide, v_wide, q_wide, qo_wide;
};

// Rows of 8-bit pages back to 16 bits.
struct Read8Args {
    const void* k_pages;        // [num_pages, kv_heads, page_size, D]
    const void* v_pages;
    const uint8_t* k_scale;     // [num_pages, kv_heads, page_size]
    const uint8_t* v_scale;
    const int32_t* page_table;  // [batch, max_pages]
    const int32_t* lens;        // [batch]
    void* k_out;                // [batch, kv_heads, n_rows, D]
    void* v_out;
    long long ko_sb, ko_sh, ko_sn, vo_sb, vo_sh, vo_sn;
    int batch, kv_heads, n_rows, page_size, num_pages, max_pages;
    bool wide;
};

// Attention of one new token per sequence.  Rows are those of a paged cache (page_table), or of a compact cache whose
// table elements name them (tok_row; one element more is the new token itself).
struct AttendArgs {
    const void* q;              // [batch, kv_heads * group, D] with strides q_sb, q_sh in elements
    long long q_sb, q_sh;
    const void* k;              // first row of the cache
    const void* v;
    void* out;                  // [batch, kv_heads * group, D]
    float* lse;                 // [batch, kv_heads * group] or null
    const int32_t* page_table;  // [batch, max_pages]
    const int32_t* lens;        // [batch]
    const int32_t* pos_pages;   // [num_pages, kv_heads, page_size] or null; < 0: masked
    const uint8_t* k_scale;     // the same, of pages in 8 bits, or null
    const uint8_t* v_scale;
    int max_pages, page_size, num_pages;
    const int32_t* tok_row;     // [batch * kv_heads, n_tok]
    const float* tok_norm;
    const float* row_norm;      // [batch * kv_heads, budget]
    const void* k_new;          // [batch * kv_heads, D]
    const void* v_new;
    int n_tok, budget;
    const int32_t* new_len;     // several new tokens a sequence: [batch] how many, or null: all `tokens`
    long long q_sn, o_sb, o_sh, o_sn, l_sb, l_sh;      // strides of their queries, outputs and log-sum-exps
    bool many;                  // whether there may be several, with strides of their own
    int tokens, heads;          // at most; q-heads of one
    int batch, kv_heads, group, head_dim;      // group: q-heads of a kv-head, of all its new tokens
    int workers;                // per kv-head and tile of q-heads: they share its sequences evenly; 0 = a block per sequence
    bool q_wide;                // q rows start at multiples of 16 bytes
    float scale_log2e;
    unsigned page_magic;        // division by page_size (set by the launcher)
    int page_shift;
    int join_q;                 // q-heads of a join block (set by the launcher)
    float* part_o;              // [kv_heads * tiles, workers, 2, 16, D] what a worker found of a sequence it shares (workspace)
    float* part_ml;             // [.., 16, 2] its maximum and sum
};
// Attention of many queries per sequence, each over the rows up to its own: whole prompts (rows with strides), or new tokens
// over a paged cache (page_table).  Strides in elements.
struct PromptArgs {
    const void* q;              // [batch, Hq, q_rows, D], or with q_start [Hq, q_rows, D]
    const void* k;              // the same of k_rows; the first row of a paged cache
    const void* v;
    void* out;
    float* lse;                 // or null
    long long q_sb, q_sh, q_sn, k_sb, k_sh, k_sn, v_sb, v_sh, v_sn, o_sb, o_sh, o_sn, l_sb, l_sh;
    const int32_t* q_start;     // [batch + 1] first rows of packed sequences, or null
    const int32_t* k_start;
    int q_rows, k_rows;
    const int32_t* page_table;  // [batch, max_pages]
    const int32_t* lens;        // [batch]
    const int32_t* new_len;     // [batch] or null: all q_rows
    const int32_t* pos_pages;   // [num_pages, kv_heads, page_size] or null; < 0: masked
    int max_pages, page_size, num_pages;
    int batch, kv_heads, group;
    long long q_tokens;         // of all sequences
    bool q_wide;                // rows start at multiples of 16 bytes
    bool kv_wide, o_wide;
    float scale_log2e;
    unsigned page_magic;        // division by page_size (set by the launcher)
    int page_shift;
    int splits;                 // blocks that share a tile's rows of keys and values
    float* part_o;              // [q_tokens, Hq, splits, D] what a block found of a tile that it shares (workspace)
    float* part_ml;             // [.., 2] its maximum and sum
};
struct PromptPlan { int waves, splits; long long tiles; };      // of a block; of a tile's rows; tiles of a kv-head at most
// `sequences` of at most `rows` query rows (tokens x q-heads of a group) each and `all_rows` together, over at most `most` rows
PromptPlan plan_prompt(long long sequences, long long rows, long long all_rows, int kv_heads, int group, int head_dim, long long most, bool paged, bool f32);
hipError_t launch_prompt(const PromptArgs& a, const PromptPlan& plan, int head_dim, bool f32, hipStream_t st);
constexpr int kAttendQ = 16;    // q-heads of a group that a block takes: the columns of a matrix product
constexpr int kAttendUnit = 128;        // rows that work is counted in
int attend_workers(int batch, int kv_heads, int group, long long max_len, int row_bytes);      // AttendArgs::workers
int append_tokens(int rows, int row_bytes);    // tokens of a block where there are many, `rows` (queries, keys, values) each
hipError_t launch_append(const AppendArgs& a, int head_dim, bool f32, hipStream_t st);
constexpr int kRead8Rows = 64;         // rows of a block
hipError_t launch_read8(const Read8Args& a, int head_dim, hipStream_t st);
hipError_t launch_attend(const AttendArgs& a, bool f32, hipStream_t st);

int score_keys_per_block(int dtype_is_f32);
// How the score passes of a launch are dealt: waves per head and stages per wave of each pass (0 waves:
// the pass takes whole items), and the floats of one partial-result array.
struct ScoreDeal { int p1_waves, p1_len, p2_waves, p2_len, p1_by_block; size_t p1_floats, p2_floats; };
ScoreDeal score_deal(int batch, int q_heads, int kv_heads, int seq_len, int head_dim, bool f32);
bool score_by_16x16x32(int batch, int q_heads, int kv_heads, int seq_len, int head_dim);       // which products 16-bit passes take
int select_chunks(int seq_len);     // blocks per head of the long-sequence select
int select_coarse_bins();
hipError_t launch_sparsity(const StatsArgs& a, hipStream_t st);
hipError_t launch_redundancy(const StatsArgs& a, bool f32, hipStream_t st);
hipError_t launch_decode_init(const DecodeInitArgs& a, bool f32, hipStream_t st);
hipError_t launch_decode_step(const DecodeStepArgs& a, bool f32, hipStream_t st);
constexpr int kDecodeMaxSlices = 32;     // slices per head of the sliced decode step
constexpr int kDecodeHandFloats = 1024;  // floats of its per-head hand-over record
struct DecodeSlices { int rows, n_rows, toks, n_toks; };   // rows and table elements per slice, slices; toks = 0: the table is not cut
bool decode_split(int heads, int budget, int n_imp, int n_tbm, int window, bool f32, DecodeSlices* s);
int decode_launches(int heads, int group, int budget, int n_imp, int n_tbm, int window, bool f32);       // of a step whose number comes with the call
hipError_t launch_expand(const ExpandArgs& a, bool f32, hipStream_t st);
hipError_t launch_score_pass1(ScoreArgs& a, bool f32, hipStream_t st);   // rows' log-sum-exp; sets a.queue_clear
hipError_t launch_score_pass2(const ScoreArgs& a, bool f32, hipStream_t st);   // column sums
hipError_t launch_select(const SelectArgs& a, hipStream_t st);
hipError_t launch_evict_merge(const MergeArgs& a, bool f32, hipStream_t st);
int dest_max_slices(int n_imp, int n_tbm, int bkv, bool f32);

}  // namespace ems
