// Host-side internals of libhata: the context and the per-stage launchers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/hata.h"

// Words between the arrival counters of consecutive units (128 bytes:
// the workgroups of different units then never queue their arrivals on one cache line).
#define HATA_COUNTER_STRIDE 32
// score values of the largest group and code: G * r + 1
#define HATA_MAX_NB 4097
// dense attention: at most this many rounds of one workgroup per CU, with a partial result each
#define HATA_DENSE_ROUNDS 4

namespace hata {
// Of a sequence in a call with groups that share rows: its rows behind the shared ones, in `runs` runs a KV head for a team each (teams
// start .. start + runs * Hkv - 1 of the launch), and the partial results of the shared rows: `splits` a KV head from item on, `step`
// apart, its query rows from `row` on
struct PrefixPlan {
    int start, runs, rows, first, item, splits, row, step;
};
}  // namespace hata

struct hata_ctx {
    hata_config cfg;
    int G;            // query heads per KV head
    int Wd;           // 32-bit words per code
    int NB;           // number of score values: G*r + 1
    int NBP;          // NB rounded up to a multiple of 8 (row pitch of the chunk histograms)
    int chunk;        // cached keys handled by one scoring / selection workgroup
    int n_chunks;     // ceil(L_cap / chunk)
    int HT;           // query heads of a group handled together by one attention workgroup
    // keys per workgroup the single-launch step may use (ascending; [0] = chunk unless the caller fixed
    // another size) and how many of its workgroups are resident at once with each (0 = unusable); a
    // call takes the size that needs the fewest launches for its batch, the smallest such
    int coop_opts, coop_opt_chunk[4], coop_opt_cap[4];
    int sparse_rows;  // selected rows per attention workgroup
    int sparse_splits;
    int64_t dense_wgs_max;  // dense attention: workgroups of a launch that the partials have room for
    // regions of the caller's workspace
    uint32_t* qcodes;      // [B_max, Hq, Wd]
    uint16_t* scores;      // [B_max, Hkv, L_cap]
    int32_t* idx;          // [B_max, Hkv, k_max]
    uint16_t* chunk_hist;  // [B_max*Hkv, n_chunks, NBP] histograms of the chunks (top-k), cumulative ones (step without waits)
    int32_t* chunk_info;   // [B_max*Hkv, n_chunks + 1, 2] = {output offset, ties taken} (top-k); estimates of the threshold [B_max*Hkv, n_chunks] (step without waits)
    int32_t* unit_info;    // [B_max*Hkv, 2] = {threshold, selected count}
    uint32_t* unit_counter;  // [B_max*Hkv, HATA_COUNTER_STRIDE] scored chunks of a unit (self-resetting)
    uint32_t* unit_hist;     // [B_max*Hkv, NB] total histogram of a unit (self-clearing)
    uint32_t* attn_counter;  // [B_max*Hq (cooperative step: per unit), attn_counter_stride] finished attention slices (self-resetting)
    int attn_counter_stride; // HATA_COUNTER_STRIDE; 1 in the static scratch of hata_sparse_decode_static
    unsigned long long* coop_cum;  // [B_max*Hkv, coop_cum_pitch()] cumulative chunk histograms, two scores and the unit's launch a word, and marks (cooperative step)
    uint32_t* unit_epoch;          // [B_max*Hkv, HATA_COUNTER_STRIDE] launches of the cooperative step on a unit, and whether chunk 0 gave the last one up
    unsigned long long* coop_qrec; // [B_max*Hkv, n_chunks, G*Wd] query code words, one copy per chunk, stamped with the unit's launch (cooperative step)
    uint32_t* plan_counter;  // [1 + groups of workgroups, HATA_COUNTER_STRIDE] finished ones of a page plan (self-resetting)
    uint32_t* error_word;    // [1] set by a cooperative launch that gave up waiting
    int spin_limit;          // polls an in-kernel wait makes before it gives up (0 = the default)
    int keep_scores;         // single-launch step also writes the score array
    int par_merge;           // single-launch step merges the heads of a unit in several workgroups
    int step_mode;           // 0 = single launch when it fits, 3 = always the form without waits
    int unit_keys;           // keys a workgroup per unit handles (0: that form is not available, or the caller asked for a launch shape)
    int shared;              // hata_tuning.shared_device
    int mode_asked;          // step_mode was set by the caller (and is not just that of a shared device)
    int cus;                 // compute units of the device that was current in hata_create
    int coop_opt_cap_paged[4];  // the same for the block-table variant of the kernel
    float* partials;       // [B_max*Hq, max(sparse_splits, n_chunks), d + 2], at least 256 * HATA_DENSE_ROUNDS * G rows
    float* prefix_part;    // partial results of rows that groups of sequences share (prefix_part_floats)
    hata::PrefixPlan* prefix_plan;  // [B_max] what is left to the sequences themselves, and where they find their own among those
    void* wplanes;               // [Hkv, r/32, 8, 2, 64] 16-byte fragments: the two scaled fp16 planes of the hash weights (prefill key encode)
    const float* prepared_W_H;   // the weight tensor those planes were made from (nullptr: none)
    size_t control_bytes;  // bytes from chunk_info up to the partials: the control words, cleared at creation and after a give-up
};

namespace hata {

// Block table of a paged cache (table == nullptr: the contiguous layout).  Page p of the pools
// holds 1 << shift rows of every KV head -- K, V [n_pages, Hkv, page_rows, d], codes [n_pages,
// Hkv, page_rows, Wd] -- and row n of sequence b lives in page table[b * max_blocks + (n >> shift)]
// at row n & (page_rows - 1).  Device code clamps the page numbers it reads to [0, n_pages).
struct PageView {
    const int32_t* table;
    int max_blocks, shift, n_pages;
};

// every launcher returns hipGetLastError() of its launches
hipError_t launch_encode_vectors(const hata_ctx* c, const void* q, uint32_t* qcodes,
                                 const void* K, const int32_t* start, const int32_t* n_new,
                                 int max_new, int from_seq_len, uint32_t* codes,
                                 const float* W_H, int B, hipStream_t s);
// K_new .. V_out non-null: fused cache fill (rows read from K_new / V_new [B, Hkv, max_new, d],
// written to the caches K_out / V_out while the key codes are computed)
hipError_t launch_encode_bulk(const hata_ctx* c, const void* K, const float* W_H,
                              const int32_t* start, const int32_t* n_new, int B, int max_new,
                              uint32_t* codes, hipStream_t s, const void* K_new = nullptr,
                              const void* V_new = nullptr, void* K_out = nullptr, void* V_out = nullptr,
                              const PageView* pages = nullptr);
hipError_t launch_split_weights(const hata_ctx* c, const float* W_H, hipStream_t s);
hipError_t launch_score(const hata_ctx* c, const uint32_t* qcodes, const uint32_t* codes, const int32_t* seq_len, int B,
                        uint16_t* scores, hipStream_t s);
hipError_t launch_score_select(const hata_ctx* c, const uint32_t* codes, const int32_t* seq_len, const int32_t* k, int B, hipStream_t s);
hipError_t launch_encode_score(const hata_ctx* c, const void* q, const void* K, const float* W_H, uint32_t* codes, int append,
                               const int32_t* seq_len, const int32_t* k, int B, hipStream_t s);
hipError_t prepare_dense();  // once per context
hipError_t launch_dense(const hata_ctx* c, const void* q, const void* K, const void* V, const int32_t* seq_len, int B,
                        float sm_scale, void* out, float* out_f32, hipStream_t s, const PageView* pages = nullptr, int pre_rows = 0);
// Rows that groups of sequences share, in front of launch_dense of the same call: partial results in prefix_part, *part_rows (which
// launch_dense is then given as pre_rows) query rows each, and prefix_plan
#define HATA_PREFIX_GROUPS 1024  // groups beyond share nothing, and neither do batches of more sequences (what a workgroup has LDS for)
#define HATA_PREFIX_MAX_B 16384
size_t prefix_part_floats(int B, int Hkv, int G);
int dense_own_wgs(int B, int Hkv, bool spare);  // workgroups of the launch behind, and waves of its teams
int dense_own_team(int B, int Hkv);
hipError_t prepare_prefix();  // once per context
hipError_t launch_prefix(const hata_ctx* c, const void* q, const void* K, const void* V, const PageView& pages, const int32_t* seq_len, int B,
                         const int32_t* group_start, const int32_t* shared_len, int n_groups, float sm_scale, int* part_rows, hipStream_t s);
// What hata_plan_pages is given, and the L_cap of its context
struct PagePlan {
    const int32_t *len_now, *len_next, *fork_from, *shared_blocks, *n_free;
    int32_t *table, *free_pages, *n_free_out, *seq_len, *token_start, *slots, *positions;
    int B, max_blocks, shift, n_pages, max_tokens, cap;
};
#define HATA_PLAN_MAX_B 8191  // sequences of a page plan (their sums lie in LDS)
#define HATA_PLAN_WGS 512     // workgroups of a plan at most, and of a group that arrives together
#define HATA_PLAN_GROUP 32
hipError_t prepare_pages();   // once per context
hipError_t launch_plan_pages(const hata_ctx* c, const PagePlan& p, hipStream_t s);
hipError_t launch_write_slots(const hata_ctx* c, const void* K_new, const void* V_new, int64_t stride_t, int64_t stride_h,
                              const int32_t* slots, int n_tokens, void* K_pool, void* V_pool, uint32_t* codes, int shift, int n_pages,
                              const float* W_H, hipStream_t s);
// Packed rows to rotate: `heads` heads into `out`, and with Hkv > 0 keys (rotated) and values (not) into the slots of the pools
struct RotateRows {
    const uint16_t* x;
    uint16_t* out;
    const uint16_t *K_new, *V_new;
    uint16_t *K, *V;
    const int32_t *positions, *slots;
    const double* freq;
    int64_t st, sh, out_st, out_sh, kv_st, kv_sh;  // strides in elements
    double magnitude;
    int n, heads, Hkv, dims, interleaved, back, shift, rows, per;  // rows: of one head in the pools; per: heads of a wave
};
hipError_t launch_rotate(const RotateRows& a, hipStream_t s);
hipError_t launch_rotate_write(const hata_ctx* c, const RotateRows& rows, uint32_t* codes, const float* W_H, hipStream_t s);
int rotary_frequencies(int pairs, double base, const hata_rotary_scaling* sc, double* freq, float* magnitude);
// Drafted tokens of B sequences over their pages
#define HATA_TREE_MAX_DRAFT 256
struct TreeSplit { int last, rows, first, h; };  // a unit that workgroup i begins and workgroup `last` ends (-1: none), its query rows, first token, KV head
struct TreeArgs {
    const uint16_t *q, *K, *V;
    const int32_t *base, *seq_len, *token_start;
    const uint32_t* mask;  // [n_tokens, words], or nullptr: a token sees those before it and itself
    uint16_t* out;
    float* out_f32;
    PageView pv;
    int B, Hq, Hkv, G, L_cap, n_tokens, max_draft, words;
    float scale_log2;
    // in the caller's scratch
    TreeSplit* splits;
    float* part;
    int part_rows;
};
size_t tree_scratch_bytes(int G, int max_draft);
hipError_t prepare_tree();  // once per context
hipError_t launch_tree(const TreeArgs& a, void* scratch, hipStream_t s);
struct KeepRows {
    uint16_t *K, *V;
    uint32_t* codes;
    const int32_t *base, *seq_len, *path, *n_path;
    int32_t* seq_len_out;
    PageView pv;
    int Hkv, Wd, L_cap, max_path, heads;  // heads: of a workgroup
};
hipError_t launch_keep_rows(const KeepRows& a, int B, hipStream_t s);
hipError_t prepare_topk();   // once per context
hipError_t prepare_attention(const hata_ctx* c);  // once per context
hipError_t launch_topk(const hata_ctx* c, const uint16_t* scores, const int32_t* seq_len,
                       const int32_t* k, int B, int32_t* idx, hipStream_t s);
// mode: 0 = rows from idx, 2 = select on the fly (writes idx)
hipError_t launch_attention(const hata_ctx* c, int mode, const void* q, const void* K,
                            const void* V, int32_t* idx, const int32_t* count_src,
                            const int32_t* seq_len, int B, float sm_scale, void* out,
                            float* out_f32, hipStream_t s);

hipError_t launch_gather_rows(const hata_ctx* c, const void* K, const void* V, const int32_t* idx,
                              const int32_t* k, int B, int max_workgroups, void* K_stage, void* V_stage,
                              hipStream_t s);

// encode + score + select + attend in one cooperative launch; returns hipErrorNotSupported if
// this shape has no cooperative kernel
hipError_t launch_coop_step(const hata_ctx* c, const void* q, const void* K, const void* V,
                            const float* W_H, uint32_t* codes, int append, const int32_t* seq_len,
                            const int32_t* k, int B, float sm_scale, void* out, float* out_f32, hipStream_t s,
                            int chunk, const PageView* pages = nullptr, int b0 = 0, int32_t* idx_only = nullptr);
// (chunk: keys per workgroup, one of the context's coop_opt_chunk; idx_only != nullptr: the launch
// stops once the index lists are written, into idx_only [B, Hkv, k_max] instead of the workspace;
// V, out and out_f32 are not touched)
// The single-launch step runs with at most HATA_COOP_CHUNKS chunks per unit, whatever the plan's chunk (on which the other kernels have
// up to 1024): marks of one reading chunk (whole cache lines), and 64-bit words of a unit's whole part of coop_cum: the chunks' rows,
// then the marks
#define HATA_COOP_CHUNKS 256
inline int coop_rows(int n_chunks) { return n_chunks < HATA_COOP_CHUNKS ? n_chunks : HATA_COOP_CHUNKS; }
inline int coop_mark_pitch(int n_chunks) { return (coop_rows(n_chunks) + 31) / 32 * 32; }
inline int coop_cum_pitch(int n_chunks, int NBP) { return coop_rows(n_chunks) * (NBP / 2 + coop_mark_pitch(n_chunks) / 2); }
// the step with a workgroup per (sequence, KV head) unit: caches of up to HATA_UNIT_KEYS_LONG rows, of up to HATA_UNIT_KEYS by
// a form of its own
#define HATA_UNIT_KEYS 4096
#define HATA_UNIT_KEYS_LONG 16384
hipError_t prepare_unit_step(hata_ctx* c);  // once per context
hipError_t launch_unit_step(const hata_ctx* c, const void* q, const void* K, const void* V, const float* W_H, uint32_t* codes,
                            int append, const int32_t* seq_len, const int32_t* k, int B, float sm_scale, void* out,
                            float* out_f32, hipStream_t s, const PageView* pages = nullptr);
int coop_capacity(const hata_ctx* c, bool paged, int chunk);

}  // namespace hata
