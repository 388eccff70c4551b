// Host interface of the 8-bit paged cache's kernels (kv8.cu, kv8_attn.cu,
// kv8_tc.cu): arguments and launches.
#pragma once

#include "internal.h"

namespace ks {

struct Kv8Args {            // cache and batch
    unsigned char* data;    // [n_pages][hk][bpp] records of kv8_record(hd) bytes
    int n_pages, bpp, hk, hd;
    const int32_t* table;   // [n_seqs][table_ld] pages
    const int32_t* offsets; // [n_seqs + 1] first row of each sequence
    const int32_t* lengths; // [n_seqs] tokens, the rows among them
    int n_seqs, table_ld, n_rows;
    int capacity;           // tokens that a sequence's pages can hold
    int* status;            // or null
    bool by_seq;            // append, read: how the grid counts blocks (set by the launch)
    const int* stop;        // draft passes: the launch does nothing when *stop != 0 (null: always runs)
    const int64_t* first_page;  // attention in two parts: where in the table a sequence's pages begin
};
struct Kv8RowArgs {         // the rows to append; strides in elements
    const void *k, *v, *q;
    int64_t k_row, k_head, v_row, v_head, q_row, q_head;
    int hq;
    const float* rope;      // [rope_rows][hd / 2][2] or null
    int rope_rows;
    __nv_bfloat16* q_out;
    int64_t q_out_row, q_out_head;
    const int32_t* shift;   // [n_seqs] what a token's position is ahead of its place in the cache, or null
};
struct Kv8AttnArgs {
    const __nv_bfloat16* q;
    int64_t q_row, q_head;
    __nv_bfloat16* out;
    int64_t out_row, out_head;
    float* lse;             // [n_rows][hq] or null
    int hq;
    float scale;
    void* workspace;
    // attention in two parts: what the rows' groups have in common gives normalised outputs and sums' logarithms to
    // base 2, which the rows of sequences with cut[s] > 0 take in
    float* common_out;      // [n_rows][hq][hd]
    float* common_lse;      // [n_rows][hq]
    const int32_t* cut;     // [n_seqs]
};
// Which part of the keys a launch attends to: all of a sequence's, those that a group of sequences has in common (its
// "sequences" are the groups, whose rows all see all of them), or what a sequence has behind these.
enum Kv8Part { kWhole = 0, kCommon = 1, kTail = 2 };
bool kv8_attention_fits(const Kv8Args& a, int hq, Kv8Part part = kWhole);      // false: too many units and tiles for one call
struct Kv8SharedArgs {      // groups of sequences with a common beginning
    const int32_t* groups;  // [n_groups + 1] first sequence of each
    const int32_t* tokens;  // [n_groups] common tokens
    int n_groups;
};

constexpr int kKv8MaxGroup = 64;    // query heads a KV head
cudaError_t launch_kv8_append(int dtype, const Kv8Args& a, const Kv8RowArgs& r, cudaStream_t s);
size_t kv8_attention_workspace(int hd, int group, int n_rows);
// A call is two launches: the units' runs, and directly behind it the merge of units that lie in several, if the
// first says that there can be any (merge; not where sequences are at most a tile long).
cudaError_t launch_kv8_attention(const Kv8Args& a, const Kv8AttnArgs& t, cudaStream_t s, bool& merge,
                                 Kv8Part part = kWhole);
cudaError_t launch_kv8_merge(const Kv8Args& a, const Kv8AttnArgs& t, cudaStream_t s, Kv8Part part = kWhole);
// Attention of groups with a common beginning (kv8_shared.cu); t.workspace has room for both parts.
size_t kv8_shared_workspace(int hd, int hk, int hq, int n_seqs, int n_rows, int n_groups);
bool kv8_shared_fits(const Kv8Args& a, const Kv8SharedArgs& g, int hq);
cudaError_t launch_kv8_shared(const Kv8Args& a, const Kv8SharedArgs& g, const Kv8AttnArgs& t, cudaStream_t s);
struct Kv8WeightArgs {      // the weight that tokens receive; scores, out: [n_seqs][hk][ld]
    const __nv_bfloat16* q;
    int64_t q_row, q_head;
    int hq;
    float scale, decay;
    const float* lse;       // [n_rows][hq]
    const float* scores;
    float* out;
    int64_t ld;
    void* workspace;        // kv8_weights_workspace() bytes
};
bool kv8_weights_fits(const Kv8Args& a, int hq);
size_t kv8_weights_workspace(int group, int64_t n_rows, int64_t n_seqs);
size_t kv8_weights_tc_workspace();
// Many query rows a sequence (kv8_weights_tc.cu); taken: false where the queries are no operand of tensor copies.
cudaError_t launch_kv8_weights_tc(const Kv8Args& a, const Kv8WeightArgs& t, cudaStream_t s, bool& taken);
// Map of rows of queries: boxes of 64 dims x box_heads heads x box_rows rows with the 128-byte swizzle (gemv.cu).
bool make_kv8_query_map(CUtensorMap* map, const void* q, uint64_t n_rows, uint32_t hq, uint32_t hd, int64_t row, int64_t head,
                        uint32_t box_heads, uint32_t box_rows);
cudaError_t launch_kv8_weights(const Kv8Args& a, const Kv8WeightArgs& t, cudaStream_t s);
struct Kv8EvictArgs {       // eviction into the pages of new_table
    const float* scores;    // [n_seqs][hk][ld]
    int64_t ld;
    const int32_t* keep;    // [n_seqs]
    int first, recent;
    const int32_t* new_table;   // [n_seqs][new_table_ld]
    int new_table_ld, new_capacity;
    int32_t* new_lengths;   // [n_seqs]
    int32_t* kept;          // [n_seqs][hk][kept_ld]
    int64_t kept_ld;
    float* new_scores;      // [n_seqs][hk][new_ld] or null
    int64_t new_ld;
};
cudaError_t launch_kv8_evict(const Kv8Args& a, const Kv8EvictArgs& t, cudaStream_t s);
// Map of the 8-bit cache's records (gemv.cu): boxes of box_records records' keys, or values.
bool make_kv8_map(CUtensorMap* map, const void* base, uint64_t records, uint32_t hd, uint32_t box_records);

}  // namespace ks
