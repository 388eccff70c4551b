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
};
struct Kv8RowArgs {         // the rows to append; strides in elements
    const void *k, *v, *q;
    int64_t k_row, k_head, v_row, v_head, q_row, q_head;
    int hq;
    const float* rope;      // [rope_rows][hd / 2][2] or null
    int rope_rows;
    __nv_bfloat16* q_out;
    int64_t q_out_row, q_out_head;
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
};

constexpr int kKv8MaxGroup = 64;    // query heads a KV head
cudaError_t launch_kv8_append(int dtype, const Kv8Args& a, const Kv8RowArgs& r, cudaStream_t s);
size_t kv8_attention_workspace(int hd, int group, int n_rows);
bool kv8_attention_fits(const Kv8Args& a, int hq);     // false: too many units and tiles for one call
// A call is two launches: the units' runs, and directly behind it the merge of units that lie in several, if the
// first says that there can be any (merge; not where sequences are at most a tile long).
cudaError_t launch_kv8_attention(const Kv8Args& a, const Kv8AttnArgs& t, cudaStream_t s, bool& merge);
cudaError_t launch_kv8_merge(const Kv8Args& a, const Kv8AttnArgs& t, cudaStream_t s);
// Map of the 8-bit cache's records (gemv.cu): boxes of box_records records' keys, or values.
bool make_kv8_map(CUtensorMap* map, const void* base, uint64_t records, uint32_t hd, uint32_t box_records);

}  // namespace ks
