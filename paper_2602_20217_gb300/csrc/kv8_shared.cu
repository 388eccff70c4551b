// Causal attention over the 8-bit paged cache for groups of sequences with a
// common beginning, which is read once for all of a group's rows.
//
// softmax over a sequence's keys, in two parts: with m_i, l_i, o_i the maximum,
// sum and weighted values of part i, o = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i -
// m) l_i.  The first launch attends from all rows of a group to what it has in
// common (no mask: every row sees all of it) and leaves normalised outputs in
// fp32 and the sums' logarithms; the second attends from each sequence's rows to
// what the sequence has by itself and takes the first part in where a row's
// output is finished.  Both are the kernels of kv8_attn.cu and kv8_tc.cu, each
// cut by its own mean rows: a group's rows fill units of 128 where a sequence's
// alone would be units of 8.  Joining in the second launch's ends saves a third one
// over all rows, and a pass over them.
//
// Measured, 64 samples of one row behind 16384 tokens, 32 heads over 8: 72 us of
// which the first launch is 40, the second 25, finding out what is shared 5; the
// cache's bytes alone would be 11 us.  The first is bound as prompts are (see
// kv8_tc.cu), the second by its units' ends: a unit has two or three tiles.  The
// plain attention of the same batch takes 275 us.  Of little that is shared it is
// faster, one launch or two against five: 4 samples behind 4096 tokens 13 us, 23 here;
// a row each, the two meet at about 32 sequences behind 4096 tokens (37 us here, 45
// there), 16 behind 8192 (35, 43), 8 behind 16384 (39, 41).
#include <algorithm>

#include "kv8_plan.cuh"

namespace ks {

namespace {

constexpr int kThreads = 1024, kNearGroups = 4096;

struct SharedPlan {             // in the workspace
    int64_t *first_common, *first_tail;     // where the pages begin in the table: groups, sequences
    int32_t *row_common, *len_common;       // [n_groups + 1], [n_groups]
    int32_t *len_tail, *cut;                // [n_seqs]
    float *lse, *out;                       // [n_rows][hq], [n_rows][hq][hd]
    void* work;                             // of the two attention launches
    size_t bytes;
};
SharedPlan shared_plan(int hd, int hk, int hq, int64_t n_seqs, int64_t n_rows, int64_t n_groups, void* at) {
    SharedPlan p{};
    char* base = static_cast<char*>(at);
    auto take = [&](size_t bytes) {
        char* r = base + p.bytes;
        p.bytes += (bytes + 255) / 256 * 256;
        return static_cast<void*>(r);
    };
    p.first_common = static_cast<int64_t*>(take(sizeof(int64_t) * n_groups));
    p.first_tail = static_cast<int64_t*>(take(sizeof(int64_t) * n_seqs));
    p.row_common = static_cast<int32_t*>(take(sizeof(int32_t) * (n_groups + 1)));
    p.len_common = static_cast<int32_t*>(take(sizeof(int32_t) * n_groups));
    p.len_tail = static_cast<int32_t*>(take(sizeof(int32_t) * n_seqs));
    p.cut = static_cast<int32_t*>(take(sizeof(int32_t) * n_seqs));
    p.lse = static_cast<float*>(take(sizeof(float) * n_rows * hq));
    p.out = static_cast<float*>(take(sizeof(float) * n_rows * hq * hd));
    p.work = take(kv8_attention_workspace(hd, hq / hk, (int)n_rows));
    return p;
}

// What the groups have in common: whole pages, as many as the caller says, and no
// token that is one of the batch's rows, so that no mask is needed there.  One
// CTA: the least over a group's sequences is an order-free minimum.  Groups that
// are no cut of the sequences, and offsets that decrease, share nothing.
__global__ void __launch_bounds__(kThreads) shared_prepare_kernel(const Kv8Args a, const Kv8SharedArgs g, const SharedPlan p) {
    __shared__ int32_t near[kNearGroups];
    const int tid = threadIdx.x, page = a.bpp * kKv8Block;
    int32_t* len = g.n_groups <= kNearGroups ? near : p.len_common;
    grid_dependency_wait();
    grid_launch_dependents();
    bool cuts = true, falls = false, bad = false;
    for (int i = tid; i <= g.n_groups; i += kThreads) {
        const int at = g.groups[i];
        cuts = cuts && at >= 0 && at <= a.n_seqs && (i == 0 || at >= g.groups[i - 1]);
    }
    for (int s = tid; s < a.n_seqs; s += kThreads) {
        falls = falls || a.offsets[s + 1] < a.offsets[s];
        bad = bad || a.lengths[s] < 0 || a.lengths[s] > a.capacity;
    }
    cuts = __syncthreads_and(cuts);
    falls = __syncthreads_or(falls);
    const bool share = cuts && !falls;
    for (int i = tid; i <= g.n_groups; i += kThreads) {
        p.row_common[i] = share ? min(max(a.offsets[g.groups[i]], 0), a.n_rows) : 0;
        if (i == g.n_groups) continue;
        const int n = g.tokens[i];
        bad = bad || n < 0 || n > a.capacity;
        len[i] = share ? min(max(n, 0), a.capacity) / page * page : 0;
        p.first_common[i] = share ? (int64_t)g.groups[i] * a.table_ld : 0;
    }
    if (bad || !cuts) kv8_flag(a, kKv8BadBatch);
    __syncthreads();
    // the last group that begins at or before s, if s is in it
    auto group_of = [&](int s) {
        int lo = 0, hi = g.n_groups;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (g.groups[mid] <= s) lo = mid;
            else hi = mid;
        }
        return g.groups[lo] <= s && s < g.groups[lo + 1] ? lo : -1;
    };
    if (share)
        for (int s = tid; s < a.n_seqs; s += kThreads) {
            const Kv8Seq q = kv8_seq(a, s);
            const int at = q.rows > 0 ? group_of(s) : -1;
            if (at >= 0) atomicMin(&len[at], max(q.len - q.rows, 0) / page * page);
        }
    __syncthreads();
    auto common = [&](int i) { return len == near ? near[i] : __ldcg(len + i); };
    for (int s = tid; s < a.n_seqs; s += kThreads) {
        const Kv8Seq q = kv8_seq(a, s);
        const int at = share ? group_of(s) : -1, cut = at >= 0 && q.rows > 0 ? common(at) : 0;
        p.cut[s] = cut;
        p.len_tail[s] = q.len - cut;
        p.first_tail[s] = (int64_t)s * a.table_ld + cut / page;
    }
    if (len == near)
        for (int i = tid; i < g.n_groups; i += kThreads) p.len_common[i] = near[i];
}

}  // namespace

size_t kv8_shared_workspace(int hd, int hk, int hq, int n_seqs, int n_rows, int n_groups) {
    return shared_plan(hd, hk, hq, n_seqs, n_rows, n_groups, nullptr).bytes;
}

bool kv8_shared_fits(const Kv8Args& a, const Kv8SharedArgs& g, int hq) {
    Kv8Args c = a;
    c.n_seqs = g.n_groups;
    return kv8_attention_fits(a, hq, kTail) && kv8_attention_fits(c, hq, kCommon);
}

cudaError_t launch_kv8_shared(const Kv8Args& a, const Kv8SharedArgs& g, const Kv8AttnArgs& t, cudaStream_t s) {
    const SharedPlan p = shared_plan(a.hd, a.hk, t.hq, a.n_seqs, a.n_rows, g.n_groups, t.workspace);
    cudaError_t e = launch_kv8(shared_prepare_kernel, dim3(1), kThreads, 0, s, a, g, p);
    if (e != cudaSuccess) return e;
    Kv8AttnArgs u = t;
    u.workspace = p.work;
    u.common_out = p.out;
    u.common_lse = p.lse;
    u.cut = p.cut;
    Kv8Args c = a;
    c.offsets = p.row_common;
    c.lengths = p.len_common;
    c.n_seqs = g.n_groups;
    c.first_page = p.first_common;
    bool merge;
    e = launch_kv8_attention(c, u, s, merge, kCommon);
    if (e == cudaSuccess && merge) e = launch_kv8_merge(c, u, s, kCommon);
    if (e != cudaSuccess) return e;
    c = a;
    c.lengths = p.len_tail;
    c.first_page = p.first_tail;
    e = launch_kv8_attention(c, u, s, merge, kTail);
    if (e == cudaSuccess && merge) e = launch_kv8_merge(c, u, s, kTail);
    return e;
}

}  // namespace ks
