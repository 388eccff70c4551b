// Causal attention over the 8-bit paged cache.
#include "kv8.cuh"

namespace ks {

namespace {

constexpr int kThreads = 128;

// One CTA per (row, query head): 128 keys at a time, a key per thread for the
// scores and a dim per thread for the values, with the running maximum and sum
// of a softmax.
template <int HD>
__global__ void __launch_bounds__(kThreads) kv8_attention_kernel(const Kv8Args a, const Kv8AttnArgs t) {
    constexpr int REC = kv8_record(HD), CODES = kKv8Block * HD;
    if (a.stop && *a.stop) return;
    const int row = blockIdx.x, h = blockIdx.y, tid = threadIdx.x, G = t.hq / a.hk;
    __shared__ float q[HD], p[kThreads], scratch[kThreads / 32 + 1];
    if (row == 0 && h == 0)
        for (int i = tid; i < a.n_seqs; i += kThreads)
            if (kv8_seq_bad(a, i)) kv8_flag(a, kKv8BadBatch);
    if (row >= kv8_row0(a, a.n_seqs)) return;
    const int s = kv8_find(a.n_seqs, row, [&](int i) { return kv8_row0(a, i); });
    const Kv8Seq seq = kv8_seq(a, s);
    if (row < seq.row0 || row >= seq.row0 + seq.rows) return;
    const int keys = seq.len - seq.rows + (row - seq.row0) + 1;     // keys the row sees
    if (tid < HD) q[tid] = __bfloat162float(t.q[row * t.q_row + h * t.q_head + tid]);
    __syncthreads();
    float m = -INFINITY, l = 0.f, o = 0.f;
    for (int j0 = 0; j0 < keys; j0 += kThreads) {
        const int j = j0 + tid;
        float sc = -INFINITY;
        const unsigned char* rec = j < keys ? kv8_record_at(a, s, j / kKv8Block, h / G, REC) : nullptr;
        if (j < keys && !rec) kv8_flag(a, kKv8BadPage);
        if (rec) {
            float x = 0.f;
            for (int d = 0; d < HD; d += 2) {
                const float2 c = from_e4m3x2(*reinterpret_cast<const uint16_t*>(rec + k_byte<HD>(j % kKv8Block, d)));
                x = fmaf(c.x, q[d], x);
                x = fmaf(c.y, q[d + 1], x);
            }
            sc = x * *reinterpret_cast<const float*>(rec + 2 * CODES) * t.scale;
        }
        __syncthreads();
        p[tid] = sc;
        __syncthreads();
        float top = m;
        for (int i = 0; i < kThreads; ++i) top = fmaxf(top, p[i]);
        const float base = top == -INFINITY ? 0.f : top, f = expf(m - base);
        const float e = rec ? expf(sc - base) : 0.f;
        l = l * f + block_sum<kThreads / 32>(e, scratch);
        o *= f;
        m = top;
        p[tid] = e;
        __syncthreads();
        if (tid < HD)
            for (int i = 0; i < kThreads && j0 + i < keys; ++i) {
                const unsigned char* r = kv8_record_at(a, s, (j0 + i) / kKv8Block, h / G, REC);
                if (!r) continue;
                const float2 c = from_e4m3x2(r[CODES + tid * 16 + v_byte((j0 + i) % kKv8Block)]);
                o = fmaf(p[i] * *reinterpret_cast<const float*>(r + 2 * CODES + 4), c.x, o);
            }
    }
    if (tid < HD) t.out[row * t.out_row + h * t.out_head + tid] = __float2bfloat16_rn(l == 0.f ? 0.f : o / l);
    if (t.lse && tid == 0) t.lse[(size_t)row * t.hq + h] = l == 0.f ? -INFINITY : m + logf(l);
}

}  // namespace

size_t kv8_attention_workspace(int, int, int, int, int) { return 256; }

cudaError_t launch_kv8_attention(const Kv8Args& a, const Kv8AttnArgs& t, cudaStream_t s) {
    const dim3 grid(a.n_rows, t.hq);
    if (a.hd == 128) kv8_attention_kernel<128><<<grid, kThreads, 0, s>>>(a, t);
    else kv8_attention_kernel<64><<<grid, kThreads, 0, s>>>(a, t);
    return cudaGetLastError();
}

}  // namespace ks
