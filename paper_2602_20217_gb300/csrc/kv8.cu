// The 8-bit paged key/value cache: appending with RoPE on the way, reading
// back, and the entry points of the family (kv8_attn.cu attends over it).
//
// Quantisation.  A block of 16 tokens of one KV head has one scale for its
// keys and one for its values, the smallest power of two 2^e (e >= -126) with
// amax <= 448 * 2^e; codes are e4m3 of x * 2^-e, nearest even.  e4m3 is a
// floating-point type, so a power of two loses nothing against amax / 448: the
// relative rounding is 2^-4 at any scale, and it makes the growth of a scale
// exact: when a later token raises it, the stored codes are multiplied by a
// power of two, which rounds only where a code becomes subnormal.
#include <algorithm>
#include <cmath>

#include "kv8.cuh"

namespace ks {

namespace {

constexpr int kAppendThreads = 128;
constexpr int kAppendQHeads = 4;     // query heads of a CTA that rotates queries

// Four codes times a power of two at most 1.
KS_DEV uint32_t rescale4(uint32_t v, float f) {
    const float2 a = from_e4m3x2((uint16_t)v), b = from_e4m3x2((uint16_t)(v >> 16));
    return (uint32_t)to_e4m3x2(a.x * f, a.y * f) | (uint32_t)to_e4m3x2(b.x * f, b.y * f) << 16;
}

// A lane's elements of a head vector: HD / 64 neighbours of the first half and
// their partners of the second.
template <int HD, typename T>
KS_DEV void load_vector(const T* p, float (&x)[HD / 32]) {
    const int lane = threadIdx.x & 31;
    constexpr int V = HD / 64;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        x[e] = to_float(p[V * lane + e]);
        x[V + e] = to_float(p[HD / 2 + V * lane + e]);
    }
}
template <int HD>
KS_DEV void rotate(const float* rope, int pos, float (&x)[HD / 32]) {
    const int lane = threadIdx.x & 31;
    constexpr int V = HD / 64;
    const float2* cs = reinterpret_cast<const float2*>(rope + (size_t)pos * HD) + V * lane;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const float2 c = __ldg(cs + e);
        const float u = x[e], w = x[V + e];
        x[e] = u * c.x - w * c.y;
        x[V + e] = w * c.x + u * c.y;
    }
}

// One CTA per (block slot, KV head): the block's new keys and values, from
// registers, into a copy of its record in shared memory, from where whole
// 16-byte pieces go out.  A block that goes on keeps its old tokens (their
// record is read while the new rows are); the tokens behind the last one are
// zeros.  Further CTAs of a slot rotate the queries of its tokens.
template <int HD, typename T>
__global__ void __launch_bounds__(kAppendThreads) kv8_append_kernel(const Kv8Args a, const Kv8RowArgs r) {
    constexpr int N = HD / 32, V = HD / 64, REC = kv8_record(HD), CODES = kKv8Block * HD;
    constexpr int WARPS = kAppendThreads / 32, PER = kKv8Block / WARPS;
    if (a.stop && *a.stop) return;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    Kv8Slot w;
    if (!kv8_slot(a, blockIdx.x, w)) return;
    const int pos0 = w.blk * kKv8Block;
    if ((int)blockIdx.y >= a.hk) {
        const int h0 = ((int)blockIdx.y - a.hk) * kAppendQHeads;
        for (int i = warp; i < kKv8Block * kAppendQHeads; i += WARPS) {
            const int t = i / kAppendQHeads, h = h0 + i % kAppendQHeads;
            if (t < w.first || t >= w.last || h >= r.hq) continue;
            float x[N];
            load_vector<HD, T>(static_cast<const T*>(r.q) + (int64_t)(w.row + t) * r.q_row + (int64_t)h * r.q_head, x);
            if (r.rope) {
                if (pos0 + t < r.rope_rows) rotate<HD>(r.rope, pos0 + t, x);
                else
                    for (int e = 0; e < N; ++e) x[e] = 0.f;
            }
            __nv_bfloat16* o = r.q_out + (int64_t)(w.row + t) * r.q_out_row + (int64_t)h * r.q_out_head;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                o[V * lane + e] = __float2bfloat16_rn(x[e]);
                o[HD / 2 + V * lane + e] = __float2bfloat16_rn(x[V + e]);
            }
        }
        return;
    }
    const int h = blockIdx.y;
    unsigned char* rec = kv8_record_at(a, w.s, w.blk, h, REC);
    if (!rec) {
        if (tid == 0) kv8_flag(a, kKv8BadPage);
        return;
    }
    __shared__ __align__(16) unsigned char codes[2 * CODES];
    __shared__ float top[2][WARPS];
    const bool goes_on = w.first > 0;
    uint4 old[2 * CODES / 16 / kAppendThreads];
    float2 stored = make_float2(0.f, 0.f);
    if (goes_on) {
        stored = *reinterpret_cast<const float2*>(rec + 2 * CODES);
#pragma unroll
        for (int i = 0; i < 2 * CODES / 16 / kAppendThreads; ++i)
            old[i] = reinterpret_cast<const uint4*>(rec)[tid + i * kAppendThreads];
    }
    float k[PER][N], v[PER][N], k_top = 0.f, v_top = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int t = warp * PER + i;
        if (t < w.first || t >= w.last) continue;
        load_vector<HD, T>(static_cast<const T*>(r.k) + (int64_t)(w.row + t) * r.k_row + (int64_t)h * r.k_head, k[i]);
        load_vector<HD, T>(static_cast<const T*>(r.v) + (int64_t)(w.row + t) * r.v_row + (int64_t)h * r.v_head, v[i]);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int t = warp * PER + i;
        if (t < w.first || t >= w.last) continue;
        if (r.rope) {
            if (pos0 + t < r.rope_rows) {
                rotate<HD>(r.rope, pos0 + t, k[i]);
            } else {
                if (lane == 0) kv8_flag(a, kKv8BadPosition);
                for (int e = 0; e < N; ++e) k[i][e] = v[i][e] = 0.f;
            }
        }
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if (finite(k[i][e])) k_top = fmaxf(k_top, fabsf(k[i][e]));
            else k[i][e] = __uint_as_float(0x7fc00000u);    // infinities too: the type has none
            if (finite(v[i][e])) v_top = fmaxf(v_top, fabsf(v[i][e]));
            else v[i][e] = __uint_as_float(0x7fc00000u);
        }
    }
    k_top = warp_max(k_top);
    v_top = warp_max(v_top);
    if (lane == 0) {
        top[0][warp] = k_top;
        top[1][warp] = v_top;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WARPS; ++i) {
        k_top = fmaxf(k_top, top[0][i]);
        v_top = fmaxf(v_top, top[1][i]);
    }
    float ks = scale_for(k_top), vs = scale_for(v_top);
    if (goes_on) {
        ks = fmaxf(ks, stored.x);
        vs = fmaxf(vs, stored.y);
    }
    const float kf = stored.x / ks, vf = stored.y / vs;
#pragma unroll
    for (int i = 0; i < 2 * CODES / 16 / kAppendThreads; ++i) {
        const int at = (tid + i * kAppendThreads) * 16;     // byte of this piece
        uint4 c = make_uint4(0, 0, 0, 0);
        if (goes_on) {
            if (at < CODES) {                               // a token's 16 dims
                const int t = (at >= CODES / 2 ? 8 : 0) + (at >> 4 & 7);
                if (t < w.first) {
                    c = old[i];
                    if (kf != 1.f)
                        c = make_uint4(rescale4(c.x, kf), rescale4(c.y, kf), rescale4(c.z, kf), rescale4(c.w, kf));
                }
            } else {                                        // a dim's 16 tokens
                c = old[i];
                if (vf != 1.f)
                    c = make_uint4(rescale4(c.x, vf), rescale4(c.y, vf), rescale4(c.z, vf), rescale4(c.w, vf));
                uint32_t* q = reinterpret_cast<uint32_t*>(&c);
#pragma unroll
                for (int j = 0; j < 4; ++j) {               // tokens 2j, 2j + 1, 8 + 2j, 9 + 2j
                    uint32_t keep = 0;
                    if (2 * j < w.first) keep |= 0xffu;
                    if (2 * j + 1 < w.first) keep |= 0xff00u;
                    if (8 + 2 * j < w.first) keep |= 0xff0000u;
                    if (9 + 2 * j < w.first) keep |= 0xff000000u;
                    q[j] &= keep;
                }
            }
        }
        reinterpret_cast<uint4*>(codes)[tid + i * kAppendThreads] = c;
    }
    __syncthreads();
    const float ki = inverse_pow2(ks), vi = inverse_pow2(vs);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int t = warp * PER + i;
        if (t < w.first || t >= w.last) continue;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int d = half * (HD / 2) + V * lane;
            if constexpr (V == 2) {
                const uint16_t kc = to_e4m3x2(k[i][2 * half] * ki, k[i][2 * half + 1] * ki);
                const uint16_t vc = to_e4m3x2(v[i][2 * half] * vi, v[i][2 * half + 1] * vi);
                *reinterpret_cast<uint16_t*>(codes + k_byte<HD>(t, d)) = kc;
                codes[CODES + d * 16 + v_byte(t)] = (unsigned char)vc;
                codes[CODES + (d + 1) * 16 + v_byte(t)] = (unsigned char)(vc >> 8);
            } else {
                codes[k_byte<HD>(t, d)] = (unsigned char)to_e4m3x2(k[i][half] * ki, 0.f);
                codes[CODES + d * 16 + v_byte(t)] = (unsigned char)to_e4m3x2(v[i][half] * vi, 0.f);
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2 * CODES / 16 / kAppendThreads; ++i)
        reinterpret_cast<uint4*>(rec)[tid + i * kAppendThreads] = reinterpret_cast<const uint4*>(codes)[tid + i * kAppendThreads];
    if (tid == 0) *reinterpret_cast<float2*>(rec + 2 * CODES) = make_float2(ks, vs);
}

// One CTA per (block slot, KV head): the record through shared memory, a
// token's dims per warp and step.
template <int HD, typename T>
__global__ void __launch_bounds__(kAppendThreads) kv8_read_kernel(const Kv8Args a, T* k_out, T* v_out, int64_t row_ld,
                                                                  int64_t head_ld) {
    constexpr int REC = kv8_record(HD), CODES = kKv8Block * HD;
    const int tid = threadIdx.x, h = blockIdx.y;
    Kv8Slot w;
    if (!kv8_slot(a, blockIdx.x, w)) return;
    const unsigned char* rec = kv8_record_at(a, w.s, w.blk, h, REC);
    if (!rec && tid == 0) kv8_flag(a, kKv8BadPage);
    __shared__ __align__(16) unsigned char codes[2 * CODES];
    float2 sc = make_float2(1.f, 1.f);
    if (rec) sc = *reinterpret_cast<const float2*>(rec + 2 * CODES);
#pragma unroll
    for (int i = 0; i < 2 * CODES / 16 / kAppendThreads; ++i)
        reinterpret_cast<uint4*>(codes)[tid + i * kAppendThreads] =
            rec ? reinterpret_cast<const uint4*>(rec)[tid + i * kAppendThreads] : make_uint4(0, 0, 0, 0);
    __syncthreads();
    constexpr int DP = HD / 2;     // pairs of dims
    for (int i = tid; i < kKv8Block * DP; i += kAppendThreads) {
        const int t = i / DP, d = 2 * (i % DP);
        if (t < w.first || t >= w.last) continue;
        const float2 kv = from_e4m3x2(*reinterpret_cast<const uint16_t*>(codes + k_byte<HD>(t, d)));
        const unsigned char* vc = codes + CODES + d * 16 + v_byte(t);
        const float2 vv = from_e4m3x2((uint16_t)(vc[0] | vc[16] << 8));
        const int64_t o = (int64_t)(w.row + t) * row_ld + (int64_t)h * head_ld + d;
        k_out[o] = from_float<T>(kv.x * sc.x);
        k_out[o + 1] = from_float<T>(kv.y * sc.x);
        v_out[o] = from_float<T>(vv.x * sc.y);
        v_out[o + 1] = from_float<T>(vv.y * sc.y);
    }
}

template <int HD>
cudaError_t append_hd(int dtype, const Kv8Args& a, const Kv8RowArgs& r, cudaStream_t s) {
    const dim3 grid(a.n_rows / kKv8Block + 2 * a.n_seqs,
                    a.hk + (r.q ? (r.hq + kAppendQHeads - 1) / kAppendQHeads : 0));
    if (dtype == KS_DTYPE_BF16) kv8_append_kernel<HD, __nv_bfloat16><<<grid, kAppendThreads, 0, s>>>(a, r);
    else kv8_append_kernel<HD, float><<<grid, kAppendThreads, 0, s>>>(a, r);
    return cudaGetLastError();
}
template <int HD, typename T>
cudaError_t read_hd(const Kv8Args& a, void* k, void* v, int64_t row_ld, int64_t head_ld, cudaStream_t s) {
    const dim3 grid(a.n_rows / kKv8Block + 2 * a.n_seqs, a.hk);
    kv8_read_kernel<HD, T><<<grid, kAppendThreads, 0, s>>>(a, static_cast<T*>(k), static_cast<T*>(v), row_ld, head_ld);
    return cudaGetLastError();
}

// ------------------------------------------------------------ entry points
constexpr int kMaxRows = 1 << 24, kMaxSeqs = 1 << 20, kMaxHeads = 1024;

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Checks of the cache and the batch, and the kernels' form of them.
ks_status kv8_args(const char* who, const ks_kv8_cache* c, const ks_kv8_batch* b, Kv8Args& a) {
    if (!c || !b) {
        set_error("%s: null argument", who);
        return KS_ERR_INVALID_ARG;
    }
    if (ks_kv8_bytes(c->n_pages, c->page_tokens, c->n_kv_heads, c->head_dim) == 0) {
        if (c->head_dim != 64 && c->head_dim != 128) {
            set_error("%s: head_dim %d (64 and 128 are supported)", who, c->head_dim);
            return KS_ERR_UNSUPPORTED;
        }
        set_error("%s: bad cache sizes: %d pages of %d tokens, %d heads", who, c->n_pages, c->page_tokens, c->n_kv_heads);
        return KS_ERR_INVALID_ARG;
    }
    if (!c->data || !aligned(c->data, 16)) {
        set_error("%s: the cache's data is null or not 16-byte aligned", who);
        return KS_ERR_INVALID_ARG;
    }
    if (b->n_seqs < 0 || b->n_seqs > kMaxSeqs || b->n_rows < 0 || b->n_rows > kMaxRows) {
        set_error("%s: %d sequences, %d rows", who, b->n_seqs, b->n_rows);
        return KS_ERR_INVALID_ARG;
    }
    if (b->n_seqs > 0) {
        if (b->table_ld < 1 || (int64_t)b->table_ld * c->page_tokens > INT32_MAX) {
            set_error("%s: a page table of %d pages of %d tokens", who, b->table_ld, c->page_tokens);
            return KS_ERR_INVALID_ARG;
        }
        for (const void* p : {(const void*)b->page_table, (const void*)b->row_offsets, (const void*)b->lengths})
            if (!p || !aligned(p, 4)) {
                set_error("%s: null or misaligned page table, row offsets or lengths", who);
                return KS_ERR_INVALID_ARG;
            }
        if (!aligned(b->status, 4)) {
            set_error("%s: misaligned status word", who);
            return KS_ERR_INVALID_ARG;
        }
    }
    a = Kv8Args{};
    a.data = static_cast<unsigned char*>(c->data);
    a.n_pages = c->n_pages;
    a.bpp = c->page_tokens / kKv8Block;
    a.hk = c->n_kv_heads;
    a.hd = c->head_dim;
    a.table = b->page_table;
    a.table_ld = b->table_ld;
    a.offsets = b->row_offsets;
    a.lengths = b->lengths;
    a.n_seqs = b->n_seqs;
    a.n_rows = b->n_rows;
    a.capacity = b->table_ld * c->page_tokens;
    a.status = b->status;
    return KS_OK;
}

bool strides_ok(int64_t row, int64_t head) {
    const int64_t most = (int64_t)1 << 40;
    return row >= 0 && head >= 0 && row <= most && head <= most;
}

ks_status launched(cudaError_t e, const char* who) {
    if (e == cudaSuccess) return KS_OK;
    set_error("%s: %s", who, cudaGetErrorString(e));
    return KS_ERR_CUDA;
}

}  // namespace

cudaError_t launch_kv8_append(int dtype, const Kv8Args& a, const Kv8RowArgs& r, cudaStream_t s) {
    return a.hd == 128 ? append_hd<128>(dtype, a, r, s) : append_hd<64>(dtype, a, r, s);
}

}  // namespace ks

using namespace ks;

extern "C" size_t ks_kv8_bytes(int32_t n_pages, int32_t page_tokens, int32_t n_kv_heads, int32_t head_dim) {
    if (n_pages < 1 || page_tokens < kKv8Block || page_tokens % kKv8Block || page_tokens > (1 << 20) || n_kv_heads < 1 ||
        n_kv_heads > kMaxHeads || (head_dim != 64 && head_dim != 128))
        return 0;
    return (size_t)n_pages * n_kv_heads * (page_tokens / kKv8Block) * kv8_record(head_dim);
}

extern "C" ks_status ks_kv8_append(const ks_kv8_cache* cache, const ks_kv8_batch* batch, const ks_kv8_rows* rows,
                                   void* stream) {
    Kv8Args a;
    ks_status st = kv8_args("ks_kv8_append", cache, batch, a);
    if (st != KS_OK) return st;
    if (!rows) {
        set_error("ks_kv8_append: null rows");
        return KS_ERR_INVALID_ARG;
    }
    if (rows->dtype != KS_DTYPE_F32 && rows->dtype != KS_DTYPE_BF16) {
        set_error("ks_kv8_append: unknown dtype %d", rows->dtype);
        return KS_ERR_INVALID_ARG;
    }
    if (a.n_seqs == 0 || a.n_rows == 0) return KS_OK;
    const size_t es = rows->dtype == KS_DTYPE_BF16 ? 2 : 4;
    if (!rows->k || !rows->v || !aligned(rows->k, es) || !aligned(rows->v, es) || !aligned(rows->q, es)) {
        set_error("ks_kv8_append: null or misaligned rows");
        return KS_ERR_INVALID_ARG;
    }
    if (!strides_ok(rows->k_row, rows->k_head) || !strides_ok(rows->v_row, rows->v_head)) {
        set_error("ks_kv8_append: bad strides");
        return KS_ERR_INVALID_ARG;
    }
    if (rows->rope && (rows->rope_rows < 1 || !aligned(rows->rope, 8))) {
        set_error("ks_kv8_append: a RoPE table of %d rows, or a misaligned one", rows->rope_rows);
        return KS_ERR_INVALID_ARG;
    }
    if (rows->q) {
        if (rows->n_q_heads < 1 || rows->n_q_heads > kMaxHeads || !rows->q_out || !aligned(rows->q_out, 2) ||
            !strides_ok(rows->q_row, rows->q_head) || !strides_ok(rows->q_out_row, rows->q_out_head) ||
            (rows->q_out_row < a.hd && a.n_rows > 1) || (rows->q_out_head < a.hd && rows->n_q_heads > 1)) {
            set_error("ks_kv8_append: bad queries: %d heads, strides, or no place for them", rows->n_q_heads);
            return KS_ERR_INVALID_ARG;
        }
    }
    Kv8RowArgs r{};
    r.k = rows->k; r.v = rows->v; r.q = rows->q;
    r.k_row = rows->k_row; r.k_head = rows->k_head;
    r.v_row = rows->v_row; r.v_head = rows->v_head;
    r.q_row = rows->q_row; r.q_head = rows->q_head;
    r.hq = rows->n_q_heads;
    r.rope = rows->rope; r.rope_rows = rows->rope_rows;
    r.q_out = static_cast<__nv_bfloat16*>(rows->q_out);
    r.q_out_row = rows->q_out_row; r.q_out_head = rows->q_out_head;
    return launched(launch_kv8_append(rows->dtype, a, r, static_cast<cudaStream_t>(stream)), "ks_kv8_append");
}

extern "C" ks_status ks_kv8_read(const ks_kv8_cache* cache, const ks_kv8_batch* batch, void* k_out, void* v_out,
                                 int32_t dtype, int64_t row_stride, int64_t head_stride, void* stream) {
    Kv8Args a;
    ks_status st = kv8_args("ks_kv8_read", cache, batch, a);
    if (st != KS_OK) return st;
    if (dtype != KS_DTYPE_F32 && dtype != KS_DTYPE_BF16) {
        set_error("ks_kv8_read: unknown dtype %d", dtype);
        return KS_ERR_INVALID_ARG;
    }
    if (a.n_seqs == 0 || a.n_rows == 0) return KS_OK;
    const size_t es = dtype == KS_DTYPE_BF16 ? 2 : 4;
    if (!k_out || !v_out || !aligned(k_out, es) || !aligned(v_out, es) || !strides_ok(row_stride, head_stride) ||
        (row_stride < a.hd && a.n_rows > 1) || (head_stride < a.hd && a.hk > 1)) {
        set_error("ks_kv8_read: null or misaligned outputs, or bad strides");
        return KS_ERR_INVALID_ARG;
    }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (dtype == KS_DTYPE_BF16)
        e = a.hd == 128 ? read_hd<128, __nv_bfloat16>(a, k_out, v_out, row_stride, head_stride, s)
                        : read_hd<64, __nv_bfloat16>(a, k_out, v_out, row_stride, head_stride, s);
    else
        e = a.hd == 128 ? read_hd<128, float>(a, k_out, v_out, row_stride, head_stride, s)
                        : read_hd<64, float>(a, k_out, v_out, row_stride, head_stride, s);
    return launched(e, "ks_kv8_read");
}

extern "C" size_t ks_kv8_attention_workspace(const ks_kv8_cache* cache, int32_t n_q_heads, int32_t n_seqs,
                                             int32_t n_rows) {
    if (!cache || ks_kv8_bytes(cache->n_pages, cache->page_tokens, cache->n_kv_heads, cache->head_dim) == 0 ||
        n_q_heads < 1 || n_q_heads > kMaxHeads || n_q_heads % cache->n_kv_heads ||
        n_q_heads / cache->n_kv_heads > kKv8MaxGroup || n_seqs < 0 || n_seqs > kMaxSeqs || n_rows < 0 || n_rows > kMaxRows)
        return 0;
    return kv8_attention_workspace(cache->head_dim, n_q_heads / cache->n_kv_heads, n_rows);
}

extern "C" ks_status ks_kv8_attention(const ks_kv8_cache* cache, const ks_kv8_batch* batch, const ks_kv8_attn* attn,
                                      void* stream) {
    Kv8Args a;
    ks_status st = kv8_args("ks_kv8_attention", cache, batch, a);
    if (st != KS_OK) return st;
    if (!attn) {
        set_error("ks_kv8_attention: null argument");
        return KS_ERR_INVALID_ARG;
    }
    if (attn->n_q_heads < 1 || attn->n_q_heads > kMaxHeads || attn->n_q_heads % a.hk) {
        set_error("ks_kv8_attention: %d query heads over %d KV heads", attn->n_q_heads, a.hk);
        return KS_ERR_INVALID_ARG;
    }
    if (attn->n_q_heads / a.hk > kKv8MaxGroup) {
        set_error("ks_kv8_attention: %d query heads a KV head (at most %d)", attn->n_q_heads / a.hk, kKv8MaxGroup);
        return KS_ERR_UNSUPPORTED;
    }
    if (!std::isfinite(attn->scale)) {
        set_error("ks_kv8_attention: the scale is not finite");
        return KS_ERR_INVALID_ARG;
    }
    if (a.n_seqs == 0 || a.n_rows == 0) return KS_OK;
    if (!attn->q || !attn->out || !aligned(attn->q, 2) || !aligned(attn->out, 2) || !aligned(attn->lse, 4) ||
        !strides_ok(attn->q_row, attn->q_head) || !strides_ok(attn->out_row, attn->out_head) ||
        (attn->out_row < a.hd && a.n_rows > 1) || (attn->out_head < a.hd && attn->n_q_heads > 1)) {
        set_error("ks_kv8_attention: null or misaligned queries or output, or bad strides");
        return KS_ERR_INVALID_ARG;
    }
    if (!kv8_attention_fits(a, attn->n_q_heads)) {
        set_error("ks_kv8_attention: %d rows over up to %d tokens are too much for one call", a.n_rows, a.capacity);
        return KS_ERR_UNSUPPORTED;
    }
    const size_t need = kv8_attention_workspace(a.hd, attn->n_q_heads / a.hk, a.n_rows);
    if (!attn->workspace || !aligned(attn->workspace, 256)) {
        set_error("ks_kv8_attention: null or misaligned workspace");
        return KS_ERR_INVALID_ARG;
    }
    if (attn->workspace_bytes < need) {
        set_error("ks_kv8_attention: a workspace of %zu bytes, %zu needed", attn->workspace_bytes, need);
        return KS_ERR_WORKSPACE;
    }
    Kv8AttnArgs t{};
    t.q = static_cast<const __nv_bfloat16*>(attn->q);
    t.q_row = attn->q_row; t.q_head = attn->q_head;
    t.out = static_cast<__nv_bfloat16*>(attn->out);
    t.out_row = attn->out_row; t.out_head = attn->out_head;
    t.lse = attn->lse;
    t.hq = attn->n_q_heads;
    t.scale = attn->scale;
    t.workspace = attn->workspace;
    return launched(launch_kv8_attention(a, t, static_cast<cudaStream_t>(stream)), "ks_kv8_attention");
}
