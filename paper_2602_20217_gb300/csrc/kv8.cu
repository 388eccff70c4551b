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
//
// Bytes bound both kernels where there are many rows: nine prompts of 40k tokens
// in all (64 query heads over 8, hd 128), append 277 us, 5.6 TB/s, and read 46 us,
// 5.3 TB/s; one prompt of 4096 tokens (32 heads) 31 us for both.  Batches of few rows
// are a chain of four dependent loads (sequence, page, record and rows, angles):
// 4 us for one token, 10 us a kernel for 96 sequences of 1 to 11 rows.
#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "kv8.cuh"

namespace ks {

namespace {

constexpr int kThreads = 128;
constexpr int kQHeads = 8;           // query heads of a CTA that rotates queries

// Four codes times a power of two at most 1.
KS_DEV uint32_t rescale4(uint32_t v, float f) {
    const float2 a = from_e4m3x2((uint16_t)v), b = from_e4m3x2((uint16_t)(v >> 16));
    return (uint32_t)to_e4m3x2(a.x * f, a.y * f) | (uint32_t)to_e4m3x2(b.x * f, b.y * f) << 16;
}

// Eight neighbouring elements, as loaded (bf16 pairs, or floats).  WIDE: 16-byte aligned.
template <typename T>
struct Raw8;
template <>
struct Raw8<__nv_bfloat16> {
    uint32_t w[4];
    KS_DEV void get(float (&x)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bf16_lo(w[i]);
            x[2 * i + 1] = bf16_hi(w[i]);
        }
    }
};
template <>
struct Raw8<float> {
    float w[8];
    KS_DEV void get(float (&x)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = w[i];
    }
};
template <bool WIDE>
KS_DEV void load8(const __nv_bfloat16* p, Raw8<__nv_bfloat16>& x) {
    if constexpr (WIDE) {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        x.w[0] = v.x; x.w[1] = v.y; x.w[2] = v.z; x.w[3] = v.w;
    } else {
        const unsigned short* e = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) x.w[i] = e[2 * i] | (uint32_t)e[2 * i + 1] << 16;
    }
}
template <bool WIDE>
KS_DEV void load8(const float* p, Raw8<float>& x) {
    if constexpr (WIDE) {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        x.w[0] = a.x; x.w[1] = a.y; x.w[2] = a.z; x.w[3] = a.w;
        x.w[4] = b.x; x.w[5] = b.y; x.w[6] = b.z; x.w[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x.w[i] = p[i];
    }
}
template <bool WIDE>
KS_DEV void store8(__nv_bfloat16* p, const float (&x)[8]) {
    if constexpr (WIDE) {
        *reinterpret_cast<uint4*>(p) =
            make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = __float2bfloat16_rn(x[i]);
    }
}
template <bool WIDE>
KS_DEV void store8(float* p, const float (&x)[8]) {
    if constexpr (WIDE) {
        reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = x[i];
    }
}
// Eight (cos, sin) of a position from dim j on.
template <bool WIDE>
KS_DEV void load_angles(const float* row, int j, float2 (&cs)[8]) {
    const float2* p = reinterpret_cast<const float2*>(row) + j;
    if constexpr (WIDE) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 v = reinterpret_cast<const float4*>(p)[i];
            cs[2 * i] = make_float2(v.x, v.y);
            cs[2 * i + 1] = make_float2(v.z, v.w);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) cs[i] = p[i];
    }
}
KS_DEV void rotate8(const float2 (&cs)[8], float (&a)[8], float (&b)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float u = a[i], w = b[i];
        a[i] = u * cs[i].x - w * cs[i].y;
        b[i] = w * cs[i].x + u * cs[i].y;
    }
}

// A record's value codes in shared memory, 16 bytes a dim and 16 unused bytes
// after every 8 dims: threads 8 dims apart use different banks.
KS_DEV int v_row(int d) { return d * 16 + (d >> 3) * 16; }

// A block of KV head blockIdx.y.
template <int HD, typename T, bool WIDE>
KS_DEV void append_block(const Kv8Args& a, const Kv8RowArgs& r, const Kv8Slot& w, int group, int d0, int d1) {
    constexpr int REC = kv8_record(HD), CODES = kKv8Block * HD, WARPS = kThreads / 32, PIECES = 2 * HD / kThreads;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, h = blockIdx.y, pos0 = w.blk * kKv8Block;
    unsigned char* rec = kv8_record_at(a, w.s, w.blk, h, REC);
    if (!rec) {
        if (tid == 0) kv8_flag(a, kKv8BadPage);
        return;
    }
    __shared__ __align__(16) unsigned char kc[CODES], vc[CODES + HD * 2];
    __shared__ float top[2][WARPS];
    const bool goes_on = w.first > 0;
    uint4 old[PIECES];
    float2 stored = make_float2(0.f, 0.f);
    if (goes_on) {
        stored = *reinterpret_cast<const float2*>(rec + 2 * CODES);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) old[i] = reinterpret_cast<const uint4*>(rec)[tid + i * kThreads];
    }
    // HD 64: the second half of the threads has no token
    const int t = group;
    const bool mine = t >= w.first && t < w.last;
    float k[2][8], v[2][8], k_top = 0.f, v_top = 0.f;
    if (mine) {
        const T* ks = static_cast<const T*>(r.k) + (int64_t)(w.row + t) * r.k_row + (int64_t)h * r.k_head;
        const T* vs = static_cast<const T*>(r.v) + (int64_t)(w.row + t) * r.v_row + (int64_t)h * r.v_head;
        Raw8<T> raw[4];
        load8<WIDE>(ks + d0, raw[0]);
        load8<WIDE>(ks + d1, raw[1]);
        load8<WIDE>(vs + d0, raw[2]);
        load8<WIDE>(vs + d1, raw[3]);
        raw[0].get(k[0]);
        raw[1].get(k[1]);
        raw[2].get(v[0]);
        raw[3].get(v[1]);
        if (r.rope) {
            if (pos0 + t < r.rope_rows) {
                float2 cs[8];
                load_angles<WIDE>(r.rope + (size_t)(pos0 + t) * HD, d0, cs);
                rotate8(cs, k[0], k[1]);
            } else {
                if (d0 == 0) kv8_flag(a, kKv8BadPosition);
#pragma unroll
                for (int e = 0; e < 8; ++e) k[0][e] = k[1][e] = v[0][e] = v[1][e] = 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
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
    if (goes_on || w.last < kKv8Block) {             // tokens that no thread brings
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int at = (tid + i * kThreads) * 16;       // byte of this piece
            uint4 c = make_uint4(0, 0, 0, 0);
            if (at < CODES) {                               // a token's 16 dims
                const int tok = (at >= CODES / 2 ? 8 : 0) + (at >> 4 & 7);
                if (goes_on && tok < w.first) {
                    c = old[i];
                    if (kf != 1.f)
                        c = make_uint4(rescale4(c.x, kf), rescale4(c.y, kf), rescale4(c.z, kf), rescale4(c.w, kf));
                }
                *reinterpret_cast<uint4*>(kc + at) = c;
            } else {                                        // a dim's 16 tokens
                if (goes_on) {
                    c = old[i];
                    if (vf != 1.f)
                        c = make_uint4(rescale4(c.x, vf), rescale4(c.y, vf), rescale4(c.z, vf), rescale4(c.w, vf));
                    uint32_t* q = reinterpret_cast<uint32_t*>(&c);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {           // tokens 2j, 2j + 1, 8 + 2j, 9 + 2j
                        uint32_t keep = 0;
                        if (2 * j < w.first) keep |= 0xffu;
                        if (2 * j + 1 < w.first) keep |= 0xff00u;
                        if (8 + 2 * j < w.first) keep |= 0xff0000u;
                        if (9 + 2 * j < w.first) keep |= 0xff000000u;
                        q[j] &= keep;
                    }
                }
                *reinterpret_cast<uint4*>(vc + v_row((at - CODES) / 16)) = c;
            }
        }
        __syncthreads();
    }
    if (mine) {
        const float ki = inverse_pow2(ks), vi = inverse_pow2(vs);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int d = i ? d1 : d0;
            uint32_t c[2];
#pragma unroll
            for (int e = 0; e < 2; ++e)
                c[e] = to_e4m3x2(k[i][4 * e] * ki, k[i][4 * e + 1] * ki) |
                       (uint32_t)to_e4m3x2(k[i][4 * e + 2] * ki, k[i][4 * e + 3] * ki) << 16;
            *reinterpret_cast<uint2*>(kc + k_byte<HD>(t, d)) = make_uint2(c[0], c[1]);
            unsigned char* to = vc + v_row(d) + v_byte(t);
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const uint16_t x = to_e4m3x2(v[i][e] * vi, v[i][e + 1] * vi);
                to[16 * e] = (unsigned char)x;
                to[16 * e + 16] = (unsigned char)(x >> 8);
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int at = (tid + i * kThreads) * 16;
        reinterpret_cast<uint4*>(rec)[tid + i * kThreads] =
            *reinterpret_cast<const uint4*>(at < CODES ? kc + at : vc + v_row((at - CODES) / 16));
    }
    if (tid == 0) *reinterpret_cast<float2*>(rec + 2 * CODES) = make_float2(ks, vs);
    __syncthreads();                                 // before the next block
}

// CTAs (., y) of a block's tokens: y below hk take KV head y, the others
// kQHeads query heads each.  HD / 16 threads share a head vector, each with eight
// neighbouring dims of the first half and their partners of the second, so that
// every access is 16 bytes and 128 contiguous ones a vector half.  Bound by bytes
// in flight: a query thread loads two vectors before it rotates the first.  Four
// of bf16 and six CTAs an SM: nine prompts, append and read, 339 us instead of 329;
// one and ten: 373.  16 heads a CTA instead of 8: 96 sequences of a few fp32 rows
// 22.6 us instead of 20.5, 32 heads 28.7.
//
// A KV head's new rows go from registers, quantised, into a copy of the block's
// record in shared memory, and from there out in 16-byte pieces.  A block that
// goes on keeps its old tokens (their record is read while the new rows are);
// the tokens behind the last one are zeros.
template <int HD, typename T, bool WIDE>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 8 : 6) kv8_append_kernel(const Kv8Args a, const Kv8RowArgs r) {
    constexpr int TH = HD / 16, GROUPS = kThreads / TH;
    grid_dependency_wait();
    grid_launch_dependents();
    if (a.stop && *a.stop) return;
    const int tid = threadIdx.x;
    const int group = tid / TH, d0 = tid % TH * 8, d1 = d0 + HD / 2;
    Kv8Slot w;
    Kv8Blocks blocks(a);
    if ((int)blockIdx.y >= a.hk) {
        const int h0 = ((int)blockIdx.y - a.hk) * kQHeads, heads = min(kQHeads, r.hq - h0);
        for (; blocks.get(w); blocks.b += blocks.step) {
            // a thread stays with one token; a block of few tokens has more threads for its heads
            const int tokens = w.last - w.first, ts = tokens > 8 ? 16 : tokens > 4 ? 8 : tokens > 2 ? 4 : tokens;
            const int t = w.first + (group & (ts - 1)), pos = w.blk * kKv8Block + t, step = GROUPS / ts;
            if (t >= w.last) continue;
            constexpr int U = 2;
            const T* src = static_cast<const T*>(r.q) + (int64_t)(w.row + t) * r.q_row;
            __nv_bfloat16* out = r.q_out + (int64_t)(w.row + t) * r.q_out_row;
            const bool turn = r.rope != nullptr, past = turn && pos >= r.rope_rows;
            float2 cs[8];
            if (turn && !past) load_angles<WIDE>(r.rope + (size_t)pos * HD, d0, cs);
            for (int i = group / ts; i < heads; i += U * step) {
                Raw8<T> xs[U], ys[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (i + u * step < heads) {
                        const T* p = src + (int64_t)(h0 + i + u * step) * r.q_head;
                        load8<WIDE>(p + d0, xs[u]);
                        load8<WIDE>(p + d1, ys[u]);
                    }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (i + u * step < heads) {
                        float x[8], y[8];
                        xs[u].get(x);
                        ys[u].get(y);
                        if (past) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) x[e] = y[e] = 0.f;
                        } else if (turn) {
                            rotate8(cs, x, y);
                        }
                        __nv_bfloat16* o = out + (int64_t)(h0 + i + u * step) * r.q_out_head;
                        store8<WIDE>(o + d0, x);
                        store8<WIDE>(o + d1, y);
                    }
            }
        }
        return;
    }
    for (; blocks.get(w); blocks.b += blocks.step) append_block<HD, T, WIDE>(a, r, w, group, d0, d1);
}

// A CTA per block and KV head: the record through shared memory, eight dims of a
// token a thread.
template <int HD, typename T, bool WIDE>
__global__ void __launch_bounds__(kThreads) kv8_read_kernel(const Kv8Args a, T* k_out, T* v_out, int64_t row_ld,
                                                            int64_t head_ld) {
    constexpr int REC = kv8_record(HD), CODES = kKv8Block * HD, PIECES = 2 * HD / kThreads, TH = HD / 8;
    const int tid = threadIdx.x, h = blockIdx.y, d = tid % TH * 8;
    __shared__ __align__(16) unsigned char kc[CODES], vc[CODES + HD * 2];
    grid_dependency_wait();
    grid_launch_dependents();
    Kv8Slot w;
    for (Kv8Blocks blocks(a); blocks.get(w); blocks.b += blocks.step) {
        const unsigned char* rec = kv8_record_at(a, w.s, w.blk, h, REC);
        if (!rec && tid == 0) kv8_flag(a, kKv8BadPage);
        float2 sc = make_float2(1.f, 1.f);
        if (rec) sc = *reinterpret_cast<const float2*>(rec + 2 * CODES);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int at = (tid + i * kThreads) * 16;
            *reinterpret_cast<uint4*>(at < CODES ? kc + at : vc + v_row((at - CODES) / 16)) =
                rec ? reinterpret_cast<const uint4*>(rec)[tid + i * kThreads] : make_uint4(0, 0, 0, 0);
        }
        __syncthreads();
        for (int t = w.first + tid / TH; t < w.last; t += kThreads / TH) {
            const int64_t o = (int64_t)(w.row + t) * row_ld + (int64_t)h * head_ld + d;
            const uint2 c = *reinterpret_cast<const uint2*>(kc + k_byte<HD>(t, d));
            const unsigned char* vb = vc + v_row(d) + v_byte(t);
            float x[8], y[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 kv = from_e4m3x2((uint16_t)((e < 2 ? c.x : c.y) >> (e & 1) * 16));
                const float2 vv = from_e4m3x2((uint16_t)(vb[32 * e] | vb[32 * e + 16] << 8));
                x[2 * e] = kv.x * sc.x; x[2 * e + 1] = kv.y * sc.x;
                y[2 * e] = vv.x * sc.y; y[2 * e + 1] = vv.y * sc.y;
            }
            store8<WIDE>(k_out + o, x);
            store8<WIDE>(v_out + o, y);
        }
        __syncthreads();
    }
}

// Sequences along x, two CTAs for their blocks, where they have at most a block's
// rows on average; else a slot a block (see Kv8Blocks).  96 sequences of 1 to 11
// rows, append and read back, with 16 query heads a CTA: 22.6 us by sequence, 24.8
// us by slots; one prompt of 4096 rows would give all its blocks to two CTAs a head
// by sequence.  The mean says nothing of uneven batches, which cost more here than
// their parts: 200 rows of 200 sequences 10 us, one sequence of 2000 rows 10 us,
// both in one call, by sequence, 145 us, and 127 sequences with the same one, by
// slots, 17 us (append, 32 heads over 8).
dim3 block_grid(Kv8Args& a, int y) {
    a.by_seq = a.n_rows <= (int64_t)kKv8Block * a.n_seqs;
    return a.by_seq ? dim3(a.n_seqs, y, 2) : dim3(a.n_rows / kKv8Block + 2 * a.n_seqs, y);
}

// 16-byte aligned, elements of es bytes, all strides whole 16 bytes
bool wide(size_t es, std::initializer_list<const void*> ptrs, std::initializer_list<int64_t> strides) {
    for (const void* p : ptrs)
        if (reinterpret_cast<uintptr_t>(p) & 15) return false;
    for (int64_t s : strides)
        if (s * es & 15) return false;
    return true;
}

template <int HD, typename T>
cudaError_t append_hd(Kv8Args a, const Kv8RowArgs& r, cudaStream_t s) {
    const dim3 grid = block_grid(a, a.hk + (r.q ? (r.hq + kQHeads - 1) / kQHeads : 0));
    const bool w = wide(sizeof(T), {r.k, r.v, r.q, r.rope}, {r.k_row, r.k_head, r.v_row, r.v_head, r.q_row, r.q_head}) &&
                   wide(2, {r.q_out}, {r.q_out_row, r.q_out_head});
    return launch_kv8(w ? kv8_append_kernel<HD, T, true> : kv8_append_kernel<HD, T, false>, grid, kThreads, 0, s, a, r);
}
template <int HD, typename T>
cudaError_t read_hd(Kv8Args a, void* k, void* v, int64_t row_ld, int64_t head_ld, cudaStream_t s) {
    const dim3 grid = block_grid(a, a.hk);
    T *ko = static_cast<T*>(k), *vo = static_cast<T*>(v);
    const bool w = wide(sizeof(T), {k, v}, {row_ld, head_ld});
    return launch_kv8(w ? kv8_read_kernel<HD, T, true> : kv8_read_kernel<HD, T, false>, grid, kThreads, 0, s, a, ko, vo,
                      row_ld, head_ld);
}

// ------------------------------------------------------------ entry points
// kMaxTokens: of a sequence; positions a tile past the last one still are ints
constexpr int kMaxRows = 1 << 24, kMaxSeqs = 1 << 20, kMaxHeads = 1024, kMaxTokens = 1 << 30;

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
        if (b->table_ld < 1 || (int64_t)b->table_ld * c->page_tokens > kMaxTokens) {
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
    if (dtype == KS_DTYPE_BF16) return a.hd == 128 ? append_hd<128, __nv_bfloat16>(a, r, s) : append_hd<64, __nv_bfloat16>(a, r, s);
    return a.hd == 128 ? append_hd<128, float>(a, r, s) : append_hd<64, float>(a, r, s);
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
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    bool merge;
    cudaError_t e = launch_kv8_attention(a, t, s, merge);
    if (e == cudaSuccess && merge) e = launch_kv8_merge(a, t, s);
    return launched(e, "ks_kv8_attention");
}
