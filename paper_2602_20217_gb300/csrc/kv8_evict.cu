// Eviction from the 8-bit paged cache: of each sequence and KV head the first
// and the most recent tokens stay, and of those between the ones with the largest
// scores, in their order, in other pages of the cache.
//
// select: the least kept score by a radix search over the scores' 32 bits, made
// whole numbers in the scores' order, 11, 11 and 10 bits at a time, then one pass
// that numbers what stays: scores above it, and as many equal ones, the earlier
// first, as there is room for.
//
// gather: a CTA writes one block of 16 kept tokens.  Their codes come from up to 16
// records with scales of their own; the new block's scale is the smallest power
// of two for their values, as an append of them would choose it, and a code is
// multiplied by a power of two, which rounds only where it becomes subnormal.  A
// token's keys are 16-byte pieces of its record; its values are one byte of every
// 16, so every sector of the record's second half is read.
#include <algorithm>

#include "kv8.cuh"

namespace ks {

namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32, kBins = 2048;

// Larger score, larger key; the two zeros are one, and NaN is below everything.
KS_DEV unsigned score_key(float v) {
    if (v != v) return 0u;
    const unsigned b = __float_as_uint(v + 0.f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// What stays of a sequence.
struct Stay {
    int len, n, first, recent;      // of len tokens n; the first and the last so many among them
    KS_DEV Stay(const Kv8Args& a, const Kv8EvictArgs& t, int s) {
        len = min(max(a.lengths[s], 0), a.capacity);
        n = min(min(max(t.keep[s], 0), len), t.new_capacity);
        recent = min(t.recent, n);
        first = min(t.first, n - recent);
    }
};

// Sum over the CTA of the counts before this thread's; total: of all.
KS_DEV int block_before(int v, int* sums, int& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int u = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int w = __shfl_up_sync(0xffffffffu, u, o);
        if (lane >= o) u += w;
    }
    if (lane == 31) sums[warp] = u;
    __syncthreads();
    int w = lane < kWarps ? sums[lane] : 0;
    total = __reduce_add_sync(0xffffffffu, w);
    const int before = __reduce_add_sync(0xffffffffu, lane < warp ? w : 0);
    __syncthreads();
    return before + u - v;
}

__global__ void __launch_bounds__(kThreads) kv8_select_kernel(const Kv8Args a, const Kv8EvictArgs t) {
    __shared__ int bins[kBins], sums[kWarps];
    __shared__ unsigned s_prefix;
    __shared__ int s_left;
    const int tid = threadIdx.x, h = blockIdx.x, s = blockIdx.y;
    grid_dependency_wait();
    grid_launch_dependents();
    const Stay w(a, t, s);
    if (h == 0 && tid == 0) {
        const int len = a.lengths[s], keep = t.keep[s];
        if (len < 0 || len > a.capacity || keep < 0 || min(keep, len) > t.new_capacity) kv8_flag(a, kKv8BadBatch);
        t.new_lengths[s] = w.n;
    }
    const float* score = t.scores + ((size_t)s * a.hk + h) * t.ld;
    int32_t* kept = t.kept + ((size_t)s * a.hk + h) * t.kept_ld;
    float* out = t.new_scores ? t.new_scores + ((size_t)s * a.hk + h) * t.new_ld : nullptr;
    if (w.n == w.len) {
        for (int i = tid; i < w.n; i += kThreads) {
            kept[i] = i;
            if (out) out[i] = score[i];
        }
        return;
    }
    const int lo = w.first, hi = w.len - w.recent, most = w.n - w.first - w.recent;      // most of [lo, hi) stay
    // the least key that stays, and how many of those equal to it
    unsigned prefix = 0;
    int left = most;
    if (most > 0) {
#pragma unroll 1
        for (int shift = 21; shift >= 0; shift -= shift == 21 ? 11 : 10) {
            const int width = shift == 0 ? 10 : 11;
            const unsigned above = shift == 21 ? 0u : 0xffffffffu << (shift + width);
            for (int i = tid; i < kBins; i += kThreads) bins[i] = 0;
            __syncthreads();
            for (int i = lo + tid; i < hi; i += kThreads) {
                const unsigned k = score_key(score[i]);
                if ((k & above) == prefix) atomicAdd(&bins[k >> shift & ((1u << width) - 1)], 1);
            }
            __syncthreads();
            // bins from the largest down, two a thread: the one in which the count passes what is left
            const int top = (1 << width) - 1, b0 = top - 2 * tid, c0 = b0 >= 0 ? bins[b0] : 0, c1 = b0 >= 1 ? bins[b0 - 1] : 0;
            int total;
            const int before = block_before(c0 + c1, sums, total);
            if (before < left && before + c0 + c1 >= left) {
                const bool second = before + c0 < left;
                s_prefix = prefix | (unsigned)(second ? b0 - 1 : b0) << shift;
                s_left = left - before - (second ? c0 : 0);
            }
            __syncthreads();
            prefix = s_prefix;
            left = s_left;
            __syncthreads();
        }
    }
    int ties = 0, done = 0;                          // equal ones, and kept ones so far
    for (int base = 0; base < w.len; base += kThreads) {
        const int i = base + tid;
        const bool inside = i >= lo && i < hi;
        const float v = i < w.len && (inside || out) ? score[i] : 0.f;
        const unsigned k = inside ? score_key(v) : 0u;
        const bool equal = inside && most > 0 && k == prefix;
        int total;
        const int tie = ties + block_before(equal, sums, total);
        ties += total;
        const bool stays = i < w.len && (!inside || (most > 0 && (k > prefix || (equal && tie < left))));
        const int o = done + block_before(stays, sums, total);
        done += total;
        if (stays) {
            kept[o] = i;
            if (out) out[o] = v;
        }
    }
}

template <int HD>
__global__ void __launch_bounds__(HD) kv8_gather_kernel(const Kv8Args a, const Kv8EvictArgs t) {
    constexpr int REC = kv8_record(HD), CODES = kKv8Block * HD, TH = HD / 16, WARPS = HD / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, b = blockIdx.x, h = blockIdx.y;
    __shared__ __align__(16) unsigned char vc[CODES + HD * 2];
    __shared__ float top[2][WARPS];
    grid_dependency_wait();
    grid_launch_dependents();
    for (int s = blockIdx.z; s < a.n_seqs; s += gridDim.z) {
        const Stay w(a, t, s);
        if (b * kKv8Block >= w.n) continue;
        const int page = t.new_table[(size_t)s * t.new_table_ld + b / a.bpp];
        if (page < 0 || page >= a.n_pages) {
            if (tid == 0) kv8_flag(a, kKv8BadPage);
            continue;
        }
        unsigned char* rec = a.data + (((size_t)page * a.hk + h) * a.bpp + b % a.bpp) * REC;
        // a sequence that keeps all of its tokens may keep its pages
        if (w.n == w.len && rec == kv8_record_at(a, s, b, h, REC)) continue;
        const int tok = tid / TH, part = tid % TH, at = b * kKv8Block + tok;
        float k[16], v[16], k_top = 0.f, v_top = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) k[i] = v[i] = 0.f;
        if (at < w.n) {
            const int from = t.kept[((size_t)s * a.hk + h) * t.kept_ld + at], ft = from % kKv8Block;
            const unsigned char* src = kv8_record_at(a, s, from / kKv8Block, h, REC);
            if (src) {
                const float2 sc = *reinterpret_cast<const float2*>(src + 2 * CODES);
                const uint4 c = *reinterpret_cast<const uint4*>(src + k_byte<HD>(ft, 16 * part));
                const unsigned char* vb = src + CODES + 16 * part * 16 + v_byte(ft);
                unsigned char e[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) e[i] = vb[16 * i];
                const uint32_t words[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float2 kv = from_e4m3x2((uint16_t)(words[i / 2] >> 16 * (i & 1)));
                    const float2 vv = from_e4m3x2((uint16_t)(e[2 * i] | e[2 * i + 1] << 8));
                    k[2 * i] = kv.x * sc.x; k[2 * i + 1] = kv.y * sc.x;
                    v[2 * i] = vv.x * sc.y; v[2 * i + 1] = vv.y * sc.y;
                }
            } else if (part == 0) {
                kv8_flag(a, kKv8BadPage);            // read as zeros
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (finite(k[i])) k_top = fmaxf(k_top, fabsf(k[i]));
            if (finite(v[i])) v_top = fmaxf(v_top, fabsf(v[i]));
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
        const float ks = scale_for(k_top), vs = scale_for(v_top), ki = inverse_pow2(ks), vi = inverse_pow2(vs);
        uint32_t c[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            c[i] = to_e4m3x2(k[4 * i] * ki, k[4 * i + 1] * ki) | (uint32_t)to_e4m3x2(k[4 * i + 2] * ki, k[4 * i + 3] * ki) << 16;
        *reinterpret_cast<uint4*>(rec + k_byte<HD>(tok, 16 * part)) = make_uint4(c[0], c[1], c[2], c[3]);
        // 16 unused bytes after every 8 dims, as in an append
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const int d = 16 * part + i;
            const uint16_t x = to_e4m3x2(v[i] * vi, v[i + 1] * vi);
            unsigned char* to = vc + d * 16 + (d >> 3) * 16 + v_byte(tok);
            to[0] = (unsigned char)x;
            to[16] = (unsigned char)(x >> 8);
        }
        __syncthreads();
        *reinterpret_cast<uint4*>(rec + CODES + tid * 16) = *reinterpret_cast<const uint4*>(vc + tid * 16 + (tid >> 3) * 16);
        if (tid == 0) *reinterpret_cast<float2*>(rec + 2 * CODES) = make_float2(ks, vs);
        __syncthreads();
    }
}

}  // namespace

cudaError_t launch_kv8_evict(const Kv8Args& a, const Kv8EvictArgs& t, cudaStream_t s) {
    cudaError_t e = cudaSuccess;
    // the grid's y and z are 65535 at most
    for (int s0 = 0; s0 < a.n_seqs && e == cudaSuccess; s0 += 65535) {
        Kv8Args b = a;
        Kv8EvictArgs u = t;
        b.n_seqs = std::min(a.n_seqs - s0, 65535);
        b.table += (size_t)s0 * a.table_ld;
        b.lengths += s0;
        u.scores += (size_t)s0 * a.hk * t.ld;
        u.keep += s0;
        u.new_table += (size_t)s0 * t.new_table_ld;
        u.new_lengths += s0;
        u.kept += (size_t)s0 * a.hk * t.kept_ld;
        if (u.new_scores) u.new_scores += (size_t)s0 * a.hk * t.new_ld;
        e = launch_kv8(kv8_select_kernel, dim3(a.hk, b.n_seqs), kThreads, 0, s, b, u);
        if (e != cudaSuccess || t.new_capacity == 0) return e;
        const dim3 grid(t.new_capacity / kKv8Block, a.hk, b.n_seqs);
        e = a.hd == 128 ? launch_kv8(kv8_gather_kernel<128>, grid, 128, 0, s, b, u)
                        : launch_kv8(kv8_gather_kernel<64>, grid, 64, 0, s, b, u);
    }
    return e;
}

}  // namespace ks
