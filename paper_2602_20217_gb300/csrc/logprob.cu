// Log probabilities of given tokens under rows of logits, the rows' entropies
// and their most likely tokens, in one pass over the logits.
//
// With m the row's largest logit and x' = (x - m) / T:
//   log p(x) = x' - log Z,  Z = sum exp x',  H = log Z - (sum x' exp x') / Z.
// The largest logit is left out of the sums and counted instead, Z = n + tail,
// so that a likely token's logarithm, -log1p(tail), keeps its digits.
//
// A cluster takes a row, each CTA every so many segments of it.  A warp reads a
// segment, 32 times 64 bytes, at a time into registers, the next one while it works
// on it, and keeps the row's maximum so far for all of its lanes: a segment that
// holds no larger logit, nearly every one, adds to the sums without a look at single
// maxima.  The
// segments' maxima stay in shared memory.  The n_top largest logits are in the
// n_top segments with the largest maxima (ties: the earlier one; every logit of
// another segment is behind each of those maxima), and at least as large as the
// least of these maxima: those segments are read again, from L2, and the few
// candidates ranked against each other.
//
// That takes n_top segments in each CTA of the row.  With fewer there is no such
// bound, and all logits of the CTA are candidates: ranked up to 1024, beyond that
// read again for each bit that the n_top-th largest is searched by.  In us, at 5,
// 20 and 64 alternatives: one row of 151936 in bf16 16, 232, 248, of 50257 in fp32
// 17, 47, 57; 251 rows of 100277 in bf16 22, 26, 1075; 4000 rows of 20000 in fp32 82,
// 95, 1066, of 5000 49, 360, 391.
//
// Measured: 1500 rows of 151936 fp32 logits 159 us, 5.7 TB/s, memory; 251 rows of
// 100277 in bf16 with 5 alternatives 20 us, 2.5 TB/s (of logits without peaks 22, and
// 18 without alternatives): 0.44 instructions a scheduler and clock, barriers the
// largest stall, as a row's end is serial and there is one partial wave of CTAs; one
// row of 128256 11 us, launch and the cluster's phases (a CTA a row 16).
#include <cmath>

#include "internal.h"
#include "tma.cuh"
#include "umma.cuh"

namespace ks {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxVocab = 1 << 22;
constexpr int kMaxTop = 64, kMaxTokens = 64;
constexpr int kCand = 1024;         // candidates that are ranked in one go
constexpr int kMaxCluster = 8, kCtas = 4;            // CTAs of a row; of an SM
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kTame = 4096.f;     // of a maximum's |m k|
constexpr float kLeast = -200.f;    // below it 2^u is 0: -inf must not be multiplied by that

struct LogprobArgs {
    const void* logits;
    int64_t ld;
    int rows, vocab;
    int n_tokens, n_top;
    float temperature;
    const int32_t* tokens;
    float *logprobs, *entropy, *top_logprobs;
    int32_t* top_ids;
};

// Larger float, larger key; the two zeros are one, and nothing is 0.
KS_DEV unsigned order_key(float v) {
    const unsigned b = __float_as_uint(v + 0.f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
KS_DEV float order_value(unsigned k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); }
// Larger first, then the lower id.
KS_DEV unsigned long long pair_key(float v, int id) {
    return ((unsigned long long)order_key(v) << 32) | (0xFFFFFFFFu - (unsigned)id);
}
KS_DEV int pair_id(unsigned long long k) { return (int)(0xFFFFFFFFu - (unsigned)k); }
KS_DEV float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Sums relative to a maximum m, u = (x - m) log2(e) / T: n logits equal to it, the
// sum of 2^u over the others and of u 2^u.
struct Sums {
    float m, t, s;
    int n;
    // the same relative to a larger maximum
    KS_DEV void raise(float top, float k) {
        if (top == m) return;
        const float u = (m - top) * k, f = exp2_approx(u), z = t + (float)n;
        s = f > 0.f ? f * fmaf(u, z, s) : 0.f;       // u may be -inf
        t = f * z;
        n = 0;
        m = top;
    }
};

// One warp: the sums of all lanes together.
KS_DEV Sums merged(Sums u, float k) {
    const float top = warp_max(u.m);
    u.raise(top, k);
    return Sums{top, warp_sum(u.t), warp_sum(u.s), (int)__reduce_add_sync(0xffffffffu, u.n)};
}

// A row as 16-byte vectors from the boundary at or before its first logit on:
// position p of them is logit p - shift.
template <typename T>
struct Row {
    static constexpr int E = 16 / sizeof(T), kVec = 4, SEG = 32 * kVec * E;
    const T* base;
    int shift, end;                 // positions [shift, end) are the row's
    KS_DEV Row(const LogprobArgs& a, int row) {
        const T* p = static_cast<const T*>(a.logits) + (int64_t)row * a.ld;
        shift = (int)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
        base = p - shift;
        end = shift + a.vocab;
    }
    KS_DEV int segments() const { return (end + SEG - 1) / SEG; }
    KS_DEV int position(int seg, int v) const { return seg * SEG + (v * 32 + (int)(threadIdx.x & 31)) * E; }
    // A lane's part of a segment, as it lies in memory; what is not the row's is -inf.
    KS_DEV void load(int seg, uint4 (&raw)[kVec]) const {
        if (seg * SEG >= shift && (seg + 1) * SEG <= end) {
#pragma unroll
            for (int v = 0; v < kVec; ++v) raw[v] = *reinterpret_cast<const uint4*>(base + position(seg, v));
        } else {
#pragma unroll
            for (int v = 0; v < kVec; ++v) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int p = position(seg, v) + i * (E / 4);
                    if constexpr (E == 4) {
                        w[i] = 0xff800000u;
                        if (p >= shift && p < end) w[i] = __float_as_uint(base[p]);
                    } else {
                        w[i] = 0xff80ff80u;
                        const unsigned short* e = reinterpret_cast<const unsigned short*>(base);
                        if (p >= shift && p < end) w[i] = (w[i] & 0xffff0000u) | e[p];
                        if (p + 1 >= shift && p + 1 < end) w[i] = (w[i] & 0xffffu) | (uint32_t)e[p + 1] << 16;
                    }
                }
                raw[v] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
    // The largest of a lane's logits; NaN is passed over.
    template <int N>
    static KS_DEV float largest(const uint4 (&raw)[N]) {
        if constexpr (E == 4) {
            float m = -INFINITY;
#pragma unroll
            for (int v = 0; v < N; ++v)
                m = fmaxf(fmaxf(fmaxf(m, __uint_as_float(raw[v].x)), __uint_as_float(raw[v].y)),
                          fmaxf(__uint_as_float(raw[v].z), __uint_as_float(raw[v].w)));
            return m;
        } else {
            __nv_bfloat162 m = pair(raw[0].x);
#pragma unroll
            for (int v = 0; v < N; ++v)
                m = __hmax2(__hmax2(__hmax2(m, pair(raw[v].x)), pair(raw[v].y)), __hmax2(pair(raw[v].z), pair(raw[v].w)));
            return fmaxf(__low2float(m), __high2float(m));
        }
    }
    static KS_DEV __nv_bfloat162 pair(uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); }
    // What is below `floor`, -inf too, as that: the exponential is 0, and times the exponent still is.  NaN stays.
    static KS_DEV uint4 raised(const uint4& r, float floor) {
        uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (E == 4) {
                asm("max.NaN.f32 %0, %0, %1;" : "+r"(w[i]) : "r"(__float_as_uint(floor)));
            } else {
                const __nv_bfloat162 f = __float2bfloat162_rn(floor), m = __hmax2_nan(pair(w[i]), f);
                w[i] = *reinterpret_cast<const uint32_t*>(&m);
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static KS_DEV void widen(const uint4& r, float* x) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (E == 4) {
                x[i] = __uint_as_float(w[i]);
            } else {
                x[2 * i] = bf16_lo(w[i]);
                x[2 * i + 1] = bf16_hi(w[i]);
            }
        }
    }
};

KS_DEV void store_cluster(void* p, int rank, unsigned long long v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(cluster_addr(p, rank)), "l"(v) : "memory");
}

struct Smem {
    unsigned long long cand[kCand];
    __align__(16) unsigned long long best[kMaxCluster][kMaxTop];      // the first CTA: every CTA's largest
    unsigned long long sums[kMaxCluster][2];            // the first CTA: (m, n), (t, s) of each
    Sums warp[kWarps];
    unsigned first[kWarps];
    int counts[2][kWarps];
    unsigned bound;
    int n_cand, n_chosen;
    int chosen[kMaxTop];
    float log_z, m;
    bool bad;
};

// The K largest pairs (value, id) among the segments at `mine`, in order, to
// out[K] (0: fewer).  maxima: the segments' largest keys, n of them, segment i
// being first + i step of the row.
template <typename T>
KS_DEV void largest(const Row<T>& row, int first, int step, int n, const unsigned* maxima, int K, Smem& sm,
                    unsigned long long* out) {
    using R = Row<T>;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        sm.n_cand = 0;
        sm.bound = 0;
    }
    __syncthreads();                                 // maxima, and the zeros behind them
    // The K segments with the largest maxima.  Up to one a thread they are ranked against each other, which is soonest
    // done; of more the K-th largest key is found bit by bit, by one warp: several microseconds, but in calls of many rows
    // next to nothing beside what the SM's other CTAs do meanwhile (1500 rows of 151936 fp32 logits 157 us, ranked 171).
    if (n <= kThreads) {
        if (const int i = tid; i < n) {
            const unsigned k = maxima[i];
            const uint4* four = reinterpret_cast<const uint4*>(maxima);      // behind the last one: zeros
            int rank = 0;
#pragma unroll 4
            for (int j = 0; j < (n + 3) / 4; ++j) {
                const uint4 o = four[j];
                rank += (o.x > k) + (o.y > k) + (o.z > k) + (o.w > k);
                // equal ones count where they are earlier
                if (o.x == k || o.y == k || o.z == k || o.w == k)
                    rank += (o.x == k && 4 * j < i) + (o.y == k && 4 * j + 1 < i) + (o.z == k && 4 * j + 2 < i) +
                            (o.w == k && 4 * j + 3 < i);
            }
            if (rank < K) sm.chosen[rank] = i;
            if (rank == K - 1) sm.bound = k;
        }
    } else if (warp == 0) {
        unsigned least = 0;
        int above = 0, at = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const unsigned t = least | (1u << bit);
            int c = 0;
            for (int i = lane; i < n; i += 32) c += maxima[i] >= t;
            c = __reduce_add_sync(0xffffffffu, c);
            if (c >= K) least = t;
            if (c == K) break;
        }
        for (int i = lane; i < n; i += 32) above += maxima[i] > least;
        int equal = K - __reduce_add_sync(0xffffffffu, above);           // of those at `least`, the first
        for (int i0 = 0; i0 < n; i0 += 32) {
            const unsigned k = i0 + lane < n ? maxima[i0 + lane] : 0u, below = (1u << lane) - 1;
            const unsigned same = __ballot_sync(0xffffffffu, i0 + lane < n && k == least);
            const bool take = i0 + lane < n && (k > least || (k == least && __popc(same & below) < equal));
            equal = max(0, equal - __popc(same));
            const unsigned taken = __ballot_sync(0xffffffffu, take);
            if (take) sm.chosen[at + __popc(taken & below)] = i0 + lane;
            at += __popc(taken);
        }
        if (lane == 0) sm.bound = least;
    }
    __syncthreads();
    const int chosen = min(n, K);
    const unsigned bound = sm.bound;
    // f for each logit of the chosen segments, of lanes that have one at least as large as `from`
    auto each = [&](float from, auto&& f) {
        uint4 next[R::kVec];
        if (warp < chosen) row.load(first + sm.chosen[warp] * step, next);
        for (int c = warp; c < chosen; c += kWarps) {
            const int seg = first + sm.chosen[c] * step;
            uint4 raw[R::kVec];
#pragma unroll
            for (int v = 0; v < R::kVec; ++v) raw[v] = next[v];
            if (c + kWarps < chosen) row.load(first + sm.chosen[c + kWarps] * step, next);
            if (R::largest(raw) < from) continue;
#pragma unroll
            for (int v = 0; v < R::kVec; ++v) {
                const uint4 one[1] = {raw[v]};
                if (R::largest(one) < from) continue;
                float x[R::E];
                R::widen(raw[v], x);
#pragma unroll
                for (int e = 0; e < R::E; ++e) {
                    const int p = row.position(seg, v) + e;
                    if (p >= row.shift && p < row.end) f(x[e], p - row.shift);
                }
            }
        }
    };
    each(order_value(bound), [&](float x, int id) {
        if (order_key(x) >= bound) {
            const int at = atomicAdd(&sm.n_cand, 1);
            if (at < kCand) sm.cand[at] = pair_key(x, id);
        }
    });
    __syncthreads();
    int found = sm.n_cand;
    if (found > kCand) {
        // too many for one go: the K-th largest pair, bit by bit (all pairs differ)
        unsigned long long least = 0;
        for (int bit = 63, turn = 0; bit >= 0; --bit, turn ^= 1) {
            const unsigned long long t = least | (1ull << bit);
            int c = 0;
            each(-INFINITY, [&](float x, int id) { c += pair_key(x, id) >= t; });
            c = __reduce_add_sync(0xffffffffu, c);
            if (lane == 0) sm.counts[turn][warp] = c;
            __syncthreads();
            c = __reduce_add_sync(0xffffffffu, lane < kWarps ? sm.counts[turn][lane] : 0);
            if (c >= K) least = t;
            if (c == K) break;
        }
        if (tid == 0) sm.n_cand = 0;
        __syncthreads();
        each(-INFINITY, [&](float x, int id) {
            const unsigned long long k = pair_key(x, id);
            if (k >= least) sm.cand[atomicAdd(&sm.n_cand, 1)] = k;
        });
        __syncthreads();
        found = sm.n_cand;
    }
    for (int i = tid; i < found; i += kThreads) {
        const unsigned long long k = sm.cand[i];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < found; ++j) rank += sm.cand[j] > k;
        if (rank < K) out[rank] = k;
    }
    if (tid >= found && tid < K) out[tid] = 0ull;
    __syncthreads();
}

template <typename T>
__global__ void __launch_bounds__(kThreads, kCtas) logprob_kernel(const LogprobArgs a, int ctas) {
    using R = Row<T>;
    extern __shared__ __align__(16) unsigned maxima[];
    __shared__ Smem sm;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = (int)blockIdx.x % ctas;
    grid_dependency_wait();
    grid_launch_dependents();
    const int r = (int)blockIdx.x / ctas;
    const R row(a, r);
    const int segs = row.segments(), mine = segs > rank ? (segs - rank - 1) / ctas + 1 : 0;
    const float k = kLog2e / a.temperature;
    if (ctas > 1) cluster_sync();                    // every CTA runs: the first one's shared memory may be written

    Sums sum{-INFINITY, 0.f, 0.f, 0};                // m is the warp's, the rest the lane's
    // Sums of segments whose logits are all below m, u taken as x k - (m k rounded): `rest` is what the rounding left.
    float2 quick_t = make_float2(0.f, 0.f), quick_s = quick_t;
    float mk = 0.f, rest = 0.f;
    bool tame = false;                               // whether m is small enough for that
    const float floor = -2.f * kTame / k;            // 2^u is 0 from there down, beside any tame maximum
    auto set = [&](float top) {
        sum.raise(top, k);
        mk = sum.m * k;
        tame = fabsf(mk) < kTame && floor > -1e38f;
        rest = tame ? fmaf(sum.m, k, -mk) : 0.f;
    };
    auto settle = [&] {
        const float t = quick_t.x + quick_t.y, f = fmaf(-rest, kLn2, 1.f);       // 2^-rest, rest under 2^-12
        sum.s = fmaf(fmaf(-rest, t, quick_s.x + quick_s.y), f, sum.s);
        sum.t = fmaf(t, f, sum.t);
        quick_t = quick_s = make_float2(0.f, 0.f);
    };
    uint4 next[R::kVec];
    if (warp < mine) row.load(rank + warp * ctas, next);
    // the tokens' logits, long before they are needed
    const bool scores = rank == 0 && tid < a.n_tokens;
    float token_x = __uint_as_float(0x7fc00000u);
    if (scores) {
        const int id = a.tokens[(size_t)r * a.n_tokens + tid];
        if (id >= 0 && id < a.vocab) token_x = to_float(row.base[row.shift + id]);
    }
    // All warps begin with the largest logit of their first segments: on its own a warp would meet a larger one than so
    // far in three of twelve segments, and looks at each of its logits then.
    {
        unsigned key = 0;                            // below that of any number
        if (warp < mine) key = __reduce_max_sync(0xffffffffu, order_key(R::largest(next)));
        if (lane == 0) sm.first[warp] = key;
        __syncthreads();
        key = __reduce_max_sync(0xffffffffu, sm.first[lane % kWarps]);
        if (key != 0) set(order_value(key));
    }
    for (int i = warp; i < mine; i += kWarps) {
        uint4 raw[R::kVec];
#pragma unroll
        for (int v = 0; v < R::kVec; ++v) raw[v] = next[v];
        if (i + kWarps < mine) row.load(rank + (i + kWarps) * ctas, next);
        const unsigned key = __reduce_max_sync(0xffffffffu, order_key(R::largest(raw)));
        if (lane == 0) maxima[i] = key;
        const float top = order_value(key);
        if (top < sum.m && tame) {
#pragma unroll
            for (int v = 0; v < R::kVec; ++v) {
                float x[R::E];
                R::widen(R::raised(raw[v], floor), x);
#pragma unroll
                for (int j = 0; j < R::E; j += 2) {
                    const float2 u = __ffma2_rn(make_float2(x[j], x[j + 1]), make_float2(k, k), make_float2(-mk, -mk));
                    const float2 e = make_float2(exp2_approx(u.x), exp2_approx(u.y));
                    quick_t = __fadd2_rn(quick_t, e);
                    quick_s = __ffma2_rn(e, u, quick_s);
                }
            }
            continue;
        }
        settle();
        if (top >= sum.m) set(top);
        const float ref = sum.m == -INFINITY ? 0.f : sum.m;
#pragma unroll
        for (int v = 0; v < R::kVec; ++v) {
            float x[R::E];
            R::widen(raw[v], x);
#pragma unroll
            for (int j = 0; j < R::E; ++j) {
                const float u = (x[j] - ref) * k, e = exp2_approx(u);
                if (x[j] == sum.m) {
                    ++sum.n;
                } else {
                    sum.t += e;
                    sum.s = fmaf(e, fmaxf(u, kLeast), sum.s);
                }
            }
        }
    }
    settle();
    sum.t = warp_sum(sum.t);
    sum.s = warp_sum(sum.s);
    sum.n = __reduce_add_sync(0xffffffffu, sum.n);
    if (lane == 0) sm.warp[warp] = sum;
    __syncthreads();
    if (tid < 4 && mine + tid < (mine + 3) / 4 * 4) maxima[mine + tid] = 0;
    if (warp == 0) {
        const Sums all = merged(lane < kWarps ? sm.warp[lane] : Sums{-INFINITY, 0.f, 0.f, 0}, k);
        const unsigned long long lo = __float_as_uint(all.m) | (unsigned long long)(unsigned)all.n << 32;
        const unsigned long long hi = __float_as_uint(all.t) | (unsigned long long)__float_as_uint(all.s) << 32;
        if (lane < 2) {
            if (ctas > 1) store_cluster(&sm.sums[rank][lane], 0, lane ? hi : lo);
            else sm.sums[0][lane] = lane ? hi : lo;
        }
    }
    if (a.n_top) {
        // this CTA's largest, in best[0] unless they go to the first CTA
        largest(row, rank, ctas, mine, maxima, a.n_top, sm, sm.best[rank]);
        if (ctas > 1 && rank > 0 && tid < a.n_top) store_cluster(&sm.best[rank][tid], 0, sm.best[rank][tid]);
    }
    if (ctas > 1) {
        cluster_sync();
        if (rank != 0) return;
    }
    __syncthreads();
    if (warp == 0) {
        Sums u{-INFINITY, 0.f, 0.f, 0};
        if (lane < ctas)
            u = Sums{__uint_as_float((unsigned)sm.sums[lane][0]), __uint_as_float((unsigned)sm.sums[lane][1]),
                     __uint_as_float((unsigned)(sm.sums[lane][1] >> 32)), (int)(sm.sums[lane][0] >> 32)};
        const Sums all = merged(u, k);
        // NaN logits are in t, an infinite one is the maximum; a row of -inf alone has no distribution
        const bool empty = all.m == -INFINITY;
        const float log_z = all.n == 1 ? log1pf(all.t) : logf((float)all.n + all.t);
        const bool bad = all.t != all.t || all.m == INFINITY;
        if (lane == 0) {
            sm.bad = bad;
            sm.m = all.m;
            sm.log_z = bad ? __uint_as_float(0x7fc00000u) : empty ? INFINITY : log_z;
        }
        if (a.entropy && lane == 0)
            a.entropy[r] = bad ? __uint_as_float(0x7fc00000u)
                                  : empty ? 0.f : log_z - all.s * kLn2 / ((float)all.n + all.t);
    }
    __syncthreads();
    const float m = sm.m == -INFINITY ? 0.f : sm.m, log_z = sm.log_z;
    if (scores) a.logprobs[(size_t)r * a.n_tokens + tid] = (token_x - m) / a.temperature - log_z;
    if (a.n_top == 0) return;
    // the CTAs' largest against each other
    const int n = ctas * a.n_top;
    for (int i = tid; i < n; i += kThreads) {
        const unsigned long long key = sm.best[i / a.n_top][i % a.n_top];
        if (key == 0ull) continue;
        // each list is in order: how many of it are larger, all lists at once
        int pos[kMaxCluster] = {}, at = 0;
#pragma unroll
        for (int step = kMaxTop; step > 0; step /= 2) {
            if (step > a.n_top) continue;
#pragma unroll
            for (int c = 0; c < kMaxCluster; ++c)
                if (c < ctas && pos[c] + step <= a.n_top && sm.best[c][pos[c] + step - 1] > key) pos[c] += step;
        }
#pragma unroll
        for (int c = 0; c < kMaxCluster; ++c) at += pos[c];
        if (at >= a.n_top) continue;
        const size_t o = (size_t)r * a.n_top + at;
        a.top_ids[o] = sm.bad ? -1 : pair_id(key);
        a.top_logprobs[o] = (order_value((unsigned)(key >> 32)) - m) / a.temperature - log_z;
    }
}

template <typename T>
cudaError_t launch(const LogprobArgs& a, cudaStream_t s) {
    auto kern = logprob_kernel<T>;
    // few rows: as many CTAs a row as are resident at once
    int ctas = 1;
    while (ctas < kMaxCluster && (int64_t)a.rows * ctas * 2 <= kCtas * sm_count() && ctas * 2 * Row<T>::SEG * 4 <= a.vocab) ctas *= 2;
    const int segs = (a.vocab + Row<T>::E - 1 + Row<T>::SEG - 1) / Row<T>::SEG;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)a.rows * ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = sizeof(unsigned) * (((segs + ctas - 1) / ctas + 3) / 4 * 4);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kern, a, ctas);
}

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

}  // namespace

}  // namespace ks

using namespace ks;

extern "C" ks_status ks_token_logprobs(const ks_logprobs* p, void* stream) {
    if (!p) {
        set_error("ks_token_logprobs: null argument");
        return KS_ERR_INVALID_ARG;
    }
    if (p->dtype != KS_DTYPE_F32 && p->dtype != KS_DTYPE_BF16) {
        set_error("ks_token_logprobs: unknown dtype %d", p->dtype);
        return KS_ERR_INVALID_ARG;
    }
    if (p->rows < 0 || p->rows > 1 << 24 || p->vocab < 1) {
        set_error("ks_token_logprobs: %d rows of %d logits", p->rows, p->vocab);
        return KS_ERR_INVALID_ARG;
    }
    if (p->vocab > kMaxVocab || p->n_tokens > kMaxTokens || p->n_top > kMaxTop) {
        set_error("ks_token_logprobs: %d logits, %d tokens, %d alternatives (at most %d, %d, %d)", p->vocab, p->n_tokens,
                  p->n_top, kMaxVocab, kMaxTokens, kMaxTop);
        return KS_ERR_UNSUPPORTED;
    }
    if (p->n_tokens < 0 || p->n_top < 0 || p->n_top > p->vocab) {
        set_error("ks_token_logprobs: %d tokens, %d alternatives of %d", p->n_tokens, p->n_top, p->vocab);
        return KS_ERR_INVALID_ARG;
    }
    if (!std::isfinite(p->temperature) || !(p->temperature > 0.f)) {
        set_error("ks_token_logprobs: the temperature is not a positive number");
        return KS_ERR_INVALID_ARG;
    }
    if (p->rows == 0) return KS_OK;
    const size_t es = p->dtype == KS_DTYPE_BF16 ? 2 : 4;
    if (!p->logits || !aligned(p->logits, es) || (p->rows > 1 && p->row_stride < p->vocab) ||
        p->row_stride < 0 || p->row_stride > (int64_t)1 << 40) {
        set_error("ks_token_logprobs: null or misaligned logits, or a bad stride");
        return KS_ERR_INVALID_ARG;
    }
    if ((p->n_tokens && (!p->tokens || !p->logprobs || !aligned(p->tokens, 4) || !aligned(p->logprobs, 4))) ||
        (p->n_top && (!p->top_ids || !p->top_logprobs || !aligned(p->top_ids, 4) || !aligned(p->top_logprobs, 4))) ||
        !aligned(p->entropy, 4)) {
        set_error("ks_token_logprobs: null or misaligned tokens or results");
        return KS_ERR_INVALID_ARG;
    }
    LogprobArgs a{};
    a.logits = p->logits;
    a.ld = p->row_stride;
    a.rows = p->rows; a.vocab = p->vocab;
    a.n_tokens = p->n_tokens; a.n_top = p->n_top;
    a.temperature = p->temperature;
    a.tokens = p->tokens;
    a.logprobs = p->logprobs; a.entropy = p->entropy;
    a.top_ids = p->top_ids; a.top_logprobs = p->top_logprobs;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = p->dtype == KS_DTYPE_BF16 ? launch<__nv_bfloat16>(a, s) : launch<float>(a, s);
    if (e == cudaSuccess) return KS_OK;
    set_error("ks_token_logprobs: %s", cudaGetErrorString(e));
    return KS_ERR_CUDA;
}
