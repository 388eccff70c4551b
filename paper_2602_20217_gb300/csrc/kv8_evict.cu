// Eviction from the 8-bit paged cache: of each sequence and KV head the first
// and the most recent tokens stay, and of those between the ones with the largest
// scores, in their order, in other pages of the cache.
//
// select: the least kept score by a radix search over the scores' 32 bits, made
// whole numbers in the scores' order, 11, 11 and 10 bits at a time, then one pass
// that numbers what stays: scores above it, and as many equal ones, the earlier
// first, as there is room for.  A cluster of up to eight CTAs takes a sequence's
// head, each a contiguous slice, in registers unless it is longer than 24 scores
// a thread; a warp has neighbouring ones, so that a ballot numbers them.  The CTAs
// add their counts that are not zero to the first one's (reading all of each
// other's counts took 25000 clocks a pass, five times the rest of it).
//
// gather: a warp writes one block of 16 kept tokens.  Their codes come from up to 16
// records with scales of their own; the new block's scale is the smallest power
// of two for their values, as an append of them would choose it, and a code is
// multiplied by a power of two, which rounds only where it becomes subnormal.  A
// token's keys are 16-byte pieces of its record.  Its values are one byte of every
// 16: a lane takes four dims (two of heads of 64), reads their bytes of each record
// that the block's tokens come from once, and has the new record's bytes of its
// dims together without any exchange.  Four warps a block, which wait for each
// other, and 16 reads of each row took 75 us where this takes 48 (24 sequences of
// 300 to 12000 tokens, 8 KV heads of 128, cut to half).
//
// Measured: gather 48 us there, 4 TB/s from DRAM beside L1's line look-ups (a lane
// with neighbouring dims took 55, the next two records in flight the same); 24 us
// for a 64k context cut to a tenth, where every kept token has a record of its own,
// 2.6 KB of 64-byte accesses, 5.7 TB/s.  select 18 us in both: about 12000 clocks of
// fixed steps, counts, sums and cluster barriers (one CTA a head took 89 for the
// 64k context; a batch that fills the GPU gains nothing from clusters).
#include <algorithm>

#include "kv8.cuh"
#include "umma.cuh"

namespace ks {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32, kBins = 2048, kPer = 24, kRound = kThreads * kPer;
constexpr int kCopies = 2;          // of a CTA's bins: scores crowd into few of them
constexpr int kMaxCluster = 8;

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

// Sum over the CTA of the values before this thread's.
KS_DEV int block_before(int v, int* sums) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int u = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int w = __shfl_up_sync(0xffffffffu, u, o);
        if (lane >= o) u += w;
    }
    if (lane == 31) sums[warp] = u;
    __syncthreads();
    const int before = __reduce_add_sync(0xffffffffu, lane < warp ? sums[lane] : 0);
    return before + u - v;
}
KS_DEV void add_cluster(int* p, int rank, int v) {
    asm volatile("red.relaxed.cluster.shared::cluster.add.s32 [%0], %1;" ::"r"(cluster_addr(p, (uint32_t)rank)), "r"(v)
                 : "memory");
}
KS_DEV void store_cluster(int* p, int rank, int v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr(p, (uint32_t)rank)), "r"(v) : "memory");
}

// Grid: a cluster of `ctas` along x per head, sequences along y.
__global__ void __launch_bounds__(kThreads, 2) kv8_select_kernel(const Kv8Args a, const Kv8EvictArgs t, int ctas) {
    __shared__ int bins[kCopies][kBins], all[3][kBins];      // this CTA's counts; the first CTA: everybody's, a pass each
    __shared__ int sums[kWarps], found[3][2];                // per pass: the least key's bits so far, what is left of its bin
    __shared__ int counts[kMaxCluster][2], in_warp[kWarps][2];       // scores that stay for sure, and equal ones
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int h = blockIdx.x / ctas, rank = blockIdx.x % ctas, s = blockIdx.y;
    grid_dependency_wait();
    grid_launch_dependents();
    const Stay w(a, t, s);
    if (blockIdx.x == 0 && tid == 0) {
        const int len = a.lengths[s], keep = t.keep[s];
        if (len < 0 || len > a.capacity || keep < 0 || min(keep, len) > t.new_capacity) kv8_flag(a, kKv8BadBatch);
        t.new_lengths[s] = w.n;
    }
    const float* score = t.scores + ((size_t)s * a.hk + h) * t.ld;
    int32_t* kept = t.kept + ((size_t)s * a.hk + h) * t.kept_ld;
    float* out = t.new_scores ? t.new_scores + ((size_t)s * a.hk + h) * t.new_ld : nullptr;
    if (w.n == w.len) {                              // the whole cluster
        for (int i = rank * kThreads + tid; i < w.n; i += ctas * kThreads) {
            kept[i] = i;
            if (out) out[i] = score[i];
        }
        return;
    }
    const int lo = w.first, hi = w.len - w.recent, most = w.n - w.first - w.recent;      // most of [lo, hi) stay
    const unsigned below = (1u << lane) - 1;
    if (w.len <= kThreads) {
        // a token a thread, ranked against all between: 1000 clocks where the passes' fixed steps take 12000
        if (rank > 0) return;
        const bool inside = tid >= lo && tid < hi;
        const float mine = tid < w.len && (inside || out) ? score[tid] : 0.f;
        const unsigned key = inside ? score_key(mine) : 0u;
        unsigned* keys = reinterpret_cast<unsigned*>(bins[0]);
        keys[tid] = key;
        __syncthreads();
        int before = 0;
        for (int i = lo; i < hi; ++i) before += keys[i] > key || (keys[i] == key && i < tid);
        const bool stays = tid < w.len && (!inside || before < most);
        const unsigned staying = __ballot_sync(0xffffffffu, stays);
        if (lane == 0) sums[warp] = __popc(staying);
        __syncthreads();
        const int o = __reduce_add_sync(0xffffffffu, lane < warp ? sums[lane] : 0) + __popc(staying & below);
        if (stays) {
            kept[o] = tid;
            if (out) out[o] = mine;
        }
        return;
    }
    const int slice = (w.len + ctas - 1) / ctas, begin = rank * slice, end = min(w.len, begin + slice);
    const int rounds = max(0, end - begin + kRound - 1) / kRound;
    // this thread's scores of a round: as many in each round as it takes, in whole threes (looked at one by one 1 us more),
    // so that short slices do not pay for the longest
    const int per = rounds ? min(kPer, ((end - begin + rounds * kThreads - 1) / (rounds * kThreads) + 2) / 3 * 3) : 0;
    float v[kPer];
    auto place = [&](int round, int e) { return begin + ((round * kWarps + warp) * per + e) * 32 + lane; };
    auto load = [&](int round) {
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            if (e % 3 == 0 && e >= per) break;
            v[e] = place(round, e) < end ? score[place(round, e)] : 0.f;
        }
    };
    if (rounds > 0) load(0);
    for (int i = tid; i < kCopies * kBins; i += kThreads) bins[0][i] = 0;
    for (int i = tid; i < 3 * kBins; i += kThreads) all[0][i] = 0;
    if (ctas > 1) cluster_sync();
    else __syncthreads();
    // the least key that stays, and how many of those equal to it
    unsigned prefix = 0;
    int left = most;
    if (most > 0) {
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11;
            const unsigned above = pass == 0 ? 0u : 0xffffffffu << (shift + width);
            for (int round = 0; round < rounds; ++round) {
                if (rounds > 1) load(round);
#pragma unroll
                for (int e = 0; e < kPer; ++e) {
                    if (e % 3 == 0 && e >= per) break;
                    const unsigned k = score_key(v[e]);
                    const int i = place(round, e);
                    if (i >= lo && i < min(hi, end) && (k & above) == prefix)
                        atomicAdd(&bins[lane % kCopies][k >> shift & ((1u << width) - 1)], 1);
                }
            }
            __syncthreads();
            for (int i = tid; i < kBins; i += kThreads) {
                const int c = bins[0][i] + bins[1][i];
                bins[0][i] = bins[1][i] = 0;
                if (ctas == 1) all[pass][i] = c;
                else if (c) add_cluster(&all[pass][i], 0, c);
            }
            if (ctas > 1) cluster_sync();
            else __syncthreads();
            if (rank == 0) {
                // bins from the largest down, four a thread: the one in which the count passes what is left
                constexpr int OWN = kBins / kThreads;
                const int b0 = (1 << width) - 1 - OWN * tid;
                int c[OWN] = {}, mine = 0;
                if (b0 > 0)
#pragma unroll
                    for (int e = 0; e < OWN; ++e) c[e] = all[pass][b0 - e];
#pragma unroll
                for (int e = 0; e < OWN; ++e) mine += c[e];
                int before = block_before(mine, sums);
                if (before < left && before + mine >= left) {
                    int e = 0;
#pragma unroll
                    for (int i = 0; i < OWN - 1; ++i)
                        if (e == i && before + c[i] < left) {
                            before += c[i];
                            ++e;
                        }
                    for (int r = 0; r < ctas; ++r) {
                        store_cluster(&found[pass][0], r, (int)(prefix | (unsigned)(b0 - e) << shift));
                        store_cluster(&found[pass][1], r, left - before);
                    }
                }
            }
            if (ctas > 1) cluster_sync();
            else __syncthreads();
            prefix = (unsigned)found[pass][0];
            left = found[pass][1];
        }
    }
    // whether a score stays for sure, and whether it is equal to the least one that stays
    auto mark = [&](int round, int e, bool& sure, bool& equal) {
        const int i = place(round, e);
        const unsigned k = score_key(v[e]);
        const bool inside = i >= lo && i < hi;
        sure = i < end && (!inside || (most > 0 && k > prefix));
        equal = i < end && inside && most > 0 && k == prefix;
    };
    int ties = 0, done = 0;                          // equal ones, and kept ones, before
    if (ctas > 1) {
        int n_sure = 0, n_equal = 0;
        for (int round = 0; round < rounds; ++round) {
            if (rounds > 1) load(round);
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                if (e % 3 == 0 && e >= per) break;
                bool sure, equal;
                mark(round, e, sure, equal);
                n_sure += sure;
                n_equal += equal;
            }
        }
        n_sure = __reduce_add_sync(0xffffffffu, n_sure);
        n_equal = __reduce_add_sync(0xffffffffu, n_equal);
        if (lane == 0) {
            in_warp[warp][0] = n_sure;
            in_warp[warp][1] = n_equal;
        }
        __syncthreads();
        if (tid < 2 * ctas) {                        // to CTA tid / 2
            int n = 0;
            for (int i = 0; i < kWarps; ++i) n += in_warp[i][tid % 2];
            store_cluster(&counts[rank][tid % 2], tid / 2, n);
        }
        cluster_sync();
        for (int r = 0; r < rank; ++r) {
            done += counts[r][0] + min(counts[r][1], max(left - ties, 0));
            ties += counts[r][1];
        }
    }
    for (int round = 0; round < rounds; ++round) {
        if (rounds > 1) load(round);
        int n_sure = 0, n_equal = 0;                 // of the warp's
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            if (e % 3 == 0 && e >= per) break;
            bool sure, equal;
            mark(round, e, sure, equal);
            n_sure += sure;
            n_equal += equal;
        }
        n_sure = __reduce_add_sync(0xffffffffu, n_sure);
        n_equal = __reduce_add_sync(0xffffffffu, n_equal);
        __syncthreads();                             // the counts of the round before are read
        if (lane == 0) {
            in_warp[warp][0] = n_sure;
            in_warp[warp][1] = n_equal;
        }
        __syncthreads();
        int o = done, tie = ties;                    // before this warp
        for (int i = 0; i < kWarps; ++i) {
            const int n = in_warp[i][0], q = in_warp[i][1], taken = min(q, max(left - ties, 0));
            if (i < warp) {
                o += n + taken;
                tie += q;
            }
            done += n + taken;
            ties += q;
        }
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            if (e % 3 == 0 && e >= per) break;
            const int rest = max(left - tie, 0);     // equal ones that there is still room for: the first of them
            bool sure, equal;
            mark(round, e, sure, equal);
            const unsigned equals = __ballot_sync(0xffffffffu, equal);
            const bool stays = sure || (equal && __popc(equals & below) < rest);
            const unsigned staying = __ballot_sync(0xffffffffu, stays);
            if (stays) {
                const int to = o + __popc(staying & below);
                kept[to] = place(round, e);
                if (out) out[to] = v[e];
            }
            o += __popc(staying);
            tie += __popc(equals);
        }
    }
    if (ctas > 1) cluster_sync();                    // nobody leaves before what it is sent has arrived
}

// A power of two f <= 2^18 as two factors of f16; below 2^-24 a code times f rounds to 0 anyway.
KS_DEV void two_factors(float f, __half& a, __half& b) {
    f = fmaxf(f, 1.f / 16777216.f);
    const float first = fminf(fmaxf(f, 1.f / 4096.f), 512.f);
    a = __float2half_rn(first);
    b = __float2half_rn(f * inverse_pow2(first));
}
KS_DEV uint32_t scaled(uint32_t halves, __half2 a, __half2 b) {
    const __half2 x = __hmul2(__hmul2(*reinterpret_cast<const __half2*>(&halves), a), b);
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(*reinterpret_cast<const uint32_t*>(&x)));
    return r;
}
KS_DEV uint32_t halves_of(uint32_t codes) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)codes));
    return h;
}

constexpr int kGatherWarps = 4;

template <int HD>
__global__ void __launch_bounds__(32 * kGatherWarps) kv8_gather_kernel(const Kv8Args a, const Kv8EvictArgs t) {
    constexpr int REC = kv8_record(HD), CODES = kKv8Block * HD, D = HD / 32, PARTS = HD / 16;    // D: dims, and pieces, of a lane
    constexpr unsigned ALL = 0xffffffffu;
    const int lane = threadIdx.x & 31, b = blockIdx.x * kGatherWarps + (threadIdx.x >> 5), h = blockIdx.y, s = blockIdx.z;
    grid_dependency_wait();
    grid_launch_dependents();
    const Stay w(a, t, s);
    if (b * kKv8Block >= w.n) return;
    // lanes 0..15: the block's tokens
    const int at = b * kKv8Block + lane;
    int place = -1;
    if (lane < kKv8Block && at < w.n) place = t.kept[((size_t)s * a.hk + h) * t.kept_ld + at];
    const int page = t.new_table[(size_t)s * t.new_table_ld + b / a.bpp];
    unsigned char* to = nullptr;
    if (page >= 0 && page < a.n_pages) to = a.data + (((size_t)page * a.hk + h) * a.bpp + b % a.bpp) * REC;
    else if (lane == 0) kv8_flag(a, kKv8BadPage);
    // a sequence that keeps all of its tokens may keep its pages
    if (to == nullptr || (w.n == w.len && to == kv8_record_at(a, s, b, h, REC))) return;
    const int block = place < 0 ? -1 : place / kKv8Block, token = place & (kKv8Block - 1);
    const unsigned char* rec = nullptr;              // null: no such page, read as zeros, or no token
    float2 scale = make_float2(0.f, 0.f);
    if (block >= 0) {
        rec = kv8_record_at(a, s, block, h, REC);
        if (rec) scale = *reinterpret_cast<const float2*>(rec + 2 * CODES);
        else kv8_flag(a, kKv8BadPage);
    }
    const unsigned there = __ballot_sync(ALL, rec != nullptr);
    const int before = __shfl_up_sync(ALL, block, 1);
    const unsigned fresh = __ballot_sync(ALL, rec != nullptr && (lane == 0 || block != before));
    auto rec_of = [&](int j) {
        return reinterpret_cast<const unsigned char*>(__shfl_sync(ALL, reinterpret_cast<unsigned long long>(rec), j));
    };
    // values of dims lane, lane + 32 ..: 16 bytes each, of a record at a time, the next one's on their way
    uint4 row[D], next[D];
    uint32_t v[D][4];
#pragma unroll
    for (int i = 0; i < D; ++i) {
        row[i] = next[i] = make_uint4(0, 0, 0, 0);
        v[i][0] = v[i][1] = v[i][2] = v[i][3] = 0;
    }
    auto fetch = [&](int j) {                        // of the j-th token's record
        const unsigned char* of = rec_of(j & 31) + CODES + lane * 16;
#pragma unroll
        for (int i = 0; i < D; ++i) next[i] = *reinterpret_cast<const uint4*>(of + 512 * i);
    };
    unsigned rest = fresh;
    if (rest) fetch(__ffs(rest) - 1);
    // pieces of keys: token (lane + 32 i) / PARTS, dims 16 ((lane + 32 i) % PARTS) ..
    uint4 k[D];
#pragma unroll
    for (int i = 0; i < D; ++i) {
        const int p = lane + 32 * i;
        const unsigned char* of = rec_of(p / PARTS);
        const int from = __shfl_sync(ALL, token, p / PARTS);
        k[i] = make_uint4(0, 0, 0, 0);
        if (of) k[i] = *reinterpret_cast<const uint4*>(of + k_byte<HD>(from, 16 * (p % PARTS)));
    }
    // the largest values: NaN is passed over, infinities there are none
    float k_top = 0.f;
#pragma unroll
    for (int i = 0; i < D; ++i) {
        const uint32_t w4[4] = {k[i].x, k[i].y, k[i].z, k[i].w};
        __half2 m = __half2(0.f, 0.f);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t x = halves_of(w4[e / 2] >> 16 * (e & 1));
            m = __hmax2(m, __habs2(*reinterpret_cast<const __half2*>(&x)));
        }
        // one scale a token
        k_top = fmaxf(k_top, fmaxf(__low2float(m), __high2float(m)) * __shfl_sync(ALL, scale.x, (lane + 32 * i) / PARTS));
    }
    k_top = warp_max(k_top);
    const float ks = scale_for(k_top);
    // lanes 0..15: both factors of a token; one past 2^18 only where all codes are zeros
    auto factors = [&](float from, float to_scale) {
        __half x, y;
        two_factors(fminf(from * inverse_pow2(to_scale), 262144.f), x, y);
        return __half2(x, y);
    };
    const __half2 kf = factors(scale.x, ks);
#pragma unroll
    for (int i = 0; i < D; ++i) {
        const int p = lane + 32 * i;
        const uint32_t f = __shfl_sync(ALL, *reinterpret_cast<const uint32_t*>(&kf), p / PARTS);
        const __half2 both = *reinterpret_cast<const __half2*>(&f), f0 = __low2half2(both), f1 = __high2half2(both);
        const uint32_t w4[4] = {k[i].x, k[i].y, k[i].z, k[i].w};
        uint32_t c[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = scaled(halves_of(w4[e]), f0, f1) | scaled(halves_of(w4[e] >> 16), f0, f1) << 16;
        *reinterpret_cast<uint4*>(to + k_byte<HD>(p / PARTS, 16 * (p % PARTS))) = make_uint4(c[0], c[1], c[2], c[3]);
    }
#pragma unroll
    for (int j = 0; j < kKv8Block; ++j) {
        if (fresh >> j & 1) {
#pragma unroll
            for (int i = 0; i < D; ++i) row[i] = next[i];
            rest &= rest - 1;
            if (rest) fetch(__ffs(rest) - 1);
        }
        if (there >> j & 1) {
            const int byte = v_byte(__shfl_sync(ALL, token, j));
            const int word = (j & 7) >> 1, place_of = 2 * (j >> 3) + (j & 1);        // where token j goes
#pragma unroll
            for (int i = 0; i < D; ++i) {
                const uint32_t lo = __byte_perm(row[i].x, row[i].y, byte & 7), hi = __byte_perm(row[i].z, row[i].w, byte & 7);
                v[i][word] |= ((byte & 8 ? hi : lo) & 0xffu) << 8 * place_of;
            }
        }
    }
    float v_top = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {                    // tokens 2 w, 2 w + 1 of word w, then 8 + 2 w, 9 + 2 w
        const int t0 = 8 * (e & 1) + 2 * (e / 2);
        const float s0 = __shfl_sync(ALL, scale.y, t0), s1 = __shfl_sync(ALL, scale.y, t0 + 1);
        __half2 m = __half2(0.f, 0.f);               // over the lane's dims, a token each
#pragma unroll
        for (int i = 0; i < D; ++i) {
            const uint32_t x = halves_of(v[i][e / 2] >> 16 * (e & 1));
            m = __hmax2(m, __habs2(*reinterpret_cast<const __half2*>(&x)));
        }
        v_top = fmaxf(v_top, fmaxf(__low2float(m) * s0, __high2float(m) * s1));
    }
    v_top = warp_max(v_top);
    const float vs = scale_for(v_top);
    const __half2 vf = factors(scale.y, vs);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int t0 = 8 * (e & 1) + 2 * (e / 2);
        const uint32_t x = __shfl_sync(ALL, *reinterpret_cast<const uint32_t*>(&vf), t0),
                       y = __shfl_sync(ALL, *reinterpret_cast<const uint32_t*>(&vf), t0 + 1);
        const uint32_t g0 = __byte_perm(x, y, 0x5410), g1 = __byte_perm(x, y, 0x7632);
        const __half2 f0 = *reinterpret_cast<const __half2*>(&g0), f1 = *reinterpret_cast<const __half2*>(&g1);
#pragma unroll
        for (int i = 0; i < D; ++i) {
            const uint32_t c = scaled(halves_of(v[i][e / 2] >> 16 * (e & 1)), f0, f1);
            v[i][e / 2] = e & 1 ? __byte_perm(v[i][e / 2], c, 0x5410) : __byte_perm(v[i][e / 2], c, 0x3254);
        }
    }
#pragma unroll
    for (int i = 0; i < D; ++i)
        *reinterpret_cast<uint4*>(to + CODES + lane * 16 + 512 * i) = make_uint4(v[i][0], v[i][1], v[i][2], v[i][3]);
    if (lane == 0) *reinterpret_cast<float2*>(to + 2 * CODES) = make_float2(ks, vs);
}

// CTAs of a head: no more than a round of scores needs, nor than fill the GPU.
cudaError_t launch_select(const Kv8Args& a, const Kv8EvictArgs& t, cudaStream_t s) {
    int ctas = 1;
    while (ctas < kMaxCluster && (int64_t)ctas * kRound < a.capacity && a.hk * a.n_seqs * ctas < sm_count()) ctas *= 2;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(a.hk * ctas, a.n_seqs);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kv8_select_kernel, a, t, ctas);
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
        e = launch_select(b, u, s);
        if (e != cudaSuccess) return e;
        const int blocks = t.new_capacity / kKv8Block;
        const dim3 grid((blocks + kGatherWarps - 1) / kGatherWarps, a.hk, b.n_seqs);
        e = a.hd == 128 ? launch_kv8(kv8_gather_kernel<128>, grid, 32 * kGatherWarps, 0, s, b, u)
                        : launch_kv8(kv8_gather_kernel<64>, grid, 32 * kGatherWarps, 0, s, b, u);
    }
    return e;
}

}  // namespace ks
