// The weights that tokens of the 8-bit paged cache receive (see kv8_weights.cu)
// from many query rows, on tcgen05: prompts, and windows of their last rows.
//
// S (128 keys x 128 queries) = K Q^T by kind::f16 in bf16: queries as they are, by
// TMA from the caller's rows, and keys converted once per tile, code times block
// scale, which bf16 holds exactly.  Keys are the rows: a thread of the softmax
// warps has one key, its weights are 2^(c s - lse2) over the columns, and their
// sum never leaves the thread.  So there is nothing to exchange between threads,
// no maximum, and the only operand beside the scores is a column's lse.
//
// A CTA holds 512 keys (128 KB), four tiles with an S in TMEM each,
// so that a chunk of queries, 32 KB from L2, is used 65536 times: at 128 keys the
// chunks alone would ask L2 for 18 TB/s.  One warp copies chunks, one issues the
// products.  A unit is (sequence, KV head, 512 keys), as long as it has chunks of
// queries that see it; the line of all units is cut into equal runs of chunks,
// one a CTA, and units in several runs leave sums that a second launch adds up in
// the runs' order: the same bits from call to call.
//
// Measured: 2001 rows over 8150 tokens, 32 heads over 8 of 128, 104 us, 1.13 PFLOP/s;
// 64 rows over 32768 tokens, 64 heads, 47.5 us.  A tile's products take 705 clocks
// (513 would be the rate: their operands are all of shared memory's bandwidth, and
// the sums that the softmax reads are there too), its 16384 exponentials 512, both
// together about 880; a unit's keys take 4 to 6 thousand clocks, which the 64 rows
// pay after every fourth chunk.  Five of the 18 warps share a scheduler, so a thread
// has 96 registers, and the compiler spills 94 bytes of it.  Tried: keys as the operand in TMEM, 513 clocks, but
// room for two S only, 122 and 47.6 us (N = 64 for four S: 217 and 77); the
// groups' exponentials in turns 116 and 50; sums read once for two tiles 141 and 50;
// the issuing loop unrolled 109 and 50 (its code is waited for).
#include <algorithm>
#include <type_traits>

#include "kv8_plan.cuh"
#include "umma.cuh"

namespace ks {

namespace {

constexpr int kTiles = 4, kTile = 128, kUnit = kTiles * kTile;     // keys
constexpr int kSoftmaxWarps = 4 * kTiles, kProductWarp = kSoftmaxWarps, kCopyWarp = kProductWarp + 1;
constexpr int kThreads = 32 * (kSoftmaxWarps + 2);
constexpr int kQueries = 128, kRing = 3, kSums = 5;
constexpr int kUnitCost = 2;            // a unit's keys, in the time of chunks: 1, 2 and 3 take 105.0, 104.1, 104.9 us

struct WeightsPlan {
    int G, tq;              // query heads a KV head; tokens of a chunk
    int block_log;          // blocks of a page, -1: no power of two
    int ctas;
    float* part;            // [2 ctas][kUnit]
    int4* desc;             // [ctas]: the unit that begins in this CTA's run and ends in a later one's: sequence, KV head,
                            // 512 keys, last CTA (-1: no such unit)
    KS_DEV int page_of(int block, int bpp) const { return block_log >= 0 ? block >> block_log : block / bpp; }
};

template <int HD>
struct Smem {
    unsigned char q[kRing][kQueries * HD * 2];  // [HD / 64][query][64], 128-byte swizzle
    unsigned char k[kTiles][kTile * HD * 2];    // [key / 8][HD / 8][8][8]
    float lse[kSums][kQueries];                 // minus the sums' logarithms, base 2
    uint64_t q_full[kRing], q_free[kRing], k_full[kTiles], s_full[kTiles], s_free[kTiles];
    uint32_t tmem;
};

KS_DEV int units_of(const Kv8Seq& q) { return q.rows > 0 ? (q.len + kUnit - 1) / kUnit : 0; }
KS_DEV int chunks_of(const Kv8Seq& q, const WeightsPlan& p) { return (q.rows + p.tq - 1) / p.tq; }
// The first chunk with a row that sees keys of unit u.
KS_DEV int first_chunk(const Kv8Seq& q, const WeightsPlan& p, int u) { return max(0, u * kUnit - (q.len - q.rows)) / p.tq; }
// What the units of one head take on the line.
KS_DEV int64_t head_length(const Kv8Seq& q, const WeightsPlan& p) {
    const int units = units_of(q), chunks = chunks_of(q, p), before = q.len - q.rows;
    const int all = min(units, before < 0 ? 0 : before / kUnit + 1);     // units that every chunk sees
    int64_t n = (int64_t)all * (kUnitCost + chunks);
    for (int u = all; u < units; ++u) n += kUnitCost + chunks - first_chunk(q, p, u);
    return n;
}

// Chunks [c, end) of a unit.
struct Segment {
    int s, h, u, c, end, c0, chunks;
    int64_t start;          // the unit's place on the line
    Kv8Seq q;
    KS_DEV void at(int64_t x0, int64_t x1, const WeightsPlan& p) {
        chunks = chunks_of(q, p);
        c0 = first_chunk(q, p, u);
        const int64_t first = start + kUnitCost - c0;            // of chunk 0
        c = (int)max((int64_t)c0, x0 - first);
        end = (int)min((int64_t)chunks, x1 - first);
    }
    KS_DEV int64_t past() const { return start + kUnitCost + chunks - c0; }
    KS_DEV bool next(const Kv8Args& a, int64_t x0, int64_t x1, const WeightsPlan& p) {
        start = past();
        if (start + kUnitCost >= x1) return false;
        if (++u >= units_of(q)) {
            u = 0;
            if (++h >= a.hk) {
                h = 0;
                do {
                    if (++s >= a.n_seqs) return false;
                    q = kv8_seq(a, s);
                } while (units_of(q) == 0);
            }
        }
        at(x0, x1, p);
        return true;
    }
};

KS_DEV int64_t shfl64(int64_t v, int i) { return (int64_t)__shfl_sync(0xffffffffu, (long long)v, i); }

// The line of all units, cut into equal runs.
struct Line {
    int64_t each, more, x0, x1;
    int ctas;
    KS_DEV int cta_of(int64_t x) const {
        const int64_t b = more * (each + 1);
        return (int)(x < b ? x / (each + 1) : more + (x - b) / each);
    }
};

// This CTA's run and its first segment; false if it has none.
KS_DEV bool find(const Kv8Args& a, const WeightsPlan& p, Line& l, Segment& k) {
    const int lane = threadIdx.x & 31, cta = blockIdx.x;
    Kv8Seq mine{};
    int64_t head = 0;
    bool falls = false;
    auto load = [&](int c) -> int64_t {
        const int s = c + lane;
        mine = Kv8Seq{};
        head = 0;
        if (s >= a.n_seqs) return 0;
        mine = kv8_seq(a, s);
        falls |= a.offsets[s + 1] < a.offsets[s];
        head = head_length(mine, p);
        return a.hk * head;
    };
    int64_t total = 0, v = 0;
    for (int c = 0; c < a.n_seqs; c += 32) {
        v = load(c);
        if (cta == 0 && c + lane < a.n_seqs && kv8_seq_bad(a, c + lane)) kv8_flag(a, kKv8BadBatch);
        int64_t u = v;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) u += (int64_t)__shfl_xor_sync(0xffffffffu, (long long)u, o);
        total += u;
    }
    if (__any_sync(0xffffffffu, falls)) return false;
    l.ctas = (int)min((int64_t)p.ctas, total);
    l.each = l.ctas ? total / l.ctas : 0;
    l.more = total - l.each * l.ctas;
    l.x0 = cta * l.each + min((int64_t)cta, l.more);
    l.x1 = l.x0 + l.each + (cta < l.more);
    if (cta >= l.ctas) return false;
    int64_t start = 0, len = 0;
    for (int c = 0;; c += 32) {
        if (c >= a.n_seqs) return false;             // not with arrays that stay what they are
        if (a.n_seqs > 32) v = load(c);
        int64_t u = v;                               // inclusive sums
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t w = (int64_t)__shfl_up_sync(0xffffffffu, (long long)u, o);
            if (lane >= o) u += w;
        }
        const unsigned past = __ballot_sync(0xffffffffu, start + u > l.x0);
        if (past) {
            const int i = __ffs(past) - 1;
            k.s = c + i;
            k.q.row0 = __shfl_sync(0xffffffffu, mine.row0, i);
            k.q.rows = __shfl_sync(0xffffffffu, mine.rows, i);
            k.q.len = __shfl_sync(0xffffffffu, mine.len, i);
            len = shfl64(head, i);
            start += shfl64(u - v, i);
            break;
        }
        start += shfl64(u, 31);
    }
    k.h = (int)((l.x0 - start) / len);
    k.start = start + k.h * len;
    // units that every chunk sees are equally long
    const int before = k.q.len - k.q.rows, all = min(units_of(k.q), before < 0 ? 0 : before / kUnit + 1);
    const int64_t one = kUnitCost + chunks_of(k.q, p);
    k.u = (int)min((int64_t)all, (l.x0 - k.start) / one);
    k.start += k.u * one;
    for (;; ++k.u) {
        if (k.u >= units_of(k.q)) return false;      // not with arrays that stay what they are
        k.at(l.x0, l.x1, p);
        if (l.x0 < k.past()) break;
        k.start = k.past();
    }
    // a run that ends before the unit's first chunk has nothing to do
    return k.end > k.c;
}

// Weights of a key that is written: of what was there before, and what it has received.
KS_DEV void put(const Kv8Args& a, const Kv8WeightArgs& t, const Kv8Seq& q, int s, int h, int key, float v) {
    if (key >= q.len) return;
    const size_t o = ((size_t)s * a.hk + h) * t.ld + key;
    if (t.decay != 0.f && key < q.len - q.rows) v = fmaf(t.decay, t.scores[o], v);
    t.out[o] = v;
}

template <int HD>
__global__ void __launch_bounds__(kThreads, 1)
    kv8_weights_tc_kernel(const Kv8Args a, const Kv8WeightArgs t, const WeightsPlan p, const __grid_constant__ CUtensorMap map) {
    constexpr int REC = kv8_record(HD);
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    Smem<HD>& sm = *reinterpret_cast<Smem<HD>*>(smem_raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (warp == kProductWarp) tmem_alloc<1>(&sm.tmem, 512);
    if (tid == 0) {
        for (int i = 0; i < kRing; ++i) {
            mbar_init(&sm.q_full[i], 1);
            mbar_init(&sm.q_free[i], 1);
        }
        for (int i = 0; i < kTiles; ++i) {
            mbar_init(&sm.k_full[i], 4);
            mbar_init(&sm.s_full[i], 2);        // the products' commit, and an arrival that orders the sums before it
            mbar_init(&sm.s_free[i], 8);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // queries that no chunk has: no NaN may come from there
    for (int i = tid; i < kRing * (HD / 64) * (kQueries - p.tq * p.G) * 8; i += kThreads) {
        const int each = (kQueries - p.tq * p.G) * 8, part = i / each;
        reinterpret_cast<uint4*>(sm.q[0])[(part * kQueries + p.tq * p.G) * 8 + i - part * each] = make_uint4(0, 0, 0, 0);
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    umma_fence_before();
    __syncthreads();
    umma_fence_after();
    const uint32_t tmem = sm.tmem;
    grid_dependency_wait();
    grid_launch_dependents();
    Line line;
    Segment at;
    const bool work = find(a, p, line, at);
    if (!work && tid == 0) p.desc[blockIdx.x] = make_int4(0, 0, 0, -1);
    // queries of a chunk
    auto columns = [&](const Segment& k, int c) { return min(p.tq, k.q.rows - c * p.tq) * p.G; };

    if (!work) {
        // nothing in this run
    } else if (warp == kCopyWarp) {
        bool alive = true;
        int it = 0;
        // four sums a lane, read a chunk ahead
        auto sums = [&](const Segment& k, int c, float (&x)[4]) {
            const int n = columns(k, c);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = 32 * i + lane, tok = j / p.G;
                x[i] = j < n ? t.lse[(size_t)(k.q.row0 + c * p.tq + tok) * t.hq + k.h * p.G + j - tok * p.G] : -INFINITY;
            }
        };
        float x[4];
        sums(at, at.c, x);
        bool more = true;
        while (more && alive) {
            const Segment k = at;
            more = at.next(a, line.x0, line.x1, p);
            for (int c = k.c; c < k.end; ++c, ++it) {
                const int st = it % kRing;
                float next[4] = {};
                if (c + 1 < k.end) sums(k, c + 1, next);
                else if (more) sums(at, at.c, next);
                alive = mbar_wait(&sm.q_free[st], ((it / kRing) & 1) ^ 1, kWaitLimitNs);
                if (!__all_sync(0xffffffffu, alive)) {
                    alive = false;
                    break;
                }
                // the products of chunk it - kRing waited until the scores of the chunk before were in registers, so
                // the weights of the one before that, which had this place, are done
                static_assert(kSums == kRing + 2, "sums outlive their queries by two chunks");
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sm.lse[it % kSums][32 * i + lane] = x[i] == -INFINITY ? -INFINITY : -x[i] * kLog2e;    // no weight
                    x[i] = next[i];
                }
                __syncwarp();
                if (lane == 0) {
                    mbar_expect_tx(&sm.q_full[st], p.tq * p.G * HD * 2);
                    for (int i = 0; i < HD / 64; ++i)
                        tma_3d(sm.q[st] + i * (kQueries * 128), &map, 64 * i, k.h * p.G, k.q.row0 + c * p.tq, &sm.q_full[st]);
                }
                __syncwarp();
            }
        }
        if (!alive && lane == 0) kv8_flag(a, kKv8Timeout);
        // no copy may be in flight when the CTA ends
        for (int i = max(0, it - kRing); i < it; ++i) mbar_wait(&sm.q_full[i % kRing], (i / kRing) & 1, kWaitLimitNs);
    } else if (warp == kProductWarp) {
        if (lane == 0) {
            bool ok = true;
            int it = 0, seg = 0;
            do {
                for (int c = at.c; c < at.end && ok; ++c, ++it) {
                    const int st = it % kRing;
                    ok = mbar_wait(&sm.q_full[st], (it / kRing) & 1, kWaitLimitNs);
                    const int n = columns(at, c);        // a whole chunk's columns behind them are zeros
                    const uint32_t idesc = umma_idesc(kTile, n == p.tq * p.G ? kQueries : (n + 15) / 16 * 16, false);
                    for (int i = 0; i < kTiles && ok; ++i) {
                        if (c == at.c) ok = mbar_wait(&sm.k_full[i], seg & 1, kWaitLimitNs);
                        ok = ok && mbar_wait(&sm.s_free[i], (it & 1) ^ 1, kWaitLimitNs);
                        if (!ok) break;
                        umma_fence_after();
                        const uint64_t ka = (uint64_t)((smem_u32(sm.k[i]) & 0x3FFFFu) >> 4) | (uint64_t)(128 >> 4) << 16 |
                                            (uint64_t)(HD * 16 >> 4) << 32 | 1ull << 46;         // without a swizzle
                        const uint64_t qb = umma_desc(smem_u32(sm.q[st]), 16, 1024);
#pragma unroll
                        for (int j = 0; j < HD / 16; ++j)
                            umma_ss<1>(tmem + kQueries * i, ka + 16 * j, qb + (j / 4 * (kQueries * 128) + j % 4 * 32) / 16, idesc,
                                       j > 0);
                        umma_commit(&sm.s_full[i]);
                        mbar_arrive(&sm.s_full[i]);
                    }
                    umma_commit(&sm.q_free[st]);
                }
                ++seg;
            } while (ok && at.next(a, line.x0, line.x1, p));
            if (!ok) kv8_flag(a, kKv8Timeout);
        }
        __syncwarp();
    } else {
        // Warps 0..7 take tiles 0 and 2, the others 1 and 3; four of the eight have the first 64 columns of a tile's
        // scores, four the others: a tile's scores are used up in half the time that four warps take, which is what
        // its next products wait for.
        const int group = warp >> 3, half = warp >> 2 & 1, row = (warp & 3) * 32 + lane;
        const int i = group + 2 * half;                                  // tile whose key this thread converts
        const uint32_t lanes = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
        const float c2 = t.scale * kLog2e;
        bool alive = true, began = false;
        int it = 0;
        // A unit's key of this thread; its page is looked up a unit ahead.
        auto look = [&](const Segment& k) {          // -1: no such key, -2: no such page
            const int key = k.u * kUnit + i * kTile + row;
            if (key >= k.q.len) return -1;
            const int page = a.table[(size_t)k.s * a.table_ld + p.page_of(key / kKv8Block, a.bpp)];
            return page < 0 ? -2 : page;
        };
        int page = look(at);
        for (;;) {
            const int key = at.u * kUnit + i * kTile + row, pos0 = at.q.len - at.q.rows;
            const bool here = page >= 0 && page < a.n_pages;
            if (!here && page != -1) kv8_flag(a, kKv8BadPage);
            uint4 raw[HD / 16];
            float scale = 0.f;
#pragma unroll
            for (int j = 0; j < HD / 16; ++j) raw[j] = make_uint4(0, 0, 0, 0);
            if (here) {
                const int b = key / kKv8Block, tok = key % kKv8Block;
                const unsigned char* rec =
                    a.data + (((size_t)page * a.hk + at.h) * a.bpp + b - p.page_of(b, a.bpp) * a.bpp) * REC;
                scale = *reinterpret_cast<const float*>(rec + 32 * HD);
#pragma unroll
                for (int j = 0; j < HD / 16; ++j)
                    raw[j] = *reinterpret_cast<const uint4*>(rec + (tok >> 3) * 8 * HD + j * 128 + (tok & 7) * 16);
            }
            // as bf16
            unsigned char* to = sm.k[i] + (row >> 3) * (HD * 16) + (row & 7) * 16;
#pragma unroll
            for (int j = 0; j < HD / 16; ++j) {
                const uint32_t w[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
                uint32_t o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 v = from_e4m3x2((uint16_t)(w[e / 2] >> 16 * (e & 1)));
                    o[e] = pack_bf16(v.x * scale, v.y * scale);
                }
                *reinterpret_cast<uint4*>(to + 256 * j) = make_uint4(o[0], o[1], o[2], o[3]);
                *reinterpret_cast<uint4*>(to + 256 * j + 128) = make_uint4(o[4], o[5], o[6], o[7]);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.k_full[i]);
            {
                Segment next = at;                   // not kept: its registers are the scores'
                page = next.next(a, line.x0, line.x1, p) ? look(next) : -1;
            }
            float sum[2] = {0.f, 0.f};               // tiles group and group + 2
            for (int c = at.c; c < at.end; ++c, ++it) {
                const int n = columns(at, c), tok0 = c * p.tq;
                const float* lse = sm.lse[it % kSums] + 64 * half;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int tile = group + 2 * u, first = at.u * kUnit + tile * kTile + (warp & 3) * 32;       // key of lane 0
                    alive = alive && mbar_wait(&sm.s_full[tile], it & 1, kWaitLimitNs);
                    __syncwarp();
                    umma_fence_after();
                    const bool edge = first + 31 > pos0 + tok0;          // a row of the chunk that does not see a key
                    float2 part[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                    const uint32_t s_at = lanes + kQueries * tile + 64 * half;
                    if (edge || n < p.tq * p.G) {
                        // columns of rows that see this key
                        const int d = max(0, first + lane - pos0 - tok0);
                        const int from = (d >= p.tq ? n : d * p.G) - 64 * half;
                        const int to = first - pos0 - tok0 < p.tq ? min(n - 64 * half, 64) : 0;
#pragma unroll 1
                        for (int j = 0; j < to; j += 32) {
                            const int here_from = from - j, here_to = to - j;
                            uint32_t s[32];
                            tmem_ld32(s, s_at + j);
                            tmem_wait_ld();
                            tmem_pin(s);
#pragma unroll
                            for (int q = 0; q < 32; q += 4) {
                                const float4 l = *reinterpret_cast<const float4*>(&lse[j + q]);
                                const float x[4] = {l.x, l.y, l.z, l.w};
                                float w[4];
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    w[e] = exp2_approx(fmaf(__uint_as_float(s[q + e]), c2, x[e]));
                                    if (q + e < here_from || q + e >= here_to) w[e] = 0.f;
                                }
                                part[0] = __fadd2_rn(part[0], make_float2(w[0], w[1]));
                                part[1] = __fadd2_rn(part[1], make_float2(w[2], w[3]));
                            }
                        }
                        umma_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&sm.s_free[tile]);
                    } else {
                        // the scores go to registers in one piece, and their place to the next products
                        uint32_t s[2][32];
                        tmem_ld32(s[0], s_at);
                        tmem_ld32(s[1], s_at + 32);
                        tmem_wait_ld();
                        tmem_pin(s[0]);
                        tmem_pin(s[1]);
                        umma_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&sm.s_free[tile]);
#pragma unroll
                        for (int q = 0; q < 64; q += 4) {
                            const uint32_t* v = s[q / 32] + q % 32;
                            const float4 l = *reinterpret_cast<const float4*>(&lse[q]);
                            const float2 x = __ffma2_rn(make_float2(__uint_as_float(v[0]), __uint_as_float(v[1])),
                                                  make_float2(c2, c2), make_float2(l.x, l.y));
                            const float2 y = __ffma2_rn(make_float2(__uint_as_float(v[2]), __uint_as_float(v[3])),
                                                  make_float2(c2, c2), make_float2(l.z, l.w));
                            part[0] = __fadd2_rn(part[0], make_float2(exp2_approx(x.x), exp2_approx(x.y)));
                            part[1] = __fadd2_rn(part[1], make_float2(exp2_approx(y.x), exp2_approx(y.y)));
                        }
                    }
                    part[0] = __fadd2_rn(part[0], part[1]);
                    sum[u] += part[0].x + part[0].y;
                }
            }
            // Both halves' sums of a tile meet where its keys were: their products are done.
            auto join = [&](int tile) { return reinterpret_cast<float*>(sm.k[tile]) + row; };
            *join(group + 2 * (half ^ 1)) = half ? sum[0] : sum[1];
            asm volatile("bar.sync %0, 256;" ::"r"(1 + group) : "memory");
            float v = (half ? sum[1] : sum[0]) + *join(i);
            asm volatile("bar.sync %0, 256;" ::"r"(1 + group) : "memory");       // before the next unit's keys
            if (!here) v = 0.f;                      // no such page: unseen
            const bool begins = at.c == at.c0, whole = begins && at.end == at.chunks;
            if (whole) {
                put(a, t, at.q, at.s, at.h, key, v);
            } else {
                p.part[(size_t)(2 * blockIdx.x + begins) * kUnit + i * kTile + row] = v;
                if (begins) {
                    began = true;
                    if (tid == 0) p.desc[blockIdx.x] = make_int4(at.s, at.h, at.u, line.cta_of(at.past() - 1));
                }
            }
            if (!at.next(a, line.x0, line.x1, p)) break;
        }
        if (tid == 0) {
            if (!began) p.desc[blockIdx.x] = make_int4(0, 0, 0, -1);
            if (!alive) kv8_flag(a, kKv8Timeout);
        }
    }
    umma_fence_before();
    __syncthreads();
    if (warp == kProductWarp) {
        umma_fence_after();
        tmem_free<1>(tmem, 512);
    }
}

// CTA x adds up the sums of the unit that begins in run x and ends in a later one.
__global__ void __launch_bounds__(kUnit) kv8_weights_merge_kernel(const Kv8Args a, const Kv8WeightArgs t, const WeightsPlan p) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int4 d = p.desc[blockIdx.x];
    if (d.w < 0) return;
    float v = p.part[(size_t)(2 * blockIdx.x + 1) * kUnit + threadIdx.x];
    for (int c = blockIdx.x + 1; c <= d.w; ++c) v += p.part[(size_t)(2 * c) * kUnit + threadIdx.x];
    put(a, t, kv8_seq(a, d.x), d.x, d.y, d.z * kUnit + threadIdx.x, v);
}

template <int HD>
cudaError_t launch_tc(const Kv8Args& a, const Kv8WeightArgs& t, const WeightsPlan& p, const CUtensorMap& map, cudaStream_t s) {
    auto kern = kv8_weights_tc_kernel<HD>;
    constexpr int bytes = sizeof(Smem<HD>);
    static_assert(bytes <= 227 * 1024, "what a CTA can have");
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    return e != cudaSuccess ? e : launch_kv8(kern, dim3(p.ctas), kThreads, bytes, s, a, t, p, map);
}

}  // namespace

size_t kv8_weights_tc_workspace() {
    return sizeof(int4) * kKv8Sms + sizeof(float) * 2 * kKv8Sms * kUnit;
}

cudaError_t launch_kv8_weights_tc(const Kv8Args& a, const Kv8WeightArgs& t, cudaStream_t s, bool& taken) {
    WeightsPlan p{};
    p.G = t.hq / a.hk;
    p.tq = kQueries / p.G;
    p.block_log = (a.bpp & (a.bpp - 1)) == 0 ? __builtin_ctz(a.bpp) : -1;
    p.ctas = std::min(sm_count(), kKv8Sms);
    p.desc = static_cast<int4*>(t.workspace);
    p.part = reinterpret_cast<float*>(p.desc + kKv8Sms);
    CUtensorMap map;
    taken = make_kv8_query_map(&map, t.q, a.n_rows, t.hq, a.hd, t.q_row, t.q_head, p.G, p.tq);
    if (!taken) return cudaSuccess;
    cudaError_t e = a.hd == 128 ? launch_tc<128>(a, t, p, map, s) : launch_tc<64>(a, t, p, map, s);
    return e != cudaSuccess ? e : launch_kv8(kv8_weights_merge_kernel, dim3(p.ctas), kUnit, 0, s, a, t, p);
}

}  // namespace ks
