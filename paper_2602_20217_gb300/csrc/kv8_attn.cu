// Causal attention over the 8-bit paged cache, any number of rows a sequence.
//
// Work.  A unit is (sequence, KV head, group of rows): a group is as many whole
// tokens as give at most RG query rows (token x query head of the KV head), and
// its keys come in tiles of 128.  The units' tiles, one after the other, are cut
// into equal runs, one per resident CTA, so a long sequence among short ones or
// few heads at a long context keep every SM busy; the lengths are read on the
// device.  A run's part of a unit is a segment.  Units that lie in several runs
// leave (m, l, o) per segment, merged in run order by a second launch; the
// result depends on the batch, never on timing.
//
// A CTA is a producer warp and four consumer warps around a ring of two tiles.
// A tile is 8 records of the cache, one contiguous copy each, wherever their
// pages are.  RG = 8 NQ WR rows: WR warps take 8 NQ rows each, and the 4 / WR
// warps with the same rows take every so many of a tile's four 32-key steps,
// with softmax statistics of their own, joined at the segment's end.
//
// A step, per 8 rows:
//   S (8 rows x 32 keys) = Q K^T by m16n8k32 e4m3: the cached codes go to the
//     tensor cores as they are (they run at four times the f16 rate of the same
//     instruction: 4000 against 1024 multiply-adds per SM and clock), and the
//     16 rows of the A operand are the queries' 8 rows in two codes each, hi =
//     e4m3(q 2^-e), lo = e4m3(q 2^-e - hi), which holds every bf16 query down
//     to 2^-10 of its row's largest element exactly;
//   online softmax in fp32, base 2, the keys' block scale folded into the
//     scores;
//   O^T (dims x 8 rows) += V^T P^T by m16n8k16 f16: P in 11 bits, times the
//     values' block scale relative to the largest seen so far and 2^14, so
//     that weights down to 2^-39 of the largest count; V^T codes converted
//     to f16 exactly in registers.  (Weights as e4m3 pairs would run at twice
//     the rate but lose everything under 2^-18 of the row's maximum, half of
//     the output where one key outweighs a flat context of 128k.)
// The record's layout makes every operand a run of ldmatrix rows without bank
// conflicts and P's accumulator layout the next product's operand.
#include <algorithm>

#include "kv8.cuh"
#include "tma.cuh"

namespace ks {

namespace {

constexpr int kConsumers = 4;
constexpr int kThreads = 32 * (kConsumers + 1);
constexpr int kTileBlocks = 8;
constexpr int kTile = kTileBlocks * kKv8Block;
constexpr int kStages = 2;
constexpr int kMaxCtas = 480;       // the workspace has room for this many
constexpr int kMaxRowsOfUnit = 64;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kWeightUp = 16384.f;

struct Plan {
    int wr;             // warps of different rows
    int tq;             // tokens of a group
    int rg;             // rows of a group, at least tq query groups
    int ctas;
    bool q_wide;        // queries can be read 8 bytes at a time
    float* part;        // [2 ctas][rg][HD + 4]: m, l, -, -, o
    int4* desc;         // [ctas]: the unit that begins in this CTA's run and ends in a later one's: s (-1: none), h, g, last CTA
};

// Tiles of group g; a group whose rows see nothing has one as well (its rows get zeros).
KS_DEV int group_tiles(const Kv8Seq& q, int tq, int g) {
    const int last = q.len - q.rows + min(q.rows, (g + 1) * tq) - 1;
    return last < 0 ? 1 : last / kTile + 1;
}
KS_DEV int groups_of(const Kv8Seq& q, int tq) { return (q.rows + tq - 1) / tq; }
KS_DEV long long head_tiles(const Kv8Seq& q, int tq) {
    long long n = 0;
    for (int g = 0; g < groups_of(q, tq); ++g) n += group_tiles(q, tq, g);
    return n;
}

// A place in the sequence of all tiles: the unit and its next tile.
struct Cursor {
    int s, h, g, tile, tiles;
    Kv8Seq q;
    KS_DEV void unit(const Kv8Args& a, int tq) { tiles = group_tiles(q, tq, g); }
    KS_DEV void next(const Kv8Args& a, int tq) {
        tile = 0;
        if (++g >= groups_of(q, tq)) {
            g = 0;
            if (++h >= a.hk) {
                h = 0;
                do {
                    if (++s >= a.n_seqs) return;
                    q = kv8_seq(a, s);
                } while (q.rows == 0);
            }
        }
        unit(a, tq);
    }
};

struct Run {
    long long total, x0, x1;    // all tiles, this CTA's
    int ctas;                   // with tiles
    Cursor at;
};

// This CTA's run: the total over the sequences, then the sequence of the first
// tile.  Every thread of the CTA takes part.
KS_DEV bool find_run(const Kv8Args& a, const Plan& p, Run& r, long long* scratch) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cta = blockIdx.x;
    auto tiles_of = [&](int s) -> long long {
        if (s >= a.n_seqs) return 0;
        if (cta == 0 && kv8_seq_bad(a, s)) kv8_flag(a, kKv8BadBatch);
        return a.hk * head_tiles(kv8_seq(a, s), p.tq);
    };
    // inclusive sums over the CTA's threads; the last is the chunk's total
    auto scan = [&](long long v) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long u = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += u;
        }
        __syncthreads();
        if (lane == 31) scratch[warp] = v;
        __syncthreads();
        for (int i = 0; i < warp; ++i) v += scratch[i];
        return v;
    };
    auto all = [&]() {
        long long t = 0;
        for (int i = 0; i < kThreads / 32; ++i) t += scratch[i];
        return t;
    };
    r.total = 0;
    long long first = 0, sum = 0;
    for (int c = 0; c < a.n_seqs; c += kThreads) {
        const long long v = tiles_of(c + tid);
        const long long u = scan(v);
        if (c == 0) first = v, sum = u;
        r.total += all();
    }
    r.ctas = (int)min((long long)p.ctas, r.total);
    if (cta >= r.ctas) return false;
    r.x0 = r.total * cta / r.ctas;
    r.x1 = r.total * (cta + 1) / r.ctas;
    int* place = reinterpret_cast<int*>(scratch + 8);
    long long* before = scratch + 9;
    long long base = 0;
    for (int c = 0;; c += kThreads) {
        const long long v = c == 0 ? first : tiles_of(c + tid), u = c == 0 ? sum : scan(v);
        if (r.x0 >= base + u - v && r.x0 < base + u) {
            *place = c + tid;
            *before = base + u - v;
        }
        if (c + kThreads >= a.n_seqs) break;
        if (c == 0) scan(v);       // scratch holds the last chunk's totals
        base += all();
    }
    __syncthreads();
    Cursor& k = r.at;
    k.s = *place;
    k.q = kv8_seq(a, k.s);
    long long rem = r.x0 - *before;
    const long long w = head_tiles(k.q, p.tq);
    k.h = (int)(rem / w);
    rem %= w;
    k.g = 0;
    k.unit(a, p.tq);
    while (rem >= k.tiles) {
        rem -= k.tiles;
        ++k.g;
        k.unit(a, p.tq);
    }
    k.tile = (int)rem;
    return true;
}

KS_DEV void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
        "l"(src), "r"(bytes), "r"(smem_u32(bar))
        : "memory");
}
KS_DEV void mma_e4m3(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
KS_DEV void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
KS_DEV uint32_t f16_of(uint16_t codes) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(codes));
    return h;
}
KS_DEV uint32_t f16_pack(float lo, float hi) {
    uint32_t h;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(hi), "f"(lo));
    return h;
}
KS_DEV float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
KS_DEV float quad_max(float v) {
    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
    return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
}
KS_DEV float quad_sum(float v) {
    v += __shfl_xor_sync(0xffffffffu, v, 1);
    return v + __shfl_xor_sync(0xffffffffu, v, 2);
}
KS_DEV void consumers_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

// A unit's rows, as its segments and the merge see them.
struct Rows {
    int n;              // query rows: tokens x G
    int row0;           // batch row of the first token
    int pos0;           // its position; negative positions see nothing
    KS_DEV Rows(const Kv8Seq& q, int tq, int g, int G) {
        const int t0 = g * tq, t = min(q.rows - t0, tq);
        n = t * G;
        row0 = q.row0 + t0;
        pos0 = q.len - q.rows + t0;
    }
};

template <int HD>
struct Smem {
    static constexpr int REC = kv8_record(HD);
    static constexpr int TILE = kTileBlocks * REC;
    static constexpr int comb(int nq) { return 8 * nq * HD * 4; }           // a warp's o
    static constexpr int bytes(int nq) {
        return kStages * TILE + 2 * comb(nq) + 2 * 8 * nq * 8 + HD * 4 + 2 * kStages * 8 + 16 * 8 + kStages * 8;
    }
};

template <int HD, int NQ>
__global__ void __launch_bounds__(kThreads, NQ == 1 ? 3 : 2)
    kv8_attention_kernel(const Kv8Args a, const Kv8AttnArgs t, const Plan p) {
    constexpr int REC = kv8_record(HD), TILE = Smem<HD>::TILE, DT = HD / 16, KJ = HD / 32;
    extern __shared__ __align__(128) unsigned char smem[];
    unsigned char* ring = smem;
    float* comb = reinterpret_cast<float*>(ring + kStages * TILE);          // [2][NQ DT 4][32]
    float2* ml = reinterpret_cast<float2*>(comb + 2 * NQ * DT * 4 * 32);    // [2][8 NQ]
    int* nan_from = reinterpret_cast<int*>(ml + 2 * 8 * NQ);                // [HD]: first key whose value is NaN
    uint64_t* full = reinterpret_cast<uint64_t*>(nan_from + HD);
    uint64_t* empty = full + kStages;
    long long* scratch = reinterpret_cast<long long*>(empty + kStages);     // [16]
    volatile int* present = reinterpret_cast<volatile int*>(scratch + 16);  // [kStages] records that were copied

    if (a.stop && *a.stop) return;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    grid_launch_dependents();
    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], kConsumers);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (int i = tid; i < HD; i += kThreads) nan_from[i] = INT32_MAX;
    Run run;
    if (!find_run(a, p, run, scratch)) {
        if (tid == 0) p.desc[blockIdx.x] = make_int4(-1, 0, 0, 0);
        return;
    }
    __syncthreads();
    Cursor at = run.at;
    long long left = run.x1 - run.x0;
    const int G = t.hq / a.hk;

    if (warp == kConsumers) {
        // ------------------------------------------------------- producer
        int it = 0;
        bool alive = true;
        while (left > 0 && alive) {
            const Rows rows(at.q, p.tq, at.g, G);
            const int last = rows.pos0 + rows.n / G - 1;         // of the group's keys
            const int end = at.tile + (int)min((long long)(at.tiles - at.tile), left);
            for (int tile = at.tile; tile < end; ++tile, ++it) {
                const int st = it % kStages, b = tile * kTileBlocks + lane;
                // the page's number is on its way while the stage is still read
                const bool wanted = lane < kTileBlocks && b * kKv8Block <= last;
                const unsigned char* rec = wanted ? kv8_record_at(a, at.s, b, at.h, REC) : nullptr;
                if (wanted && !rec) kv8_flag(a, kKv8BadPage);
                const unsigned have = __ballot_sync(0xffffffffu, rec != nullptr);
                alive = mbar_wait(&empty[st], ((it / kStages) & 1) ^ 1, kWaitLimitNs);
                if (!alive) break;
                if (lane == 0) {
                    present[st] = (int)have;
                    mbar_expect_tx(&full[st], __popc(have) * REC);
                }
                __syncwarp();
                if (rec) bulk_load(ring + st * TILE + lane * REC, rec, REC, &full[st]);
            }
            left -= end - at.tile;
            if (left > 0) at.next(a, p.tq);
        }
        if (!alive && lane == 0) kv8_flag(a, kKv8Timeout);
        // no copy may be in flight when the CTA ends
        for (int i = max(0, it - kStages); i < it; ++i) mbar_wait(&full[i % kStages], (i / kStages) & 1, kWaitLimitNs);
        return;
    }

    // ----------------------------------------------------------- consumers
    const int g = lane >> 2, q4 = lane & 3;
    const int wri = warp % p.wr, wk = warp / p.wr, WK = kConsumers / p.wr;
    const int m0 = wri * 8 * NQ;
    int it = 0;
    bool alive = true, began = false;
    while (left > 0) {
        const Rows rows(at.q, p.tq, at.g, G);
        const int t0 = at.tile, t1 = at.tile + (int)min((long long)(at.tiles - at.tile), left);
        // this warp's queries, in two codes
        uint32_t qa[NQ][KJ][4];
        float qf[NQ];
        int lim[NQ];                                             // last key that the row sees
        const int wn = min(rows.n - m0, 8 * NQ);                 // rows of this warp
        const int lim_first = rows.pos0 + m0 / G, lim_last = rows.pos0 + (m0 + wn - 1) / G;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int m = m0 + 8 * n + g;
            const bool valid = m < rows.n;
            const int tok = valid ? m / G : 0, head = at.h * G + (valid ? m - tok * G : 0);
            const __nv_bfloat16* src = t.q + (int64_t)(rows.row0 + tok) * t.q_row + (int64_t)head * t.q_head;
            lim[n] = valid ? rows.pos0 + tok : INT32_MAX;
            float x[KJ * 2][4], top = 0.f;
#pragma unroll
            for (int j = 0; j < 2 * KJ; ++j) {
                const __nv_bfloat16* e = src + 16 * j + 4 * q4;
                if (!valid) {
                    x[j][0] = x[j][1] = x[j][2] = x[j][3] = 0.f;
                } else if (p.q_wide) {
                    const uint2 v = *reinterpret_cast<const uint2*>(e);
                    x[j][0] = bf16_lo(v.x); x[j][1] = bf16_hi(v.x);
                    x[j][2] = bf16_lo(v.y); x[j][3] = bf16_hi(v.y);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[j][i] = __bfloat162float(e[i]);
                }
            }
#pragma unroll
            for (int j = 0; j < 2 * KJ; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (finite(x[j][i])) top = fmaxf(top, fabsf(x[j][i]));
                    else x[j][i] = __uint_as_float(0x7fc00000u);     // the row becomes NaN, as its scores are
                }
            const float sc = scale_for(quad_max(top)), inv = inverse_pow2(sc);
            qf[n] = sc * (t.scale * kLog2e);
#pragma unroll
            for (int j = 0; j < KJ; ++j)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const float* v = x[2 * j + half];
                    const uint16_t h0 = to_e4m3x2(v[0] * inv, v[1] * inv), h1 = to_e4m3x2(v[2] * inv, v[3] * inv);
                    const float2 f0 = from_e4m3x2(h0), f1 = from_e4m3x2(h1);
                    qa[n][j][2 * half] = h0 | (uint32_t)h1 << 16;
                    qa[n][j][2 * half + 1] = to_e4m3x2(v[0] * inv - f0.x, v[1] * inv - f0.y) |
                                             (uint32_t)to_e4m3x2(v[2] * inv - f1.x, v[3] * inv - f1.y) << 16;
                }
        }
        float m[NQ], l[NQ], vref = 0.f, o[NQ][DT][4];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            m[n] = -INFINITY;
            l[n] = 0.f;
#pragma unroll
            for (int i = 0; i < DT; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.f;
        }

        for (int tile = t0; tile < t1; ++tile, ++it) {
            const int st = it % kStages;
            if (alive) alive = mbar_wait(&full[st], (it / kStages) & 1, kWaitLimitNs);
            const int have = alive && wn > 0 ? present[st] : 0;
            for (int step = wk; step < 4; step += WK) {
                const int got = have >> (2 * step) & 3, key0 = tile * kTile + 32 * step;
                if (got == 0 || key0 > lim_last) continue;
                const unsigned char* rec = ring + st * TILE + 2 * step * REC;
                const uint32_t base = smem_u32(rec);
                const bool edge = got != 3 || key0 + 31 > lim_first;
                float2 sc[2];                                    // key and value scales
                sc[0] = *reinterpret_cast<const float2*>(rec + 32 * HD);
                sc[1] = *reinterpret_cast<const float2*>(rec + REC + 32 * HD);
                float s[NQ][4][4];
#pragma unroll
                for (int nb = 0; nb < 4; ++nb) {
                    const uint32_t kb = base + (nb >> 1) * REC + (nb & 1) * 8 * HD + lane * 16;
#pragma unroll
                    for (int n = 0; n < NQ; ++n) s[n][nb][0] = s[n][nb][1] = s[n][nb][2] = s[n][nb][3] = 0.f;
#pragma unroll
                    for (int j = 0; j < KJ / 2; ++j) {
                        uint32_t kf[4];
                        ldsm_x4(kf, kb + j * 512);
#pragma unroll
                        for (int n = 0; n < NQ; ++n) {
                            mma_e4m3(s[n][nb], qa[n][2 * j], kf[0], kf[1]);
                            mma_e4m3(s[n][nb], qa[n][2 * j + 1], kf[2], kf[3]);
                        }
                    }
                }
                // values of a record that is not there count for nothing
                const float v0 = got & 1 ? sc[0].y : 0.f, v1 = got & 2 ? sc[1].y : 0.f;
                const float vnew = fmaxf(vref, fmaxf(v0, v1)), vinv = inverse_pow2(vnew), vfac = vref * vinv;
                const float w0 = v0 * vinv * kWeightUp, w1 = v1 * vinv * kWeightUp;
                vref = vnew;
                uint32_t pb[NQ][4];
                float fac[NQ];
                bool same = true;
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    const float f0 = qf[n] * sc[0].x, f1 = qf[n] * sc[1].x;
                    float x[4][2], top = m[n];
#pragma unroll
                    for (int nb = 0; nb < 4; ++nb)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            x[nb][e] = (s[n][nb][e] + s[n][nb][2 + e]) * (nb < 2 ? f0 : f1);
                            if (edge && (key0 + 8 * nb + 2 * q4 + e > lim[n] || !(got >> (nb >> 1) & 1)))
                                x[nb][e] = -INFINITY;
                            top = fmaxf(top, x[nb][e]);
                        }
                    top = quad_max(top);
                    const float ref = top == -INFINITY ? 0.f : top;
                    const float al = exp2_approx(m[n] - ref);
                    m[n] = top;
                    float sum = 0.f;
#pragma unroll
                    for (int nb = 0; nb < 4; ++nb) {
                        const float p0 = exp2_approx(x[nb][0] - ref), p1 = exp2_approx(x[nb][1] - ref);
                        sum += p0 + p1;
                        const float w = nb < 2 ? w0 : w1;
                        pb[n][nb] = f16_pack(p0 * w, p1 * w);
                    }
                    l[n] = l[n] * al + sum;
                    fac[n] = al * vfac;
                    same = same && fac[n] == 1.f;
                }
                if (!__all_sync(0xffffffffu, same)) {
#pragma unroll
                    for (int n = 0; n < NQ; ++n) {
                        const float a0 = __shfl_sync(0xffffffffu, fac[n], 8 * q4), a1 = __shfl_sync(0xffffffffu, fac[n], 8 * q4 + 4);
#pragma unroll
                        for (int i = 0; i < DT; ++i) {
                            o[n][i][0] *= a0; o[n][i][1] *= a1;
                            o[n][i][2] *= a0; o[n][i][3] *= a1;
                        }
                    }
                }
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    if (!(got >> kb & 1)) continue;
#pragma unroll
                    for (int dd = 0; dd < DT / 2; ++dd) {
                        uint32_t vf[4];
                        ldsm_x4(vf, base + kb * REC + 16 * HD + dd * 512 + lane * 16);
                        if (edge) {
                            // tokens that not every row sees: a NaN would pass through a weight of zero.  It is
                            // taken out, and the rows that do see it get their NaN at the end.
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                uint32_t nan = ((vf[i] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
                                if (nan) {
                                    for (int c = 0; c < 4; ++c)
                                        if (nan >> (8 * c + 7) & 1)
                                            atomicMin(&nan_from[32 * dd + 8 * i + g],
                                                      key0 + 16 * kb + 2 * q4 + (c & 1) + 8 * (c >> 1));
                                    vf[i] &= ~((nan >> 7) * 0xffu);
                                }
                            }
                        }
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            const uint32_t r0 = vf[2 * half], r1 = vf[2 * half + 1];
                            const uint32_t af[4] = {f16_of((uint16_t)r0), f16_of((uint16_t)r1), f16_of((uint16_t)(r0 >> 16)),
                                                    f16_of((uint16_t)(r1 >> 16))};
#pragma unroll
                            for (int n = 0; n < NQ; ++n) mma_f16(o[n][2 * dd + half], af, pb[n][2 * kb], pb[n][2 * kb + 1]);
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty[st]);
        }

        // ------------------------------------------------- segment's end
        const float up = vref / kWeightUp;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            l[n] = quad_sum(l[n]);
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) o[n][i][c] *= up;
        }
        // join the warps with the same rows, halving their number each time
        consumers_sync();
        for (int d = WK / 2; d > 0; d >>= 1) {
            const int buf = (wk & (d - 1)) * p.wr + wri;         // of the pair
            float* mine = comb + buf * NQ * DT * 4 * 32 + lane;
            if (wk >= d && wk < 2 * d) {
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
#pragma unroll
                    for (int i = 0; i < DT; ++i)
#pragma unroll
                        for (int c = 0; c < 4; ++c) mine[((n * DT + i) * 4 + c) * 32] = o[n][i][c];
                    if (q4 == 0) ml[buf * 8 * NQ + 8 * n + g] = make_float2(m[n], l[n]);
                }
            }
            consumers_sync();
            if (wk < d) {
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    const float2 u = ml[buf * 8 * NQ + 8 * n + g];
                    const float top = fmaxf(m[n], u.x), ref = top == -INFINITY ? 0.f : top;
                    const float fa = exp2_approx(m[n] - ref), fb = exp2_approx(u.x - ref);
                    m[n] = top;
                    l[n] = l[n] * fa + u.y * fb;
                    const float a0 = __shfl_sync(0xffffffffu, fa, 8 * q4), a1 = __shfl_sync(0xffffffffu, fa, 8 * q4 + 4);
                    const float b0 = __shfl_sync(0xffffffffu, fb, 8 * q4), b1 = __shfl_sync(0xffffffffu, fb, 8 * q4 + 4);
#pragma unroll
                    for (int i = 0; i < DT; ++i)
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            o[n][i][c] = o[n][i][c] * (c & 1 ? a1 : a0) + mine[((n * DT + i) * 4 + c) * 32] * (c & 1 ? b1 : b0);
                }
            }
            consumers_sync();
        }
        const bool whole = t0 == 0 && t1 == at.tiles;
        if (wk == 0 && wn > 0) {
            float* slot = p.part + (size_t)(2 * blockIdx.x + (t0 == 0)) * p.rg * (HD + 4);
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                const int m_row = m0 + 8 * n + g;
                if (q4 == 0 && m_row < rows.n) {
                    if (!whole) {
                        *reinterpret_cast<float2*>(slot + (size_t)m_row * (HD + 4)) = make_float2(m[n], l[n]);
                    } else if (t.lse) {
                        const int tok = m_row / G;
                        t.lse[(size_t)(rows.row0 + tok) * t.hq + at.h * G + m_row - tok * G] =
                            l[n] == 0.f ? -INFINITY : (m[n] + log2f(l[n])) * kLn2;
                    }
                }
                const float inv = whole ? (l[n] == 0.f ? 0.f : 1.f / l[n]) : 1.f;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float f = __shfl_sync(0xffffffffu, inv, 8 * q4 + 4 * e);
                    const int r = m0 + 8 * n + 2 * q4 + e;
                    if (r >= rows.n) continue;
                    const int tok = r / G, seen = rows.pos0 + tok;
                    __nv_bfloat16* out = t.out + (int64_t)(rows.row0 + tok) * t.out_row + (int64_t)(at.h * G + r - tok * G) * t.out_head;
#pragma unroll
                    for (int i = 0; i < DT; ++i)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const int d = 16 * i + 8 * c + g;
                            float v = o[n][i][2 * c + e] * f;
                            if (nan_from[d] <= seen) v = __uint_as_float(0x7fc00000u);
                            if (whole) out[d] = __float2bfloat16_rn(v);
                            else slot[(size_t)r * (HD + 4) + 4 + d] = v;
                        }
                }
            }
        }
        if (!whole && t0 == 0) {
            began = true;
            if (tid == 0) {
                const long long end = run.x1 - left + at.tiles;        // first tile after the unit
                p.desc[blockIdx.x] = make_int4(at.s, at.h, at.g, (int)((end * run.ctas - 1) / run.total));
            }
        }
        left -= t1 - t0;
        if (left > 0) {
            consumers_sync();                                    // nan_from is read
            for (int i = tid; i < HD; i += 32 * kConsumers) nan_from[i] = INT32_MAX;
            consumers_sync();
            at.next(a, p.tq);
        }
    }
    if (tid == 0) {
        if (!began) p.desc[blockIdx.x] = make_int4(-1, 0, 0, 0);
        if (!alive) kv8_flag(a, kKv8Timeout);
    }
}

// Merge of the units that lie in several runs: CTA (x, y) takes kMergeRows rows
// of the unit that begins in run x; the two warps of a row take every other
// segment and meet in shared memory.
constexpr int kMergeRows = 4, kMergeThreads = 64 * kMergeRows;
template <int HD>
__global__ void __launch_bounds__(kMergeThreads) kv8_merge_kernel(const Kv8Args a, const Kv8AttnArgs t, const Plan p) {
    constexpr int V = HD / 32;
    grid_dependency_wait();
    if (a.stop && *a.stop) return;
    const int4 u = p.desc[blockIdx.x];
    if (u.x < 0) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = warp & 1, G = t.hq / a.hk;
    const Rows rows(kv8_seq(a, u.x), p.tq, u.z, G);
    const int r = blockIdx.y * kMergeRows + (warp >> 1), parts = u.w - (int)blockIdx.x + 1;
    __shared__ float other[kMergeRows][HD];
    // segment i: run x + i; the first one is its run's second slot, a later one its first
    auto part = [&](int i) {
        return p.part + ((size_t)(2 * (blockIdx.x + i) + (i == 0)) * p.rg + r) * (HD + 4);
    };
    float acc[V], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.f;
    if (r < rows.n) {
        for (int i = lane; i < parts; i += 32) m = fmaxf(m, part(i)[0]);
        m = warp_max(m);
        const float ref = m == -INFINITY ? 0.f : m;
        for (int c = 0; c < parts; c += 32) {
            float w = 0.f;
            if (c + lane < parts) {
                const float2 x = *reinterpret_cast<const float2*>(part(c + lane));
                w = exp2_approx(x.x - ref);
                l += x.y * w;
            }
            const int n = min(32, parts - c);
#pragma unroll 8
            for (int i = half; i < n; i += 2) {
                const float f = __shfl_sync(0xffffffffu, w, i);
                const float* o = part(c + i) + 4 + V * lane;
                if constexpr (V == 4) {
                    const float4 x = *reinterpret_cast<const float4*>(o);
                    acc[0] = fmaf(f, x.x, acc[0]); acc[1] = fmaf(f, x.y, acc[1]);
                    acc[2] = fmaf(f, x.z, acc[2]); acc[3] = fmaf(f, x.w, acc[3]);
                } else {
                    const float2 x = *reinterpret_cast<const float2*>(o);
                    acc[0] = fmaf(f, x.x, acc[0]); acc[1] = fmaf(f, x.y, acc[1]);
                }
            }
        }
        l = warp_sum(l);
    }
    if (half == 1)
#pragma unroll
        for (int i = 0; i < V; ++i) other[warp >> 1][V * lane + i] = acc[i];
    __syncthreads();
    if (half == 1 || r >= rows.n) return;
    const int tok = r / G, head = u.y * G + r - tok * G;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    __nv_bfloat16* out = t.out + (int64_t)(rows.row0 + tok) * t.out_row + (int64_t)head * t.out_head + V * lane;
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = __float2bfloat16_rn((acc[i] + other[warp >> 1][V * lane + i]) * inv);
    if (t.lse && lane == 0) t.lse[(size_t)(rows.row0 + tok) * t.hq + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// Rows of a group: the next of 8, 16, 32, 64 at or above the batch's average of
// query rows per sequence and KV head, and above G (whole tokens).
int rows_of_unit(int G, int64_t n_rows, int64_t n_seqs) {
    const int64_t avg = n_seqs > 0 ? (n_rows * G + n_seqs - 1) / n_seqs : 0;
    int rg = 8;
    while (rg < kMaxRowsOfUnit && (rg < avg || rg < G)) rg *= 2;
    return rg;
}

template <int HD, int NQ>
cudaError_t launch_hd(const Kv8Args& a, const Kv8AttnArgs& t, Plan p, bool split, cudaStream_t s) {
    const int bytes = Smem<HD>::bytes(NQ);
    static const cudaError_t set = cudaFuncSetAttribute(kv8_attention_kernel<HD, NQ>,
                                                        cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (set != cudaSuccess) return set;
    kv8_attention_kernel<HD, NQ><<<p.ctas, kThreads, bytes, s>>>(a, t, p);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || !split) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(p.ctas, (p.rg + kMergeRows - 1) / kMergeRows);
    cfg.blockDim = dim3(kMergeThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kv8_merge_kernel<HD>, a, t, p);
}

}  // namespace

size_t kv8_attention_workspace(int hd, int G, int n_rows) {
    const int64_t rows = (int64_t)n_rows * G;
    const int rg = rows >= kMaxRowsOfUnit ? kMaxRowsOfUnit : rows_of_unit(G, n_rows, 1);
    return sizeof(float) * 2 * kMaxCtas * (size_t)rg * (hd + 4) + sizeof(int4) * kMaxCtas;
}

cudaError_t launch_kv8_attention(const Kv8Args& a, const Kv8AttnArgs& t, cudaStream_t s) {
    const int G = t.hq / a.hk;
    Plan p{};
    p.rg = rows_of_unit(G, a.n_rows, a.n_seqs);
    p.tq = p.rg / G;
    p.wr = p.rg <= 16 ? 1 : p.rg / 16;
    const int64_t tiles = (a.capacity + kTile - 1) / kTile;
    const int64_t most = (int64_t)a.hk * (a.n_rows / p.tq + a.n_seqs) * std::max<int64_t>(tiles, 1);
    p.ctas = (int)std::min<int64_t>(std::min(kMaxCtas, sm_count() * (p.rg == 8 ? 3 : 2)), most);
    p.q_wide = reinterpret_cast<uintptr_t>(t.q) % 8 == 0 && t.q_row % 4 == 0 && t.q_head % 4 == 0;
    p.desc = static_cast<int4*>(t.workspace);
    p.part = reinterpret_cast<float*>(p.desc + kMaxCtas);
    const bool split = tiles > 1;
    if (a.hd == 128)
        return p.rg == 8 ? launch_hd<128, 1>(a, t, p, split, s) : launch_hd<128, 2>(a, t, p, split, s);
    return p.rg == 8 ? launch_hd<64, 1>(a, t, p, split, s) : launch_hd<64, 2>(a, t, p, split, s);
}

}  // namespace ks
