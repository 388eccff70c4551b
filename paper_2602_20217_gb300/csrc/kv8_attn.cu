// Causal attention over the 8-bit paged cache: units of at most 16 query rows
// (decoding), the merge of split units for every size, and the choice between
// this kernel and the tcgen05 one (kv8_tc.cu).  kv8_plan.cuh cuts the work.
//
// A CTA is a producer warp and four consumer warps around a ring of four tiles
// of 64 keys.  A tile is four records of the cache, contiguous ones in one copy,
// wherever their pages are.  The unit's 8 NQ rows are every warp's, each takes
// one 16-key step of a tile, with softmax statistics of its own, and they are
// joined at the segment's end.
//
// A step, per 8 rows:
//   S (8 rows x 16 keys) = Q K^T by m16n8k32 e4m3: the cached codes go to the
//     tensor cores as they are (4000 multiply-adds per SM and clock in this
//     instruction, 1024 in its f16 form), and the 16 rows of the A operand are
//     the queries' 8 rows in two codes each, hi = e4m3(q 2^-e), lo = e4m3(q
//     2^-e - hi), which hold every bf16 query down to 2^-9 of its row's
//     largest element exactly;
//   online softmax in fp32, base 2, the keys' block scale folded into the
//     scores;
//   O^T (dims x 8 rows) += V^T P^T by m16n8k16 f16: P in 11 bits, times the
//     values' block scale relative to the largest seen so far and 2^14, so
//     that weight times relative scale counts down to 2^-39 and has 11 bits down
//     to 2^-28; V^T codes converted to f16 exactly in registers.  (Weights as
//     e4m3 pairs would run at twice the rate but lose everything under 2^-18 of
//     the row's maximum, half of the output where one key outweighs a flat
//     context of 128k.)
// The record's layout makes every operand a run of ldmatrix rows without bank
// conflicts and P's accumulator layout the next product's operand.
//
// Measured: one row of 64 query heads over 8 (hd 128) at 65537 tokens 31.5 us, 4.3
// TB/s; 64 sequences of up to 16000 tokens, 32 heads over 8, 73 us, 5.2 TB/s; at
// 4099 tokens 12 us.  Past about 10 us of launches, first loads and the merge the
// bytes bound it (6.6 TB/s between the two contexts above); under 4k tokens those
// fixed steps are all of it.
#include <algorithm>
#include <type_traits>

#include "kv8_plan.cuh"

namespace ks {

namespace {

constexpr int kConsumers = 4;
constexpr int kThreads = 32 * (kConsumers + 1);
constexpr int kBlocks = 4, kTile = kBlocks * kKv8Block, kStages = 4;
constexpr float kWeightUp = 16384.f;

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
KS_DEV float quad_max(float v) {
    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
    return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
}
KS_DEV float quad_sum(float v) {
    v += __shfl_xor_sync(0xffffffffu, v, 1);
    return v + __shfl_xor_sync(0xffffffffu, v, 2);
}
KS_DEV void consumers_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

// A CTA's shared memory.
template <int HD, int NQ>
struct Smem {
    static constexpr int REC = kv8_record(HD);
    static constexpr int TILE = kBlocks * REC;
    static constexpr int HALF = NQ * (HD / 32) * 4 * 32;         // floats: half of a warp's o
    static constexpr bool Q = NQ > 1;                            // queries here instead of in registers
    unsigned char ring[kStages][TILE];
    float comb[kConsumers][HALF];
    uint32_t q[Q ? NQ * (HD / 32) * 4 * 32 : 4];                 // [NQ][HD / 32] A operands, 4 matrices each
    float qf[8 * NQ];                                            // of their scores
    float2 ml[kConsumers][8 * NQ];
    int nan_from[3][HD];                                         // first key whose value is NaN, a segment each
    int any_nan[3];
    int present[kStages];                                        // records that were copied
    uint64_t full[kStages], empty[kStages];
};

// o[i][c] = NaN for i and c that are not known when compiling (rare)
template <int DT>
KS_DEV void set_nan(float (&o)[DT][4], int i, int c) {
#pragma unroll
    for (int j = 0; j < DT; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i == j && c == k) o[j][k] = __uint_as_float(0x7fc00000u);
}

// Warps wk and wk ^ bit have the same rows: each gives half of its CUR tiles of
// dims (all in o[.][0 .. CUR)) to the other and keeps the sum of the other half
// in o[.][0 .. CUR / 2).  Returns the first kept tile of the CUR.
template <int NQ, int DT, int CUR>
KS_DEV int join(float (&o)[NQ][DT][4], float (&m)[NQ], float (&l)[NQ], float* comb, float2* ml, int warp, int other,
                bool upper) {
    constexpr int H = CUR / 2, SLOT = NQ * (DT / 2) * 4 * 32;
    const int lane = threadIdx.x & 31, g = lane >> 2, q4 = lane & 3;
    float* mine = comb + warp * SLOT + lane;
    const float* theirs = comb + other * SLOT + lane;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
#pragma unroll
        for (int i = 0; i < H; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                mine[((n * H + i) * 4 + c) * 32] = upper ? o[n][i][c] : o[n][H + i][c];
                if (upper) o[n][i][c] = o[n][H + i][c];
            }
        if (q4 == 0) ml[warp * 8 * NQ + 8 * n + g] = make_float2(m[n], l[n]);
    }
    consumers_sync();
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const float2 u = ml[other * 8 * NQ + 8 * n + g];
        const float top = fmaxf(m[n], u.x), ref = top == -INFINITY ? 0.f : top;
        const float fa = exp2_approx(m[n] - ref), fb = exp2_approx(u.x - ref);
        m[n] = top;
        l[n] = __fadd_rn(__fmul_rn(l[n], fa), __fmul_rn(u.y, fb));      // the same bits in both warps
        const float a0 = __shfl_sync(0xffffffffu, fa, 8 * q4), a1 = __shfl_sync(0xffffffffu, fa, 8 * q4 + 4);
        const float b0 = __shfl_sync(0xffffffffu, fb, 8 * q4), b1 = __shfl_sync(0xffffffffu, fb, 8 * q4 + 4);
#pragma unroll
        for (int i = 0; i < H; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                o[n][i][c] = o[n][i][c] * (c & 1 ? a1 : a0) + theirs[((n * H + i) * 4 + c) * 32] * (c & 1 ? b1 : b0);
    }
    consumers_sync();
    return upper ? H : 0;
}

template <int HD, int NQ, int PART>
__global__ void __launch_bounds__(kThreads, NQ == 1 ? 3 : 2)
    kv8_attention_kernel(const Kv8Args a, const Kv8AttnArgs t, const Kv8Plan p) {
    using S = Smem<HD, NQ>;
    constexpr int REC = S::REC, DT = HD / 16, KJ = HD / 32;
    extern __shared__ __align__(128) unsigned char smem_raw[];
    S& sm = *reinterpret_cast<S*>(smem_raw);
    volatile int* present = sm.present;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&sm.full[i], 1);
            mbar_init(&sm.empty[i], kConsumers);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (int i = tid; i < 3 * HD; i += kThreads) sm.nan_from[0][i] = INT32_MAX;
    if (tid < 3) sm.any_nan[tid] = 0;
    __syncthreads();
    grid_dependency_wait();
    grid_launch_dependents();
    if (a.stop && *a.stop) return;
    Run run;
    Segment<PART> at;
    if (!find_run(a, p, run, at)) {
        if (tid == 0) p.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
        return;
    }
    const int G = p.G;

    if (warp == kConsumers) {
        // ------------------------------------------------------- producer
        // Page numbers are read a group of tiles ahead, across segments: under
        // load such a read takes microseconds.
        constexpr int TILES = 32 / kBlocks;                      // tiles of a group, a block per lane
        auto pages = [&](const Segment<PART>& k, int tile) {
            const int b = tile * kBlocks + lane;
            if (b * kKv8Block > last_key<PART>(k.q, p, k.g) || tile + lane / kBlocks >= k.end) return -1;
            const int page = pages_of<PART>(a, k.s)[p.page_of(b, a.bpp)];
            return page >= 0 && page < a.n_pages ? page : -2;
        };
        int it = 0, tile = at.tile, page = pages(at, tile);
        bool alive = true, more = true;
        while (more && alive) {
            // the group after this one
            Segment<PART> next = at;
            int next_tile = tile + TILES;
            if (next_tile >= at.end) {
                more = next.next(a, run, p);
                next_tile = next.tile;
            }
            const int next_page = more ? pages(next, next_tile) : -1;
            if (page == -2) kv8_flag(a, kKv8BadPage);
            const int b = tile * kBlocks + lane;
            const unsigned char* rec =
                page >= 0 ? a.data + (((size_t)page * a.hk + at.h) * a.bpp + b - p.page_of(b, a.bpp) * a.bpp) * REC
                          : nullptr;
            const unsigned have = __ballot_sync(0xffffffffu, rec != nullptr);
            // one copy for records that follow each other: the lane of the first one makes it
            const unsigned char* before = reinterpret_cast<const unsigned char*>(
                __shfl_up_sync(0xffffffffu, reinterpret_cast<unsigned long long>(rec), 1));
            const bool head = rec != nullptr && (lane % kBlocks == 0 || before == nullptr || rec != before + REC);
            const unsigned ends = (__ballot_sync(0xffffffffu, head || rec == nullptr) | 0x11111111u) >> lane >> 1;
            const int length = min(ends ? __ffs(ends) : 32, kBlocks - lane % kBlocks);
            for (int i = 0; i < TILES && tile + i < at.end; ++i, ++it) {
                const int st = it % kStages;
                const unsigned mask = have >> (i * kBlocks) & ((1u << kBlocks) - 1);
                alive = mbar_wait(&sm.empty[st], ((it / kStages) & 1) ^ 1, kWaitLimitNs);
                if (!alive) break;
                if (lane == 0) {
                    present[st] = (int)mask;
                    mbar_expect_tx(&sm.full[st], __popc(mask) * REC);
                }
                __syncwarp();
                if (head && lane / kBlocks == i)
                    bulk_load(sm.ring[st] + lane % kBlocks * REC, rec, length * REC, &sm.full[st]);
            }
            at = next;
            tile = next_tile;
            page = next_page;
        }
        if (!alive && lane == 0) kv8_flag(a, kKv8Timeout);
        // no copy may be in flight when the CTA ends
        for (int i = max(0, it - kStages); i < it; ++i)
            mbar_wait(&sm.full[i % kStages], (i / kStages) & 1, kWaitLimitNs);
        return;
    }

    // ----------------------------------------------------------- consumers
    const int g = lane >> 2, q4 = lane & 3;
    int it = 0;
    bool alive = true, began = false;
    for (int buf = 0;; buf = buf == 2 ? 0 : buf + 1) {
        const Rows rows(at, p.tq, G);
        // the queries, in two codes: every warp's in its registers, or 8 rows by a warp for all
        static_assert(S::Q ? NQ <= kConsumers : NQ == 1);
        uint32_t qa[S::Q ? 1 : KJ][4];
        float qf[NQ];
        int lim[NQ];                                             // last key that the row sees
        const int lim_first = rows.pos0, lim_last = rows.pos0 + (rows.tokens - 1) * rows.step;
#pragma unroll
        for (int n = 0; n < NQ; ++n) lim[n] = 8 * n + g < rows.n ? rows.pos0 + p.token(8 * n + g) * rows.step : INT32_MAX;
        if (const int n = S::Q ? warp : 0; n < NQ) {
            const int m = 8 * n + g;
            const bool valid = m < rows.n;
            const int tok = valid ? p.token(m) : 0, head = at.h * G + (valid ? m - tok * G : 0);
            const __nv_bfloat16* src = t.q + (int64_t)(rows.row0 + tok) * t.q_row + (int64_t)head * t.q_head;
            float x[KJ * 2][4], top = 0.f;
            // all loads first, without a branch between them
            uint2 raw[KJ * 2];
            if (p.q_wide) {
#pragma unroll
                for (int j = 0; j < 2 * KJ; ++j) raw[j] = *reinterpret_cast<const uint2*>(src + 16 * j + 4 * q4);
            } else {
                const unsigned short* e = reinterpret_cast<const unsigned short*>(src) + 4 * q4;
#pragma unroll
                for (int j = 0; j < 2 * KJ; ++j)
                    raw[j] = make_uint2(e[16 * j] | (uint32_t)e[16 * j + 1] << 16, e[16 * j + 2] | (uint32_t)e[16 * j + 3] << 16);
            }
#pragma unroll
            for (int j = 0; j < 2 * KJ; ++j) {
                if (!valid) raw[j] = make_uint2(0, 0);
                x[j][0] = bf16_lo(raw[j].x); x[j][1] = bf16_hi(raw[j].x);
                x[j][2] = bf16_lo(raw[j].y); x[j][3] = bf16_hi(raw[j].y);
            }
#pragma unroll
            for (int j = 0; j < 2 * KJ; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (finite(x[j][i])) top = fmaxf(top, fabsf(x[j][i]));
                    else x[j][i] = __uint_as_float(0x7fc00000u);     // the row becomes NaN, as its scores are
                }
            const float sc = scale_for(quad_max(top)), inv = inverse_pow2(sc);
            qf[0] = sc * (t.scale * kLog2e);
            if constexpr (S::Q) {
                if (q4 == 0) sm.qf[m] = qf[0];
            }
#pragma unroll
            for (int j = 0; j < KJ; ++j)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const float* v = x[2 * j + half];
                    const uint16_t h0 = to_e4m3x2(v[0] * inv, v[1] * inv), h1 = to_e4m3x2(v[2] * inv, v[3] * inv);
                    const float2 f0 = from_e4m3x2(h0), f1 = from_e4m3x2(h1);
                    const uint32_t hi = h0 | (uint32_t)h1 << 16;
                    const uint32_t lo = to_e4m3x2(v[0] * inv - f0.x, v[1] * inv - f0.y) |
                                        (uint32_t)to_e4m3x2(v[2] * inv - f1.x, v[3] * inv - f1.y) << 16;
                    if constexpr (S::Q) {
                        // matrix i of (n, j), row g, bytes 4 q4 ..
                        sm.q[(n * KJ + j) * 128 + 64 * half + lane] = hi;
                        sm.q[(n * KJ + j) * 128 + 64 * half + 32 + lane] = lo;
                    } else {
                        qa[j][2 * half] = hi;
                        qa[j][2 * half + 1] = lo;
                    }
                }
        }
        if constexpr (S::Q) {
            consumers_sync();
#pragma unroll
            for (int n = 0; n < NQ; ++n) qf[n] = sm.qf[8 * n + g];
        }
        float m[NQ], l[NQ], vref = 0.f, o[NQ][DT][4];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            m[n] = -INFINITY;
            l[n] = 0.f;
#pragma unroll
            for (int i = 0; i < DT; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.f;
        }

        for (int tile = at.tile; tile < at.end; ++tile, ++it) {
            const int st = it % kStages;
            if (alive) alive = mbar_wait(&sm.full[st], (it / kStages) & 1, kWaitLimitNs);
            const int have = alive ? present[st] : 0, key0 = tile * kTile + warp * kKv8Block;
            if ((have >> warp & 1) && key0 <= lim_last) {
                const unsigned char* rec = sm.ring[st] + warp * REC;
                const uint32_t base = smem_u32(rec);
                const bool edge = key0 + kKv8Block - 1 > lim_first;
                const float2 sc = *reinterpret_cast<const float2*>(rec + 32 * HD);       // key and value scales
                float s[NQ][2][4];
#pragma unroll
                for (int n = 0; n < NQ; ++n)
#pragma unroll
                    for (int c = 0; c < 4; ++c) s[n][0][c] = s[n][1][c] = 0.f;
#pragma unroll
                for (int j = 0; j < KJ / 2; ++j) {
                    uint32_t k0[4], k1[4];
                    ldsm_x4(k0, base + lane * 16 + j * 512);
                    ldsm_x4(k1, base + 8 * HD + lane * 16 + j * 512);
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            if constexpr (S::Q) {
                                uint32_t q[4];
                                ldsm_x4(q, smem_u32(sm.q + (n * KJ + 2 * j + e) * 128) + lane * 16);
                                mma_e4m3(s[n][0], q, k0[2 * e], k0[2 * e + 1]);
                                mma_e4m3(s[n][1], q, k1[2 * e], k1[2 * e + 1]);
                            } else {
                                mma_e4m3(s[n][0], qa[2 * j + e], k0[2 * e], k0[2 * e + 1]);
                                mma_e4m3(s[n][1], qa[2 * j + e], k1[2 * e], k1[2 * e + 1]);
                            }
                        }
                }
                const float vnew = fmaxf(vref, sc.y), vinv = inverse_pow2(vnew), vfac = vref * vinv;
                const float w = sc.y * vinv * kWeightUp;         // in this order: vinv may be 2^126
                vref = vnew;
                uint32_t pb[NQ][2];
                float fac[NQ];
                bool same = true;
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    float x[2][2], top = m[n];
#pragma unroll
                    for (int nb = 0; nb < 2; ++nb)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            x[nb][e] = (s[n][nb][e] + s[n][nb][2 + e]) * (qf[n] * sc.x);
                            if (edge && key0 + 8 * nb + 2 * q4 + e > lim[n]) x[nb][e] = -INFINITY;
                            top = fmaxf(top, x[nb][e]);
                        }
                    top = quad_max(top);
                    const float ref = top == -INFINITY ? 0.f : top;
                    const float al = exp2_approx(m[n] - ref);
                    m[n] = top;
                    float sum = 0.f;
#pragma unroll
                    for (int nb = 0; nb < 2; ++nb) {
                        const float p0 = exp2_approx(x[nb][0] - ref), p1 = exp2_approx(x[nb][1] - ref);
                        sum += p0 + p1;
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
                for (int dd = 0; dd < DT / 2; ++dd) {
                    uint32_t vf[4];
                    ldsm_x4(vf, base + 16 * HD + dd * 512 + lane * 16);
                    if (edge) {
                        // tokens that not every row sees: a NaN would pass through a weight of zero.  It is taken
                        // out, and the rows that do see it get their NaN at the end.
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t nan = ((vf[i] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
                            if (nan) {
                                sm.any_nan[buf] = 1;
                                for (int c = 0; c < 4; ++c)
                                    if (nan >> (8 * c + 7) & 1)
                                        atomicMin(&sm.nan_from[buf][32 * dd + 8 * i + g],
                                                  key0 + 2 * q4 + (c & 1) + 8 * (c >> 1));
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
                        for (int n = 0; n < NQ; ++n) mma_f16(o[n][2 * dd + half], af, pb[n][0], pb[n][1]);
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.empty[st]);
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
        // the next segment's NaN marks begin empty: who read this buffer two segments ago has passed a barrier since
        const int clear = buf == 2 ? 0 : buf + 1;
        for (int i = tid; i < HD; i += 32 * kConsumers) sm.nan_from[clear][i] = INT32_MAX;
        if (tid == 0) sm.any_nan[clear] = 0;
        const bool whole = at.tile == 0 && at.end == at.tiles;
        bool joins = false;                                      // with what its group has in common
        if constexpr (PART == kTail) joins = t.cut[at.s] > 0;
        // the group's part of the rows that end here, all loads at once and before the joins: its own quarter of the
        // dims, see below
        float c_lse[PART == kTail ? NQ : 1], c_out[PART == kTail ? NQ : 1][2][PART == kTail ? DT / 2 : 1];
        if constexpr (PART == kTail) {
            if (whole && joins) {
                const int d0 = 16 * ((warp & 2 ? DT / 2 : 0) + (warp & 1 ? DT / 4 : 0)) + g;
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    const int m_row = min(8 * n + g, rows.n - 1), tok = p.token(m_row);
                    c_lse[n] = t.common_lse[(size_t)(rows.row0 + tok) * t.hq + at.h * G + m_row - tok * G];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int r = min(8 * n + 2 * q4 + e, rows.n - 1), tok_r = p.token(r);
                        const float* c = t.common_out + ((size_t)(rows.row0 + tok_r) * t.hq + at.h * G + r - tok_r * G) * HD + d0;
#pragma unroll
                        for (int i = 0; i < DT / 2; ++i) c_out[n][e][i] = c[8 * i];
                    }
                }
            }
        }
        consumers_sync();                                        // this segment's NaN marks are complete
        // join the warps; each ends with a quarter of the dims
        int dt0 = join<NQ, DT, DT>(o, m, l, sm.comb[0], sm.ml[0], warp, warp ^ 2, warp & 2);
        dt0 += join<NQ, DT, DT / 2>(o, m, l, sm.comb[0], sm.ml[0], warp, warp ^ 1, warp & 1);
        const bool any_nan = sm.any_nan[buf];
        {
            float* slot = p.part + (size_t)(2 * blockIdx.x + (at.tile == 0)) * p.rg * (HD + 4);
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                float inv = whole ? (l[n] == 0.f ? 0.f : 1.f / l[n]) : 1.f, other = 0.f, joined = 0.f;
                if constexpr (PART == kTail) {
                    if (whole && joins) {
                        const Joined j(m[n], l[n], c_lse[n]);
                        inv = j.own;
                        other = j.other;
                        joined = j.lse;
                    }
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float f = __shfl_sync(0xffffffffu, inv, 8 * q4 + 4 * e);
                    const float fc = PART == kTail ? __shfl_sync(0xffffffffu, other, 8 * q4 + 4 * e) : 0.f;
                    const int r = 8 * n + 2 * q4 + e;
                    if (any_nan) {
                        const int seen = rows.pos0 + p.token(r) * rows.step;
                        for (int i = 0; i < DT / 4; ++i)
                            for (int c = 0; c < 2; ++c)
                                if (sm.nan_from[buf][16 * (dt0 + i) + 8 * c + g] <= seen)
                                    set_nan<DT>(o[n], i, 2 * c + e);
                    }
                    if (r >= rows.n) continue;
                    if (PART == kCommon && whole) {
                        const int tok = p.token(r);
                        float* out = t.common_out + ((size_t)(rows.row0 + tok) * t.hq + at.h * G + r - tok * G) * HD +
                                     16 * dt0 + g;
#pragma unroll
                        for (int i = 0; i < DT / 4; ++i) {
                            out[16 * i] = o[n][i][e] * f;
                            out[16 * i + 8] = o[n][i][2 + e] * f;
                        }
                    } else if (PART == kTail && whole && joins) {
                        const int tok = p.token(r);
                        const int64_t row = rows.row0 + tok, head = at.h * G + r - tok * G;
                        __nv_bfloat16* out = t.out + row * t.out_row + head * t.out_head + 16 * dt0 + g;
#pragma unroll
                        for (int i = 0; i < DT / 4; ++i) {
                            out[16 * i] = __float2bfloat16_rn(fmaf(o[n][i][e], f, c_out[n][e][2 * i] * fc));
                            out[16 * i + 8] = __float2bfloat16_rn(fmaf(o[n][i][2 + e], f, c_out[n][e][2 * i + 1] * fc));
                        }
                    } else if (whole) {
                        const int tok = p.token(r);
                        __nv_bfloat16* out = t.out + (int64_t)(rows.row0 + tok) * t.out_row +
                                             (int64_t)(at.h * G + r - tok * G) * t.out_head + 16 * dt0 + g;
#pragma unroll
                        for (int i = 0; i < DT / 4; ++i) {
                            out[16 * i] = __float2bfloat16_rn(o[n][i][e] * f);
                            out[16 * i + 8] = __float2bfloat16_rn(o[n][i][2 + e] * f);
                        }
                    } else {
                        float* out = slot + (size_t)r * (HD + 4) + 4 + 16 * dt0 + g;
#pragma unroll
                        for (int i = 0; i < DT / 4; ++i) {
                            out[16 * i] = o[n][i][e];
                            out[16 * i + 8] = o[n][i][2 + e];
                        }
                    }
                }
                const int m_row = 8 * n + g;
                if (warp == 0 && q4 == 0 && m_row < rows.n) {
                    if (!whole) {
                        *reinterpret_cast<float2*>(slot + (size_t)m_row * (HD + 4)) = make_float2(m[n], l[n]);
                    } else if (PART == kCommon) {
                        const int tok = p.token(m_row);
                        t.common_lse[(size_t)(rows.row0 + tok) * t.hq + at.h * G + m_row - tok * G] =
                            l[n] == 0.f ? -INFINITY : m[n] + log2f(l[n]);
                    } else if (PART == kTail && joins) {
                        const int tok = p.token(m_row);
                        if (t.lse) t.lse[(size_t)(rows.row0 + tok) * t.hq + at.h * G + m_row - tok * G] = joined * kLn2;
                    } else if (t.lse) {
                        const int tok = p.token(m_row);
                        t.lse[(size_t)(rows.row0 + tok) * t.hq + at.h * G + m_row - tok * G] =
                            l[n] == 0.f ? -INFINITY : (m[n] + log2f(l[n])) * kLn2;
                    }
                }
            }
        }
        if (!whole && at.tile == 0) {
            began = true;
            if (tid == 0)
                p.desc[blockIdx.x] =
                    make_int4(rows.row0, rows.n, joins ? ~at.h : at.h, run.cta_of(at.first + at.tiles - 1));
        }
        if (!at.next(a, run, p)) break;
    }
    if (tid == 0) {
        if (!began) p.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
        if (!alive) kv8_flag(a, kKv8Timeout);
    }
}

// Merge of the units that lie in several runs: CTA (x, y) takes the x-th such
// unit and 16 / MW of its rows.  The MW warps of a row take every so many of its
// segments, each with its own maximum, and meet in shared memory.  A row of few
// units is up to 64 segments, 34 KB that one SM takes 0.5 us for: all 16 warps are
// one row's while there are at most as many rows as SMs, 8 where there are fewer
// units than segments of one, else 2.  Attention and merge in us with 16, 8 and 2:
// one row at 64k tokens 31.5, 31.9, -; five rows (128 of a unit) at 128k 82.9, 80.1,
// 80.9; a batch of 64 sequences 90.7, 80.5, 72.9.
constexpr int kMergeThreads = 512;
template <int HD, int MW, int PART>
__global__ void __launch_bounds__(kMergeThreads) kv8_merge_kernel(const Kv8Args a, const Kv8AttnArgs t, const Kv8Plan p) {
    constexpr int V = HD / 32, BATCH = 8, RW = kMergeThreads / 32 / MW;
    using Vec = typename std::conditional<V == 4, float4, float2>::type;
    static_assert(kKv8MaxCtas <= kMergeThreads, "a thread per run");
    __shared__ float acc_s[RW][MW][HD];
    __shared__ float2 ml_s[RW][MW];
    __shared__ int counts[kMergeThreads / 32];
    __shared__ int4 unit;
    __shared__ int run_x;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, wm = warp % MW, G = p.G;
    if (tid == 0) unit = make_int4(0, 0, 0, 0);
    grid_dependency_wait();
    if (a.stop && *a.stop) return;
    // the x-th run in which such a unit begins
    const int4 mine = tid < p.ctas ? p.desc[tid] : make_int4(0, 0, 0, 0);
    const unsigned begins = __ballot_sync(0xffffffffu, mine.y > 0);
    if (lane == 0) counts[warp] = __popc(begins);
    __syncthreads();
    int rank = __popc(begins & ((1u << lane) - 1));
    for (int i = 0; i < warp; ++i) rank += counts[i];
    if (mine.y > 0 && rank == (int)blockIdx.x) {
        unit = mine;
        run_x = tid;
    }
    __syncthreads();
    const int4 u = unit;
    const int rr = warp / MW, r = blockIdx.y * RW + rr;
    if ((int)blockIdx.y * RW >= u.y) return;
    const int first = run_x;
    // segment i: run first + i; the first one is its run's second slot, a later one its first
    auto part = [&](int i) {
        return p.part + ((size_t)(2 * (first + i) + (i == 0)) * p.rg + r) * (HD + 4);
    };
    const int parts = u.w - first + 1, n = r < u.y && parts > wm ? (parts - wm - 1) / MW + 1 : 0;
    float acc[V], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.f;
    for (int c = 0; c < n; c += BATCH) {
        float2 x = make_float2(-INFINITY, 0.f);
        float o[BATCH][V];
        if (lane < BATCH && c + lane < n) x = *reinterpret_cast<const float2*>(part(wm + (c + lane) * MW));
#pragma unroll
        for (int i = 0; i < BATCH; ++i)
            if (c + i < n)
                *reinterpret_cast<Vec*>(o[i]) =
                    *reinterpret_cast<const Vec*>(part(wm + (c + i) * MW) + 4 + V * lane);
        const float top = fmaxf(m, warp_max(x.x)), ref = top == -INFINITY ? 0.f : top;
        const float old = exp2_approx(m - ref), w = exp2_approx(x.x - ref);
        m = top;
        l = l * old + warp_sum(x.y * w);
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] *= old;
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const float f = __shfl_sync(0xffffffffu, w, i);
            if (c + i < n)
#pragma unroll
                for (int j = 0; j < V; ++j) acc[j] = fmaf(f, o[i][j], acc[j]);
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) acc_s[rr][wm][V * lane + i] = acc[i];
    if (lane == 0) ml_s[rr][wm] = make_float2(m, l);
    __syncthreads();
    if (wm != 0 || r >= u.y) return;
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int i = 0; i < MW; ++i) top = fmaxf(top, ml_s[rr][i].x);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.f;
#pragma unroll
    for (int i = 0; i < MW; ++i) {
        const float f = exp2_approx(ml_s[rr][i].x - ref);
        sum = fmaf(ml_s[rr][i].y, f, sum);
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = fmaf(acc_s[rr][i][V * lane + j], f, acc[j]);
    }
    const bool joins = PART == kTail && u.z < 0;     // a head below zero: ~head, see the units' end
    const int tok = p.token(r), head = (joins ? ~u.z : u.z) * G + r - tok * G;
    float inv = sum == 0.f ? 0.f : 1.f / sum;
    if constexpr (PART == kCommon) {
        const size_t at = (size_t)(u.x + tok) * t.hq + head;
#pragma unroll
        for (int i = 0; i < V; ++i) t.common_out[at * HD + V * lane + i] = acc[i] * inv;
        if (lane == 0) t.common_lse[at] = sum == 0.f ? -INFINITY : top + log2f(sum);
        return;
    }
    if (joins) {
        const size_t at = (size_t)(u.x + tok) * t.hq + head;
        const Joined j(top, sum, t.common_lse[at]);
        __nv_bfloat16* out = t.out + (int64_t)(u.x + tok) * t.out_row + (int64_t)head * t.out_head + V * lane;
#pragma unroll
        for (int i = 0; i < V; ++i)
            out[i] = __float2bfloat16_rn(fmaf(acc[i], j.own, t.common_out[at * HD + V * lane + i] * j.other));
        if (t.lse && lane == 0) t.lse[at] = j.lse * kLn2;
        return;
    }
    __nv_bfloat16* out = t.out + (int64_t)(u.x + tok) * t.out_row + (int64_t)head * t.out_head + V * lane;
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = __float2bfloat16_rn(acc[i] * inv);
    if (t.lse && lane == 0) t.lse[(size_t)(u.x + tok) * t.hq + head] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

// The same for the parts of an attention over common beginnings, where there are
// many such units of few segments each: a warp takes a row, with all of its
// segments, and then the next, so that a CTA's search for its unit is done once.
// 200 rows of 64 heads in five groups, prefix of 4400 tokens: 9 us, and 26 with two
// warps a row and eight rows a CTA.
template <int HD, int PART>
__global__ void __launch_bounds__(kMergeThreads) kv8_rows_merge_kernel(const Kv8Args a, const Kv8AttnArgs t, const Kv8Plan p) {
    constexpr int V = HD / 32, BATCH = 4, WARPS = kMergeThreads / 32;
    using Vec = typename std::conditional<V == 4, float4, float2>::type;
    __shared__ int counts[WARPS];
    __shared__ int4 unit;
    __shared__ int run_x;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, G = p.G;
    if (tid == 0) unit = make_int4(0, 0, 0, 0);
    grid_dependency_wait();
    grid_launch_dependents();
    // the x-th run in which such a unit begins
    const int4 mine = tid < p.ctas ? p.desc[tid] : make_int4(0, 0, 0, 0);
    const unsigned begins = __ballot_sync(0xffffffffu, mine.y > 0);
    if (lane == 0) counts[warp] = __popc(begins);
    __syncthreads();
    int rank = __popc(begins & ((1u << lane) - 1));
    for (int i = 0; i < warp; ++i) rank += counts[i];
    if (mine.y > 0 && rank == (int)blockIdx.x) {
        unit = mine;
        run_x = tid;
    }
    __syncthreads();
    const int4 u = unit;
    const int first = run_x, parts = u.w - first + 1;
    const bool joins = PART == kTail && u.z < 0;     // a head below zero: ~head, see the units' end
    for (int r = blockIdx.y * WARPS + warp; r < u.y; r += gridDim.y * WARPS) {
        const int tok = p.token(r), head = (joins ? ~u.z : u.z) * G + r - tok * G;
        const size_t at = (size_t)(u.x + tok) * t.hq + head;
        Vec common{};
        float common_lse = -INFINITY;
        if (joins) {
            common = *reinterpret_cast<const Vec*>(t.common_out + at * HD + V * lane);
            common_lse = t.common_lse[at];
        }
        // segment i: run first + i; the first one is its run's second slot, a later one its first
        auto part = [&](int i) { return p.part + ((size_t)(2 * (first + i) + (i == 0)) * p.rg + r) * (HD + 4); };
        float acc[V], m = -INFINITY, l = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = 0.f;
        for (int c = 0; c < parts; c += BATCH) {
            float2 x[BATCH];
            float o[BATCH][V];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                x[i] = make_float2(-INFINITY, 0.f);
                if (c + i < parts) {
                    x[i] = *reinterpret_cast<const float2*>(part(c + i));
                    *reinterpret_cast<Vec*>(o[i]) = *reinterpret_cast<const Vec*>(part(c + i) + 4 + V * lane);
                }
            }
            float top = m;
#pragma unroll
            for (int i = 0; i < BATCH; ++i) top = fmaxf(top, x[i].x);
            const float ref = top == -INFINITY ? 0.f : top, old = exp2_approx(m - ref);
            m = top;
            l *= old;
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] *= old;
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
                if (c + i < parts) {
                    const float f = exp2_approx(x[i].x - ref);
                    l = fmaf(x[i].y, f, l);
#pragma unroll
                    for (int j = 0; j < V; ++j) acc[j] = fmaf(f, o[i][j], acc[j]);
                }
        }
        const Joined j(m, l, common_lse);            // -inf: nothing to join with
        const float* other = reinterpret_cast<const float*>(&common);
        if constexpr (PART == kCommon) {
            Vec out;
#pragma unroll
            for (int i = 0; i < V; ++i) reinterpret_cast<float*>(&out)[i] = acc[i] * j.own;
            *reinterpret_cast<Vec*>(t.common_out + at * HD + V * lane) = out;
            if (lane == 0) t.common_lse[at] = j.lse;
        } else {
            __nv_bfloat16* out = t.out + (int64_t)(u.x + tok) * t.out_row + (int64_t)head * t.out_head + V * lane;
#pragma unroll
            for (int i = 0; i < V; ++i)
                out[i] = __float2bfloat16_rn(joins ? fmaf(acc[i], j.own, other[i] * j.other) : acc[i] * j.own);
            if (t.lse && lane == 0) t.lse[at] = j.lse * kLn2;
        }
    }
}

// Query rows of a unit by the batch's average per sequence and KV head, and at
// least G (whole tokens): 8 or 16 for this file's kernel, else the tcgen05
// kernel's 128.  On the Qwen3-32B shape at 64k, 16 rows take 41 us here and 49 us
// there; 24 rows take 74 us here (three row tiles of registers spill), 32 in two
// warps of 16 rows 65 us, and 56 us there.  One size serves the whole call, so an
// uneven batch costs more than its parts: 200 single rows at 4000 tokens 268 us,
// one sequence of 2000 rows at 4000 tokens 201 us, both in one call 811 us (32
// heads over 8); two calls over disjoint sequences are faster there.
int rows_of_unit(int G, int64_t n_rows, int64_t n_seqs, Kv8Part part = kWhole) {
    const int64_t avg = n_seqs > 0 ? (n_rows * G + n_seqs - 1) / n_seqs : 0;
    const int64_t need = std::max<int64_t>(avg, G);
    // What sequences have behind a common beginning is short: two units of 16 rows there read it twice, but begin
    // sooner than one of 128: 60 samples of one to six rows in five groups take 123 us so, 130 with that.
    if (part == kTail && G <= 16 && need > 16 && need <= 32) return 16;
    return need <= 8 ? 8 : need <= 16 ? 16 : kKv8TcRows;
}
// CTAs of an SM
int resident(int rg) { return rg == kKv8TcRows ? 1 : rg == 8 ? 3 : 2; }

template <int HD, int NQ, int PART>
cudaError_t launch_few(const Kv8Args& a, const Kv8AttnArgs& t, const Kv8Plan& p, cudaStream_t s) {
    auto kern = kv8_attention_kernel<HD, NQ, PART>;
    constexpr int bytes = sizeof(Smem<HD, NQ>);
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    return e != cudaSuccess ? e : launch_kv8(kern, dim3(p.ctas), kThreads, bytes, s, a, t, p);
}

template <int HD, int PART>
cudaError_t launch_merge(const Kv8Args& a, const Kv8AttnArgs& t, const Kv8Plan& p, int64_t units, cudaStream_t s) {
    const int x = (int)std::min<int64_t>(p.ctas, units), rows = p.tq * p.G;
    if (units * rows <= kKv8Sms)
        return launch_kv8(kv8_merge_kernel<HD, 16, PART>, dim3(x, rows), kMergeThreads, 0, s, a, t, p);
    if (units * units < p.ctas)
        return launch_kv8(kv8_merge_kernel<HD, 8, PART>, dim3(x, (rows + 1) / 2), kMergeThreads, 0, s, a, t, p);
    if (PART != kWhole) {
        const int most = (rows + kMergeThreads / 32 - 1) / (kMergeThreads / 32);
        return launch_kv8(kv8_rows_merge_kernel<HD, PART == kWhole ? kCommon : PART>,
                          dim3(x, std::min(most, std::max(1, 2 * kKv8Sms / x))), kMergeThreads, 0, s, a, t, p);
    }
    return launch_kv8(kv8_merge_kernel<HD, 2, PART>, dim3(x, (rows + 7) / 8), kMergeThreads, 0, s, a, t, p);
}

// The plan of a call; false if its line of tiles is too long for 32 bits.
bool make_plan(const Kv8Args& a, int hq, Kv8Plan& p, int64_t& units, int64_t& tiles, Kv8Part part) {
    const int G = hq / a.hk;
    p = Kv8Plan{};
    p.rg = rows_of_unit(G, a.n_rows, a.n_seqs, part);
    p.G = G;
    p.token_mul = (65536 + G - 1) / G;
    p.tq = p.rg / G;
    p.tile_log = p.rg == kKv8TcRows ? 7 : 6;
    // A part's ends read or write fp32 rows as well.  64 samples behind 16384 tokens take 72.8, 71.5, 74.0 and 75.6 us at
    // 1, 1.5, 2 and 2.5 times the cost.
    p.cost = (128 * kUnitCost * (part == kWhole ? 2 : 3) / 2) >> p.tile_log;
    p.block_log = (a.bpp & (a.bpp - 1)) == 0 ? __builtin_ctz(a.bpp) : -1;
    tiles = (a.capacity + (1ll << p.tile_log) - 1) >> p.tile_log;
    units = (int64_t)a.hk * (a.n_rows / p.tq + a.n_seqs);
    return units * (tiles + p.cost) <= INT32_MAX;
}

// The plan with what depends on the launch's pointers and device.
bool make_launch(const Kv8Args& a, const Kv8AttnArgs& t, Kv8Plan& p, int64_t& units, int64_t& tiles, Kv8Part part) {
    if (!make_plan(a, t.hq, p, units, tiles, part)) return false;
    p.ctas = (int)std::min<int64_t>(std::min(sm_count(), kKv8Sms) * resident(p.rg), units * (tiles + p.cost));
    p.q_wide = reinterpret_cast<uintptr_t>(t.q) % 16 == 0 && t.q_row % 8 == 0 && t.q_head % 8 == 0;
    p.out_wide = reinterpret_cast<uintptr_t>(t.out) % 16 == 0 && t.out_row % 8 == 0 && t.out_head % 8 == 0;
    p.desc = static_cast<int4*>(t.workspace);
    p.part = reinterpret_cast<float*>(p.desc + kKv8MaxCtas);
    return true;
}

}  // namespace

size_t kv8_attention_workspace(int hd, int group, int n_rows) {
    // A call with more sequences may have smaller units, whose CTAs are more: the largest of all up to this size.
    const int most = rows_of_unit(group, n_rows, 1);
    size_t rows = 0;
    for (int rg : {8, 16, kKv8TcRows})
        if (rg <= most) rows = std::max(rows, (size_t)2 * kKv8Sms * resident(rg) * rg);
    return sizeof(float) * rows * (hd + 4) + sizeof(int4) * kKv8MaxCtas;
}

bool kv8_attention_fits(const Kv8Args& a, int hq, Kv8Part part) {
    Kv8Plan p;
    int64_t units, tiles;
    return make_plan(a, hq, p, units, tiles, part);
}

namespace {

// f with the part as a constant
template <class F>
cudaError_t with_part(Kv8Part part, F&& f) {
    switch (part) {
        case kCommon: return f(std::integral_constant<int, kCommon>{});
        case kTail: return f(std::integral_constant<int, kTail>{});
        default: return f(std::integral_constant<int, kWhole>{});
    }
}

}  // namespace

cudaError_t launch_kv8_attention(const Kv8Args& a, const Kv8AttnArgs& t, cudaStream_t s, bool& merge, Kv8Part part) {
    Kv8Plan p;
    int64_t units, tiles;
    merge = false;
    if (!make_launch(a, t, p, units, tiles, part)) return cudaErrorInvalidValue;
    merge = tiles > 1;
    if (p.rg == kKv8TcRows) return launch_kv8_tc(a, t, p, s, part);
    return with_part(part, [&](auto c) {
        constexpr int PART = decltype(c)::value;
        auto few = [&](auto hd) {
            constexpr int HD = decltype(hd)::value;
            return p.rg == 8 ? launch_few<HD, 1, PART>(a, t, p, s) : launch_few<HD, 2, PART>(a, t, p, s);
        };
        return a.hd == 128 ? few(std::integral_constant<int, 128>{}) : few(std::integral_constant<int, 64>{});
    });
}

cudaError_t launch_kv8_merge(const Kv8Args& a, const Kv8AttnArgs& t, cudaStream_t s, Kv8Part part) {
    Kv8Plan p;
    int64_t units, tiles;
    if (!make_launch(a, t, p, units, tiles, part)) return cudaErrorInvalidValue;
    return with_part(part, [&](auto c) {
        constexpr int PART = decltype(c)::value;
        return a.hd == 128 ? launch_merge<128, PART>(a, t, p, units, s) : launch_merge<64, PART>(a, t, p, units, s);
    });
}

}  // namespace ks
