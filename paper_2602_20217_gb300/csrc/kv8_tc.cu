// Causal attention over the 8-bit paged cache with units of 128 query rows:
// verify passes of many rows and prompts, on tcgen05.
//
// S (128 rows x 128 keys) = Q K^T by kind::f8f6f4, with the cached key codes as
// they are and the queries in two e4m3 codes each, hi and lo (see
// kv8_attn.cu), two products into one accumulator: as many tensor cycles as one
// f16 product, without converting K.  O (rows x dims) += P V by kind::f16, P from
// TMEM in 11 bits, V converted to f16 once per tile by four warps.
// Shared memory carries per 128-key tile 64 KB of the first product's operands,
// 32 KB of the second's and 48 KB of the conversion: 1150 clocks at 128 bytes,
// against 1340 clocks in which 33 KB of the cache arrive at the HBM's rate, so
// padding the rows up to 128 costs nothing that bytes do not; with all 128 rows
// in use the tensor pipe has 1024 clocks of work and the softmax about as many.
//
// Warps 0..3 and 4..7 are two softmax streams, a thread per row each: the CTA's
// even tiles and the odd ones, with a maximum, a sum and an accumulator each
// (TMEM: S0 S1 O0 O1, P in the first half of its S), joined at a segment's end,
// so that one stream's softmax runs under the other's products.  Warps 8
// to 11 convert V, warp 12 issues the products, warp 13 the copies: a record's
// keys, values and scales go to three places, keys and values of a tile
// contiguous, which is the layout that the descriptors without a swizzle take.
//
// The weights are 2^(x - m + 7) with a reference m that is the maximum seen when
// it was set, rounded up to a whole number, not the running one: a row's m is
// raised (and its l, O and the weights of the tile so far multiplied down by a
// power of two, without rounding) only when its weights of 32 keys add up to
// more than 2^15.5.  A raise finishes its 32 keys itself, so no score, however
// far, keeps a row raising.  So most tiles need no maximum at all, no weight
// passes f16, and weights count down to f16's 2^-24, at least 2^-30 of the
// largest (2^-39 where the reference lags behind it): what 128k keys below that
// add up to is under 2^-13 of the row, a sixteenth of the output's rounding.
//
// Measured: 2001 rows of a prompt at 8150 tokens (64 query heads over 8, hd 128)
// 592 us, 790 TFLOP/s; 5 rows of 32 heads over 8 at 131077 tokens 75 us, 3.6
// TB/s; 24 sequences of 2 to 11 rows at up to 16000 tokens 125 us.  What bounds
// it is the round trip of a stream's tile, products to softmax and back, about
// 5000 clocks of which the two products are 1350 and the softmax 2200; the two
// streams hide half.  Taking out the conversion, half of Q K^T and most of P V
// together saves 19 % of the prompt, three quarters of the weights another 26 %.
// All roles share the instruction cache: code in the loops that seldom runs cost
// more than anything it did (raises and quiet blocks in the softmax loop 6 %).  A
// third stream has no TMEM (S and O of two fill it).  Other arrangements of two
// were slower: tiles of 64 keys, two threads a row on one tile, the two products
// issued by two warps, 64 scores at a time or 16.
#include "kv8_plan.cuh"
#include "umma.cuh"

namespace ks {

namespace {

constexpr int kSoftmaxWarps = 8, kConvertWarps = 4, kProductWarp = 12, kCopyWarp = 13;
constexpr int kThreads = 32 * (kSoftmaxWarps + kConvertWarps + 2);
constexpr int kRows = kKv8TcRows, kTile = 128, kBlocks = kTile / kKv8Block;
constexpr int kRing = 3;            // tiles of keys, and of values
constexpr int kNear = 8;            // tiles whose scales are kept
constexpr float kUp = 7.f, kMost = 46340.f;
constexpr float kQuiet = 1.f / 16384.f;
constexpr float kFar = 4194304.f;   // 2^22

// Values' scales are taken relative to vref, which follows the tiles of a
// segment in order: four times the loudest block seen, raised when one passes
// it.  The f16 values carry a block's relative scale down to 2^-14 (codes of
// 2^-9 and more stay exact there), the weights the rest of a quieter block's:
// with a weight of 1 it has 11 bits down to 2^-32 of the loudest block's.
KS_DEV uint32_t f16_times(uint32_t v, __half2 f) {
    const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&v), f);
    return *reinterpret_cast<const uint32_t*>(&r);
}

template <int HD>
struct Smem {
    static constexpr int TILE = kTile * HD;
    unsigned char q[2][kRows * HD];             // hi, lo: [row / 8][HD / 16][8][16]
    unsigned char k[kRing][TILE];               // [key / 8][HD / 16][8][16]
    unsigned char v[kRing][TILE];               // [key / 16][HD][16]
    unsigned char v16[2][2 * TILE];             // f16 [key / 8][HD][8]
    float2 scale[kNear][kBlocks];               // key scale, value scale
    __half2 factor[kNear][kBlocks];             // of the values
    float4 join[2][kRows];                      // m, l, vref of a stream
    float qf[kRows];
    float vref[kNear];                          // of a tile; negative: one of its blocks is quiet
    int nan_from[4][HD];                        // first key whose value is NaN, a segment each
    int any_nan[4];
    int present[kNear];
    uint64_t scales[kNear], k_full[kRing], k_free[kRing], v_full[kRing], v_free[kRing], v16_full[2];
    uint64_t q_full, s_full[2], p_full[2], o_full[2], o_free;
    uint32_t tmem;
};

KS_DEV void umma_e4m3(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{ .reg .pred p; setp.ne.u32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p; }" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}
// K-major operand without a swizzle: 8-row x 16-byte matrices of 128 contiguous
// bytes, lbo apart along K and sbo apart along M or N.
KS_DEV uint64_t desc_plain(uint32_t addr, uint32_t lbo, uint32_t sbo) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(lbo >> 4) << 16) | ((uint64_t)(sbo >> 4) << 32) | (1ull << 46);
}
// fp32 accumulators; e4m3 for kind::f8f6f4 and f16 for kind::f16 are both type 0
__host__ __device__ constexpr uint32_t idesc_of(int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kRows >> 4) << 24); }

// Whether three phases have ended, without waiting: a look takes a hundred clocks, the three overlap.
KS_DEV void mbar_look(const uint64_t* a, int pa, const uint64_t* b, int pb, const uint64_t* c, int pc, bool& ra, bool& rb,
                      bool& rc) {
    uint32_t x, y, z;
    asm volatile(
        "{ .reg .pred p, q, r;\n"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%3], %4;\n"
        "mbarrier.test_wait.parity.shared::cta.b64 q, [%5], %6;\n"
        "mbarrier.test_wait.parity.shared::cta.b64 r, [%7], %8;\n"
        "selp.u32 %0, 1, 0, p;\nselp.u32 %1, 1, 0, q;\nselp.u32 %2, 1, 0, r; }"
        : "=r"(x), "=r"(y), "=r"(z)
        : "r"(smem_u32(a)), "r"(pa), "r"(smem_u32(b)), "r"(pb), "r"(smem_u32(c)), "r"(pc)
        : "memory");
    ra = x;
    rb = y;
    rc = z;
}
KS_DEV void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// v[i] of a register array, for an i that is not known when compiling
KS_DEV float pick(const float (&v)[kBlocks], int i) {
    const float a = i & 1 ? v[1] : v[0], b = i & 1 ? v[3] : v[2], c = i & 1 ? v[5] : v[4], d = i & 1 ? v[7] : v[6];
    const float e = i & 2 ? b : a, f = i & 2 ? d : c;
    return i & 4 ? f : e;
}
// 2^d for a whole d <= 0 (-inf: 0)
KS_DEV float pow2_below(float d) { return d < -126.f ? 0.f : __uint_as_float((uint32_t)(127 + (int)d) << 23); }
// The first n x 32 weights of a row, in TMEM, times f <= 1, in two factors: below
// 2^-24 f is no f16 number, but its products with weights up to 2^15.5 are.
KS_DEV void scale_weights(uint32_t at, int n, float f) {
    const float f1 = fmaxf(f, kQuiet);
    const __half2 w1 = __float2half2_rn(f1), w2 = __float2half2_rn(f / f1);
#pragma unroll 1
    for (int c = 0; c < n; ++c) {
        uint32_t x[16];
        tmem_wait_st();
        tmem_ld16(x, at + 16 * c);
        tmem_wait_ld();
        tmem_pin(x);
#pragma unroll
        for (int q = 0; q < 16; ++q) x[q] = f16_times(f16_times(x[q], w1), w2);
        tmem_st16(at + 16 * c, x);
    }
}
// Whether the weights of a row with this reference need products that are rounded
// before the reference is taken off.  s f - (m - 7) in one rounding keeps the whole
// product, and m came from rounded ones: that differs by half a unit in the last
// place of the product, 16 at scores of 2^28, and m - 7 is m from there on.
KS_DEV bool far(float m) { return fabsf(m) >= kFar && m != -INFINITY; }
KS_DEV void softmax_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
KS_DEV void convert_sync() { asm volatile("bar.sync 2, 128;" ::: "memory"); }

template <int HD, int KIND>
__global__ void __launch_bounds__(kThreads, 1)
    kv8_tc_kernel(const Kv8Args a, const Kv8AttnArgs t, const Kv8Plan p, const __grid_constant__ CUtensorMap map) {
    using S = Smem<HD>;
    constexpr int REC = kv8_record(HD), PART = kKv8Block * HD;   // a record's keys (or values)
    extern __shared__ __align__(128) unsigned char smem_raw[];
    S& sm = *reinterpret_cast<S*>(smem_raw);
    volatile int* present = sm.present;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (warp == kProductWarp) tmem_alloc<1>(&sm.tmem, 512);
    if (tid == 0) {
        for (int i = 0; i < kNear; ++i) mbar_init(&sm.scales[i], 1);
        for (int i = 0; i < kRing; ++i) {
            mbar_init(&sm.k_full[i], 1);
            mbar_init(&sm.k_free[i], 1);
            mbar_init(&sm.v_full[i], 1);
            mbar_init(&sm.v_free[i], kConvertWarps / 2);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sm.v16_full[i], kConvertWarps / 2);
            mbar_init(&sm.s_full[i], 1);
            mbar_init(&sm.p_full[i], 4);
            mbar_init(&sm.o_full[i], 2);        // the products' commit, and an arrival that orders nan_from before it
        }
        mbar_init(&sm.q_full, kSoftmaxWarps);
        mbar_init(&sm.o_free, kSoftmaxWarps);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (int i = tid; i < 4 * HD; i += kThreads) sm.nan_from[0][i] = INT32_MAX;
    if (tid < 4) sm.any_nan[tid] = 0;
    umma_fence_before();
    __syncthreads();
    umma_fence_after();
    const uint32_t tmem = sm.tmem;
    grid_dependency_wait();
    grid_launch_dependents();
    Run run;
    Segment<KIND> at;
    const bool stopped = a.stop && *a.stop;
    const bool work = !stopped && find_run(a, p, run, at);
    if (!work && !stopped && tid == 0) p.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
    const int G = p.G;

    if (!work) {
        // nothing in this run
    } else if (warp == kCopyWarp) {
        // ---------------------------------------------------------- copies
        // Page numbers are read a group of tiles ahead, across segments.
        constexpr int TILES = 32 / kBlocks;
        auto pages = [&](const Segment<KIND>& k, int tile) {
            const int b = tile * kBlocks + lane;
            if (b * kKv8Block > last_key<KIND>(k.q, p, k.g) || tile + lane / kBlocks >= k.end) return -1;
            const int page = pages_of<KIND>(a, k.s)[p.page_of(b, a.bpp)];
            return page >= 0 && page < a.n_pages ? page : -2;
        };
        // a run of p.run records is one copy of keys and one of values
        const int r = lane % kBlocks;
        const unsigned heads = p.run == 8 ? 0x01u : p.run == 4 ? 0x11u : p.run == 2 ? 0x55u : 0xffu;
        int it = 0, tile = at.tile, page = pages(at, tile);
        float vref = 0.f;
        bool alive = true, more = true;
        while (more && alive) {
            Segment<KIND> next = at;
            int next_tile = tile + TILES;
            if (next_tile >= at.end) {
                more = next.next(a, run, p);
                next_tile = next.tile;
            }
            const int next_page = more ? pages(next, next_tile) : -1;
            if (page == -2) kv8_flag(a, kKv8BadPage);
            const int b = tile * kBlocks + lane;
            const int record = page >= 0 ? (page * a.hk + at.h) * a.bpp + b - p.page_of(b, a.bpp) * a.bpp : -1;
            // the scales come by ordinary loads, behind the first copies
            float2 scale = make_float2(0.f, 0.f);
            if (record >= 0) scale = *reinterpret_cast<const float2*>(a.data + (size_t)record * REC + 2 * PART);
            const unsigned have = __ballot_sync(0xffffffffu, record >= 0);
            float top = scale.y;                     // of the lane's tile
#pragma unroll
            for (int o = 1; o < kBlocks; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            if (tile == at.tile) vref = 0.f;
            for (int i = 0; i < TILES && tile + i < at.end; ++i, ++it) {
                const int st = it % kRing, near = it % kNear, odd = ((it / kRing) & 1) ^ 1;
                const unsigned mask = have >> (i * kBlocks) & ((1u << kBlocks) - 1);
                alive = mbar_wait(&sm.k_free[st], odd, kWaitLimitNs) && mbar_wait(&sm.v_free[st], odd, kWaitLimitNs);
                if (!__all_sync(0xffffffffu, alive)) {
                    alive = false;
                    break;
                }
                if (lane == 0) {
                    const uint32_t bytes = __popc(mask & heads) * p.run * PART;
                    present[near] = (int)mask;
                    mbar_expect_tx(&sm.k_full[st], bytes);
                    mbar_expect_tx(&sm.v_full[st], bytes);
                }
                __syncwarp();
                if (lane / kBlocks == i && record >= 0 && (heads >> r & 1)) {
                    tma_2d(sm.k[st] + r * PART, &map, 0, record, &sm.k_full[st]);
                    tma_2d(sm.v[st] + r * PART, &map, PART / 8, record, &sm.v_full[st]);
                }
                const float loudest = __shfl_sync(0xffffffffu, top, i * kBlocks);
                if (loudest > vref) vref = 4.f * loudest;
                const float rel = scale.y * inverse_pow2(vref);
                const bool own = lane / kBlocks == i && record >= 0;
                const unsigned quiet = __ballot_sync(0xffffffffu, own && rel < kQuiet);
                if (own) {
                    sm.scale[near][r] = scale;
                    sm.factor[near][r] = __float2half2_rn(fmaxf(rel, kQuiet));
                }
                if (lane == 0) sm.vref[near] = quiet ? -vref : vref;
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm.scales[near]);
            }
            at = next;
            tile = next_tile;
            page = next_page;
        }
        if (!alive && lane == 0) kv8_flag(a, kKv8Timeout);
        // no copy may be in flight when the CTA ends
        for (int i = max(0, it - kRing); i < it; ++i) {
            mbar_wait(&sm.k_full[i % kRing], (i / kRing) & 1, kWaitLimitNs);
            mbar_wait(&sm.v_full[i % kRing], (i / kRing) & 1, kWaitLimitNs);
        }
    } else if (warp == kProductWarp) {
        // -------------------------------------------------------- products
        if (lane == 0) {
            constexpr uint32_t kIdS = idesc_of(kTile), kIdO = idesc_of(HD);
            bool ok = true;
            int it0 = 0, seg = 0, n[2] = {0, 0};     // tiles before the segment, segments, tiles of each stream
            do {
                const int cnt = at.end - at.tile;
                ok = mbar_wait(&sm.q_full, seg & 1, kWaitLimitNs);
                auto scores = [&](int j, bool here) {
                    const int st = (it0 + j) % kRing, i = (it0 + j) & 1;
                    ok = ok && (here || mbar_wait(&sm.k_full[st], ((it0 + j) / kRing) & 1, kWaitLimitNs));
                    if (!ok) return;
                    umma_fence_after();
                    // hi, then lo; a step of 256 bytes is 16 in a descriptor
                    const uint64_t q0 = desc_plain(smem_u32(sm.q[0]), 128, 8 * HD), k0 = desc_plain(smem_u32(sm.k[st]), 128, 8 * HD);
#pragma unroll
                    for (int c = 0; c < HD / 16; ++c) {
                        const int k = c % (HD / 32);
                        umma_e4m3(tmem + 128 * i, q0 + (c / (HD / 32) * (kRows * HD / 16) + 16 * k), k0 + 16 * k, kIdS, c > 0);
                    }
                    umma_commit(&sm.s_full[i]);
                };
                scores(0, false);
                if (cnt > 1) scores(1, false);
                if (seg > 0) ok = ok && mbar_wait(&sm.o_free, (seg - 1) & 1, kWaitLimitNs);
                for (int j = 0; j < cnt && ok; ++j) {
                    const int i = (it0 + j) & 1;
                    const int next = it0 + j + 2;
                    bool weights, values, keys;
                    mbar_look(&sm.p_full[i], n[i] & 1, &sm.v16_full[i], ((it0 + j) >> 1) & 1, &sm.k_full[next % kRing],
                              (next / kRing) & 1, weights, values, keys);
                    ok = (values || mbar_wait(&sm.v16_full[i], ((it0 + j) >> 1) & 1, kWaitLimitNs)) &&
                         (weights || mbar_wait(&sm.p_full[i], n[i] & 1, kWaitLimitNs));
                    if (!ok) break;
                    ++n[i];
                    umma_fence_after();
                    const uint64_t v0 = desc_plain(smem_u32(sm.v16[i]), 16 * HD, 128);
#pragma unroll
                    for (int c = 0; c < kTile / 16; ++c)
                        umma_ts(tmem + 256 + 128 * i, tmem + 128 * i + 8 * c, v0 + 2 * HD * c, kIdO, j > 1 || c > 0);
                    umma_commit(&sm.o_full[i]);
                    mbar_arrive(&sm.o_full[i]);
                    if (j + 2 < cnt) scores(j + 2, keys);
                }
                it0 += cnt;
                ++seg;
            } while (ok && at.next(a, run, p));
            if (!ok) kv8_flag(a, kKv8Timeout);
        }
        __syncwarp();
    } else if (warp >= kSoftmaxWarps) {
        // ------------------------------------------------------ V to f16
        // two warps a tile, even and odd ones: a tile's fixed latencies pass under the other's work
        const int mine = (warp - kSoftmaxWarps) / (kConvertWarps / 2), ct = tid % (16 * kConvertWarps);
        bool alive = true;
        int it = 0, seg = 0;
        do {
            const Rows rows(at, p.tq, G);
            for (int tile = at.tile; tile < at.end; ++tile, ++it) {
                const int st = it % kRing, b = it & 1, near = it % kNear;
                if (b == mine) alive = alive && mbar_wait(&sm.o_full[b], ((it >> 1) & 1) ^ 1, kWaitLimitNs);
                if (tile == at.tile) {
                    // Clear the next segment's marks.  The products of the tile two before are done, so those of
                    // the segment two back have begun and the readers of the one three back, who had this
                    // buffer, have left; and nobody marks the next segment before all have cleared.
                    convert_sync();
                    for (int i = tid - 32 * kSoftmaxWarps; i < HD; i += 32 * kConvertWarps)
                        sm.nan_from[(seg + 1) & 3][i] = INT32_MAX;
                    if (tid == 32 * kSoftmaxWarps) sm.any_nan[(seg + 1) & 3] = 0;
                    convert_sync();
                }
                if (b != mine) continue;
                alive = alive && mbar_wait(&sm.scales[near], (it / kNear) & 1, kWaitLimitNs);
                const int have = present[near];
                alive = alive && mbar_wait(&sm.v_full[st], (it / kRing) & 1, kWaitLimitNs);
                const bool edge = have != (1 << kBlocks) - 1 || tile * kTile + kTile - 1 > rows.pos0;
                const unsigned char* src = sm.v[st];
                unsigned char* dst = sm.v16[b];
                auto convert = [&](int r, int d, uint4 x, __half2 f) {
                    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
                    uint32_t lo[4], hi[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        lo[j] = f16_times(f16_of((uint16_t)w[j]), f);
                        hi[j] = f16_times(f16_of((uint16_t)(w[j] >> 16)), f);
                    }
                    *reinterpret_cast<uint4*>(dst + (2 * r * HD + d) * 16) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                    *reinterpret_cast<uint4*>(dst + ((2 * r + 1) * HD + d) * 16) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                };
                constexpr int STEP = 16 * kConvertWarps, N = kBlocks * HD / STEP, PER = HD / STEP;   // passes a record
                // the next loads first: they wait behind the products' reads of shared memory
                constexpr int AHEAD = 4;
                uint4 x[AHEAD], next[AHEAD];
                auto load = [&](int c) {
#pragma unroll
                    for (int i = 0; i < AHEAD; ++i)
                        next[i] = *reinterpret_cast<const uint4*>(src + ((c + i) * STEP + ct) * 16);
                };
                load(0);
#pragma unroll 1
                for (int c = 0; c < N; c += AHEAD) {
                    __half2 f[AHEAD];
#pragma unroll
                    for (int i = 0; i < AHEAD; ++i) {
                        x[i] = next[i];
                        f[i] = sm.factor[near][(c + i) / PER];
                    }
                    if (c + AHEAD < N) load(c + AHEAD);
                    if (edge) {
                        // absent records are zeros; a NaN that not every row sees would pass through a weight of
                        // zero: it is taken out, and the rows that do see it get their NaN at the end
                        uint32_t any = 0;
#pragma unroll
                        for (int i = 0; i < AHEAD; ++i) {
                            const bool here = have >> (c + i) / PER & 1;
                            uint32_t* w = reinterpret_cast<uint32_t*>(&x[i]);
                            if (!here) f[i] = __half2(0.f, 0.f);
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                if (!here) w[j] = 0;
                                const uint32_t nan = ((w[j] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
                                any |= nan;
                                w[j] &= ~((nan >> 7) * 0xffu);
                            }
                        }
                        if (any) {
                            sm.any_nan[seg & 3] = 1;
#pragma unroll 1
                            for (int k = 0; k < 16 * AHEAD; ++k) {           // bytes: tokens in the records' order
                                const int at = (c + k / 16) * STEP + ct, r = at / HD, byte = k & 15;
                                if ((have >> r & 1) && (src[at * 16 + byte] & 0x7f) == 0x7f)
                                    atomicMin(&sm.nan_from[seg & 3][at % HD], tile * kTile + 16 * r + 2 * (byte >> 2) +
                                                                                  (byte & 1) + 8 * (byte >> 1 & 1));
                            }
                        }
                    }
#pragma unroll
                    for (int i = 0; i < AHEAD; ++i) convert((c + i) / PER, (i % PER) * STEP + ct, x[i], f[i]);
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&sm.v16_full[b]);
                    mbar_arrive(&sm.v_free[st]);
                }
            }
            ++seg;
        } while (at.next(a, run, p));
        if (!alive && lane == 0) kv8_flag(a, kKv8Timeout);
    } else {
        // --------------------------------------------------------- softmax
        const int i = warp >> 2, quad = warp & 3, lane_row = 32 * quad + lane;
        const uint32_t lanes = tmem + ((uint32_t)(32 * quad) << 16);
        const uint32_t s_at = lanes + 128 * i, o_at = lanes + 256 + 128 * i;
        bool alive = true, began = false;
        int it0 = 0, seg = 0, n = 0;                 // tiles before the segment, segments, tiles of this stream
        for (;;) {
            const Rows rows(at, p.tq, G);
            const int cnt = at.end - at.tile;
            // Few rows: they stand in the 128 two or four times, and the warps of a copy take 64 or 32 of a tile's keys
            // (TMEM lanes belong to warps: the other warps could not help with them).  Their weights of the other
            // keys are zeros, and the copies' O are added at the end.
            const int copies = rows.n <= 32 ? 4 : rows.n <= 64 ? 2 : 1, per = 4 / copies;
            const int row = 32 * (quad % per) + lane, c0 = quad / per * per, c1 = c0 + per;     // own 32-key chunks
            {
                // the unit's queries in two codes: two threads a row
                const int qr = tid >> 1, half = tid & 1, ur = qr & (kRows / copies - 1);
                const bool valid = ur < rows.n;
                const int tok = valid ? p.token(ur) : 0, head = at.h * G + (valid ? ur - tok * G : 0);
                const __nv_bfloat16* src = t.q + (int64_t)(rows.row0 + tok) * t.q_row + (int64_t)head * t.q_head + half * (HD / 2);
                uint4 raw[HD / 16];
                if (p.q_wide) {
#pragma unroll
                    for (int c = 0; c < HD / 16; ++c) raw[c] = *reinterpret_cast<const uint4*>(src + 8 * c);
                } else {
                    const unsigned short* e = reinterpret_cast<const unsigned short*>(src);
#pragma unroll
                    for (int c = 0; c < HD / 16; ++c)
                        raw[c] = make_uint4(e[8 * c] | (uint32_t)e[8 * c + 1] << 16, e[8 * c + 2] | (uint32_t)e[8 * c + 3] << 16,
                                            e[8 * c + 4] | (uint32_t)e[8 * c + 5] << 16, e[8 * c + 6] | (uint32_t)e[8 * c + 7] << 16);
                }
                float top = 0.f;
                const uint32_t* w = reinterpret_cast<const uint32_t*>(raw);
#pragma unroll
                for (int c = 0; c < HD / 4; ++c) {
                    const float x0 = bf16_lo(w[c]), x1 = bf16_hi(w[c]);
                    if (finite(x0)) top = fmaxf(top, fabsf(x0));
                    if (finite(x1)) top = fmaxf(top, fabsf(x1));
                }
                if (!valid) top = 0.f;
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                // a scale below zero goes into the codes' sign, so that the factors of the scores are positive
                const float sc = scale_for(top), inv = t.scale < 0.f ? -inverse_pow2(sc) : inverse_pow2(sc);
                if (half == 0 && qr < kRows / copies) sm.qf[qr] = sc * (fabsf(t.scale) * kLog2e);
#pragma unroll
                for (int c = 0; c < HD / 32; ++c) {
                    uint32_t hi[4], lo[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float x[4] = {bf16_lo(w[8 * c + 2 * j]), bf16_hi(w[8 * c + 2 * j]),
                                      bf16_lo(w[8 * c + 2 * j + 1]), bf16_hi(w[8 * c + 2 * j + 1])};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (!finite(x[e])) x[e] = __uint_as_float(0x7fc00000u);   // the row becomes NaN
                            x[e] = valid ? x[e] * inv : 0.f;
                        }
                        const uint16_t h0 = to_e4m3x2(x[0], x[1]), h1 = to_e4m3x2(x[2], x[3]);
                        const float2 f0 = from_e4m3x2(h0), f1 = from_e4m3x2(h1);
                        hi[j] = h0 | (uint32_t)h1 << 16;
                        lo[j] = to_e4m3x2(x[0] - f0.x, x[1] - f0.y) | (uint32_t)to_e4m3x2(x[2] - f1.x, x[3] - f1.y) << 16;
                    }
                    const int to = (qr >> 3) * 8 * HD + (half * (HD / 32) + c) * 128 + (qr & 7) * 16;
                    *reinterpret_cast<uint4*>(sm.q[0] + to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                    *reinterpret_cast<uint4*>(sm.q[1] + to) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                }
                fence_async_smem();
                softmax_sync();                      // qf too
                if (lane == 0) mbar_arrive(&sm.q_full);
            }
            const float qf = sm.qf[row];
            const int lim = row < rows.n ? rows.pos0 + p.token(row) * rows.step : INT32_MAX;
            float m = -INFINITY, l = 0.f, vref = 0.f;
            bool first = true;
            auto rescale = [&](float fac) {           // O, once the products before are in it
                alive = alive && mbar_wait(&sm.o_full[i], (n - 1) & 1, kWaitLimitNs);
                __syncwarp();
                umma_fence_after();
#pragma unroll 1
                for (int c = 0; c < HD / 16; ++c) {
                    uint32_t o[16];
                    tmem_ld16(o, o_at + 16 * c);
                    tmem_wait_ld();
                    tmem_pin(o);
#pragma unroll
                    for (int q = 0; q < 16; ++q) o[q] = __float_as_uint(__uint_as_float(o[q]) * fac);
                    tmem_st16(o_at + 16 * c, o);
                }
                tmem_wait_st();
            };
            for (int j = (it0 ^ i) & 1; j < cnt; j += 2, ++n) {
                const int tile = at.tile + j, near = (it0 + j) % kNear;
                alive = alive && mbar_wait(&sm.scales[near], ((it0 + j) / kNear) & 1, kWaitLimitNs);
                // read before the scores are there: shared memory is the products' while they run, and a load
                // between them takes hundreds of clocks
                float f[kBlocks];
#pragma unroll
                for (int c = 0; c < kBlocks; ++c) f[c] = fmaxf(qf * sm.scale[near][c].x, 1e-36f);   // above zero: -inf stays
                const int have = present[near];
                const float vnow = sm.vref[near], vnew = fabsf(vnow);
                const bool edge = have != (1 << kBlocks) - 1 || tile * kTile + kTile - 1 > rows.pos0;
                const bool fresh = __any_sync(0xffffffffu, m == -INFINITY);
                const bool special = edge || fresh || vnew != vref;
                alive = alive && mbar_wait(&sm.s_full[i], n & 1, kWaitLimitNs);
                __syncwarp();
                if (quad == 0 && lane == 0) mbar_arrive(&sm.k_free[(it0 + j) % kRing]);      // spares the issuing thread a commit
                umma_fence_after();
                if (32 * (quad % per) >= rows.n) {   // no row: P stays what it is, in lanes that nobody reads
                    if (lane == 0) mbar_arrive(&sm.p_full[i]);
                    continue;
                }
                if (special) {
                    if (edge) {
                        // what a row does not see becomes -inf where it lies, so that the pass below needs no mask
#pragma unroll 1
                        for (int c = c0; c < c1; ++c) {
                            uint32_t x[32];
                            tmem_ld32(x, s_at + 32 * c);
                            tmem_wait_ld();
                            tmem_pin(x);
#pragma unroll
                            for (int q = 0; q < 32; ++q)
                                if (tile * kTile + 32 * c + q > lim || !(have >> (2 * c + q / 16) & 1)) x[q] = 0xff800000u;
                            tmem_st32(s_at + 32 * c, x);
                        }
                        tmem_wait_st();
                    }
                    if (vnew != vref) {
                        if (!first) rescale(vref * inverse_pow2(vnew));
                        vref = vnew;
                    }
                    if (fresh) {
                        float top = m;
#pragma unroll 1
                        for (int c = c0; c < c1; ++c) {
                            uint32_t x[32];
                            tmem_ld32(x, s_at + 32 * c);
                            const float f0 = pick(f, 2 * c), f1 = pick(f, 2 * c + 1);
                            tmem_wait_ld();
                            tmem_pin(x);
#pragma unroll
                            for (int q = 0; q < 32; ++q) top = fmaxf(top, __uint_as_float(x[q]) * (q < 16 ? f0 : f1));
                        }
                        if (m == -INFINITY) m = ceilf(top);          // l and O are still zero
                    }
                }
                // 32 scores at a time, in a short loop: unrolled, or with what is rare in it, the roles' code together
                // no longer fits the instruction cache, and a tile of the softmax takes up to 6700 clocks.
                for (int c = c0; c < c1; ++c) {
                    // no sum of weights is below zero: a row of far scores leaves the loop at every chunk
                    const float most = far(m) ? -1.f : kMost;
                    bool raise = false;
#pragma unroll 1
                    for (; c < c1; ++c) {
                        uint32_t s[32], pk[16];
                        tmem_ld32(s, s_at + 32 * c);
                        const float f0 = pick(f, 2 * c), f1 = pick(f, 2 * c + 1);
                        const float ref = (m == -INFINITY ? 0.f : m) - kUp;
                        tmem_wait_ld();
                        tmem_pin(s);
                        float2 part[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                        for (int q = 0; q < 32; q += 2) {
                            const float fq = q < 16 ? f0 : f1;
                            const float2 x = fma2(make_float2(__uint_as_float(s[q]), __uint_as_float(s[q + 1])),
                                                  make_float2(fq, fq), make_float2(-ref, -ref));
                            const float2 y = make_float2(exp2_approx(x.x), exp2_approx(x.y));
                            part[q / 2 & 1] = add2(part[q / 2 & 1], y);
                            pk[q / 2] = f16_pack(y.x, y.y);
                        }
                        part[0] = add2(part[0], part[1]);
                        const float sum = part[0].x + part[0].y;
                        raise = sum > most;          // else no weight passes f16
                        if (__any_sync(0xffffffffu, raise)) break;
                        l += sum;
                        tmem_st16(s_at + 16 * c, pk);                    // over scores that are used
                    }
                    if (c >= c1) break;
                    // A chunk in which a row is raised is done here, whatever comes of it: one visit a chunk.  Only that
                    // row's own reference moves, to a whole number: the factor is exact.  A product below 2^22 rounds by a
                    // quarter at most, so no weight of the row is above 2^(kUp + 1/4) then; those of far scores (see far())
                    // come from rounded products, as the reference did, and are at most 2^kUp.  A block at a time keeps
                    // this short: 32 scores in one go take the batch of verify passes from 127 to 130 us.
                    float top = m;
#pragma unroll 1
                    for (int b = 2 * c; b < 2 * c + 2; ++b) {
                        uint32_t s[16];
                        tmem_ld16(s, s_at + 16 * b);
                        const float fq = pick(f, b);
                        tmem_wait_ld();
                        tmem_pin(s);
#pragma unroll
                        for (int q = 0; q < 16; ++q) top = fmaxf(top, __uint_as_float(s[q]) * fq);
                    }
                    const float mnew = raise ? fmaxf(m, ceilf(top)) : m;
                    const float fac = m == mnew ? 1.f : pow2_below(m - mnew);
                    l *= fac;
                    m = mnew;
                    if (!first) rescale(fac);
                    scale_weights(s_at + 16 * c0, c - c0, fac);          // of this tile so far
                    const float base = m == -INFINITY ? 0.f : m, ref = base - kUp;
                    const bool apart = far(m);
                    float2 part[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll 1
                    for (int b = 2 * c; b < 2 * c + 2; ++b) {
                        uint32_t s[16], pk[8];
                        tmem_ld16(s, s_at + 16 * b);
                        const float fq = pick(f, b);
                        tmem_wait_ld();
                        tmem_pin(s);
#pragma unroll
                        for (int q = 0; q < 16; q += 2) {
                            const float s0 = __uint_as_float(s[q]), s1 = __uint_as_float(s[q + 1]);
                            float2 x = fma2(make_float2(s0, s1), make_float2(fq, fq), make_float2(-ref, -ref));
                            if (apart)
                                x = make_float2(__fsub_rn(__fmul_rn(s0, fq), base) + kUp,
                                                __fsub_rn(__fmul_rn(s1, fq), base) + kUp);
                            const float2 y = make_float2(exp2_approx(x.x), exp2_approx(x.y));
                            part[q / 2 & 1] = add2(part[q / 2 & 1], y);
                            pk[q / 2] = f16_pack(y.x, y.y);
                        }
                        tmem_st8(s_at + 8 * b, pk);
                    }
                    part[0] = add2(part[0], part[1]);                    // as in the loop: a row's sum is its own affair
                    l += part[0].x + part[0].y;
                }
                if (vnow < 0.f) {                    // a quiet block
                    const float vinv = inverse_pow2(vref);
#pragma unroll 1
                    for (int c = c0; c < c1; ++c) {
                        uint32_t x[16];
                        tmem_wait_st();
                        tmem_ld16(x, s_at + 16 * c);
                        tmem_wait_ld();
                        tmem_pin(x);
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int b = 2 * c + e;
                            const float y = have >> b & 1 ? sm.scale[near][b].y * vinv : 1.f;
                            const __half2 w = __float2half2_rn(fminf(y * (1.f / kQuiet), 1.f));
#pragma unroll
                            for (int q = 0; q < 8; ++q) x[8 * e + q] = f16_times(x[8 * e + q], w);
                        }
                        tmem_st16(s_at + 16 * c, x);
                    }
                }
                if (copies > 1) {                    // zeros for the other chunks: one pair, and half of the own one
                    uint32_t zero[32], half[16];
#pragma unroll
                    for (int q = 0; q < 32; ++q) zero[q] = half[q / 2] = 0;
                    tmem_st32(s_at + 32 * (c0 < 2), zero);
                    if (per == 1) tmem_st16(s_at + 16 * (c0 ^ 1), half);
                }
                first = false;
                tmem_wait_st();
                umma_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm.p_full[i]);
            }
            // ---------------------------------------------- segment's end
            const bool mine = cnt > ((it0 ^ i) & 1);                     // this stream had a tile
            const bool has0 = cnt > 1 || !(it0 & 1), has1 = cnt > 1 || (it0 & 1);
            if (mine) alive = alive && mbar_wait(&sm.o_full[i], (n - 1) & 1, kWaitLimitNs);
            sm.join[i][lane_row] = make_float4(m, l, vref, 0.f);
            umma_fence_before();
            softmax_sync();
            umma_fence_after();
            // both streams' O over half of the dims each, relative to the maximum over streams and copies
            float top = -INFINITY, sum = 0.f;
            for (int c = 0; c < copies; ++c)
                top = fmaxf(top, fmaxf(sm.join[0][row + c * per * 32].x, sm.join[1][row + c * per * 32].x));
            const float ref = top == -INFINITY ? 0.f : top;
            for (int c = 0; c < copies; ++c)
                for (int k = 0; k < 2; ++k) {
                    const float4 u = sm.join[k][row + c * per * 32];
                    sum = fmaf(u.y, exp2_approx(u.x - ref), sum);
                }
            const float4 u0 = sm.join[0][lane_row], u1 = sm.join[1][lane_row];
            const float o0 = exp2_approx(u0.x - ref) * u0.z, o1 = exp2_approx(u1.x - ref) * u1.z;
            const bool whole = at.tile == 0 && at.end == at.tiles;
            float inv = whole ? (sum == 0.f ? 0.f : 1.f / sum) : 1.f;
            const bool valid = row < rows.n, any_nan = sm.any_nan[seg & 3];
            const int tok = valid ? p.token(row) : 0, head = at.h * G + (valid ? row - tok * G : 0);
            const size_t common_at = (size_t)(rows.row0 + tok) * t.hq + head;
            bool joins = false;                      // with what its group has in common
            float other = 0.f, joined = 0.f;
            if constexpr (KIND == kTail) {
                joins = t.cut[at.s] > 0;
                if (whole && joins) {
                    const Joined j(top - kUp, sum, t.common_lse[common_at]);
                    inv = j.own;
                    other = j.other;
                    joined = j.lse;
                }
            }
            float* slot = p.part + ((size_t)(2 * blockIdx.x + (at.tile == 0)) * p.rg + row) * (HD + 4);
            __nv_bfloat16* out = t.out + (int64_t)(rows.row0 + tok) * t.out_row + (int64_t)head * t.out_head;
            float* pile = reinterpret_cast<float*>(sm.q);        // free: every product with it is done
#pragma unroll 1
            for (int c = 0; c < HD / 64; ++c) {
                const int d0 = i * (HD / 2) + 32 * c;
                uint32_t x[32], y[32];
                tmem_ld32(x, lanes + 256 + d0);
                tmem_ld32(y, lanes + 384 + d0);
                tmem_wait_ld();
                tmem_pin(x);
                tmem_pin(y);
#pragma unroll
                for (int q = 0; q < 32; ++q) {
                    float v = has0 ? __uint_as_float(x[q]) * o0 : 0.f;   // a stream without a tile has no O
                    if (has1) v = fmaf(__uint_as_float(y[q]), o1, v);
                    x[q] = __float_as_uint(v);
                }
                // add the copies, half of them at a time: 32 x 32 values a warp
                for (int n = copies / 2; n > 0; n /= 2) {
                    const int copy = quad / per;
                    softmax_sync();
                    if (copy >= n && copy < 2 * n) {
                        float* to = pile + (i * 2 + (quad - n * per)) * 1024 + lane;
#pragma unroll
                        for (int q = 0; q < 32; ++q) to[32 * q] = __uint_as_float(x[q]);
                    }
                    softmax_sync();
                    if (copy < n) {
                        const float* from = pile + (i * 2 + quad) * 1024 + lane;
#pragma unroll
                        for (int q = 0; q < 32; ++q) x[q] = __float_as_uint(__uint_as_float(x[q]) + from[32 * q]);
                    }
                }
                if (quad >= per || !valid) continue;
#pragma unroll
                for (int q = 0; q < 32; ++q) {
                    float v = __uint_as_float(x[q]) * inv;
                    if (any_nan && sm.nan_from[seg & 3][d0 + q] <= lim) v = __uint_as_float(0x7fc00000u);
                    x[q] = __float_as_uint(v);
                }
                if constexpr (KIND == kCommon) {
                    if (whole) {
                        float* to = t.common_out + common_at * HD + d0;
#pragma unroll
                        for (int q = 0; q < 8; ++q)
                            *reinterpret_cast<uint4*>(to + 4 * q) = make_uint4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
                        continue;
                    }
                }
                if constexpr (KIND == kTail) {
                    if (whole && joins) {
                        const float* from = t.common_out + common_at * HD + d0;
#pragma unroll
                        for (int q = 0; q < 8; ++q) {
                            const float4 u = *reinterpret_cast<const float4*>(from + 4 * q);
                            x[4 * q] = __float_as_uint(fmaf(u.x, other, __uint_as_float(x[4 * q])));
                            x[4 * q + 1] = __float_as_uint(fmaf(u.y, other, __uint_as_float(x[4 * q + 1])));
                            x[4 * q + 2] = __float_as_uint(fmaf(u.z, other, __uint_as_float(x[4 * q + 2])));
                            x[4 * q + 3] = __float_as_uint(fmaf(u.w, other, __uint_as_float(x[4 * q + 3])));
                        }
                    }
                }
                if (!whole) {
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        *reinterpret_cast<uint4*>(slot + 4 + d0 + 4 * q) = make_uint4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
                } else if (p.out_wide) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t b[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            b[k] = pack_bf16(__uint_as_float(x[8 * q + 2 * k]), __uint_as_float(x[8 * q + 2 * k + 1]));
                        *reinterpret_cast<uint4*>(out + d0 + 8 * q) = make_uint4(b[0], b[1], b[2], b[3]);
                    }
                } else {
#pragma unroll
                    for (int q = 0; q < 32; ++q) out[d0 + q] = __float2bfloat16_rn(__uint_as_float(x[q]));
                }
            }
            if (valid && i == 0 && quad < per) {
                // l and o carry the factor 2^kUp
                if (!whole) *reinterpret_cast<float2*>(slot) = make_float2(top - kUp, sum);
                else if (KIND == kCommon) t.common_lse[common_at] = sum == 0.f ? -INFINITY : top - kUp + log2f(sum);
                else if (KIND == kTail && joins) {
                    if (t.lse) t.lse[common_at] = joined * kLn2;
                } else if (t.lse) t.lse[(size_t)(rows.row0 + tok) * t.hq + head] = sum == 0.f ? -INFINITY : (top - kUp + log2f(sum)) * kLn2;
            }
            if (!whole && at.tile == 0) {
                began = true;
                if (tid == 0) p.desc[blockIdx.x] = make_int4(rows.row0, rows.n, joins ? ~at.h : at.h, run.cta_of(at.first + at.tiles - 1));
            }
            if (copies > 1) softmax_sync();          // the pile is read: the next queries may go there
            umma_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.o_free);
            it0 += cnt;
            ++seg;
            if (!at.next(a, run, p)) break;
        }
        if (tid == 0) {
            if (!began) p.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
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

template <int HD, int KIND>
cudaError_t launch_tc(const Kv8Args& a, const Kv8AttnArgs& t, Kv8Plan p, cudaStream_t s) {
    auto kern = kv8_tc_kernel<HD, KIND>;
    constexpr int bytes = sizeof(Smem<HD>);
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return e;
    // records of a page in one copy, as many as divide a page's and a tile's: a copy costs its unit about 78 clocks,
    // and 24 small ones a tile (keys, values and scales of each record) took 1870, more than the tile's bytes
    p.run = a.bpp % 8 == 0 ? 8 : a.bpp % 4 == 0 ? 4 : a.bpp % 2 == 0 ? 2 : 1;
    CUtensorMap map;
    if (!make_kv8_map(&map, a.data, (uint64_t)a.n_pages * a.hk * a.bpp, HD, p.run)) return cudaErrorInvalidValue;
    return launch_kv8(kern, dim3(p.ctas), kThreads, bytes, s, a, t, p, map);
}

}  // namespace

cudaError_t launch_kv8_tc(const Kv8Args& a, const Kv8AttnArgs& t, const Kv8Plan& p, cudaStream_t s, Kv8Part part) {
    switch (part) {
        case kCommon: return a.hd == 128 ? launch_tc<128, kCommon>(a, t, p, s) : launch_tc<64, kCommon>(a, t, p, s);
        case kTail: return a.hd == 128 ? launch_tc<128, kTail>(a, t, p, s) : launch_tc<64, kTail>(a, t, p, s);
        default: return a.hd == 128 ? launch_tc<128, kWhole>(a, t, p, s) : launch_tc<64, kWhole>(a, t, p, s);
    }
}

}  // namespace ks
