// The attention weight that each cached token of the 8-bit paged cache receives
// from the batch's rows:
//   out[t] = decay scores[t] + sum over rows i >= t and query heads g of exp(scale q_ig k_t - lse_ig)
// for a sequence and KV head, the softmax's own sums lse given by the attention.
//
// Only keys are read, and only once.  A CTA is a producer warp, which copies the
// keys of 128 tokens at a time into a ring (a record's first half and its
// scales), and four consumer warps, each with 32 of the keys in registers as the
// A operand of m16n8k32 e4m3 products; all rows of the sequence pass by as B,
// eight at a time and in two codes each (see kv8_attn.cu).  A thread's
// accumulators are two rows' scores of each of its keys, so the sum over the
// rows stays in the thread until the end; one warp writes a token, in an order
// of its own: no atomics, and the same bits from call to call.
//
// Measured: 24 sequences of 500 to 16000 tokens, a row of 32 heads over 8 each, 28
// us for 106 MB, 3.8 TB/s: 6 us until runs are found, first keys there and queries
// in codes, then 22 for the bytes, 4.8 TB/s.  Three CTAs an SM of three stages; two
// take 30.2 us, four 28.2, eight warps a CTA 33.9.
//
// Calls of many rows a sequence, on average, go to kv8_weights_tc.cu.  One long chunk
// among single rows does not, and its queries are converted again for each tile:
// 63 single rows and a chunk of 400 over 4000 tokens each take 4.5 ms, 0.063 and
// 0.026 ms in two calls.  So do queries that no tensor map takes (2001 rows over 8150
// tokens 2.1 ms, 0.10 there).
#include <algorithm>
#include <type_traits>

#include "kv8_plan.cuh"

namespace ks {

namespace {

constexpr int kWarps = 4, kThreads = 32 * (kWarps + 1), kCtas = 3;  // consumers; CTAs an SM
constexpr int kWarpBlocks = 2;                      // blocks of 16 keys a warp
constexpr int kTileLog = 7, kTile = 1 << kTileLog, kBlocks = kTile / kKv8Block, kStages = 3;
constexpr int kUnitTiles = 2;                       // a unit's fixed cost, in tiles: 1, 2 and 3 take 29.0, 28.2, 28.9 us
constexpr int kChunkBlocks = 4, kChunk = 8 * kChunkBlocks;      // queries in shared memory
static_assert(kBlocks == kWarps * kWarpBlocks && kWarpBlocks == 2, "a tile is what the warps hold, a key a lane");

KS_DEV void mma_e4m3(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int HD>
struct Smem {
    unsigned char keys[kStages][kBlocks][kKv8Block * HD];
    float4 scales[kStages][kBlocks];                // key scale, value scale, unused
    uint4 code[kChunkBlocks][2][HD / 64][32];       // [hi, lo]: B operands of two products, as a lane holds them
    float2 factor[kChunk];                          // of the scores, and minus the sum's logarithm; base 2
    int lim[kChunk];                                // last key that the row sees
    int present[kStages];                           // records that were copied
    uint64_t full[kStages], empty[kStages];
};
KS_DEV void consumers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory"); }

// Queries first .. of a unit's n, eight a warp and turn, in two codes.
template <int HD, bool WIDE>
KS_DEV void convert(Smem<HD>& sm, const Kv8Args& a, const Kv8WeightArgs& t, const Rows& rows, int h, int G, int first) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q4 = lane & 3;
    constexpr int P = HD / 64;
    for (int b = warp; b < kChunkBlocks; b += kWarps) {
        const int i = first + 8 * b + g;
        if (first + 8 * b >= rows.n) break;
        const bool valid = i < rows.n;
        const int tok = valid ? i / G : 0, head = h * G + (valid ? i - tok * G : 0);
        const __nv_bfloat16* src = t.q + (int64_t)(rows.row0 + tok) * t.q_row + (int64_t)head * t.q_head + 16 * q4;
        uint32_t raw[P][8];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if constexpr (WIDE) {
                const uint4 u = reinterpret_cast<const uint4*>(src + 64 * p)[0], v = reinterpret_cast<const uint4*>(src + 64 * p)[1];
                raw[p][0] = u.x; raw[p][1] = u.y; raw[p][2] = u.z; raw[p][3] = u.w;
                raw[p][4] = v.x; raw[p][5] = v.y; raw[p][6] = v.z; raw[p][7] = v.w;
            } else {
                const unsigned short* e = reinterpret_cast<const unsigned short*>(src + 64 * p);
#pragma unroll
                for (int j = 0; j < 8; ++j) raw[p][j] = e[2 * j] | (uint32_t)e[2 * j + 1] << 16;
            }
        }
        float x[P][16], top = 0.f;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float v = valid ? (j & 1 ? bf16_hi(raw[p][j / 2]) : bf16_lo(raw[p][j / 2])) : 0.f;
                x[p][j] = finite(v) ? v : __uint_as_float(0x7fc00000u);      // the row becomes NaN
                if (finite(v)) top = fmaxf(top, fabsf(v));
            }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const float sc = scale_for(top), inv = inverse_pow2(sc);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float* v = x[p] + 4 * j;
                const uint16_t h0 = to_e4m3x2(v[0] * inv, v[1] * inv), h1 = to_e4m3x2(v[2] * inv, v[3] * inv);
                const float2 f0 = from_e4m3x2(h0), f1 = from_e4m3x2(h1);
                hi[j] = h0 | (uint32_t)h1 << 16;
                lo[j] = to_e4m3x2(v[0] * inv - f0.x, v[1] * inv - f0.y) |
                        (uint32_t)to_e4m3x2(v[2] * inv - f1.x, v[3] * inv - f1.y) << 16;
            }
            // dims 16 q4 + 4 j: the product's lane j of row g has them, as word q4 of its operands
            uint32_t *hi_at = reinterpret_cast<uint32_t*>(sm.code[b][0][p]), *lo_at = reinterpret_cast<uint32_t*>(sm.code[b][1][p]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                hi_at[(4 * g + j) * 4 + q4] = hi[j];
                lo_at[(4 * g + j) * 4 + q4] = lo[j];
            }
        }
        if (q4 == 0) {
            const float lse = valid ? t.lse[(size_t)(rows.row0 + tok) * t.hq + head] : INFINITY;
            // a row that sees nothing, and none: no weight
            const bool none = !valid || lse == -INFINITY;
            sm.factor[8 * b + g] = none ? make_float2(0.f, -INFINITY) : make_float2(sc * (t.scale * kLog2e), -lse * kLog2e);
            sm.lim[8 * b + g] = none ? -1 : rows.pos0 + tok;
        }
    }
}

template <int HD, bool WIDE>
__global__ void __launch_bounds__(kThreads, kCtas)
    kv8_weights_kernel(const Kv8Args a, const Kv8WeightArgs t, const Kv8Plan p) {
    constexpr int REC = kv8_record(HD), P = HD / 64, KEYS = kKv8Block * HD;
    extern __shared__ __align__(128) unsigned char smem_raw[];
    Smem<HD>& sm = *reinterpret_cast<Smem<HD>*>(smem_raw);
    volatile int* present = sm.present;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q4 = lane & 3;
    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&sm.full[i], 1);
            mbar_init(&sm.empty[i], kWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    grid_dependency_wait();
    grid_launch_dependents();
    Run run;
    Segment<> at;
    if (!find_run(a, p, run, at)) return;
    const int G = p.G;

    if (warp == kWarps) {
        // ------------------------------------------------------- producer
        // Page numbers are read a group of tiles ahead, across segments.
        constexpr int TILES = 32 / kBlocks;
        auto pages = [&](const Segment<>& k, int tile) {             // -1: no such block, -2: no such page
            const int b = tile * kBlocks + lane;
            if (b * kKv8Block >= k.q.len || tile + lane / kBlocks >= k.end) return -1;
            const int page = a.table[(size_t)k.s * a.table_ld + p.page_of(b, a.bpp)];
            return page >= 0 && page < a.n_pages ? page : -2;
        };
        int it = 0, tile = at.tile, page = pages(at, tile);
        bool alive = true, more = true;
        while (more && alive) {
            Segment<> next = at;
            int next_tile = tile + TILES;
            if (next_tile >= at.end) {
                more = next.next(a, run, p);
                next_tile = next.tile;
            }
            const int next_page = more ? pages(next, next_tile) : -1;
            if (page == -2) kv8_flag(a, kKv8BadPage);
            const int b = tile * kBlocks + lane;
            const unsigned char* rec =
                page >= 0 ? a.data + (((size_t)page * a.hk + at.h) * a.bpp + b - p.page_of(b, a.bpp) * a.bpp) * REC : nullptr;
            const unsigned have = __ballot_sync(0xffffffffu, rec != nullptr);
            for (int i = 0; i < TILES && tile + i < at.end; ++i, ++it) {
                const int st = it % kStages;
                const unsigned mask = have >> (i * kBlocks) & ((1u << kBlocks) - 1);
                alive = mbar_wait(&sm.empty[st], ((it / kStages) & 1) ^ 1, kWaitLimitNs);
                if (!__all_sync(0xffffffffu, alive)) {
                    alive = false;
                    break;
                }
                if (lane == 0) {
                    present[st] = (int)mask;
                    mbar_expect_tx(&sm.full[st], __popc(mask) * (KEYS + 16));
                }
                __syncwarp();
                if (lane / kBlocks == i && rec != nullptr) {
                    bulk_load(sm.keys[st][lane % kBlocks], rec, KEYS, &sm.full[st]);
                    bulk_load(&sm.scales[st][lane % kBlocks], rec + 2 * KEYS, 16, &sm.full[st]);
                }
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
    int it = 0;
    bool alive = true;
    do {
        const Rows rows(at, p.tq, G);
        const int chunks = (rows.n + kChunk - 1) / kChunk;
        const size_t score0 = ((size_t)at.s * a.hk + at.h) * t.ld;
        const int older = t.decay != 0.f ? at.q.len - at.q.rows : 0;         // tokens whose scores count
        auto score_of = [&](int tile) {              // of this lane's key, a tile ahead
            const int key = tile * kTile + warp * kWarpBlocks * kKv8Block + lane;
            return tile < at.end && key < older ? t.scores[score0 + key] : 0.f;
        };
        float next_old = score_of(at.tile);
        int held = -1;                               // chunk in shared memory
        for (int tile = at.tile; tile < at.end; ++tile, ++it) {
            const int st = it % kStages;
            const float old = next_old;
            next_old = score_of(tile + 1);
            const int key0 = tile * kTile + warp * kWarpBlocks * kKv8Block;
            if (alive) alive = mbar_wait(&sm.full[st], (it / kStages) & 1, kWaitLimitNs);
            const int have = alive ? present[st] >> (warp * kWarpBlocks) : 0;
            float sum[kWarpBlocks][2] = {};
            // rows before the tile's first key see nothing of it
            for (int c = (int)(max(0, tile * kTile - rows.pos0) * (int64_t)G / kChunk); c < chunks; ++c) {
                if (held != c) {
                    consumers_sync();
                    convert<HD, WIDE>(sm, a, t, rows, at.h, G, c * kChunk);
                    consumers_sync();
                    held = c;
                }
                const bool edge = key0 + kWarpBlocks * kKv8Block - 1 > rows.pos0 + c * kChunk / G;
                const int blocks = min(kChunkBlocks, (rows.n - c * kChunk + 7) / 8);
                // a block of keys at a time: its registers are what bounds the CTAs of an SM
#pragma unroll
                for (int kb = 0; kb < kWarpBlocks; ++kb) {
                    // matrices (tokens 0..7, dims 32 j ..), (tokens 8.., same), (tokens 0..7, dims 32 j + 16 ..), (tokens 8.., same)
                    const uint32_t base = smem_u32(sm.keys[st][warp * kWarpBlocks + kb]) + (lane >> 3 & 1) * (8 * HD) +
                                          (lane >> 4) * 128 + (lane & 7) * 16;
                    uint32_t k[2 * P][4];
#pragma unroll
                    for (int j = 0; j < 2 * P; ++j) ldsm_x4(k[j], base + j * 256);
                    const float scale = sm.scales[st][warp * kWarpBlocks + kb].x;
                    const int key = key0 + 16 * kb + g;
                    float part[2] = {};              // of a chunk: sums of many rows keep their digits
                    for (int b = 0; b < blocks; ++b) {
                        const float4 f = *reinterpret_cast<const float4*>(&sm.factor[8 * b + 2 * q4]);
                        float s[2][4] = {};          // of the two codes: two chains of products
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int j = 0; j < P; ++j) {
                                const uint4 q = sm.code[b][i][j][lane];
                                mma_e4m3(s[i], k[2 * j], q.x, q.y);
                                mma_e4m3(s[i], k[2 * j + 1], q.z, q.w);
                            }
                        const float f0 = f.x * scale, f1 = f.z * scale;
                        float x[4] = {fmaf(s[0][0] + s[1][0], f0, f.y), fmaf(s[0][1] + s[1][1], f1, f.w),
                                      fmaf(s[0][2] + s[1][2], f0, f.y), fmaf(s[0][3] + s[1][3], f1, f.w)};
                        if (edge) {
                            const int lim0 = sm.lim[8 * b + 2 * q4], lim1 = sm.lim[8 * b + 2 * q4 + 1];
                            if (key > lim0) x[0] = -INFINITY;
                            if (key > lim1) x[1] = -INFINITY;
                            if (key + 8 > lim0) x[2] = -INFINITY;
                            if (key + 8 > lim1) x[3] = -INFINITY;
                        }
                        part[0] += exp2_approx(x[0]) + exp2_approx(x[1]);
                        part[1] += exp2_approx(x[2]) + exp2_approx(x[3]);
                    }
                    sum[kb][0] += part[0];
                    sum[kb][1] += part[1];
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.empty[st]);
#pragma unroll
            for (int kb = 0; kb < kWarpBlocks; ++kb)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    sum[kb][half] += __shfl_xor_sync(0xffffffffu, sum[kb][half], 1);
                    sum[kb][half] += __shfl_xor_sync(0xffffffffu, sum[kb][half], 2);
                    if (!(have >> kb & 1)) sum[kb][half] = 0.f;          // no such page: unseen
                }
            // a quad has the sums of keys g, g + 8, g + 16 and g + 24: one to each of its lanes, then lane i gets key i
            float v = q4 < 2 ? (q4 == 0 ? sum[0][0] : sum[0][1]) : q4 == 2 ? sum[1][0] : sum[1][1];
            v = __shfl_sync(0xffffffffu, v, 4 * (lane & 7) + (lane >> 3));
            const int key = key0 + lane;
            if (key < at.q.len) t.out[score0 + key] = key < older ? fmaf(t.decay, old, v) : v;
        }
        consumers_sync();                            // the next segment's queries
    } while (at.next(a, run, p));
    if (!alive && lane == 0) kv8_flag(a, kKv8Timeout);
}

bool make_plan(const Kv8Args& a, int hq, Kv8Plan& p) {
    p = Kv8Plan{};
    p.G = hq / a.hk;
    p.tq = INT32_MAX / 2;                            // a unit has all rows of its sequence
    p.tile_log = kTileLog;
    p.cost = kUnitTiles;
    p.block_log = (a.bpp & (a.bpp - 1)) == 0 ? __builtin_ctz(a.bpp) : -1;
    const int64_t tiles = ((int64_t)a.capacity + kTile - 1) / kTile, total = (int64_t)a.hk * a.n_seqs * (tiles + p.cost);
    p.ctas = (int)std::min<int64_t>(sm_count() * kCtas, total);
    return total <= INT32_MAX;
}

// Query rows a KV head and sequence, on average, from which on the tcgen05 kernel takes the call: what this one holds in
// shared memory at once is read again for every tile behind that.  At 24, 32, 40 and 48 rows here and there, us: 24
// sequences of 8000 tokens, 32 heads over 8, 81, 99, -, 208 and 121, 121, -, 130; 8 of 16000, 64 heads, 56, 68, 124, 139
// and 85, 85, 90, 90.
constexpr int kManyRows = kChunk + 1;
bool many_rows(int64_t group, int64_t n_rows, int64_t n_seqs) { return group * n_rows >= kManyRows * n_seqs; }

}  // namespace

size_t kv8_weights_workspace(int group, int64_t n_rows, int64_t n_seqs) {
    return many_rows(group, n_rows, n_seqs) ? kv8_weights_tc_workspace() : 0;
}

bool kv8_weights_fits(const Kv8Args& a, int hq) {
    const int64_t tiles = ((int64_t)a.capacity + kTile - 1) / kTile;
    return hq > 0 && (int64_t)a.hk * a.n_seqs * (tiles + kUnitTiles) <= INT32_MAX;
}

cudaError_t launch_kv8_weights(const Kv8Args& a, const Kv8WeightArgs& t, cudaStream_t s) {
    if (many_rows(t.hq / a.hk, a.n_rows, a.n_seqs)) {
        bool taken;
        const cudaError_t e = launch_kv8_weights_tc(a, t, s, taken);
        if (taken) return e;
    }
    Kv8Plan p;
    if (!make_plan(a, t.hq, p)) return cudaErrorInvalidValue;
    const bool wide = reinterpret_cast<uintptr_t>(t.q) % 16 == 0 && t.q_row % 8 == 0 && t.q_head % 8 == 0;
    auto go = [&](auto hd) {
        constexpr int HD = decltype(hd)::value;
        auto kern = wide ? kv8_weights_kernel<HD, true> : kv8_weights_kernel<HD, false>;
        constexpr int bytes = sizeof(Smem<HD>);
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        return e != cudaSuccess ? e : launch_kv8(kern, dim3(p.ctas), kThreads, bytes, s, a, t, p);
    };
    return a.hd == 128 ? go(std::integral_constant<int, 128>{}) : go(std::integral_constant<int, 64>{});
}

}  // namespace ks
