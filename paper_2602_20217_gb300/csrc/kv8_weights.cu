// The attention weight that each cached token of the 8-bit paged cache receives
// from the batch's rows:
//   out[t] = decay scores[t] + sum over rows i >= t and query heads g of exp(scale q_ig k_t - lse_ig)
// for a sequence and KV head, the softmax's own sums lse given by the attention.
//
// Only keys are read, and only once: a warp holds 32 of them, in registers, as
// the A operand of m16n8k32 e4m3 products, and all rows of the sequence pass by
// as B, eight at a time and in two codes each (see kv8_attn.cu).  A thread's
// accumulators are two rows' scores of each of its keys, so the sum over the
// rows stays in the thread until the end; one warp writes a token, in an order
// of its own: no atomics, and the same bits from call to call.
//
// The dot product goes over the dims in any order, as long as both operands have
// the same: a lane's 16 contiguous bytes of a token are its four k-slices of four
// products, so a record's keys come by 16-byte loads, all of a line used, and
// straight from memory, without shared memory or ldmatrix.
#include <algorithm>
#include <type_traits>

#include "kv8_plan.cuh"

namespace ks {

namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kWarpBlocks = 2;                      // blocks of 16 keys a warp
constexpr int kTileLog = 7, kTile = 1 << kTileLog;
constexpr int kChunkBlocks = 8, kChunk = 8 * kChunkBlocks;      // queries in shared memory
static_assert(kTile == kWarps * kWarpBlocks * kKv8Block, "a tile is what the warps hold");

KS_DEV void mma_e4m3(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Of a block of keys, or of eight queries in one code: 16 bytes of dims 64 i + 16 q4 .. of row g, and of row g + 8.
template <int HD>
struct Keys {
    static constexpr int P = HD / 64;
    uint4 x[2][P];              // [token half]
    float scale;
    KS_DEV void load(const unsigned char* rec) {
        const int lane = threadIdx.x & 31, at = (lane & 3) * 128 + (lane >> 2) * 16;
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int i = 0; i < P; ++i) {
                x[half][i] = make_uint4(0, 0, 0, 0);
                if (rec) x[half][i] = *reinterpret_cast<const uint4*>(rec + half * 8 * HD + i * 512 + at);
            }
        scale = rec ? *reinterpret_cast<const float*>(rec + 32 * HD) : 0.f;
    }
};
KS_DEV uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

template <int HD>
struct Smem {
    uint4 code[kChunkBlocks][2][HD / 64][32];       // [hi, lo], a lane's dims as in Keys
    float2 factor[kChunk];                          // of the scores, and minus the sum's logarithm; base 2
    int lim[kChunk];                                // last key that the row sees
};

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
            sm.code[b][0][p][lane] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            sm.code[b][1][p][lane] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
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
__global__ void __launch_bounds__(kThreads, 4) kv8_weights_kernel(const Kv8Args a, const Kv8WeightArgs t, const Kv8Plan p) {
    constexpr int REC = kv8_record(HD), P = HD / 64;
    __shared__ Smem<HD> sm;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q4 = lane & 3;
    grid_dependency_wait();
    grid_launch_dependents();
    Run run;
    Segment<> at;
    if (!find_run(a, p, run, at)) return;
    const int G = p.G;
    do {
        const Rows rows(at, p.tq, G);
        const int chunks = (rows.n + kChunk - 1) / kChunk;
        // the pages of this warp's blocks of a tile (-1: no such block), two tiles ahead: an address that waits for
        // its page holds up everything behind it
        int page[kWarpBlocks];
        auto look = [&](int tile) {
#pragma unroll
            for (int kb = 0; kb < kWarpBlocks; ++kb) {
                const int b = tile * (kTile / kKv8Block) + warp * kWarpBlocks + kb;
                page[kb] = -1;
                if (tile < at.end && b * kKv8Block < at.q.len) {
                    page[kb] = a.table[(size_t)at.s * a.table_ld + p.page_of(b, a.bpp)];
                    if (page[kb] < 0) page[kb] = -2;
                }
            }
        };
        Keys<HD> next[kWarpBlocks];
        bool next_there[kWarpBlocks];
        auto fetch = [&](int tile) {
#pragma unroll
            for (int kb = 0; kb < kWarpBlocks; ++kb) {
                const int b = tile * (kTile / kKv8Block) + warp * kWarpBlocks + kb;
                next_there[kb] = page[kb] >= 0 && page[kb] < a.n_pages;
                if (!next_there[kb] && page[kb] != -1 && lane == 0) kv8_flag(a, kKv8BadPage);
                next[kb].load(next_there[kb] ? a.data + (((size_t)page[kb] * a.hk + at.h) * a.bpp + b -
                                                         p.page_of(b, a.bpp) * a.bpp) * REC : nullptr);
            }
        };
        look(at.tile);
        fetch(at.tile);
        look(at.tile + 1);
        int held = -1;                               // chunk in shared memory
        for (int tile = at.tile; tile < at.end; ++tile) {
            Keys<HD> k[kWarpBlocks];
            bool there[kWarpBlocks];
#pragma unroll
            for (int kb = 0; kb < kWarpBlocks; ++kb) {
                k[kb] = next[kb];
                there[kb] = next_there[kb];
            }
            fetch(tile + 1);
            look(tile + 2);
            const int key0 = tile * kTile + warp * kWarpBlocks * kKv8Block;
            float sum[kWarpBlocks][2] = {};
            // rows before the tile's first key see nothing of it
            for (int c = max(0, tile * kTile - rows.pos0) * (int64_t)G / kChunk; c < chunks; ++c) {
                if (held != c) {
                    __syncthreads();
                    convert<HD, WIDE>(sm, a, t, rows, at.h, G, c * kChunk);
                    __syncthreads();
                    held = c;
                }
                const bool edge = key0 + kWarpBlocks * kKv8Block - 1 > rows.pos0 + c * kChunk / G;
                float part[kWarpBlocks][2] = {};     // of a chunk: sums of many rows keep their digits
                const int blocks = min(kChunkBlocks, (rows.n - c * kChunk + 7) / 8);
                for (int b = 0; b < blocks; ++b) {
                    uint4 q[2][P];
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int j = 0; j < P; ++j) q[i][j] = sm.code[b][i][j][lane];
                    const float4 f = *reinterpret_cast<const float4*>(&sm.factor[8 * b + 2 * q4]);
                    int lim[2] = {INT32_MAX, INT32_MAX};
                    if (edge) {
                        lim[0] = sm.lim[8 * b + 2 * q4];
                        lim[1] = sm.lim[8 * b + 2 * q4 + 1];
                    }
#pragma unroll
                    for (int kb = 0; kb < kWarpBlocks; ++kb) {
                        float s[4] = {};
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int j = 0; j < 2 * P; ++j) {
                                // two words of 16 bytes a product
                                constexpr int W = 2;
                                const int part16 = j / 2, w = j % 2 * W;
                                const uint32_t ka[4] = {word(k[kb].x[0][part16], w), word(k[kb].x[1][part16], w),
                                                        word(k[kb].x[0][part16], w + 1), word(k[kb].x[1][part16], w + 1)};
                                mma_e4m3(s, ka, word(q[i][part16], w), word(q[i][part16], w + 1));
                            }
                        const float f0 = f.x * k[kb].scale, f1 = f.z * k[kb].scale;
                        const int key = key0 + 16 * kb + g;
                        float x[4] = {fmaf(s[0], f0, f.y), fmaf(s[1], f1, f.w), fmaf(s[2], f0, f.y), fmaf(s[3], f1, f.w)};
                        if (edge) {
                            if (key > lim[0]) x[0] = -INFINITY;
                            if (key > lim[1]) x[1] = -INFINITY;
                            if (key + 8 > lim[0]) x[2] = -INFINITY;
                            if (key + 8 > lim[1]) x[3] = -INFINITY;
                        }
                        part[kb][0] += exp2_approx(x[0]) + exp2_approx(x[1]);
                        part[kb][1] += exp2_approx(x[2]) + exp2_approx(x[3]);
                    }
                }
#pragma unroll
                for (int kb = 0; kb < kWarpBlocks; ++kb) {
                    sum[kb][0] += part[kb][0];
                    sum[kb][1] += part[kb][1];
                }
            }
#pragma unroll
            for (int kb = 0; kb < kWarpBlocks; ++kb)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    float v = sum[kb][half];
                    v += __shfl_xor_sync(0xffffffffu, v, 1);
                    v += __shfl_xor_sync(0xffffffffu, v, 2);
                    const int key = key0 + 16 * kb + 8 * half + g;
                    if (q4 == 0 && key < at.q.len) {
                        const size_t o = ((size_t)at.s * a.hk + at.h) * t.ld + key;
                        if (!there[kb]) v = 0.f;                 // its page is not there: unseen
                        if (t.decay != 0.f && key < at.q.len - at.q.rows) v = fmaf(t.decay, t.scores[o], v);
                        t.out[o] = v;
                    }
                }
        }
        __syncthreads();                             // the next segment's queries
    } while (at.next(a, run, p));
}

bool make_plan(const Kv8Args& a, int hq, Kv8Plan& p) {
    p = Kv8Plan{};
    p.G = hq / a.hk;
    p.tq = INT32_MAX / 2;                            // a unit has all rows of its sequence
    p.tile_log = kTileLog;
    p.cost = 1;
    p.block_log = (a.bpp & (a.bpp - 1)) == 0 ? __builtin_ctz(a.bpp) : -1;
    const int64_t tiles = ((int64_t)a.capacity + kTile - 1) / kTile, total = (int64_t)a.hk * a.n_seqs * (tiles + p.cost);
    p.ctas = (int)std::min<int64_t>(sm_count() * 4, total);
    return total <= INT32_MAX;
}

// Query rows a KV head and sequence, on average, from which on the tcgen05 kernel takes the call.
constexpr int kManyRows = 17;
bool many_rows(int64_t group, int64_t n_rows, int64_t n_seqs) { return group * n_rows >= kManyRows * n_seqs; }

}  // namespace

size_t kv8_weights_workspace(int group, int64_t n_rows, int64_t n_seqs) {
    // a call with fewer sequences may be one of many rows
    (void)n_seqs;
    return group * n_rows >= kManyRows ? kv8_weights_tc_workspace() : 0;
}

bool kv8_weights_fits(const Kv8Args& a, int hq) {
    const int64_t tiles = ((int64_t)a.capacity + kTile - 1) / kTile;
    return hq > 0 && (int64_t)a.hk * a.n_seqs * (tiles + 1) <= INT32_MAX;
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
        return launch_kv8(wide ? kv8_weights_kernel<HD, true> : kv8_weights_kernel<HD, false>, dim3(p.ctas), kThreads, 0, s,
                          a, t, p);
    };
    return a.hd == 128 ? go(std::integral_constant<int, 128>{}) : go(std::integral_constant<int, 64>{});
}

}  // namespace ks
