// How the attention over the 8-bit cache is cut into work for the resident
// CTAs, and what its kernels share.
//
// A unit is (sequence, KV head, group of rows): a group is as many whole tokens
// as give at most rg query rows (token x query head of the KV head), and its
// keys come in tiles.  The units' tiles, one after the other, are cut into equal
// runs, one per CTA, so a long sequence among short ones or few heads at a long
// context keep every SM busy; the lengths are read on the device.  A run's part
// of a unit is a segment.  Units that lie in several runs leave (m, l, o) per
// segment, merged in run order by a second launch: the result depends on the
// batch, never on timing.
#pragma once

#include "kv8.cuh"

namespace ks {

constexpr int kKv8Sms = 160, kKv8MaxCtas = 3 * kKv8Sms;    // the workspace has room for this many
constexpr int kKv8TcRows = 128;     // query rows of a unit of the tcgen05 kernel
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// A unit's fixed cost (queries, joining its warps, output) in the time of 128
// keys, for the cut into runs.
constexpr int kUnitCost = 2;

struct Kv8Plan {
    int tile_log;       // keys of a tile
    int block_log;      // blocks of a page, -1: no power of two
    int G;              // query heads a KV head
    int token_mul;      // see token()
    int cost;           // a unit's fixed cost in tiles
    int tq;             // tokens of a group
    int rg;             // rows of a group, at least tq query groups
    int ctas;
    int run;            // records of a copy (tcgen05 kernel)
    bool q_wide, out_wide;  // queries can be read, the output written 16 bytes at a time
    float* part;        // [2 ctas][rg][HD + 4]: m, l, -, -, o
    int4* desc;         // [ctas]: the unit that begins in this CTA's run and ends in a later one's: first batch row,
                        // query rows (0: no such unit), KV head, last CTA
    // The kernels' fixed steps are chains of a few hundred clocks each, in which a division by a number that is not
    // known when compiling takes about 150: tiles and pages go by shifts, and row r < 128 of a group is of token
    // r / G = r token_mul >> 16, token_mul = 2^16 / G rounded up (r (G - 1) < 2^16).
    KS_DEV int token(int r) const { return r * token_mul >> 16; }
    KS_DEV int page_of(int block, int bpp) const { return block_log >= 0 ? block >> block_log : block / bpp; }
};

// A sequence of a launch.  A group with nothing in common has no units.
template <int PART>
KS_DEV Kv8Seq seq_of(const Kv8Args& a, int s) {
    Kv8Seq q = kv8_seq(a, s);
    if (PART == kCommon && q.len == 0) q.rows = 0;
    return q;
}
// Last key of group g.
template <int PART>
KS_DEV int last_key(const Kv8Seq& q, const Kv8Plan& p, int g) {
    return PART == kCommon ? q.len - 1 : q.len - q.rows + min(q.rows, (g + 1) * p.tq) - 1;
}
// Tiles of group g; a group whose rows see nothing has one as well (its rows get zeros).
template <int PART>
KS_DEV int group_tiles(const Kv8Seq& q, const Kv8Plan& p, int g) {
    const int last = last_key<PART>(q, p, g);
    return last < 0 ? 1 : (last >> p.tile_log) + 1;
}
// Where a sequence's pages begin in the table.
template <int PART>
KS_DEV const int32_t* pages_of(const Kv8Args& a, int s) {
    return a.table + (PART == kWhole ? (int64_t)s * a.table_ld : a.first_page[s]);
}
KS_DEV int groups_of(const Kv8Seq& q, int tq) { return q.rows <= tq ? q.rows > 0 : (q.rows + tq - 1) / tq; }
// What the units of one head of a sequence take on the line of all units.
template <int PART>
KS_DEV int head_length(const Kv8Seq& q, const Kv8Plan& p) {
    if (PART == kCommon) return groups_of(q, p.tq) * (group_tiles<PART>(q, p, 0) + p.cost);
    int n = 0;
    for (int g = 0, groups = groups_of(q, p.tq); g < groups; ++g) n += group_tiles<PART>(q, p, g) + p.cost;
    return n;
}

// The line of all units, each its fixed cost and its tiles long, cut into equal runs
// [x0, x1): a CTA works on the tiles in its run.
struct Run {
    int ctas, each, more;       // runs of each + 1 (the first `more`), then of each
    int x0, x1;
    KS_DEV void cut(int total, int most, int cta) {
        ctas = min(most, total);
        each = ctas ? total / ctas : 0;
        more = total - each * ctas;
        x0 = cta * each + min(cta, more);
        x1 = x0 + each + (cta < more);
    }
    KS_DEV int cta_of(int x) const {
        const int b = more * (each + 1);
        return x < b ? x / (each + 1) : more + (x - b) / each;
    }
};

// A segment: tiles [tile, end) of a unit, whose first tile is at `first` on the line.
template <int PART = kWhole>
struct Segment {
    int s, h, g, tile, end, tiles, first;
    Kv8Seq q;
    KS_DEV void at(const Run& r, const Kv8Plan& p, int start) {
        tiles = group_tiles<PART>(q, p, g);
        first = start + p.cost;
        tile = max(0, r.x0 - first);
        end = min(tiles, r.x1 - first);
    }
    // the next unit, if a tile of it is in the run
    KS_DEV bool next(const Kv8Args& a, const Run& r, const Kv8Plan& p) {
        const int start = first + tiles;
        if (start + p.cost >= r.x1) return false;
        if (++g >= groups_of(q, p.tq)) {
            g = 0;
            if (++h >= a.hk) {
                h = 0;
                do {
                    if (++s >= a.n_seqs) return false;
                    q = seq_of<PART>(a, s);
                } while (q.rows == 0);
            }
        }
        at(r, p, start);
        return true;
    }
};

// This CTA's run and its first segment; false if it has none.  Every warp finds
// it by itself, 32 sequences at a time.  Where offsets decrease, no CTA has one:
// sequences that share rows could be more units than the host counted, and their
// line longer than an int.
template <int PART>
KS_DEV bool find_run(const Kv8Args& a, const Kv8Plan& p, Run& r, Segment<PART>& k) {
    const int lane = threadIdx.x & 31, cta = blockIdx.x;
    Kv8Seq mine{};
    int head = 0;                                // length of one of its heads' units
    bool falls = false;
    auto load = [&](int c) {
        const int s = c + lane;
        if (s >= a.n_seqs) {
            mine = Kv8Seq{};
            return 0;
        }
        mine = seq_of<PART>(a, s);
        falls |= a.offsets[s + 1] < a.offsets[s];
        head = head_length<PART>(mine, p);
        return a.hk * head;
    };
    int total = 0, v = 0;
    for (int c = 0; c < a.n_seqs; c += 32) {
        v = load(c);
        if (cta == 0 && c + lane < a.n_seqs && kv8_seq_bad(a, c + lane)) kv8_flag(a, kKv8BadBatch);
        total += __reduce_add_sync(0xffffffffu, v);
    }
    if (__any_sync(0xffffffffu, falls)) return false;
    r.cut(total, p.ctas, cta);
    if (cta >= r.ctas) return false;
    int start = 0, len = 0;                      // of the sequence's units on the line; a head's length
    for (int c = 0;; c += 32) {
        if (c >= a.n_seqs) return false;         // not with arrays that stay what they are
        if (a.n_seqs > 32) v = load(c);
        int u = v;                               // inclusive sums
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int w = __shfl_up_sync(0xffffffffu, u, o);
            if (lane >= o) u += w;
        }
        const unsigned past = __ballot_sync(0xffffffffu, start + u > r.x0);
        if (past) {
            const int i = __ffs(past) - 1;
            k.s = c + i;
            k.q.row0 = __shfl_sync(0xffffffffu, mine.row0, i);
            k.q.rows = __shfl_sync(0xffffffffu, mine.rows, i);
            k.q.len = __shfl_sync(0xffffffffu, mine.len, i);
            len = __shfl_sync(0xffffffffu, head, i);
            start += __shfl_sync(0xffffffffu, u - v, i);
            break;
        }
        start += __shfl_sync(0xffffffffu, u, 31);
    }
    k.h = (r.x0 - start) / len;
    start += k.h * len;
    k.g = 0;
    for (;;) {
        k.at(r, p, start);
        if (r.x0 < k.first + k.tiles) break;
        start = k.first + k.tiles;
        ++k.g;
    }
    // a run that ends before the unit's first tile has nothing to do
    return k.end > k.tile;
}

KS_DEV void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
        "l"(src), "r"(bytes), "r"(smem_u32(bar))
        : "memory");
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
// Two fp32 operations in one instruction.
KS_DEV float2 fma2(float2 a, float2 b, float2 c) {
    uint64_t r;
    asm("{ .reg .b64 x, y, z; mov.b64 x, {%1, %2}; mov.b64 y, {%3, %4}; mov.b64 z, {%5, %6}; fma.rn.f32x2 %0, x, y, z; }"
        : "=l"(r)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return make_float2(__uint_as_float((uint32_t)r), __uint_as_float((uint32_t)(r >> 32)));
}
KS_DEV float2 add2(float2 a, float2 b) {
    uint64_t r;
    asm("{ .reg .b64 x, y; mov.b64 x, {%1, %2}; mov.b64 y, {%3, %4}; add.rn.f32x2 %0, x, y; }"
        : "=l"(r)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return make_float2(__uint_as_float((uint32_t)r), __uint_as_float((uint32_t)(r >> 32)));
}
// A unit's rows, as its segments and the merge see them.
struct Rows {
    int tokens;
    int n;              // query rows: tokens x G
    int row0;           // batch row of the first token
    int pos0;           // its position; negative positions see nothing
    int step;           // from a token's position to the next one's: 0 where all see the same
    template <int PART>
    KS_DEV Rows(const Segment<PART>& at, int tq, int G) : step(PART != kCommon) {
        const Kv8Seq& q = at.q;
        const int g = at.g;
        const int t0 = g * tq;
        tokens = min(q.rows - t0, tq);
        n = tokens * G;
        row0 = q.row0 + t0;
        pos0 = PART == kCommon ? q.len - 1 : q.len - q.rows + t0;
    }
};
// A row's sums m, l (base 2) of its own part joined with the common part's: the factors of the two outputs (own not
// normalised, the other normalised) and the sum's logarithm.
struct Joined {
    float own, other, lse;
    KS_DEV Joined(float m, float l, float common) {
        const float top = fmaxf(m, common), ref = top == -INFINITY ? 0.f : top;
        const float a = exp2_approx(m - ref), b = exp2_approx(common - ref), sum = fmaf(a, l, b);
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        own = a * inv;
        other = b * inv;
        lse = sum == 0.f ? -INFINITY : ref + log2f(sum);
    }
};

// kv8_tc.cu
cudaError_t launch_kv8_tc(const Kv8Args& a, const Kv8AttnArgs& t, const Kv8Plan& p, cudaStream_t s, Kv8Part part);

}  // namespace ks
