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

// Tiles of group g; a group whose rows see nothing has one as well (its rows get zeros).
KS_DEV int group_tiles(const Kv8Seq& q, const Kv8Plan& p, int g) {
    const int last = q.len - q.rows + min(q.rows, (g + 1) * p.tq) - 1;
    return last < 0 ? 1 : (last >> p.tile_log) + 1;
}
KS_DEV int groups_of(const Kv8Seq& q, int tq) { return q.rows <= tq ? q.rows > 0 : (q.rows + tq - 1) / tq; }
// What the units of one head of a sequence take on the line of all units.
KS_DEV int head_length(const Kv8Seq& q, const Kv8Plan& p) {
    int n = 0;
    for (int g = 0, groups = groups_of(q, p.tq); g < groups; ++g) n += group_tiles(q, p, g) + p.cost;
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
struct Segment {
    int s, h, g, tile, end, tiles, first;
    Kv8Seq q;
    KS_DEV void at(const Run& r, const Kv8Plan& p, int start) {
        tiles = group_tiles(q, p, g);
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
                    q = kv8_seq(a, s);
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
KS_DEV bool find_run(const Kv8Args& a, const Kv8Plan& p, Run& r, Segment& k) {
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
        mine = kv8_seq(a, s);
        falls |= a.offsets[s + 1] < a.offsets[s];
        head = head_length(mine, p);
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
// A unit's rows, as its segments and the merge see them.
struct Rows {
    int tokens;
    int n;              // query rows: tokens x G
    int row0;           // batch row of the first token
    int pos0;           // its position; negative positions see nothing
    KS_DEV Rows(const Kv8Seq& q, int tq, int g, int G) {
        const int t0 = g * tq;
        tokens = min(q.rows - t0, tq);
        n = tokens * G;
        row0 = q.row0 + t0;
        pos0 = q.len - q.rows + t0;
    }
};

cudaError_t launch_kv8_tc(const Kv8Args& a, const Kv8AttnArgs& t, const Kv8Plan& p, cudaStream_t s);   // kv8_tc.cu

}  // namespace ks
