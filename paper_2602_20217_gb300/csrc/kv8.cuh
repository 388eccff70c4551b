// The 8-bit paged key/value cache: record layout, code conversions and the
// batch's sequences, shared by the kernels that write and read it.
//
// A record holds one block of kKv8Block tokens of one KV head: e4m3 key codes
// as [2][HD / 16][8 tokens][16 dims] and value codes as [HD dims][16 tokens]
// (token t at byte v_byte(t)), so that every 8 x 16-byte matrix that the
// attention feeds to the tensor cores is 128 contiguous bytes and no
// transposition or swizzle is left to do, then the two scales (fp32 powers of
// two) and 24 unused bytes.  Keys, values and scales of a block are one
// contiguous piece: one asynchronous copy brings them.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"
#include "kv8.h"
#include "tma.cuh"

namespace ks {

constexpr int kKv8Block = 16;
__host__ __device__ constexpr int kv8_record(int hd) { return 2 * kKv8Block * hd + 32; }
constexpr int kKv8BadPage = 1, kKv8BadBatch = 2, kKv8BadPosition = 4, kKv8Timeout = 8;

// Byte of token t in a row of value codes: lane t of a quad of the score
// product holds tokens 2t, 2t + 1, 8 + 2t, 9 + 2t, and the value product takes
// four neighbouring bytes of a lane.
KS_DEV int v_byte(int t) { return 4 * ((t & 7) >> 1) + 2 * (t >> 3) + (t & 1); }
// Byte of (token, dim) among a record's key codes.
template <int HD>
KS_DEV int k_byte(int t, int d) {
    return ((t >> 3) * (HD / 16) + (d >> 4)) * 128 + (t & 7) * 16 + (d & 15);
}

// Two floats as e4m3 codes, nearest even (lo in the low byte).
KS_DEV uint16_t to_e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
KS_DEV float2 from_e4m3x2(uint16_t v) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(v));
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

KS_DEV bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }
// Smallest 2^e, e >= -126, with amax <= 448 * 2^e (448 = 1.75 * 2^8).
KS_DEV float scale_for(float amax) {
    const unsigned b = __float_as_uint(amax);
    const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u);
    return __uint_as_float((unsigned)(max(e, -126) + 127) << 23);
}
// 1 / s for a power of two from 2^-126 to 2^127
KS_DEV float inverse_pow2(float s) { return __uint_as_float((254u << 23) - __float_as_uint(s)); }

KS_DEV void kv8_flag(const Kv8Args& a, int code) {
    if (a.status) atomicOr(a.status, code);
}

// Sequence s of the batch: its rows [row0, row0 + rows) and its length, the
// rows among it.  Row i is token len - rows + i.  Values outside the batch's
// own sizes are brought inside (and flagged): nothing is addressed by them
// that does not exist.
struct Kv8Seq {
    int row0, rows, len;
};
KS_DEV int kv8_row0(const Kv8Args& a, int s) { return min(max(a.offsets[s], 0), a.n_rows); }
KS_DEV Kv8Seq kv8_seq(const Kv8Args& a, int s) {
    const int o0 = a.offsets[s], o1 = a.offsets[s + 1], n = a.lengths[s];
    Kv8Seq q;
    q.row0 = min(max(o0, 0), a.n_rows);
    q.rows = min(max(o1, q.row0), a.n_rows) - q.row0;
    q.len = min(max(n, 0), a.capacity);
    return q;
}
KS_DEV bool kv8_seq_bad(const Kv8Args& a, int s) {
    const int o0 = a.offsets[s], o1 = a.offsets[s + 1], n = a.lengths[s];
    return o0 < 0 || o1 < o0 || o1 > a.n_rows || n < 0 || n > a.capacity;
}

// The last sequence s with first(s) <= x (0 if there is none), first not
// decreasing, found by one warp with 32 probes a round.
template <class F>
KS_DEV int kv8_find(int n_seqs, int x, F&& first) {
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = n_seqs;
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, i = lo + step * lane;
        const unsigned yes = __ballot_sync(0xffffffffu, i < hi && (lane == 0 || first(i) <= x));
        lo += step * (__popc(yes) - 1);
        hi = min(hi, lo + step);
    }
    return lo;
}

// The record of block b of sequence s and head h, or null for a page that the
// pool does not have.
KS_DEV unsigned char* kv8_record_at(const Kv8Args& a, int s, int b, int h, int rec) {
    const int page = a.table[(size_t)s * a.table_ld + b / a.bpp];
    if (page < 0 || page >= a.n_pages) return nullptr;
    return a.data + (((size_t)page * a.hk + h) * a.bpp + b % a.bpp) * rec;
}

// The touched blocks of a batch, over the grid's x and z.  Batches of few rows a
// sequence (by_seq): x is the sequence, z counts its blocks, so that a CTA reads
// the sequence's numbers at once.  Others: x is a block slot; the slots of
// sequence s begin at row0 / 16 + 2 s, which leaves room for every block that its
// rows can touch (r rows touch at most (r + 30) / 16) without a sum over the
// sequences, and the sequence is searched for.
struct Kv8Slot {
    int s, blk, first, last;   // sequence, block; tokens [first, last) of the block are the batch's rows
    int row;                   // batch row of the block's token 0 (it may be before the sequence's rows)
};
struct Kv8Blocks {
    Kv8Seq q;
    int s, start, b, step;
    KS_DEV Kv8Blocks(const Kv8Args& a) {
        if (a.by_seq) {
            s = blockIdx.x;
            b = blockIdx.z;
            step = gridDim.z;
        } else {
            auto first = [&](int i) { return kv8_row0(a, i) / kKv8Block + 2 * i; };
            s = kv8_find(a.n_seqs, blockIdx.x, first);
            b = (int)blockIdx.x - first(s);      // below 0 for slots before the first sequence's
            step = 1 << 30;
        }
        q = kv8_seq(a, s);
        start = max(q.len - q.rows, 0);
        // x is at least n_seqs wide either way, and offsets that decrease may hide a sequence from the search
        if ((int)blockIdx.x < a.n_seqs && blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x == 0) {
            const Kv8Seq own = kv8_seq(a, blockIdx.x);
            if (kv8_seq_bad(a, blockIdx.x)) kv8_flag(a, kKv8BadBatch);
            if (own.len < own.rows) kv8_flag(a, kKv8BadPosition);
        }
    }
    KS_DEV bool get(Kv8Slot& w) const {
        w.s = s;
        w.blk = start / kKv8Block + b;
        if (b < 0 || q.rows == 0 || b >= 1 << 28 || w.blk * kKv8Block >= q.len) return false;
        w.first = max(start - w.blk * kKv8Block, 0);
        w.last = min(q.len - w.blk * kKv8Block, kKv8Block);
        w.row = q.row0 + w.blk * kKv8Block - (q.len - q.rows);
        return true;
    }
};

// Programmatic launch: the kernel waits for what is before it by itself.  It may
// be resident while its predecessor still writes, so nothing that a caller may
// write is read by non-coherent loads.
template <class K, class... Args>
cudaError_t launch_kv8(K kern, dim3 grid, int threads, int smem, cudaStream_t s, const Args&... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, args...);
}

}  // namespace ks
