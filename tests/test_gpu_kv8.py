"""The 8-bit paged cache on the GPU against its fp64 restatement (oracle/kv8.py).

Tolerances.
Without RoPE a value is x * 2^-e, exact in fp32 (bf16 and fp32 inputs of the
magnitudes here), and its code is the nearest one: bytes are compared for
equality, tails included.  With RoPE the rotated key has an fp32 error, so a
code next to a rounding border may fall to either side: the stored value is
within half a step of the code (2^-4 relative, 2^-10 of the scale where codes
are subnormal) of the fp64 key, plus 2^-21 |x| of the pair for three fp32
roundings; a scale may differ only if amax is that close to its border.
Rotated queries: half a bf16 step, 2^-8 relative, plus the same.
Attention: the output's own rounding, 2^-8 |out|; the probabilities go to the
tensor cores in 11 bits, which moves the average of |v| under the softmax
(``mag``) by at most 2^-11 each for the probabilities and, with their fp32
sums and exponents over at most 20000 keys (scores up to 40 in fp32: 40 * 2^-22
relative in a probability), less than 2^-11 for the rest: 2^-10 mag.  Queries
are split into two codes, exact for bf16 values down to 2^-10 of the row's
largest and off by 2^-18 of it below: a few dims of a row, each moving its
scores by at most 2^-18 max|q| |k| scale < 2^-15 for the inputs here.
lse: that and fp32 rounding, 2e-4 absolute at |lse| <= 64.
"""
import math

import numpy as np
import pytest

from helpers import need_gpu
from oracle import kv8 as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()


class Pool:
    """A cache whose records the host knows: pages in random order, unused ones and tails full of NaN codes."""

    def __init__(self, lens, hk, hd, page, seed=0, spare=2, garbage=0x7f):
        self.rng = np.random.default_rng(seed)
        self.hk, self.hd, self.page, self.bpp = hk, hd, page, page // 16
        self.lens = list(lens)
        self.per = [-(-n // page) for n in lens]
        self.n_pages = max(1, sum(self.per)) + spare
        self.ld = max(1, max(self.per, default=1))
        order = self.rng.permutation(self.n_pages)
        self.table = np.zeros((len(lens), self.ld), np.int32)
        at = 0
        for s, c in enumerate(self.per):
            self.table[s, :c] = order[at:at + c]
            at += c
        self.data = np.full((self.n_pages, hk, self.bpp, O.record_bytes(hd)), garbage, np.uint8)

    def block(self, s, b):
        """The records [hk, bytes] of block b of sequence s."""
        return self.data[self.table[s, b // self.bpp], :, b % self.bpp]

    def fill(self, std=1.0, spread=2.0):
        """Random tokens up to each length (the codes' tails stay garbage)."""
        self.kv = []
        for s, n in enumerate(self.lens):
            kv = np.zeros((2, n, self.hk, self.hd))
            for b in range(-(-n // 16)):
                last = min(16, n - 16 * b)
                for h in range(self.hk):
                    x = self.rng.standard_normal((2, last, self.hd)) * std * np.exp2(self.rng.uniform(-spread, spread, (2, 1, 1)))
                    kc, vc, ks, vs = O.append_block(None, 0, x[0], x[1])
                    kc[last:] = 0x7f
                    vc[last:] = 0xff
                    self.block(s, b)[h] = O.pack_record(kc, vc, ks, vs)
                    kv[0, 16 * b:16 * b + last, h] = O.VALUES[kc[:last]] * ks
                    kv[1, 16 * b:16 * b + last, h] = O.VALUES[vc[:last]] * vs
            self.kv.append(kv)
        return self

    def token(self, s, t, h):
        """(K, V) values of a token as the records hold them."""
        kc, vc, ks, vs = O.unpack_record(self.block(s, t // 16)[h])
        return O.VALUES[kc[t % 16]] * ks, O.VALUES[vc[t % 16]] * vs

    def device(self, rows, lengths=None, pad=0, offsets=None):
        import torch

        from paper_2602_20217_gb300 import kv8
        off = np.concatenate(([0], np.cumsum(rows))) if offsets is None else np.asarray(offsets)
        self.n_rows = int(off[-1]) + pad
        self.offsets = off
        dev = {}
        dev["data"] = torch.tensor(self.data, device="cuda").reshape(-1)
        dev["table"] = torch.tensor(self.table, device="cuda")
        dev["offsets"] = torch.tensor(off.astype(np.int32), device="cuda")
        dev["lengths"] = torch.tensor(np.asarray(self.lens if lengths is None else lengths, np.int32), device="cuda")
        dev["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        dev["cache"] = kv8.Cache8(self.n_pages, self.page, self.hk, self.hd, data=dev["data"])
        dev["batch"] = kv8.Batch8(dev["table"], dev["offsets"], dev["lengths"], self.n_rows, dev["status"])
        return dev


# ---------------------------------------------------------------- attention
def attend(pool, rows, hq, seed=1, pad=0, lengths=None, q=None, scale=None, want=0, status=0, offsets=None, ld=None):
    """Runs the attention; checks every row against the oracle, padding untouched, the status word."""
    import torch
    d = pool.device(rows, lengths, pad, offsets)
    rng = np.random.default_rng(seed)
    n, hd = pool.n_rows, pool.hd
    if q is None:
        q = rng.standard_normal((n, hq, hd)) * 2
    qt = torch.tensor(q, dtype=torch.bfloat16, device="cuda")
    out = torch.full((n, hq, hd), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n, hq), 7.0, device="cuda")
    work = d["cache"].attention_workspace(hq, len(pool.lens), n)
    work.fill_(0xff)
    scale = hd ** -0.5 if scale is None else scale
    d["cache"].attention(d["batch"], qt, scale=scale, out=out, lse=lse, workspace=work)
    torch.cuda.synchronize()
    assert int(d["status"]) == status
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    check(pool, rows, qt.double().cpu().numpy(), got, got_lse, scale, lengths)
    end = int(pool.offsets[-1])
    assert np.all(got[end:] == 7) and np.all(got_lse[end:] == 7)
    return d, qt, out, lse, work


def check(pool, rows, q, got, got_lse, scale, lengths=None):
    for s, r in enumerate(rows):
        n = pool.lens[s] if lengths is None else lengths[s]
        o0 = int(pool.offsets[s])
        kv = pool.kv[s][:, :n]
        ref, ref_lse, mag = O.attention(q[o0:o0 + r], kv[0], kv[1], scale)
        g = got[o0:o0 + r]
        assert np.array_equal(np.isnan(g), np.isnan(ref)), s
        ok = ~np.isnan(ref)
        err = np.abs(g - ref)[ok] - (2.0 ** -8 * np.abs(ref) + 2.0 ** -10 * mag)[ok]
        assert err.size == 0 or err.max() <= 1e-30, (s, n, r, float(err.max()))
        gl = got_lse[o0:o0 + r]
        assert np.array_equal(np.isnan(gl), np.isnan(ref_lse))
        fin = np.isfinite(ref_lse)
        assert np.array_equal(gl[~fin & ~np.isnan(gl)], ref_lse[~fin & ~np.isnan(ref_lse)])
        far = np.abs(gl[fin] - ref_lse[fin])
        assert far.size == 0 or far.max() <= 2e-4, (s, far.max())


@pytest.mark.parametrize("hq,hk,hd,page", [(2, 1, 64, 16), (4, 2, 128, 64), (8, 1, 128, 48)])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 130, 255, 257, 1000])
def test_one_token(hq, hk, hd, page, n):
    attend(Pool([n], hk, hd, page, seed=n).fill(), [1], hq)


@pytest.mark.parametrize("hq,hk,hd,page", [(3, 1, 64, 32), (32, 8, 128, 64), (64, 8, 128, 128), (8, 8, 64, 16),
                                           (12, 4, 128, 16), (17, 1, 64, 64), (64, 1, 128, 256), (10, 2, 128, 80)])
@pytest.mark.parametrize("rows", [[1], [2], [5], [11], [16], [37]])
def test_rows_and_groups(hq, hk, hd, page, rows):
    attend(Pool([421 + rows[0]], hk, hd, page, seed=rows[0]).fill(), rows, hq)


@pytest.mark.parametrize("hd,page", [(64, 16), (128, 64)])
def test_ragged_batch_with_empty_parts(hd, page):
    """No rows, no tokens, more rows than tokens (the first rows see nothing), whole prompts, padding rows."""
    lens = [300, 0, 77, 5, 3, 129, 1, 640, 16, 50]
    rows = [3, 2, 0, 5, 7, 129, 1, 9, 16, 1]
    attend(Pool(lens, 2, hd, page, seed=3).fill(), rows, 8, pad=5)


def test_many_sequences():
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 300, 200)
    attend(Pool(lens, 2, 64, 32, seed=5).fill(), [int(r) for r in rng.integers(0, 4, 200)], 4)


def test_long_and_short_together():
    attend(Pool([20000, 3, 700, 4097], 2, 128, 64, seed=6).fill(), [2, 1, 5, 1], 8)


def test_prompt_rows():
    attend(Pool([700, 450], 2, 64, 32, seed=7).fill(), [600, 450], 6)


def test_offsets_that_do_not_begin_at_zero():
    import torch
    pool = Pool([40, 50], 1, 64, 16, seed=8).fill()
    d, q, out, lse, _ = attend(pool, [3, 2], 2, offsets=[4, 7, 9], pad=1)
    assert bool((out[:4] == 7).all()) and bool((lse[:4] == 7).all())


@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-3, 0.5])
def test_scales(scale):
    attend(Pool([200], 1, 64, 16, seed=9).fill(), [4], 4, scale=scale)


def test_a_peak_over_a_long_flat_tail():
    """Half of the weight on one key and the rest spread over 20000: the tail's small probabilities count."""
    n, hd = 20001, 64
    pool = Pool([n], 1, hd, 128, seed=10).fill(spread=0)
    for b in range(-(-n // 16)):           # keys: zeros but for the first, values of one sign
        kc, vc, ks, vs = O.unpack_record(pool.block(0, b)[0])
        kc, vc = np.zeros_like(kc), vc & 0x7f
        last = min(16, n - 16 * b)
        if b == 0:
            kc[0, 0] = 0x7e
            vc[0] = 0
        pool.block(0, b)[0] = O.pack_record(kc, vc, 1.0, vs)
        pool.kv[0][0, 16 * b:16 * b + last, 0] = O.VALUES[kc[:last]]
        pool.kv[0][1, 16 * b:16 * b + last, 0] = O.VALUES[vc[:last]] * vs
    q = np.zeros((1, 2, hd))
    q[0, :, 0] = 0.0234375                 # 448 * q * 1 = 10.5 = ln 36000
    attend(pool, [1], 2, q=q, scale=1.0)


def test_blocks_of_far_scales():
    """Values of a block 2^20 below its neighbours', which holds the weight of one row; blocks of zeros."""
    pool = Pool([96], 1, 64, 16, seed=11).fill(spread=0)
    for b, f in ((0, 2.0 ** -20), (2, 0.0), (4, 2.0 ** 9)):
        kc, vc, ks, vs = O.unpack_record(pool.block(0, b)[0])
        vs = vs * f if f else 2.0 ** -126
        vc = vc if f else vc & 0x80
        pool.block(0, b)[0] = O.pack_record(kc, vc, ks, vs)
        pool.kv[0][1, 16 * b:16 * b + 16, 0] = O.VALUES[vc] * vs
    attend(pool, [3], 2)
    q = pool.kv[0][0, 5, 0]
    q = q / (q @ q) * 40                   # all on token 5, of the quiet block
    attend(pool, [1], 1, q=q[None, None], scale=1.0)


def test_nan_tokens_stay_with_the_rows_that_see_them():
    """A NaN value makes one dim of the rows from its token on NaN, a NaN key the whole rows."""
    pool = Pool([150], 1, 64, 16, seed=12).fill()
    for t, d, which in ((141, 7, 1), (147, 3, 0), (146, 7, 1)):
        rec = pool.block(0, t // 16)[0]
        kc, vc, ks, vs = O.unpack_record(rec)
        (kc, vc)[which][t % 16, d] = 0xff
        pool.block(0, t // 16)[0] = O.pack_record(kc, vc, ks, vs)
        pool.kv[0][which, t, 0, d] = np.nan
    attend(pool, [16], 8)
    attend(pool, [1], 8)


def test_nan_in_a_value_that_every_row_sees():
    pool = Pool([400], 1, 128, 64, seed=13).fill()
    kc, vc, ks, vs = O.unpack_record(pool.block(0, 3)[0])
    vc[4, 100] = 0x7f
    pool.block(0, 3)[0] = O.pack_record(kc, vc, ks, vs)
    pool.kv[0][1, 52, 0, 100] = np.nan
    attend(pool, [5], 4)


def test_queries_that_are_not_finite():
    pool = Pool([60], 1, 64, 16, seed=14).fill()
    import torch
    d = pool.device([3])
    q = torch.randn(3, 4, 64, device="cuda").to(torch.bfloat16)
    q[0, 1, 5], q[1, 2, 60], q[2, 3, 0] = math.inf, -math.inf, math.nan
    out = d["cache"].attention(d["batch"], q)
    bad = torch.isnan(out.float())
    rows = {(int(i), int(h)) for i, h in bad.any(-1).nonzero()}
    assert rows == {(0, 1), (1, 2), (2, 3)} and bool(bad[0, 1].all() & bad[1, 2].all() & bad[2, 3].all())


def test_strided_queries_and_outputs():
    import torch
    pool = Pool([333, 90], 2, 128, 64, seed=15).fill()
    d = pool.device([4, 2])
    wide = torch.randn(6, 12, 128 + 6, device="cuda").to(torch.bfloat16)
    q = wide[:, 2:10, 3:131]                            # 2-byte aligned rows
    place = torch.full((6, 9, 136), 7.0, dtype=torch.bfloat16, device="cuda")
    out = place[:, 1:9, 5:133]
    d["cache"].attention(d["batch"], q, out=out)
    ref = torch.zeros(6, 8, 128, dtype=torch.bfloat16, device="cuda")
    d["cache"].attention(d["batch"], q.contiguous(), out=ref)
    assert bool((out == ref).all())
    keep = torch.ones_like(place, dtype=torch.bool)
    keep[:, 1:9, 5:133] = False
    assert bool((place[keep] == 7).all())
    # the same query for every head: a stride of zero
    one = wide[:, :1, :128]
    d["cache"].attention(d["batch"], one.expand(6, 8, 128), out=ref)
    again = torch.zeros_like(ref)
    d["cache"].attention(d["batch"], one.repeat(1, 8, 1), out=again)
    assert bool((ref == again).all())


def test_shared_pages():
    """Two sequences with the same first pages."""
    pool = Pool([64 + 20, 64 + 50], 1, 64, 64, seed=16).fill()
    pool.table[1, 0] = pool.table[0, 0]
    pool.kv[1][:, :64] = pool.kv[0][:, :64]
    attend(pool, [1, 2], 4)


def test_bad_pages_and_lengths_are_flagged():
    """Tokens of a page outside the pool are not seen; lengths and offsets out of range are brought inside."""
    import torch
    pool = Pool([200, 60], 1, 64, 16, seed=17).fill()
    good = pool.table.copy()
    for bad in (-1, pool.n_pages, 2 ** 31 - 1, -2 ** 31):
        pool.table[:] = good
        pool.table[0, 3] = bad
        pool_kv = pool.kv[0]
        seen = np.r_[0:48, 64:200]
        q = np.random.default_rng(1).standard_normal((3, 4, 64)) * 2
        d = pool.device([1, 2])
        qt = torch.tensor(q, dtype=torch.bfloat16, device="cuda")
        out = d["cache"].attention(d["batch"], qt)
        torch.cuda.synchronize()
        assert int(d["status"]) == 1
        ref, _, mag = O.attention(qt.double().cpu().numpy()[:1], pool_kv[0, seen], pool_kv[1, seen], 0.125)
        assert np.all(np.abs(out[:1].double().cpu().numpy() - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -10 * mag)
    pool.table[:] = good
    for lengths, offsets in (([10 ** 6, 60], [0, 1, 3]), ([-5, 60], [0, 1, 3]), ([200, 60], [0, 5, 3]),
                             ([200, 60], [-4, 1, 3]), ([200, 60], [0, 1, 1000])):
        d = pool.device([1, 2], lengths=lengths)
        d["offsets"].copy_(torch.tensor(offsets, dtype=torch.int32))
        out = d["cache"].attention(d["batch"], torch.ones(3, 4, 64, dtype=torch.bfloat16, device="cuda"))
        torch.cuda.synchronize()
        assert int(d["status"]) & 2
        if lengths[1] == 60 and offsets[1:] == [1, 3]:
            assert bool(torch.isfinite(out[1:].float()).all())


def test_results_do_not_change_from_call_to_call():
    import torch
    pool = Pool([5000, 40, 900], 2, 128, 64, seed=18).fill()
    d, q, out, lse, work = attend(pool, [3, 1, 2], 8)
    for _ in range(5):
        again = d["cache"].attention(d["batch"], q, scale=128 ** -0.5, workspace=work)
        assert bool((again == out).all())
    # a larger workspace, dirty from other calls, is as good
    big = d["cache"].attention_workspace(8, 50, 400)
    d["cache"].attention(d["batch"], q * 2, workspace=big)
    assert bool((d["cache"].attention(d["batch"], q, scale=128 ** -0.5, workspace=big) == out).all())


def test_captured_call_follows_the_arrays():
    """A graph's replays see new lengths, pages and queries; two graphs share the workspace one after the other."""
    import torch
    pool = Pool([700, 300], 1, 64, 32, seed=19).fill()
    d = pool.device([2, 1])
    hq = 4
    work = d["cache"].attention_workspace(hq, 2, 3)
    q = torch.randn(3, hq, 64, device="cuda").to(torch.bfloat16)
    outs, graphs = [], []
    for _ in range(2):
        out = torch.zeros(3, hq, 64, dtype=torch.bfloat16, device="cuda")
        d["cache"].attention(d["batch"], q, out=out, workspace=work)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            d["cache"].attention(d["batch"], q, out=out, workspace=work)
        outs.append(out)
        graphs.append(g)
    for lengths in ([700, 300], [33, 300], [2, 1], [511, 7]):
        d["lengths"].copy_(torch.tensor(lengths, dtype=torch.int32))
        q.copy_(torch.randn(3, hq, 64, device="cuda"))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert bool((outs[0] == outs[1]).all())
        check_rows = outs[0].double().cpu().numpy()
        pool.offsets = np.array([0, 2, 3])
        for s, r in enumerate([2, 1]):
            n, o0 = lengths[s], int(pool.offsets[s])
            ref, _, mag = O.attention(q.double().cpu().numpy()[o0:o0 + r], *pool.kv[s][:, :n], 64 ** -0.5)
            assert np.all(np.abs(check_rows[o0:o0 + r] - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -10 * mag)


def test_on_two_streams_at_once():
    import torch
    pool = Pool([3000], 2, 128, 64, seed=20).fill()
    d, q, out, lse, work = attend(pool, [2], 8)
    streams = [torch.cuda.Stream() for _ in range(2)]
    works = [d["cache"].attention_workspace(8, 1, 2) for _ in streams]
    outs = [torch.zeros_like(out) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, w, o in zip(streams, works, outs):
            d["cache"].attention(d["batch"], q, out=o, workspace=w, stream=s)
    torch.cuda.synchronize()
    assert all(bool((o == out).all()) for o in outs)


# ------------------------------------------------------------------- append
def angles(n, hd):
    a = np.arange(n)[:, None] * 10000.0 ** (-2 * np.arange(hd // 2) / hd)
    return np.stack((np.cos(a), np.sin(a)), -1).astype(np.float32)


def new_rows(pool, n_rows, hq, dtype, seed, std=1.0):
    import torch
    g = np.random.default_rng(seed)
    x = g.standard_normal((n_rows, hq + 2 * pool.hk, pool.hd)) * std * np.exp2(g.uniform(-3, 3, (n_rows, 1, 1)))
    return torch.tensor(x, device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def expect_append(pool, rows, k, v):
    """The records after appending k, v (fp64 [row, head, hd], already rotated): {(s, b, h): block}."""
    want = {}
    for s, r in enumerate(rows):
        n = pool.lens[s]
        start, o0 = max(n - r, 0), int(pool.offsets[s]) + r - n
        for b in range(start // 16, -(-n // 16) if r else 0):
            first, last = max(start - 16 * b, 0), min(n - 16 * b, 16)
            at = o0 + 16 * b
            for h in range(pool.hk):
                old = O.unpack_record(pool.block(s, b)[h]) if first else None
                want[s, b, h] = O.append_block(old, first, k[at + first:at + last, h], v[at + first:at + last, h])
    return want


LAYOUTS = [([1], [1]), ([17], [1]), ([16], [16]), ([33, 250, 9, 64], [5, 250, 0, 16]), ([300, 1, 31], [11, 1, 31]),
           ([95, 15, 48], [40, 2, 33])]


@pytest.mark.parametrize("hk,hd,page", [(2, 64, 16), (1, 128, 48), (8, 128, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,rows", LAYOUTS)
def test_append_bytes(hk, hd, page, dtype, lens, rows):
    """Without rotation: every touched record byte for byte, everything else as it was."""
    import torch
    pool = Pool(lens, hk, hd, page, seed=len(lens)).fill()
    d = pool.device(rows, pad=3)
    x = new_rows(pool, pool.n_rows, 0, dtype, 3)
    before = d["data"].clone()
    d["cache"].append(d["batch"], x[:, :hk], x[:, hk:])
    torch.cuda.synchronize()
    assert int(d["status"]) == 0
    xs = x.double().cpu().numpy()
    want = expect_append(pool, rows, xs[:, :hk], xs[:, hk:])
    for (s, b, h), blk in want.items():
        rec = O.pack_record(*blk)
        rec[-24:] = pool.block(s, b)[h][-24:]
        pool.block(s, b)[h] = rec
    assert np.array_equal(d["data"].cpu().numpy().reshape(pool.data.shape), pool.data)
    assert len(want) or bool((d["data"] == before).all())


@pytest.mark.parametrize("hq,hk,hd,page", [(4, 2, 64, 32), (32, 8, 128, 64), (5, 1, 128, 16)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,rows", LAYOUTS)
def test_append_rotates(hq, hk, hd, page, dtype, lens, rows):
    import torch
    pool = Pool(lens, hk, hd, page, seed=7).fill()
    d = pool.device(rows, pad=2)
    x = new_rows(pool, pool.n_rows, hq, dtype, 4)
    table = angles(max(lens), hd)
    rope = torch.tensor(table, device="cuda")
    q_out = torch.full((pool.n_rows, hq, hd), 7.0, dtype=torch.bfloat16, device="cuda")
    d["cache"].append(d["batch"], x[:, hq:hq + hk], x[:, hq + hk:], rope=rope, q=x[:, :hq], q_out=q_out)
    k_out = torch.full((pool.n_rows, hk, hd), 7.0, device="cuda")
    v_out = torch.full_like(k_out, 7.0)
    d["cache"].read(d["batch"], k_out, v_out)
    torch.cuda.synchronize()
    assert int(d["status"]) == 0
    xs = x.double().cpu().numpy()
    pos = np.concatenate([np.arange(n - r, n) for n, r in zip(lens, rows)])
    end = int(pool.offsets[-1])
    rot = O.rope(xs[:end, :hq + hk], table[pos][:, None].astype(np.float64))
    pair = np.abs(xs[:end, :hq + hk])
    pair = np.tile(pair[..., :hd // 2] + pair[..., hd // 2:], 2) * 2.0 ** -21
    got = q_out.double().cpu().numpy()
    assert np.all(np.abs(got[:end] - rot[:, :hq]) <= 2.0 ** -8 * np.abs(rot[:, :hq]) + pair[:, :hq])
    assert np.all(got[end:] == 7)
    after = d["data"].cpu().numpy().reshape(pool.data.shape)
    gk, gv = k_out.double().cpu().numpy(), v_out.double().cpu().numpy()
    assert np.all(gk[end:] == 7) and np.all(gv[end:] == 7)
    want = expect_append(pool, rows, rot[:, hq:], xs[:end, hq + hk:])
    for (s, b, h), (kc, vc, ks, vs) in want.items():
        rec = after[pool.table[s, b // pool.bpp], h, b % pool.bpp]
        rk, rv, rks, rvs = O.unpack_record(rec)
        assert np.array_equal(rv, vc) and rvs == vs
        n, r = lens[s], rows[s]
        first, last = max(n - r - 16 * b, 0), min(n - 16 * b, 16)
        at = int(pool.offsets[s]) + r - n + 16 * b
        new, slack = rot[at + first:at + last, hq + h], pair[at + first:at + last, hq + h]
        if rks != ks:
            top = np.abs(new).max()
            assert rks in (ks / 2, 2 * ks) and abs(top / (448 * min(ks, rks)) - 1) < 1e-5
        else:
            assert np.array_equal(rk[:first], kc[:first]) and not rk[last:].any()
        stored = O.VALUES[rk[first:last]] * rks
        assert np.all(np.abs(stored - new) <= np.maximum(2.0 ** -4 * np.abs(new), 2.0 ** -10 * rks) + slack)
        assert np.array_equal(gk[at + first:at + last, h], stored)
        assert np.array_equal(gv[at + first:at + last, h], O.VALUES[rv[first:last]] * rvs)


def test_append_values_out_of_the_ordinary():
    """Zeros, the smallest and largest values, infinities and NaN."""
    import torch
    pool = Pool([40], 1, 64, 16, seed=1)
    d = pool.device([40])
    x = torch.zeros(40, 2, 64, device="cuda")
    x[0:16] = 0.0
    x[16, :, 3], x[17, :, 4], x[18, :, 5] = math.inf, -math.inf, math.nan
    x[19, :, 6] = -1.5
    x[32, :, 0], x[33, :, 1], x[34, :, 2] = 3.0e38, 1e-30, -0.0
    x[35] = 1e-42
    d["cache"].append(d["batch"], x[:, :1], x[:, 1:])
    torch.cuda.synchronize()
    pool.offsets = np.array([0, 40])
    xs = x.double().cpu().numpy()
    for (s, b, h), blk in expect_append(pool, [40], xs[:, :1], xs[:, 1:]).items():
        rec = d["data"].cpu().numpy().reshape(pool.data.shape)[pool.table[0, b], 0, 0]
        got = O.unpack_record(rec)
        assert got[2:] == blk[2:]
        assert np.array_equal(O.VALUES[got[0]], O.VALUES[blk[0]], equal_nan=True)
        assert np.array_equal(O.VALUES[got[1]], O.VALUES[blk[1]], equal_nan=True)


def test_append_token_by_token_and_over_rejected_drafts():
    """One token a call, a scale that grows; a rejected draft's tokens are overwritten; the block's start resets it."""
    import torch
    hd = 64
    pool = Pool([64], 2, hd, 32, seed=2)
    d = pool.device([1], lengths=[1])
    rng = np.random.default_rng(3)
    state = {}

    def step(length, r, std):
        x = torch.tensor(rng.standard_normal((r, 4, hd)) * std, device="cuda").to(torch.bfloat16)
        d["offsets"][1] = r
        d["lengths"][0] = length
        from paper_2602_20217_gb300 import kv8
        kv8_batch = kv8.Batch8(d["table"], d["offsets"], d["lengths"], r)
        d["cache"].append(kv8_batch, x[:, :2], x[:, 2:])
        xs = x.double().cpu().numpy()
        for b in range((length - r) // 16, -(-length // 16)):
            first, last = max(length - r - 16 * b, 0), min(length - 16 * b, 16)
            at = 16 * b - (length - r)
            for h in range(2):
                state[b, h] = O.append_block(state.get((b, h)), first, xs[at + first:at + last, h],
                                             xs[at + first:at + last, 2 + h])
        data = d["data"].cpu().numpy().reshape(pool.data.shape)
        for (b, h), blk in state.items():
            got = O.unpack_record(data[pool.table[0, b // 2], h, b % 2])
            assert got[2:] == blk[2:] and np.array_equal(got[0], blk[0]) and np.array_equal(got[1], blk[1]), (length, b, h)

    for n in range(1, 20):
        step(n, 1, 2.0 ** (n % 5))
    step(24, 5, 100.0)
    step(21, 2, 0.01)      # the drafts from token 19 on were wrong
    step(35, 19, 1.0)
    step(33, 17, 0.5)      # block 1 begins anew


def test_append_and_read_with_strides():
    import torch
    pool = Pool([30, 5], 2, 64, 16, seed=4).fill()
    d = pool.device([9, 5])
    n = pool.n_rows
    big = torch.randn(2, 3, n, 70, device="cuda").to(torch.bfloat16)      # [k, v][head][row]
    k, v = (big[i, :2, :, 3:67].transpose(0, 1) for i in range(2))
    d["cache"].append(d["batch"], k, v)
    first = d["data"].clone()
    d["cache"].append(d["batch"], k.contiguous(), v.contiguous())
    assert bool((first == d["data"]).all())
    place = [torch.full((n, 5, 66), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ko, vo = (p[:, 1:5:2, 1:65] for p in place)
    d["cache"].read(d["batch"], ko, vo)
    kr, vr = torch.zeros(n, 2, 64, device="cuda"), torch.zeros(n, 2, 64, device="cuda")
    d["cache"].read(d["batch"], kr, vr)
    assert bool((ko.float() == kr).all() & (vo.float() == vr).all())     # codes times powers of two are bf16 values
    for p in place:
        m = torch.ones_like(p, dtype=torch.bool)
        m[:, 1:5:2, 1:65] = False
        assert bool((p[m] == 7).all())


def test_append_flags_what_it_cannot_place():
    import torch
    pool = Pool([40, 20], 1, 64, 16, seed=5).fill()
    good = pool.table.copy()
    x = torch.randn(8, 3, 64, device="cuda").to(torch.bfloat16)
    for bad in (-1, pool.n_pages, 2 ** 31 - 1):
        pool.table[:] = good
        pool.table[0, 2] = bad
        d = pool.device([5, 3])
        before = d["data"].clone().reshape(pool.data.shape)
        d["cache"].append(d["batch"], x[:, :1], x[:, 1:2])
        ko, vo = torch.full((8, 1, 64), 7.0, device="cuda"), torch.full((8, 1, 64), 7.0, device="cuda")
        d["cache"].read(d["batch"], ko, vo)
        torch.cuda.synchronize()
        assert int(d["status"]) == 1
        after = d["data"].reshape(pool.data.shape)
        changed = (before != after).any(-1).nonzero()[:, 0].unique().tolist()
        assert changed == [int(good[1, 1])]            # rows 0..4 are tokens 35..39, all of block 2
        assert not ko[:5].any() and not vo[:5].any() and bool((ko[5:] != 7).all())
    pool.table[:] = good
    # a table that ends before the token: stored as zeros, the query too
    d = pool.device([5, 3])
    rope = torch.tensor(angles(38, 64), device="cuda")
    q_out = torch.full((8, 1, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    d["cache"].append(d["batch"], x[:, :1], x[:, 1:2], rope=rope, q=x[:, 2:], q_out=q_out)
    ko, vo = torch.empty(8, 1, 64, device="cuda"), torch.empty(8, 1, 64, device="cuda")
    d["cache"].read(d["batch"], ko, vo)
    torch.cuda.synchronize()
    assert int(d["status"]) == 4
    assert not ko[3:5].any() and not vo[3:5].any() and not q_out[3:5].any() and bool((q_out[:3] != 0).any())
    # more rows than tokens
    d = pool.device([5, 3], lengths=[3, 20])
    before = d["data"].clone()
    d["cache"].append(d["batch"], x[:, :1], x[:, 1:2])
    torch.cuda.synchronize()
    assert int(d["status"]) == 4
    # lengths and offsets out of range
    for lengths, offsets in (([10 ** 7, 20], [0, 5, 8]), ([-1, 20], [0, 5, 8]), ([40, 20], [0, 9, 4]),
                             ([40, 20], [-3, 5, 8]), ([40, 20], [0, 5, 10 ** 6])):
        d = pool.device([5, 3], lengths=lengths)
        d["offsets"].copy_(torch.tensor(offsets, dtype=torch.int32))
        d["cache"].append(d["batch"], x[:, :1], x[:, 1:2])
        torch.cuda.synchronize()
        assert int(d["status"]) & 2


def test_append_then_attend_as_a_decoder_does():
    """Prompts, then decode steps and verify passes of several rows on the cache's own bytes, in a captured graph too."""
    import torch
    hq, hk, hd, page = 8, 2, 128, 32
    lens = [130, 45]
    pool = Pool([200, 200], hk, hd, page, seed=6)
    pool.lens = lens
    rng = np.random.default_rng(8)
    table = torch.tensor(angles(256, hd), device="cuda")
    from paper_2602_20217_gb300 import kv8
    d = pool.device(lens, lengths=lens)

    def one(rows, lengths):
        n = sum(rows)
        d["offsets"].copy_(torch.tensor(np.concatenate(([0], np.cumsum(rows))), dtype=torch.int32))
        d["lengths"].copy_(torch.tensor(lengths, dtype=torch.int32))
        batch = kv8.Batch8(d["table"], d["offsets"], d["lengths"], n, d["status"])
        x = torch.tensor(rng.standard_normal((n, hq + 2 * hk, hd)) * 1.5, device="cuda", dtype=torch.float32)
        q_out = torch.empty(n, hq, hd, dtype=torch.bfloat16, device="cuda")
        d["cache"].append(batch, x[:, hq:hq + hk], x[:, hq + hk:], rope=table, q=x[:, :hq], q_out=q_out)
        out = torch.zeros(n, hq, hd, dtype=torch.bfloat16, device="cuda")
        lse = torch.zeros(n, hq, device="cuda")
        d["cache"].attention(batch, q_out, out=out, lse=lse)
        torch.cuda.synchronize()
        assert int(d["status"]) == 0
        pool.data = d["data"].cpu().numpy().reshape(pool.data.shape)
        pool.lens = lengths
        pool.kv = [np.stack([np.stack([np.stack(pool.token(s, t, h)) for h in range(hk)], 1) for t in range(m)], 1)
                   for s, m in enumerate(lengths)]
        pool.offsets = np.concatenate(([0], np.cumsum(rows)))
        check(pool, rows, q_out.double().cpu().numpy(), out.double().cpu().numpy(), lse.double().cpu().numpy(), hd ** -0.5)

    one(lens, lens)                      # prompts
    one([1, 1], [131, 46])               # a token each
    one([5, 11], [136, 57])              # verify passes
    one([1, 2], [133, 50])               # after rejections
