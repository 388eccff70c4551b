"""The 8-bit cache attention where a unit has more than 16 query rows: 17 to 32
(four copies of them in a tile), up to 64 (two) and more, with the tolerances
of test_gpu_kv8.  What is special there: weights are relative to a reference
that is raised now and then, values to the loudest block so far, tiles hold 128
keys, and a raise or a NaN may come in any of a tile's parts."""
import math

import numpy as np
import pytest

from helpers import need_gpu
from oracle import kv8 as O
from test_gpu_kv8 import Pool, angles, attend, expect_append

pytestmark = pytest.mark.gpu

HQ = 4
ROWS = [5, 12, 32, 45]          # 20, 48, 128 and 180 query rows of one KV head


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()


def put(pool, s, k, v):
    """Tokens k, v [n, hd] of sequence s, head 0."""
    for b in range(-(-len(k) // 16)):
        last = min(16, len(k) - 16 * b)
        kc, vc, ks, vs = O.append_block(None, 0, k[16 * b:16 * b + last], v[16 * b:16 * b + last])
        kc[last:] = 0x7f
        vc[last:] = 0xff
        pool.block(s, b)[0] = O.pack_record(kc, vc, ks, vs)
        pool.kv[s][0, 16 * b:16 * b + last, 0] = O.VALUES[kc[:last]] * ks
        pool.kv[s][1, 16 * b:16 * b + last, 0] = O.VALUES[vc[:last]] * vs


def mark(pool, t, d, which):
    """A NaN in token t of sequence 0: its value (1) or its key (0)."""
    rec = O.unpack_record(pool.block(0, t // 16)[0])
    rec[which][t % 16, d] = 0xff
    pool.block(0, t // 16)[0] = O.pack_record(*rec)
    pool.kv[0][which, t, 0, d] = math.nan


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("shape", ["rising", "steps", "falling", "late peak", "alternating"])
def test_scores_that_move(rows, shape):
    """Scores along one direction of the head: the reference is raised often, seldom, in every part of a tile."""
    n, hd = 900, 64
    t = np.arange(n)
    x = {"rising": -30 + 60 * t / n, "falling": 30 - 60 * t / n,
         "steps": 12.0 * ((t > 130).astype(int) + (t > 200) + (t > 210) + (t > 500)) - 20,
         "late peak": np.where(t == n - rows - 40, 30.0, -10.0),
         "alternating": np.where(t // 37 % 2, 20.0, -20.0) * (t / n)}[shape]
    rng = np.random.default_rng(rows)
    u = rng.standard_normal(hd)
    u /= np.linalg.norm(u)
    pool = Pool([n], 1, hd, 64, seed=1).fill()
    put(pool, 0, x[:, None] * u + 0.1 * rng.standard_normal((n, hd)), rng.standard_normal((n, hd)))
    q = u + 0.02 * rng.standard_normal((rows, HQ, hd))
    q[::3] *= 0.5                                    # rows that are raised at other keys
    attend(pool, [rows], HQ, q=q, scale=1.0)


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("hd,page", [(64, 16), (128, 128)])
def test_blocks_of_far_scales(rows, hd, page):
    """Values 2^-20 and 2^9 of their neighbours', zeros; all weight on a token of a quiet block behind a loud one."""
    pool = Pool([500], 1, hd, page, seed=2).fill(spread=0)
    for b, f in ((0, 2.0 ** -20), (2, 0.0), (4, 2.0 ** 9), (9, 2.0 ** -20), (17, 2.0 ** 14), (20, 2.0 ** -18)):
        kc, vc, ks, vs = O.unpack_record(pool.block(0, b)[0])
        vs = vs * f if f else 2.0 ** -126
        vc = vc if f else vc & 0x80
        pool.block(0, b)[0] = O.pack_record(kc, vc, ks, vs)
        pool.kv[0][1, 16 * b:16 * b + 16, 0] = O.VALUES[vc] * vs
    attend(pool, [rows], HQ)
    for token in (5, 150, 325):
        k = pool.kv[0][0, token, 0]
        q = np.broadcast_to(k / (k @ k) * 60, (rows, HQ, hd))
        attend(pool, [rows], HQ, q=q, scale=1.0)


@pytest.mark.parametrize("rows", ROWS)
def test_a_long_flat_tail_behind_a_peak(rows):
    n, hd = 20000 + rows, 64
    pool = Pool([n], 1, hd, 128, seed=3).fill(spread=0)
    k = np.zeros((n, hd))
    k[0, 0] = 448.0
    v = np.abs(np.random.default_rng(4).standard_normal((n, hd)))
    v[0] = 0
    put(pool, 0, k, v)
    q = np.zeros((rows, HQ, hd))
    q[:, :, 0] = 0.0234375                           # 10.5: half of the weight on token 0
    attend(pool, [rows], HQ, q=q, scale=1.0)


@pytest.mark.parametrize("rows", ROWS)
def test_nan_tokens_stay_with_the_rows_that_see_them(rows):
    n = 400
    pool = Pool([n], 1, 64, 16, seed=5).fill()
    mark(pool, n - rows + 2, 7, 1)                   # seen from row 2 on
    mark(pool, n - 2, 3, 0)                          # a key: whole rows
    mark(pool, n - 1, 9, 1)
    attend(pool, [rows], HQ)
    pool = Pool([n], 1, 64, 16, seed=6).fill()
    mark(pool, 77, 5, 1)                             # seen by all: one dim
    attend(pool, [rows], HQ)


@pytest.mark.parametrize("rows", ROWS)
def test_queries_that_are_not_finite(rows):
    import torch
    pool = Pool([200], 1, 64, 16, seed=7).fill()
    d = pool.device([rows])
    q = torch.randn(rows, HQ, 64, device="cuda").to(torch.bfloat16)
    ref = d["cache"].attention(d["batch"], q)
    q[0, 1, 5], q[2, 2, 60], q[rows - 1, 3, 0] = math.inf, -math.inf, math.nan
    out = d["cache"].attention(d["batch"], q)
    bad = torch.isnan(out.float())
    assert {(int(i), int(h)) for i, h in bad.any(-1).nonzero()} == {(0, 1), (2, 2), (rows - 1, 3)}
    assert bool((bad.any(-1) == bad.all(-1)).all()) and bool((out[~bad] == ref[~bad]).all())


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("scale", [0.0, -0.3, 0.5])
def test_scales(rows, scale):
    attend(Pool([300], 1, 64, 32, seed=8).fill(), [rows], HQ, scale=scale)


@pytest.mark.parametrize("rows", ROWS)
def test_queries_of_zeros_and_of_far_elements(rows):
    """A row of zeros, rows whose elements lie 2^20 apart (the small ones are below what the codes hold)."""
    rng = np.random.default_rng(9)
    q = rng.standard_normal((rows, HQ, 64))
    q[1] = 0
    q[2, :, ::2] *= 2.0 ** -20
    q[3] *= 2.0 ** -100
    attend(Pool([300], 1, 64, 32, seed=9).fill(spread=0), [rows], HQ, q=q)


@pytest.mark.parametrize("rows", [[20, 7], [45, 33]])
def test_strided_queries_and_outputs(rows):
    import torch
    n = sum(rows)
    pool = Pool([333, 90], 2, 128, 64, seed=15).fill()
    d = pool.device(rows)
    wide = torch.randn(n, 12, 128 + 6, device="cuda").to(torch.bfloat16)
    q = wide[:, 2:10, 3:131]                         # 2-byte aligned rows
    place = torch.full((n, 9, 136), 7.0, dtype=torch.bfloat16, device="cuda")
    out = place[:, 1:9, 5:133]
    d["cache"].attention(d["batch"], q, out=out)
    ref = torch.zeros(n, 8, 128, dtype=torch.bfloat16, device="cuda")
    d["cache"].attention(d["batch"], q.contiguous(), out=ref)
    assert bool((out == ref).all())
    keep = torch.ones_like(place, dtype=torch.bool)
    keep[:, 1:9, 5:133] = False
    assert bool((place[keep] == 7).all())


def test_bad_pages_are_not_seen():
    import torch
    pool = Pool([300, 60], 1, 64, 16, seed=17).fill()
    for bad in (-1, pool.n_pages, 2 ** 31 - 1, -2 ** 31):
        pool.table[0, 3], keep = bad, pool.table[0, 3]
        seen = np.r_[0:48, 64:300]
        q = np.random.default_rng(1).standard_normal((45, HQ, 64)) * 2
        d = pool.device([40, 5])
        qt = torch.tensor(q, dtype=torch.bfloat16, device="cuda")
        out = d["cache"].attention(d["batch"], qt)
        torch.cuda.synchronize()
        assert int(d["status"]) == 1
        ref, _, mag = O.attention(qt.double().cpu().numpy()[:40], pool.kv[0][0, seen], pool.kv[0][1, seen], 0.125)
        assert np.all(np.abs(out[:40].double().cpu().numpy() - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -10 * mag)
        pool.table[0, 3] = keep


def test_replays_of_a_padded_batch():
    """Two graphs of one workspace, padded to 60 rows; offsets, lengths and queries change between replays."""
    import torch
    pool = Pool([700, 300, 90], 1, 64, 32, seed=19).fill()
    d = pool.device([40, 9, 1], pad=10)
    n, work = 60, d["cache"].attention_workspace(HQ, 3, 60)
    q = torch.randn(n, HQ, 64, device="cuda").to(torch.bfloat16)
    outs = [torch.zeros(n, HQ, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    graphs = []
    for out in outs:
        d["cache"].attention(d["batch"], q, out=out, workspace=work)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            d["cache"].attention(d["batch"], q, out=out, workspace=work)
        graphs.append(g)
    for lengths, rows in (([700, 300, 90], [40, 9, 1]), ([33, 300, 1], [1, 1, 1]), ([511, 7, 0], [50, 7, 0]),
                          ([129, 128, 90], [0, 60, 0])):
        off = np.concatenate(([0], np.cumsum(rows)))
        d["lengths"].copy_(torch.tensor(lengths, dtype=torch.int32))
        d["offsets"].copy_(torch.tensor(off, dtype=torch.int32))
        q.copy_(torch.randn(n, HQ, 64, device="cuda"))
        for out, g in zip(outs, graphs):
            out.fill_(7.0)
            g.replay()
        torch.cuda.synchronize()
        assert bool((outs[0] == outs[1]).all()) and bool((outs[0][off[-1]:] == 7).all())
        assert int(d["status"]) == 0
        got, qn = outs[0].double().cpu().numpy(), q.double().cpu().numpy()
        for s, r in enumerate(rows):
            o0 = off[s]
            ref, _, mag = O.attention(qn[o0:o0 + r], *pool.kv[s][:, :lengths[s]], 64 ** -0.5)
            assert np.all(np.abs(got[o0:o0 + r] - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -10 * mag)


def test_on_two_streams_at_once():
    import torch
    pool = Pool([3000, 500], 2, 128, 64, seed=20).fill()
    d, q, out, lse, work = attend(pool, [40, 13], 8)
    streams = [torch.cuda.Stream() for _ in range(2)]
    works = [d["cache"].attention_workspace(8, 2, 53) for _ in streams]
    outs = [torch.zeros_like(out) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, w, o in zip(streams, works, outs):
            d["cache"].attention(d["batch"], q, out=o, workspace=w, stream=s)
    torch.cuda.synchronize()
    assert all(bool((o == out).all()) for o in outs)


@pytest.mark.parametrize("rows", [1, 40])
def test_a_cache_larger_than_32_bit_offsets(rows):
    """Pages at both ends of a pool of 5 GB: bytes appended there are read back and attended over."""
    import torch
    from paper_2602_20217_gb300 import kv8
    hk, hd, page, hq = 8, 128, 128, 32
    per_page = hk * (page // 16) * O.record_bytes(hd)
    n_pages = 5 * 2 ** 30 // per_page
    cache = kv8.Cache8(n_pages, page, hk, hd)
    n = 300
    table = torch.tensor([[n_pages - 1, 0, n_pages // 2 + 1]], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def batch(r):
        return kv8.Batch8(table, torch.tensor([0, r], dtype=torch.int32, device="cuda"),
                          torch.tensor([n], dtype=torch.int32, device="cuda"), r, status)
    x = torch.randn(2, n, hk, hd, device="cuda").to(torch.bfloat16)
    cache.append(batch(n), x[0], x[1])
    ko, vo = torch.empty(2, n, hk, hd, device="cuda")
    cache.read(batch(n), ko, vo)
    # a code is within half a step, 2^-4, or 2^-10 of the scale, at most 2^-8 |x|max of the block
    assert bool(((ko - x[0].float()).abs() <= 2.0 ** -4 * x[0].float().abs() + 2.0 ** -16 * 8).all())
    assert bool(((vo - x[1].float()).abs() <= 2.0 ** -4 * x[1].float().abs() + 2.0 ** -16 * 8).all())
    q = torch.randn(rows, hq, hd, device="cuda").to(torch.bfloat16)
    out = cache.attention(batch(rows), q).double().cpu().numpy()
    ref, _, mag = O.attention(q.double().cpu().numpy(), ko.double().cpu().numpy(), vo.double().cpu().numpy(), hd ** -0.5)
    assert int(status) == 0
    assert np.all(np.abs(out - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -10 * mag)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_from_unaligned_rows(dtype, hd):
    """Rows, queries and outputs at odd elements give the bytes of aligned ones."""
    import torch
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    pool = Pool([70, 5, 33], 2, hd, 16, seed=21).fill()
    rows = [30, 5, 1]
    d = pool.device(rows)
    n, hq = sum(rows), 6
    table = torch.tensor(angles(80, hd), device="cuda")
    x = torch.randn(n, hq + 4, hd + 3, device="cuda").to(td)[:, :, 1:hd + 1]
    start = d["data"].clone()
    place = torch.full((n, hq + 1, hd + 5), 7.0, dtype=torch.bfloat16, device="cuda")
    q_out = place[:, 1:, 3:hd + 3]
    d["cache"].append(d["batch"], x[:, hq:hq + 2], x[:, hq + 2:], rope=table, q=x[:, :hq], q_out=q_out)
    first = d["data"].clone()
    d["data"].copy_(start)
    y = x.contiguous()
    ref = torch.zeros(n, hq, hd, dtype=torch.bfloat16, device="cuda")
    d["cache"].append(d["batch"], y[:, hq:hq + 2], y[:, hq + 2:], rope=table, q=y[:, :hq], q_out=ref)
    assert bool((first == d["data"]).all()) and bool((q_out == ref).all())
    keep = torch.ones_like(place, dtype=torch.bool)
    keep[:, 1:, 3:hd + 3] = False
    assert bool((place[keep] == 7).all()) and int(d["status"]) == 0


def test_append_many_blocks_of_few_sequences():
    """Batches cut by sequence whose rows still touch more blocks than a sequence has CTAs for."""
    import torch
    lens = [500] + [40] * 40
    rows = [450] + [1] * 40
    pool = Pool(lens, 2, 64, 32, seed=22).fill()
    d = pool.device(rows)
    x = torch.tensor(np.random.default_rng(23).standard_normal((sum(rows), 4, 64)), device="cuda").to(torch.bfloat16)
    xs = x.double().cpu().numpy()
    want = expect_append(pool, rows, xs[:, :2], xs[:, 2:])
    d["cache"].append(d["batch"], x[:, :2], x[:, 2:])
    ko, vo = torch.empty(2, sum(rows), 2, 64, device="cuda")
    d["cache"].read(d["batch"], ko, vo)
    data = d["data"].cpu().numpy().reshape(pool.data.shape)
    assert int(d["status"]) == 0
    for (s, b, h), blk in want.items():
        got = O.unpack_record(data[pool.table[s, b // 2], h, b % 2])
        assert got[2:] == blk[2:] and np.array_equal(got[0], blk[0]) and np.array_equal(got[1], blk[1]), (s, b, h)
    o0 = int(pool.offsets[0])
    for t in range(50, 500):
        blk = want[0, t // 16, 1]
        assert np.array_equal(ko[o0 + t - 50, 1].cpu().numpy(), O.VALUES[blk[0][t % 16]] * blk[2])
        assert np.array_equal(vo[o0 + t - 50, 1].cpu().numpy(), O.VALUES[blk[1][t % 16]] * blk[3])


@pytest.mark.parametrize("offsets", [[100, 3, 60], [0, 80, 70], [-3, 50, 100], [0, 50, 101]])
def test_append_flags_offsets_in_batches_of_many_rows(offsets):
    import torch
    pool = Pool([100, 100], 1, 64, 16, seed=24).fill()
    d = pool.device([50, 50])
    d["offsets"].copy_(torch.tensor(offsets, dtype=torch.int32))
    x = torch.randn(100, 2, 64, device="cuda").to(torch.bfloat16)
    d["cache"].append(d["batch"], x[:, :1], x[:, 1:])
    torch.cuda.synchronize()
    assert int(d["status"]) & 2
    d["status"].zero_()
    out = torch.empty(2, 100, 1, 64, device="cuda")
    d["cache"].read(d["batch"], out[0], out[1])
    torch.cuda.synchronize()
    assert int(d["status"]) & 2


@pytest.mark.parametrize("rows", [1, 20])
def test_calls_in_a_row_see_each_others_writes(rows):
    """Steps of append and attention without a pause between launches give the bits of steps with one after each
    call: scales that grow, rows written over, a workspace and query buffer used by every step, a layer after the
    other."""
    import torch
    from paper_2602_20217_gb300 import kv8
    hq, hk, hd, page, steps, layers = 8, 2, 128, 32, 40, 3
    n_pages = (rows * steps + 200) // page + 1
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    x = torch.randn(steps, layers, rows, hq + 2 * hk, hd, generator=g, device="cuda")
    x *= torch.exp2(torch.arange(steps, device="cuda") % 7 - 3.0)[:, None, None, None, None]
    x = x.to(torch.bfloat16)
    table = torch.tensor(angles(rows * steps + 200, hd), device="cuda")
    pages = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)[None]
    offsets = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def run(pause):
        caches = [kv8.Cache8(n_pages, page, hk, hd, data=torch.zeros(kv8.Cache8(n_pages, page, hk, hd).nbytes,
                                                                    dtype=torch.uint8, device="cuda"))
                  for _ in range(layers)]
        lengths = torch.full((1,), 100, dtype=torch.int32, device="cuda")
        batch = kv8.Batch8(pages, offsets, lengths, rows, status)
        work = caches[0].attention_workspace(hq, 1, rows)
        q = torch.empty(rows, hq, hd, dtype=torch.bfloat16, device="cuda")
        outs = torch.zeros(steps, layers, rows, hq, hd, dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        for s in range(steps):
            lengths += rows if s % 3 else rows - rows // 2      # every third step writes over half of the last one
            for i, c in enumerate(caches):
                y = x[s, i]
                c.append(batch, y[:, hq:hq + hk], y[:, hq + hk:], rope=table, q=y[:, :hq], q_out=q)
                if pause:
                    torch.cuda.synchronize()
                c.attention(batch, q, out=outs[s, i], workspace=work)
                if pause:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        return outs, torch.stack([c.data for c in caches])

    want = run(True)
    for _ in range(3):
        got = run(False)
        assert torch.equal(got[0].view(torch.int16), want[0].view(torch.int16)) and torch.equal(got[1], want[1])
    assert int(status) == 0
