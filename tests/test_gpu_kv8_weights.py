"""The weights that tokens of the 8-bit cache receive, against the fp64 restatement.

Tolerance of a term exp(s - lse), relative (oracle/kv8_evict.py computes it): the
score's error, 2^-17 max|q| sum|k| over the dims below 2^-9 of the row's largest
element (queries in two codes) and 2^-16 sum|q k| (128 products added in fp32),
times the scale; three roundings of the score and of lse; 2^-22 of the
exponential.  A token's sum adds 2^-24 of itself for each addition: 2 rows of a
block, 8 blocks, then the chunks of 64 queries, the decayed score and 2 joins.
Terms below 2^-126 are zeros.
"""
import math

import numpy as np
import pytest

from helpers import need_gpu
from oracle import kv8 as K
from oracle import kv8_evict as O
from test_gpu_kv8 import Pool

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()


def receive(pool, rows, hq, decay=1.0, seed=1, lengths=None, pad=0, status=0, offsets=None, q=None, place="new",
            lse=None, extra=0, scale=None):
    import torch
    d = pool.device(rows, lengths, pad, offsets)
    rng = np.random.default_rng(seed)
    n, hd, n_seqs = pool.n_rows, pool.hd, len(pool.lens)
    qt = torch.tensor(rng.standard_normal((n, hq, hd)) * 2 if q is None else q, dtype=torch.bfloat16, device="cuda")
    ld = pool.ld * pool.page + extra
    old = torch.tensor(rng.exponential(1.0, (n_seqs, pool.hk, ld)), dtype=torch.float32, device="cuda")
    scale = hd ** -0.5 if scale is None else scale
    qd = qt.double().cpu().numpy()
    lens = [min(max(x, 0), pool.ld * pool.page) for x in (pool.lens if lengths is None else lengths)]
    if lse is None:
        lse = np.zeros((n, hq), np.float32)
        for s, r in enumerate(rows):
            o = int(pool.offsets[s])
            if r and offsets is None:
                kv = pool.kv[s][:, :lens[s]]
                lse[o:o + r] = K.attention(qd[o:o + r], kv[0], kv[1], scale)[1]
    lse = np.asarray(lse, np.float32)
    if decay == 0:
        old[:] = math.nan
    out = old if place == "same" else torch.full_like(old, 7.0)
    before = out.double().cpu().numpy()
    given = old.double().cpu().numpy()
    got = d["cache"].attention_weights(d["batch"], qt, torch.tensor(lse, device="cuda"),
                                       None if decay == 0 and place == "none" else old, scale=scale, decay=decay, out=out)
    torch.cuda.synchronize()
    assert int(d["status"]) == status and got is out
    got = out.double().cpu().numpy()
    for s, r in enumerate(rows):
        if offsets is not None or r == 0:
            assert np.array_equal(got[s], before[s], equal_nan=True)
            continue
        o, m = int(pool.offsets[s]), lens[s]
        ref, off = O.weights(qd[o:o + r], pool.kv[s][0][:m], lse[o:o + r].astype(np.float64), scale, r)
        older = max(m - r, 0)
        adds = 2 + 8 + (r * hq // pool.hk + 63) // 64 + 3
        if decay != 0:
            add = np.float64(np.float32(decay)) * given[s][:, :older]
            ref[:, :older] += add
        bound = off + 2.0 ** -24 * adds * np.abs(ref) + r * hq * 2.0 ** -125
        assert np.array_equal(np.isnan(got[s][:, :m]), np.isnan(ref)), s
        ok = ~np.isnan(ref)
        err = np.abs(got[s][:, :m] - ref)[ok] - bound[ok]
        assert err.size == 0 or err.max() <= 0, (s, float(err.max()))
        assert np.array_equal(got[s][:, m:], before[s][:, m:], equal_nan=True)
    return d, qt, out


@pytest.mark.parametrize("hq,hk,hd,page", [(2, 1, 64, 16), (32, 8, 128, 64), (12, 4, 128, 48), (64, 1, 128, 32), (4, 2, 64, 16)])
@pytest.mark.parametrize("n", [1, 15, 16, 17, 127, 128, 129, 300, 1000])
def test_one_row(hq, hk, hd, page, n):
    receive(Pool([n], hk, hd, page, seed=n).fill(), [1], hq)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("rows", [2, 7, 16, 33, 130])
@pytest.mark.parametrize("decay", [0.0, 0.9, 1.0])
def test_rows(hd, rows, decay):
    """Several rows, whole prompts, chunks of 64 queries that end inside a row's heads."""
    receive(Pool([rows, rows + 1, rows + 200], 2, hd, 16, seed=rows).fill(), [rows] * 3, 6, decay=decay,
            place="none" if decay == 0 and rows == 7 else "new")


def test_ragged_batch():
    receive(Pool([300, 5, 64, 700, 17, 1], 2, 64, 32).fill(), [1, 5, 0, 12, 3, 1], 8, pad=3, place="same")
    receive(Pool([300, 5, 64, 700, 17, 1], 2, 64, 32).fill(), [1, 5, 0, 12, 3, 1], 8, pad=3, extra=5, decay=-0.5)


def test_many_sequences():
    rng = np.random.default_rng(0)
    lens = [int(x) for x in rng.integers(1, 90, 70)]
    receive(Pool(lens, 2, 64, 16).fill(), [min(n, 1 + i % 3) for i, n in enumerate(lens)], 4)


def test_more_rows_than_tokens():
    """Rows before position 0 see nothing: their sums are -inf, and they give no weight."""
    receive(Pool([10, 40], 2, 64, 16).fill(), [14, 2], 8)


def test_lengths_and_offsets_out_of_range():
    receive(Pool([90, 64], 2, 64, 16).fill(), [1, 1], 8, lengths=[90, -5], status=2)
    receive(Pool([96, 96], 2, 64, 16).fill(), [1, 1], 8, lengths=[96, 5000], status=2)
    receive(Pool([90, 64, 50], 2, 64, 16).fill(), [1, 1, 1], 8, offsets=[0, 2, 1, 3], status=2)


def test_pages_outside_the_pool():
    """Their tokens receive nothing; the others' weights are what lse makes of them."""
    import torch
    pool = Pool([100], 2, 64, 16).fill()
    d, q, want = receive(pool, [2], 4, decay=0.5)
    pool.table[0, 2] = 999
    lse = np.full((2, 4), 3.0, np.float32)
    plain = Pool([100], 2, 64, 16).fill()
    _, _, a = receive(plain, [2], 4, decay=0.5, lse=lse)
    dev = pool.device([2])
    old = torch.tensor(np.random.default_rng(1).exponential(1.0, (1, 2, pool.ld * 16)), dtype=torch.float32, device="cuda")
    old = torch.rand_like(old)
    out = torch.full_like(old, 7.0)
    dev["cache"].attention_weights(dev["batch"], q, torch.tensor(lse, device="cuda"), old, decay=0.5, out=out)
    ref = torch.full_like(old, 7.0)
    d["cache"].attention_weights(d["batch"], q, torch.tensor(lse, device="cuda"), old, decay=0.5, out=ref)
    torch.cuda.synchronize()
    assert int(dev["status"]) == 1
    ref[:, :, 32:48] = 0.5 * old[:, :, 32:48]
    assert torch.equal(out, ref)


def test_not_finite():
    """A NaN key, query or sum spoils what it enters; sums of -inf and +inf give nothing."""
    pool = Pool([200, 60], 2, 64, 16).fill()
    pool.block(0, 3)[1][0] = 0x7f                    # token 48, dim 0, head 1
    pool.kv[0][0, 48, 1, 0] = math.nan
    receive(pool, [3, 2], 8, lse=np.full((5, 8), 2.0))
    q = np.random.default_rng(0).standard_normal((5, 8, 64))
    q[1, 2, 5] = math.inf
    q[3, 7, 0] = math.nan
    pool = Pool([200, 60], 2, 64, 16).fill()
    q[1, 2] = math.nan                               # infinities are NaN there
    receive(pool, [3, 2], 8, lse=np.full((5, 8), 2.0), q=q)
    lse = np.full((5, 8), 2.0)
    lse[0, 0], lse[2, 3], lse[4, 5] = -math.inf, math.inf, math.nan
    receive(pool, [3, 2], 8, lse=lse)


def test_scales():
    for scale in (0.0, -0.2, 1.5):
        receive(Pool([200, 60], 2, 64, 16).fill(), [3, 2], 8, scale=scale)


def test_strides_streams_and_graphs():
    import torch
    pool = Pool([300, 5, 64], 2, 64, 32).fill()
    d, q, out = receive(pool, [1, 5, 2], 8)
    lse = torch.full((8, 8), 3.0, device="cuda")
    old = torch.rand(3, 2, pool.ld * 32, device="cuda")
    want = d["cache"].attention_weights(d["batch"], q, lse, old, out=torch.zeros_like(old))
    odd = torch.zeros(8, 9, 67, dtype=torch.bfloat16, device="cuda")[:, 1:, 1:65]
    odd.copy_(q)
    got = d["cache"].attention_weights(d["batch"], odd, lse, old, out=torch.zeros_like(old))
    assert torch.equal(got, want)
    torch.cuda.synchronize()
    got = d["cache"].attention_weights(d["batch"], q, lse, old, out=torch.zeros_like(old), stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    out = torch.zeros_like(old)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        d["cache"].attention_weights(d["batch"], q, lse, old, out=out)
    d["lengths"][1] = 0                              # its rows see nothing now
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[0], want[0]) and torch.equal(out[2], want[2]) and bool((out[1] == 0).all())


def test_many_rows_of_many_sequences():
    """Calls for the tcgen05 kernel with more sequences than a warp looks at in one go, some without rows or tokens."""
    rng = np.random.default_rng(3)
    lens = [int(x) for x in rng.integers(0, 700, 50)]
    rows = [int(min(n, x)) for n, x in zip(lens, rng.integers(0, 60, 50))]
    receive(Pool(lens, 2, 64, 16, seed=2).fill(), rows, 8, pad=2, decay=0.5)


@pytest.mark.parametrize("n", [511, 512, 513, 1024, 1500])
@pytest.mark.parametrize("rows", [40, 300])
def test_units_of_512_keys(n, rows):
    """Lengths around a unit of the tcgen05 kernel; rows in one chunk of queries and in several; runs that cut units."""
    receive(Pool([n], 8, 128, 64, seed=n).fill(), [rows], 32, decay=0.9, place="same")


@pytest.mark.parametrize("group", [5, 12, 48])
def test_groups_that_do_not_fill_a_chunk(group):
    """Whole chunks of fewer than 128 queries, and the rows of a sequence behind them, which are not finite."""
    for rows in (3 * (128 // group), 3 * (128 // group) + 1):
        q, lse = np.random.default_rng(group).standard_normal((rows + 20, 2 * group, 64)), np.full((rows + 20, 2 * group), 5.0)
        q[rows:rows + 2] = math.nan
        receive(Pool([700, 40], 2, 64, 16).fill(), [rows, 20], 2 * group, decay=0.5, lse=lse, q=q)


def test_many_rows_out_of_range():
    receive(Pool([90, 64, 50], 2, 64, 16).fill(), [20, 20, 20], 8, lengths=[90, -5, 50], status=2)
    receive(Pool([96, 96], 2, 64, 16).fill(), [30, 8], 8, lengths=[96, 5000], status=2)
    receive(Pool([90, 64, 50], 2, 64, 16).fill(), [20, 20, 20], 8, offsets=[0, 40, 20, 60], status=2)


def test_many_rows_not_finite():
    for what in ("key", "query", "lse"):
        pool = Pool([700, 60], 2, 64, 16).fill()
        q, lse = np.random.default_rng(0).standard_normal((90, 8, 64)), np.full((90, 8), 2.0)
        if what == "key":
            pool.block(0, 3)[1][0] = 0x7f
            pool.kv[0][0, 48, 1, 0] = math.nan
        if what == "query":
            q[1, 2, 9] = q[70, 7, 0] = math.nan
        if what == "lse":
            lse[0, 0], lse[30, 3], lse[80, 5] = -math.inf, math.inf, math.nan
        receive(pool, [50, 40], 8, lse=lse, q=q)


def test_many_rows_with_pages_outside_the_pool():
    import torch
    pool = Pool([600], 2, 64, 16).fill()
    lse = torch.full((40, 8), 3.0, device="cuda")
    q = torch.randn(40, 8, 64, device="cuda").to(torch.bfloat16)
    old = torch.rand(1, 2, pool.ld * 16, device="cuda")
    d = pool.device([40])
    want = d["cache"].attention_weights(d["batch"], q, lse, old, decay=0.5, out=torch.full_like(old, 7.0))
    pool.table[0, 3], pool.table[0, 20] = 10 ** 6, -1
    d = pool.device([40])
    got = d["cache"].attention_weights(d["batch"], q, lse, old, decay=0.5, out=torch.full_like(old, 7.0))
    torch.cuda.synchronize()
    assert int(d["status"]) == 1
    for a, b in ((48, 64), (320, 336)):
        want[:, :, a:b] = 0.5 * old[:, :, a:b]
    assert torch.equal(got, want)


def test_many_rows_strides_streams_and_graphs():
    """Queries that tensor copies cannot take go through the other kernel; calls at once have a workspace each."""
    import torch
    pool = Pool([900, 40, 333], 2, 64, 32).fill()
    d, q, out = receive(pool, [100, 40, 33], 8)
    n = q.shape[0]
    lse = torch.full((n, 8), 3.0, device="cuda")
    old = torch.rand(3, 2, pool.ld * 32, device="cuda")
    want = d["cache"].attention_weights(d["batch"], q, lse, old, out=torch.zeros_like(old))
    odd = torch.zeros(n, 9, 67, dtype=torch.bfloat16, device="cuda")[:, 1:, 1:65]
    odd.copy_(q)
    got = d["cache"].attention_weights(d["batch"], odd, lse, old, out=torch.zeros_like(old))
    assert float(((got - want).abs() / want.abs().clamp(min=1e-3)).max()) < 2.0 ** -9     # each within its own bound
    wide = torch.zeros(n, 16, 72, dtype=torch.bfloat16, device="cuda")[:, 8:, :64]
    wide.copy_(q)
    got = d["cache"].attention_weights(d["batch"], wide, lse, old, out=torch.zeros_like(old))
    assert torch.equal(got, want)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros_like(old) for _ in range(6)]
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        d["cache"].attention_weights(d["batch"], q, lse, old, out=o, stream=streams[i % 2])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    with pytest.raises(ValueError):
        d["cache"].attention_weights(d["batch"], q, lse, old, out=outs[0], stream=streams[0].cuda_stream)
    work, out = d["cache"].weights_workspace(8, n), torch.zeros_like(old)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        d["cache"].attention_weights(d["batch"], q, lse, old, out=out, workspace=work)
    work.fill_(0xff)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    d["lengths"][0] = 517
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[1:], want[1:]) and not torch.equal(out[0], want[0])


def test_refusals_of_the_python_face():
    import torch
    pool = Pool([50], 2, 64, 16).fill()
    d = pool.device([1])
    q, lse = torch.zeros(1, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 8, device="cuda")
    ok = torch.zeros(1, 2, pool.ld * 16, device="cuda")
    c, b = d["cache"], d["batch"]
    for bad in [(q.float(), lse, ok), (q, lse[:, :7], ok), (q, lse.double(), ok), (q, lse, ok[:, :1]),
                (q, lse, ok[:, :, 1:]), (q, lse, ok.double()), (q, lse, ok.cpu()), (q, lse, None)]:
        with pytest.raises(ValueError):
            c.attention_weights(b, *bad)
    with pytest.raises(ValueError):
        c.attention_weights(b, q, lse, None, out=ok)             # a decay of 1 needs scores
    with pytest.raises(ValueError):
        c.attention_weights(b, q, lse, torch.zeros(1, 2, pool.ld * 16 + 1, device="cuda"), out=ok)
