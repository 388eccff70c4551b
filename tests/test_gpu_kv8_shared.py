"""Attention of sequences with a common beginning against the fp64 restatement
of the plain attention: what a group shares is only where its tokens lie.

Tolerances are those of test_gpu_kv8.py.  Joining the two parts rounds each
part's output and factors in fp32, a few 2^-24 of the average of |v|, which the
2^-10 of it that the probabilities' 11 bits are given does not leave: the bound
there allows 2^-11 for sums and exponents of 20000 keys, of which the scores
here, under 40, use less than half.
"""
import math

import numpy as np
import pytest

from helpers import need_gpu
from test_gpu_kv8 import Pool, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()


def share(pool, groups, tokens, garbage=True):
    """Sequences groups[g] .. groups[g + 1] begin with the first one's tokens[g] tokens (whole pages); the others'
    tables say nothing of them."""
    for g, n in enumerate(tokens):
        n = n // pool.page * pool.page
        for s in range(groups[g] + 1, groups[g + 1]):
            m = min(n, pool.lens[s] // pool.page * pool.page)
            pool.kv[s][:, :m] = pool.kv[groups[g]][:, :m]
            pool.table[s, :m // pool.page] = -7 if garbage else pool.table[groups[g], :m // pool.page]
    return pool


def attend(pool, rows, hq, groups, tokens, seed=1, pad=0, status=0, offsets=None, lengths=None, lse=True, q=None,
           lens_checked=None, scale=None):
    import torch

    from paper_2602_20217_gb300 import kv8
    d = pool.device(rows, lengths, pad, offsets)
    n, hd = pool.n_rows, pool.hd
    if q is None:
        q = np.random.default_rng(seed).standard_normal((n, hq, hd)) * 2
    qt = torch.tensor(q, dtype=torch.bfloat16, device="cuda")
    out = torch.full((n, hq, hd), 7.0, dtype=torch.bfloat16, device="cuda")
    sums = torch.full((n, hq), 7.0, device="cuda")
    shared = kv8.Shared8(torch.tensor(groups, dtype=torch.int32, device="cuda"),
                         torch.tensor(tokens, dtype=torch.int32, device="cuda"))
    work = d["cache"].attention_workspace(hq, len(pool.lens), n, shared=shared)
    work.fill_(0xff)
    scale = hd ** -0.5 if scale is None else scale
    d["cache"].attention(d["batch"], qt, scale=scale, out=out, lse=sums if lse else None, workspace=work, shared=shared)
    torch.cuda.synchronize()
    assert int(d["status"]) == status
    got, got_lse = out.double().cpu().numpy(), sums.double().cpu().numpy()
    if lse:
        check(pool, rows, qt.double().cpu().numpy(), got, got_lse, scale, lengths if lens_checked is None else lens_checked)
    end = int(pool.offsets[-1])
    assert np.all(got[end:] == 7) and np.all(got_lse[end:] == 7)
    return d, qt, out, sums, work, shared


def near(a, b, pool):
    """Each is within 2^-8 of itself (a bf16 rounding) and 2^-10 of the average of |v|, at most the largest, of the
    exact output: two of them lie within the sum of both."""
    v = max(float(np.abs(kv[1]).max()) for kv in pool.kv)
    a, b = a.double(), b.double()
    return bool(((a - b).abs() <= 2.0 ** -8 * (a.abs() + b.abs()) + 2 * 2.0 ** -10 * v).all())


def pool_of(groups, tokens, tails, hk, hd, page, seed=0, **kw):
    lens = [0] * groups[-1]
    for g, n in enumerate(tokens):
        for s in range(groups[g], groups[g + 1]):
            lens[s] = n // page * page + tails[s]
    return share(Pool(lens, hk, hd, page, seed).fill(**kw), groups, tokens)


@pytest.mark.parametrize("hq,hk,hd", [(8, 2, 64), (32, 8, 128), (12, 4, 128), (16, 1, 64), (64, 8, 128)])
@pytest.mark.parametrize("page", [16, 48, 64])
@pytest.mark.parametrize("seqs", [1, 2, 5])
def test_one_group(hq, hk, hd, page, seqs):
    tails = [1 + 13 * s for s in range(seqs)]
    attend(pool_of([0, seqs], [4 * page + 3], tails, hk, hd, page, seed=seqs), [1] * seqs, hq, [0, seqs],
           [4 * page + 3], pad=2)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("rows", [1, 3, 11, 40])
def test_groups_of_rows(hd, rows):
    """Several groups of uneven sizes; one row a sequence to units of many rows."""
    groups, tokens = [0, 3, 4, 12], [130, 64, 700]
    rng = np.random.default_rng(rows)
    tails = [rows + int(rng.integers(0, 150)) for _ in range(12)]
    each = [int(rng.integers(1, rows + 1)) for _ in range(12)]
    attend(pool_of(groups, tokens, tails, 2, hd, 32, seed=rows), each, 16, groups, tokens, pad=1)


@pytest.mark.parametrize("tokens", [16, 128, 1024, 9008])
def test_lengths_of_the_beginning(tokens):
    attend(pool_of([0, 20], [tokens], [1 + 7 * (s % 4) for s in range(20)], 2, 64, 16, seed=tokens), [1] * 20, 8,
           [0, 20], [tokens])


def test_sequences_without_a_group_without_rows_and_empty_groups():
    pool = Pool([100, 90, 120, 130, 64, 77], 2, 64, 16).fill()
    share(pool, [1, 1, 3, 5], [0, 64, 48])
    attend(pool, [2, 1, 1, 0, 3, 2], 8, [1, 1, 3, 5, 5], [48, 64, 48, 32], pad=1)


def test_nothing_in_common():
    attend(pool_of([0, 2, 3], [0, 0], [40, 50, 33], 2, 128, 16), [1, 2, 3], 8, [0, 2, 3], [15, 0])


def test_rows_within_the_beginning():
    """A group with a row among its common tokens shares only what is before that row."""
    groups, tokens = [0, 3], [320]
    pool = Pool([400, 100, 330], 2, 64, 32).fill()
    share(pool, groups, [96], garbage=False)         # the second sequence has 100 tokens: 97 before its rows
    attend(pool, [2, 3, 4], 8, groups, tokens)
    pool = Pool([400, 2, 330], 2, 64, 32).fill()     # and here none: a row at the very beginning
    attend(pool, [2, 2, 4], 8, groups, tokens)


def test_groups_that_are_none():
    """Offsets of groups that decrease or leave the batch: nothing is shared, and the batch is flagged."""
    for groups in ([0, 3, 2], [-1, 3, 3], [0, 1, 9]):
        attend(Pool([100, 90, 120], 2, 64, 16).fill(), [1, 1, 2], 8, groups, [64, 64], status=2)


def test_tokens_out_of_range():
    pool = share(Pool([100, 90], 2, 64, 16).fill(), [0, 2], [80])
    attend(pool, [1, 1], 8, [0, 2], [100000], status=2)
    attend(Pool([100, 90], 2, 64, 16).fill(), [1, 1], 8, [0, 2], [-5], status=2)


def test_offsets_that_decrease_write_nothing():
    import torch
    pool = share(Pool([100, 90, 70], 2, 64, 16).fill(), [0, 3], [48])
    d, q, out, lse, _, _ = attend(pool, [1, 1, 1], 8, [0, 3], [48], offsets=[0, 2, 1, 3], status=2, lse=False)
    assert bool((out == 7).all())


def test_bad_lengths():
    """Lengths below 0 or above the pages are taken as the nearest possible ones, and flagged."""
    pool = Pool([96, 96, 96], 2, 64, 16).fill()
    share(pool, [0, 2], [32], garbage=False)
    attend(pool, [1, 1, 1], 8, [0, 2, 3], [32, 0], lengths=[96, 500, 96], lens_checked=[96, 96, 96], status=2)
    # a length of -4 hides its row's tokens, and the group's: its rows see nothing
    attend(pool, [1, 1, 1], 8, [0, 2, 3], [32, 0], lengths=[96, -4, 96], lens_checked=[96, 0, 96], status=2)


def test_pages_outside_the_pool():
    """Their tokens are unseen by the whole group."""
    pool = pool_of([0, 3], [160], [20, 30, 40], 2, 64, 32)
    pool.table[0, 2] = 10000
    for s in range(3):
        pool.kv[s] = np.delete(pool.kv[s], range(64, 96), axis=1)
    lens = list(pool.lens)
    pool_lens, pool.lens = pool.lens, [n - 32 for n in lens]
    attend(pool, [1, 1, 1], 8, [0, 3], [160], lengths=lens, lens_checked=[n - 32 for n in lens], status=1)
    pool.lens = pool_lens


@pytest.mark.parametrize("rows", [1, 20])
def test_nan_in_either_part(rows):
    """A NaN value spoils its dim, a NaN key the row; in the common part for every row of the group."""
    for where, what in ((5, 1), (5, 0), (130, 1), (130, 0)):
        pool = Pool([128 + 40, 128 + 50, 60], 2, 64, 16, seed=rows).fill()
        rec = pool.block(0, where // 16)[1]
        at = (where % 16 // 8 * 4 + 2) * 128 + where % 8 * 16 + 1 if what == 0 else 16 * 64 + 33 * 16 + _v_byte(where % 16)
        rec[at] = 0x7f
        pool.kv[0][what, where, 1, 33] = math.nan
        share(pool, [0, 2, 3], [128, 0])
        attend(pool, [rows, rows, 3], 8, [0, 2, 3], [128, 0])


def _v_byte(t):
    return 4 * (t % 8 // 2) + 2 * (t // 8) + t % 2


@pytest.mark.parametrize("rows", [1, 9])
def test_far_scores(rows):
    """One part outweighs the other, either way: scores up to 12 |k|^2 scale = 12 * 64 * 16 * 0.003 = 37."""
    for loud in (0, 1):
        pool = pool_of([0, 4], [96], [30, 40, 50, 60], 2, 64, 16, seed=loud)
        q = np.random.default_rng(3).standard_normal((4 * rows, 8, 64)) * 0.3
        r = 0
        for s in range(4):
            k = pool.kv[s][0]
            far = k[:96] if loud == 0 else k[96:96 + 30 + 10 * s - rows]
            for i in range(rows):
                for h in range(8):
                    q[r, h] += 12 * far[(7 * r + h) % len(far), h // 4]
                r += 1
        attend(pool, [rows] * 4, 8, [0, 4], [96], q=q, scale=0.003)


def test_strides_of_queries_and_output():
    import torch
    pool = pool_of([0, 3], [64], [20, 30, 40], 2, 64, 16)
    d, q, out, lse, work, shared = attend(pool, [1, 2, 3], 8, [0, 3], [64])
    wide_q = torch.full((6, 9, 67), 5.0, dtype=torch.bfloat16, device="cuda")[:, 1:, 2:66]
    wide_q.copy_(q)
    got = torch.full((6, 10, 71), 3.0, dtype=torch.bfloat16, device="cuda")
    view = got[:, 2:, 1:65]
    d["cache"].attention(d["batch"], wide_q, out=view, workspace=work, shared=shared)
    assert torch.equal(view, out)
    got[:, 2:, 1:65] = 3.0
    assert bool((got == 3).all())


def test_same_as_the_plain_attention_of_the_same_batch():
    """Within the two calls' roundings, and bit for bit from call to call."""
    import torch
    pool = pool_of([0, 7], [1024], [11 * s + 1 for s in range(7)], 8, 128, 64)
    share(pool, [0, 7], [1024], garbage=False)
    d, q, out, lse, work, shared = attend(pool, [1] * 7, 32, [0, 7], [1024])
    plain = d["cache"].attention(d["batch"], q)
    assert near(plain, out, pool)
    again = torch.zeros_like(out)
    d["cache"].attention(d["batch"], q, out=again, workspace=work, shared=shared)
    assert torch.equal(again, out)


def test_graph_follows_the_groups_and_streams_have_their_own_workspaces():
    import torch

    from paper_2602_20217_gb300 import kv8
    pool = pool_of([0, 3, 6], [96, 64], [9, 20, 31, 42, 53, 64], 2, 64, 16)
    share(pool, [0, 3, 6], [96, 64], garbage=False)
    d, q, out, lse, work, shared = attend(pool, [1] * 6, 8, [0, 3, 6], [96, 64])
    want = out.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        d["cache"].attention(d["batch"], q, out=out, workspace=work, shared=shared)
    shared._keep[1].copy_(torch.tensor([32, 0], dtype=torch.int32))       # the same rows, less in common
    out.fill_(7)
    g.replay()
    assert near(want, out, pool) and bool((out != 7).any())
    shared._keep[1].copy_(torch.tensor([96, 64], dtype=torch.int32))
    g.replay()
    assert torch.equal(out, want)
    # two calls at once, each with what it allocates by itself
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = [d["cache"].attention(d["batch"], q, stream=streams[i % 2], shared=shared) for i in range(8)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_thousands_of_groups():
    """More groups than the preparation keeps in shared memory, of one and two sequences."""
    import torch

    from paper_2602_20217_gb300 import kv8
    n_groups, page = 5000, 16
    sizes = np.random.default_rng(0).integers(1, 3, n_groups)
    groups = np.concatenate(([0], np.cumsum(sizes)))
    n = int(groups[-1])
    cache = kv8.Cache8(n_groups + n, page, 1, 64)
    cache.data.random_(0, 100)
    cache.data.view(-1, 2080)[:, -32:-24] = torch.full((2,), 2.0 ** -5, device="cuda").view(torch.uint8)
    table = np.stack((np.repeat(np.arange(n_groups), sizes), n_groups + np.arange(n)), 1).astype(np.int32)
    i32 = dict(dtype=torch.int32, device="cuda")
    lens = torch.randint(17, 33, (n,), **i32)
    batch = kv8.Batch8(torch.tensor(table, device="cuda"), torch.arange(n + 1, **i32), lens, n, torch.zeros(1, **i32))
    shared = kv8.Shared8(torch.tensor(groups, **i32), torch.full((n_groups,), 16, **i32))
    q = torch.randn(n, 4, 64, device="cuda").to(torch.bfloat16)
    out = cache.attention(batch, q, shared=shared)
    plain = cache.attention(batch, q)
    assert int(batch._keep[3]) == 0
    v = 2.0 ** -5 * 448                              # the largest value that a code times the scale can be
    a, b = out.double(), plain.double()
    assert bool(((a - b).abs() <= 2.0 ** -8 * (a.abs() + b.abs()) + 2.0 ** -9 * v).all()) and bool((a != 0).any())


def test_refusals_of_the_python_face():
    import torch

    from paper_2602_20217_gb300 import kv8

    def i32(*v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")
    for bad in [(i32(0, 2).long(), i32(5)), (i32(0, 2), i32(5, 6)), (i32(0), i32()), (i32(0, 2).cpu(), i32(5)),
                (i32(0, 0, 2, 2)[::2], i32(5)), (i32(0, 2)[None], i32(5))]:
        with pytest.raises(ValueError):
            kv8.Shared8(*bad)
