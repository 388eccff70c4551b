"""Eviction from the 8-bit cache against its restatement: places, scores and
lengths are equal, and so are the new pages' bytes to an append of the kept
values; and a run of the operators around it, as a serving loop would make it.
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


def evict(pool, scores, keep, first=0, recent=0, new_pages=None, status=0, lengths=None, with_scores=True, spoil=None):
    """Evicts into spare pages of the pool and checks everything against the restatement."""
    import torch
    n_seqs, page, bpp = len(pool.lens), pool.page, pool.bpp
    lens = [min(max(x, 0), pool.ld * page) for x in (pool.lens if lengths is None else lengths)]
    ld = new_pages if new_pages is not None else max(1, max(-(-min(max(k, 0), n) // page) for k, n in zip(keep, lens)))
    used = set()
    for s in range(n_seqs):
        used |= set(pool.table[s, :pool.per[s]].tolist())
    free = [p for p in range(pool.n_pages) if p not in used]
    assert len(free) >= n_seqs * ld, (len(free), n_seqs, ld)
    table = np.array(free[:n_seqs * ld], np.int32).reshape(n_seqs, ld)
    if spoil is not None:
        table[spoil] = 10 ** 6
    d = pool.device([1] * n_seqs, lengths)
    room = ld * page
    old = np.full((n_seqs, pool.hk, pool.ld * page), np.nan, np.float32)
    old[:, :, :scores.shape[2]] = scores
    kept = torch.full((n_seqs, pool.hk, room), -9, dtype=torch.int32, device="cuda")
    new_scores = torch.full((n_seqs, pool.hk, room), 7.0, device="cuda") if with_scores else None
    new_lengths = torch.full((n_seqs,), -9, dtype=torch.int32, device="cuda")
    st = torch.tensor(old, device="cuda")
    before = d["data"].clone()
    d["cache"].evict(d["batch"], st, torch.tensor(keep, dtype=torch.int32, device="cuda"),
                     torch.tensor(table, device="cuda"), new_lengths, kept, new_scores=new_scores, first=first,
                     recent=recent)
    torch.cuda.synchronize()
    assert int(d["status"]) == status
    got_kept = kept.cpu().numpy()
    data = d["data"].cpu().numpy().reshape(pool.data.shape)
    want_data = before.cpu().numpy().reshape(pool.data.shape).copy()
    for s in range(n_seqs):
        n = O.stay(lens[s], keep[s], first, recent, room)[0]
        assert int(new_lengths[s]) == n
        for h in range(pool.hk):
            want = O.kept(old[s, h], lens[s], keep[s], first, recent, room)
            assert np.array_equal(got_kept[s, h, :n], want), (s, h)
            assert np.all(got_kept[s, h, n:] == -9)
            if with_scores:
                ns = new_scores[s, h].cpu().numpy()
                assert np.array_equal(ns[:n], old[s, h][want], equal_nan=True) and np.all(ns[n:] == 7)
            for b in range(-(-n // 16)):
                p = table[s, b // bpp]
                if p >= pool.n_pages:
                    continue
                at = want[16 * b:16 * b + 16]
                kv = [pool.token(s, t, h) if pool.table[s, t // page] < pool.n_pages else
                      (np.zeros(pool.hd), np.zeros(pool.hd)) for t in at]
                rec = K.pack_record(*K.append_block(None, 0, np.array([x[0] for x in kv]), np.array([x[1] for x in kv])))
                rec[-24:] = want_data[p, h, b % bpp, -24:]       # unused bytes
                want_data[p, h, b % bpp] = rec
    assert np.array_equal(data, want_data)
    return d, table, new_lengths, kept, new_scores


def scores_of(pool, seed=0, kind="heavy"):
    rng = np.random.default_rng(seed)
    shape = (len(pool.lens), pool.hk, max(pool.lens, default=1))
    x = np.exp(rng.standard_normal(shape) * 2)
    if kind == "ties":
        x = np.round(x)
    return x.astype(np.float32)


@pytest.mark.parametrize("hk,hd,page", [(2, 64, 16), (8, 128, 64), (1, 128, 48)])
@pytest.mark.parametrize("n,keep", [(1, 1), (2, 1), (17, 16), (100, 37), (129, 128), (1000, 100), (1025, 700)])
def test_one_sequence(hk, hd, page, n, keep):
    pool = Pool([n], hk, hd, page, seed=n, spare=20 + 1000 // page).fill()
    evict(pool, scores_of(pool, n), [keep], first=min(4, keep // 4), recent=keep // 3)


@pytest.mark.parametrize("kind", ["heavy", "ties"])
@pytest.mark.parametrize("first,recent", [(0, 0), (4, 0), (0, 32), (16, 50), (1000, 1000)])
def test_ragged_batch(kind, first, recent):
    pool = Pool([300, 5, 64, 700, 17, 1], 2, 64, 16, spare=300).fill()
    evict(pool, scores_of(pool, 3, kind), [100, 5, 3, 350, 16, 4], first, recent)


def test_orders_of_scores():
    """All equal, rising, falling, negative, both zeros, infinities and NaN, the smallest and largest numbers."""
    pool = Pool([500] * 8, 1, 64, 16, spare=120).fill()
    x = np.zeros((8, 1, 500), np.float32)
    x[1, 0] = np.arange(500)
    x[2, 0] = -np.arange(500)
    x[3, 0] = np.where(np.arange(500) % 2, -0.0, 0.0)
    x[4, 0] = np.random.default_rng(0).standard_normal(500)
    x[4, 0, [3, 77]], x[4, 0, [5, 300]], x[4, 0, 100:140] = math.inf, -math.inf, math.nan
    x[5, 0] = math.nan
    x[6, 0] = np.nextafter(np.float32(0), np.float32(1)) * np.arange(500)
    x[7, 0] = np.random.default_rng(1).choice([3.4e38, -3.4e38, 1e-45, 1.0], 500)
    evict(pool, x, [200] * 8, first=2, recent=3)


def test_all_stay_or_none():
    pool = Pool([100, 33], 2, 64, 16, spare=40).fill()
    evict(pool, scores_of(pool), [100, 500])
    evict(pool, scores_of(pool), [0, 0], new_pages=1)
    evict(pool, scores_of(pool), [0, 10], first=5, recent=5, with_scores=False)


def test_counts_out_of_range():
    pool = Pool([100, 90], 2, 64, 16, spare=40).fill()
    evict(pool, scores_of(pool), [-5, 20], new_pages=2, status=2)
    evict(pool, scores_of(pool), [60, 20], new_pages=2, status=2)            # room for 32
    evict(pool, scores_of(pool), [20, 20], lengths=[-1, 90], new_pages=2, status=2)


def test_pages_outside_the_pool():
    pool = Pool([100, 90], 2, 64, 16, spare=40).fill()
    pool.table[1, 2] = 10 ** 6                       # read as zeros
    evict(pool, scores_of(pool), [100, 60], status=1)
    pool = Pool([100, 90], 2, 64, 16, spare=40).fill()
    evict(pool, scores_of(pool), [60, 60], status=1, spoil=(0, 1))           # not written


def test_quiet_and_loud_blocks():
    """Blocks far apart in scale meet in one: codes that become subnormal round as an append would; NaN stays."""
    pool = Pool([400], 2, 64, 16, spare=30).fill(spread=8.0)
    pool.block(0, 5)[0][3 * 16] = 0x7f
    pool.block(0, 6)[1][16 * 64 + 7] = 0xff
    evict(pool, scores_of(pool, 1), [150])
    evict(pool, scores_of(pool, 2, "ties"), [390])


def test_keeps_its_pages():
    """A sequence that keeps all of its tokens may keep its pages; another is evicted in the same call."""
    import torch
    pool = Pool([50, 80], 2, 64, 16, spare=10).fill()
    d = pool.device([1, 1])
    table = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    table[0, :4] = d["table"][0, :4]
    free = [p for p in range(pool.n_pages) if p not in set(pool.table[0, :4]) | set(pool.table[1, :5])]
    table[1, :2] = torch.tensor(free[:2], dtype=torch.int32)
    x = torch.rand(2, 2, pool.ld * 16, device="cuda")
    kept = torch.zeros(2, 2, 64, dtype=torch.int32, device="cuda")
    lengths = torch.zeros(2, dtype=torch.int32, device="cuda")
    before = d["data"].clone().view(pool.n_pages, -1)
    d["cache"].evict(d["batch"], x, torch.tensor([64, 20], dtype=torch.int32, device="cuda"), table, lengths, kept)
    after = d["data"].view(pool.n_pages, -1)
    torch.cuda.synchronize()
    assert lengths.tolist() == [50, 20] and int(d["status"]) == 0
    changed = (before != after).any(1).nonzero().flatten().tolist()
    assert sorted(changed) == sorted(free[:2])


def test_many_sequences_and_a_graph():
    import torch
    rng = np.random.default_rng(0)
    lens = [int(x) for x in rng.integers(1, 120, 90)]
    pool = Pool(lens, 2, 64, 16, spare=90 * 4).fill()
    x = scores_of(pool, 5)
    d, table, lengths, kept, new_scores = evict(pool, x, [50] * 90, 1, 5, new_pages=4)
    st = torch.zeros(90, 2, pool.ld * 16, device="cuda")
    st[:, :, :x.shape[2]] = torch.tensor(x)
    keep = torch.full((90,), 50, dtype=torch.int32, device="cuda")
    table = torch.tensor(table, device="cuda")
    again, n = torch.full_like(kept, -9), torch.zeros_like(lengths)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        d["cache"].evict(d["batch"], st, keep, table, n, again, first=1, recent=5)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(again, kept) and torch.equal(n, lengths)
    keep.fill_(3)
    again.fill_(-9)
    g.replay()
    torch.cuda.synchronize()
    assert n.tolist() == [min(3, m) for m in lens]
    assert all(int(again[s, 0, min(3, m) - 1]) == m - 1 for s, m in enumerate(lens))


@pytest.mark.parametrize("n", [40000, 131072])
def test_long_sequence(n):
    """Selection alone over long contexts, with ties: the pages are zeros."""
    import torch

    from paper_2602_20217_gb300 import kv8
    page, pages = 256, n // 256 + 1
    cache = kv8.Cache8(2 * pages, page, 2, 64)
    cache.data.zero_()
    i32 = dict(dtype=torch.int32, device="cuda")
    table = torch.arange(pages, **i32)[None].contiguous()
    batch = kv8.Batch8(table, torch.tensor([0, 1], **i32), torch.tensor([n], **i32), 1)
    x = torch.round(torch.exp(torch.randn(1, 2, pages * page, device="cuda") * 3) * 4)
    kept, lengths = torch.zeros(1, 2, pages * page, **i32), torch.zeros(1, **i32)
    for keep in (1, n // 10, n // 2, n - 1):
        cache.evict(batch, x, torch.tensor([keep], **i32), table + pages, lengths, kept, first=3, recent=100)
        for h in range(2):
            assert np.array_equal(kept[0, h, :keep].cpu().numpy(),
                                  O.kept(x[0, h].cpu().numpy(), n, keep, 3, 100, 1 << 30)), keep


def test_more_sequences_than_a_grid_has():
    """70000 sequences of at most 16 tokens, a page each."""
    import torch

    from paper_2602_20217_gb300 import kv8
    n = 70000
    cache = kv8.Cache8(2 * n, 16, 1, 64)
    cache.data.random_(0, 100)
    rec = cache.data.view(2 * n, 2080)
    rec[:, -32:-24] = torch.ones(2, device="cuda").view(torch.uint8)
    i32 = dict(dtype=torch.int32, device="cuda")
    table = torch.arange(n, **i32)[:, None].contiguous()
    lens = torch.randint(1, 17, (n,), **i32)
    batch = kv8.Batch8(table, torch.arange(n + 1, **i32), lens, n, torch.zeros(1, **i32))
    x = torch.rand(n, 1, 16, device="cuda")
    kept, lengths = torch.full((n, 1, 16), -1, **i32), torch.zeros(n, **i32)
    cache.evict(batch, x, torch.full((n,), 9, **i32), table + n, lengths, kept, recent=2)
    assert torch.equal(lengths, lens.clamp(max=9)) and int(batch._keep[3]) == 0
    t = torch.arange(16, device="cuda")
    key = torch.where(t >= lens[:, None] - 2, 2.0, x[:, 0]).masked_fill(t >= lens[:, None], -1.0)
    want = torch.where(t[:9] < lengths[:, None], key.topk(9).indices, 99).sort(1).values
    assert torch.equal(kept[:, 0, :9].long().masked_fill(t[:9] >= lengths[:, None], 99), want)
    k, v = (torch.zeros(n * 16, 1, 64, device="cuda") for _ in range(2))
    offs = torch.cat((torch.zeros(1, **i32), lens.cumsum(0).int()))
    cache.read(kv8.Batch8(table, offs, lens, n * 16), k, v)
    k2, v2 = torch.zeros_like(k), torch.zeros_like(v)
    offs2 = torch.cat((torch.zeros(1, **i32), lengths.cumsum(0).int()))
    cache.read(kv8.Batch8((table + n).contiguous(), offs2, lengths, n * 16), k2, v2)
    seq = torch.repeat_interleave(torch.arange(n, device="cuda"), lengths.long())
    at = torch.arange(len(seq), device="cuda") - offs2.long()[seq]
    src = offs.long()[seq] + kept[seq, 0, at].long()
    assert torch.equal(k2[:len(seq)], k[src]) and torch.equal(v2[:len(seq)], v[src])


def test_append_goes_on_at_the_old_positions():
    """After an eviction rows are rotated by their positions, and stored at their places."""
    import torch

    from paper_2602_20217_gb300 import kv8
    page, hk, hd, hq = 16, 2, 64, 4
    rng = np.random.default_rng(0)
    i32 = dict(dtype=torch.int32, device="cuda")
    angle = rng.uniform(0, 6, (500, hd // 2))
    rope = torch.tensor(np.stack((np.cos(angle), np.sin(angle)), -1), dtype=torch.float32, device="cuda")
    rows = torch.tensor(rng.standard_normal((2, 3, hk, hd)), dtype=torch.bfloat16, device="cuda")
    q = torch.tensor(rng.standard_normal((3, hq, hd)), dtype=torch.bfloat16, device="cuda")
    got = {}
    for name, lens, shift, offs in (("evicted", [25, 33], [100, 400], [0, 2, 3]), ("whole", [125, 433], None, [0, 2, 3])):
        cache = kv8.Cache8(80, page, hk, hd)
        cache.data.zero_()
        table = torch.arange(2 * 30, **i32).view(2, 30).contiguous()
        batch = kv8.Batch8(table, torch.tensor(offs, **i32), torch.tensor(lens, **i32), 3, torch.zeros(1, **i32))
        out = torch.zeros(3, hq, hd, dtype=torch.bfloat16, device="cuda")
        kw = {} if shift is None else {"shift": torch.tensor(shift, **i32)}
        cache.append(batch, rows[0], rows[1], rope=rope, q=q, q_out=out, **kw)
        k, v = torch.zeros(3, hk, hd, device="cuda"), torch.zeros(3, hk, hd, device="cuda")
        cache.read(batch, k, v)
        got[name] = (out, k, v, batch._keep[3].item())
    assert got["evicted"][3] == got["whole"][3] == 0
    assert all(torch.equal(a, b) for a, b in zip(got["evicted"][:3], got["whole"][:3]))
    # positions outside the table are flagged and stored as zeros
    for shift in ([-30, 0], [500, 0], [2 ** 31 - 1, -(2 ** 31)]):
        batch._keep[3].zero_()
        batch._keep[2].copy_(torch.tensor([25, 33]))
        cache.append(batch, rows[0], rows[1], rope=rope, q=q, q_out=out, shift=torch.tensor(shift, **i32))
        cache.read(batch, k, v)
        assert int(batch._keep[3]) == 4 and bool((out[:2] == 0).all()) and bool((k[:2] == 0).all())


def test_a_serving_loop():
    """A prompt is appended and attended, its tokens' weights taken, the cache cut, four samples share what stays, and
    the sampled tokens are scored: each step is that of the restatements on what the cache holds."""
    import torch

    from oracle import logprobs as L
    from paper_2602_20217_gb300 import kv8, logprobs
    from test_gpu_logprobs import EPS, bounds
    hq, hk, hd, page, n, keep = 8, 2, 64, 16, 150, 64
    i32 = dict(dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(7)

    def bf(*shape):
        return torch.tensor(rng.standard_normal(shape), dtype=torch.bfloat16, device="cuda")
    cache = kv8.Cache8(40, page, hk, hd)
    cache.data.fill_(0x7f)
    status = torch.zeros(1, **i32)
    prompt = kv8.Batch8(torch.arange(10, **i32)[None].contiguous(), torch.tensor([0, n], **i32), torch.tensor([n], **i32),
                        n, status)
    q = bf(n, hq, hd) * 2
    cache.append(prompt, bf(n, hk, hd), bf(n, hk, hd))
    lse = torch.zeros(n, hq, device="cuda")
    cache.attention(prompt, q, lse=lse)
    scores = torch.zeros(1, hk, 160, device="cuda")
    cache.attention_weights(prompt, q, lse, scores)
    assert float((scores.sum() - n * hq).abs()) < 1e-3 * n * hq          # every row gives weight 1
    small = torch.arange(10, 14, **i32)[None].contiguous()
    lengths, kept = torch.zeros(1, **i32), torch.zeros(1, hk, 64, **i32)
    less = torch.zeros(1, hk, 64, device="cuda")
    cache.evict(prompt, scores, torch.tensor([keep], **i32), small, lengths, kept, new_scores=less, first=2, recent=16)
    for h in range(hk):
        want = O.kept(scores[0, h].cpu().numpy(), n, keep, 2, 16, 64)
        assert np.array_equal(kept[0, h].cpu().numpy(), want)
        assert torch.equal(less[0, h], scores[0, h][kept[0, h].long()])
    # four samples, a token each, behind what stays
    tables = torch.cat((small.expand(4, 4), torch.arange(20, 24, **i32)[:, None]), 1).contiguous()
    samples = kv8.Batch8(tables, torch.arange(5, **i32), torch.full((4,), keep + 1, **i32), 4, status)
    group = kv8.Shared8(torch.tensor([0, 4], **i32), torch.tensor([keep], **i32))
    q1, k1, v1 = bf(4, hq, hd) * 2, bf(4, hk, hd), bf(4, hk, hd)
    cache.append(samples, k1, v1, shift=torch.full((4,), n - keep, **i32))
    out = cache.attention(samples, q1, shared=group)
    everything = kv8.Batch8(tables, torch.arange(5, **i32) * (keep + 1), torch.full((4,), keep + 1, **i32), 4 * (keep + 1))
    k, v = (torch.zeros(4 * (keep + 1), hk, hd, device="cuda") for _ in range(2))
    cache.read(everything, k, v)
    for s in range(4):
        rows = slice(s * (keep + 1), (s + 1) * (keep + 1))
        ref, _, mag = K.attention(q1[s:s + 1].double().cpu().numpy(), k[rows].double().cpu().numpy(),
                                  v[rows].double().cpu().numpy(), hd ** -0.5)
        err = np.abs(out[s:s + 1].double().cpu().numpy() - ref)
        assert np.all(err <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -10 * mag)
    head = torch.tensor(rng.standard_normal((1000, hq * hd)), dtype=torch.float32, device="cuda")
    logits = out.float().view(4, -1) @ head.T
    tokens = logits.argmax(1).int()
    got = logprobs.token_logprobs(logits, tokens, n_top=3)
    for s in range(4):
        x = logits[s].double().cpu().numpy()
        lp, _, ids, _ = L.row(x, [int(tokens[s])], 3, 1.0)
        assert got.top_ids[s].tolist() == list(ids)
        assert abs(float(got.logprobs[s, 0]) - lp[0]) <= bounds(x, 1.0)[0] + 3 * EPS * abs(lp[0])
    assert int(status) == 0
