"""The 8-bit cache attention where a CTA's run of tiles holds several of one
sequence: many sequences over the same pages, with the tolerances and inputs of
test_gpu_kv8.  A single short sequence is cut to one tile a CTA, so what moves
from tile to tile (references, value scales, marks of NaN) needs these."""
import math

import numpy as np
import pytest

from helpers import need_gpu
from oracle import kv8 as O
from test_gpu_kv8 import Pool, attend
from test_gpu_kv8_many_rows import mark, put

pytestmark = pytest.mark.gpu

HQ, N = 4, 900
# rows a sequence and sequences: units of 8, 16 and, on tcgen05, 20, 48, 128 and 180 (two units) query rows
BATCHES = [(1, 400), (4, 300), (5, 120), (12, 60), (32, 40), (45, 30)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()


def together(pool, rows, seqs, q, **more):
    pool.lens, pool.kv, pool.table = pool.lens * seqs, pool.kv * seqs, np.repeat(pool.table, seqs, 0)
    return attend(pool, [rows] * seqs, HQ, q=np.tile(q, (seqs, 1, 1)), **more)


@pytest.mark.parametrize("rows,seqs", BATCHES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("shape", ["rising", "steps", "falling", "late peak", "alternating"])
def test_scores_that_move(rows, seqs, hd, shape):
    t = np.arange(N)
    x = {"rising": -30 + 60 * t / N, "falling": 30 - 60 * t / N,
         "steps": 12.0 * ((t > 130).astype(int) + (t > 200) + (t > 210) + (t > 500)) - 20,
         "late peak": np.where(t == N - rows - 40, 30.0, -10.0),
         "alternating": np.where(t // 37 % 2, 20.0, -20.0) * (t / N)}[shape]
    rng = np.random.default_rng(rows)
    u = rng.standard_normal(hd)
    u /= np.linalg.norm(u)
    pool = Pool([N], 1, hd, 64, seed=1).fill()
    put(pool, 0, x[:, None] * u + 0.1 * rng.standard_normal((N, hd)), rng.standard_normal((N, hd)))
    q = u + 0.02 * rng.standard_normal((rows, HQ, hd))
    q[::3] *= 0.5                                    # rows that are raised at other keys
    together(pool, rows, seqs, q, scale=1.0)


@pytest.mark.parametrize("rows,seqs", BATCHES)
@pytest.mark.parametrize("hd", [64, 128])
def test_blocks_of_far_scales(rows, seqs, hd):
    pool = Pool([N], 1, hd, 64, seed=2).fill(spread=0)
    rng = np.random.default_rng(rows)
    for b in range(N // 16 + 1):
        f = 2.0 ** rng.integers(-12, 13) if b % 7 else 0.0
        kc, vc, ks, vs = O.unpack_record(pool.block(0, b)[0])
        vs = vs * f if f else 2.0 ** -126
        if not f:
            vc = vc & 0x80
            vc[N - 16 * b:] = 0xff
        pool.block(0, b)[0] = O.pack_record(kc, vc, ks, vs)
        last = min(16, N - 16 * b)
        pool.kv[0][1, 16 * b:16 * b + last, 0] = O.VALUES[vc[:last]] * vs
    together(pool, rows, seqs, rng.standard_normal((rows, HQ, hd)) * 2)


@pytest.mark.parametrize("rows,seqs", BATCHES)
def test_nan_tokens_and_missing_pages(rows, seqs):
    """Marks of one segment do not reach the next one of the CTA: every other sequence sees none."""
    import torch
    rng = np.random.default_rng(rows)
    clean, dirty = Pool([N], 1, 64, 64, seed=3).fill(), Pool([N], 1, 64, 64, seed=3).fill()
    mark(dirty, N - 1, 9, 1)
    mark(dirty, 300, 5, 1)
    if rows > 2:
        mark(dirty, N - rows + 2, 7, 1)
        mark(dirty, N - 2, 3, 0)
    pool = Pool([N] * seqs, 1, 64, 64, seed=4)
    pages = clean.per[0]
    pool.n_pages = 2 * pages
    pool.data = np.concatenate((clean.data[clean.table[0]], dirty.data[dirty.table[0]]))
    pool.table = np.stack([np.arange(pages) + pages * (s % 3 == 1) for s in range(seqs)]).astype(np.int32)
    pool.kv = [dirty.kv[0] if s % 3 == 1 else clean.kv[0] for s in range(seqs)]
    q = np.tile(rng.standard_normal((rows, HQ, 64)) * 2, (seqs, 1, 1))
    _, _, out, _, _ = attend(pool, [rows] * seqs, HQ, q=q)
    out = out.view(seqs, rows, HQ, 64)
    plain = [s for s in range(seqs) if s % 3 != 1]
    assert bool(torch.isfinite(out[plain].float()).all())
    # every other sequence lacks a page: its tokens are not seen
    pool.table[1::2, 5] = -1
    d = pool.device([rows] * seqs)
    qt = torch.tensor(q, dtype=torch.bfloat16, device="cuda")
    got = d["cache"].attention(d["batch"], qt).view(seqs, rows, HQ, 64)
    torch.cuda.synchronize()
    assert int(d["status"]) == 1
    seen = np.r_[0:320, 384:N]
    ref, _, mag = O.attention(qt[:rows].double().cpu().numpy(), *(clean.kv[0][i, seen] for i in (0, 1)), 64 ** -0.5)
    for s in plain:
        if s % 2:
            assert np.all(np.abs(got[s].double().cpu().numpy() - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -10 * mag)
        else:
            assert np.all(np.abs((got[s] - out[s]).double().cpu().numpy()) <=
                          2.0 ** -7 * np.abs(out[s].double().cpu().numpy()) + 2.0 ** -9 * mag + math.ulp(0))
