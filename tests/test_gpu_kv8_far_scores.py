"""The 8-bit cache attention at scores far beyond what fp32 resolves to a unit
(finite queries and keys of some 10^4, a large scale): which key is largest is
all that matters there, and every loop has to end.

Tolerances.  A score is off by at most
    2^-17 max|q| sum|k|    (queries in two e4m3 codes: an element is off by 2^-10
                            where the row's largest is above 224)
  + 2^-16 sum|q k|         (128 products added in fp32)
  + 2^-22 |q k|            (two products with the scales)
times the scale.  Rows whose two largest scores lie closer than twice that and
40 are left out; the others' output is the value of the largest one, e^-40
being nothing.  lse: the same bound.
"""
import numpy as np
import pytest

from helpers import need_gpu
from oracle import kv8 as O
from test_gpu_kv8 import Pool
from test_gpu_kv8_many_rows import put

pytestmark = pytest.mark.gpu

HQ, HD, N = 4, 64, 700
ROWS = [1, 4, 5, 12, 45]        # units of 8, 16 and, on tcgen05, 20, 48 and 128 query rows


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()


def run(pool, rows, q, scale):
    import torch
    d = pool.device([rows])
    qt = torch.tensor(q, dtype=torch.bfloat16, device="cuda")
    out = torch.full((rows, HQ, HD), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((rows, HQ), 7.0, device="cuda")
    d["cache"].attention(d["batch"], qt, scale=scale, out=out, lse=lse)
    torch.cuda.synchronize()
    assert int(d["status"]) == 0
    return qt.double().cpu().numpy(), out.double().cpu().numpy(), lse.double().cpu().numpy()


def inputs(rows, exponent, scale, order):
    """Scores with a standard deviation of 2^exponent (base 2)."""
    rng = np.random.default_rng(rows + exponent)
    std = 2.0 ** ((exponent - 3.5) / 2) / scale ** 0.5
    k, v = rng.standard_normal((2, N, HD))
    q = rng.standard_normal((rows, HQ, HD))
    if order != "mixed":
        u = rng.standard_normal(HD)
        k = k[np.argsort(k @ u * (1 if order == "rising" else -1))]
        q = u + 0.3 * q
    pool = Pool([N], 1, HD, 64, seed=1).fill()
    put(pool, 0, k * std, v)
    return pool, q * std


def expected(pool, rows, q, scale):
    """(rows that can be told, value of the largest score, lse, its bound)"""
    k, v = pool.kv[0][0, :, 0], pool.kv[0][1, :, 0]
    told, out, lse = np.zeros((rows, HQ), bool), np.zeros((rows, HQ, HD)), np.zeros((rows, HQ))
    bound = np.zeros((rows, HQ))
    for i in range(rows):
        seen = k[:N - rows + i + 1]
        for h in range(HQ):
            x = q[i, h]
            s = seen @ x * scale
            err = abs(scale) * (2.0 ** -17 * np.abs(x).max() * np.abs(seen).sum(-1) +
                                2.0 ** -16 * np.abs(seen) @ np.abs(x)) + 2.0 ** -22 * np.abs(s)
            a, b = np.argsort(s)[:-3:-1]
            told[i, h] = s[a] - s[b] > 2 * err.max() + 40
            out[i, h], lse[i, h], bound[i, h] = v[a], s[a], err.max() + 2e-4
    return told, out, lse, bound


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("order", ["mixed", "rising", "falling"])
@pytest.mark.parametrize("exponent", [20, 21, 24, 28, 30, 36, 60, 100])
def test_the_largest_score_wins(rows, order, exponent):
    pool, q = inputs(rows, exponent, 1.0, order)
    q, got, got_lse = run(pool, rows, q, 1.0)
    told, out, lse, bound = expected(pool, rows, q, 1.0)
    assert told.mean() >= 0.75
    assert np.isfinite(got).all() and np.isfinite(got_lse).all()
    assert np.all(np.abs(got - out)[told] <= 2.0 ** -8 * np.abs(out)[told] + 2.0 ** -10 * np.abs(out)[told])
    assert np.all(np.abs(got_lse - lse)[told] <= bound[told])


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("scale", [2.0 ** 30, -2.0 ** 30])
def test_a_far_scale(rows, scale):
    pool, q = inputs(rows, 4, 1.0, "mixed")
    q, got, got_lse = run(pool, rows, q, scale)
    told, out, lse, bound = expected(pool, rows, q, scale)
    assert told.mean() >= 0.75
    assert np.isfinite(got).all()
    assert np.all(np.abs(got - out)[told] <= (2.0 ** -8 + 2.0 ** -10) * np.abs(out)[told])
    assert np.all(np.abs(got_lse - lse)[told] <= bound[told])


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("exponent", [22, 28, 40])
def test_equal_far_scores_share_the_weight(rows, exponent):
    """One key over and over: the mean of the values that a row sees."""
    rng = np.random.default_rng(exponent)
    std = 2.0 ** ((exponent - 3) / 2)
    k = np.broadcast_to(rng.standard_normal(HD) * std, (N, HD))
    v = rng.standard_normal((N, HD))
    pool = Pool([N], 1, HD, 64, seed=2).fill()
    put(pool, 0, k, v)
    _, got, _ = run(pool, rows, rng.standard_normal((rows, HQ, HD)) * std, 1.0)
    for i in range(rows):
        seen = pool.kv[0][1, :N - rows + i + 1, 0]
        ref, mag = seen.mean(0), np.abs(seen).mean(0)
        assert np.all(np.abs(got[i] - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -10 * mag)


@pytest.mark.parametrize("rows,seqs", [(1, 300), (4, 300), (5, 200), (12, 100), (45, 40)])
@pytest.mark.parametrize("order", ["mixed", "rising", "falling"])
@pytest.mark.parametrize("exponent", [22, 28, 60])
def test_far_scores_in_runs_of_many_tiles(rows, seqs, order, exponent):
    """So many sequences of the same pages that a CTA's run holds several tiles of one: raises move what is summed."""
    pool, q = inputs(rows, exponent, 1.0, order)
    pool.lens, pool.kv, pool.table = [N] * seqs, pool.kv * seqs, np.repeat(pool.table, seqs, 0)
    import torch
    d = pool.device([rows] * seqs)
    qt = torch.tensor(np.tile(q, (seqs, 1, 1)), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(rows * seqs, HQ, device="cuda")
    got = d["cache"].attention(d["batch"], qt, scale=1.0, lse=lse)
    torch.cuda.synchronize()
    assert int(d["status"]) == 0
    told, out, want_lse, bound = expected(pool, rows, qt[:rows].double().cpu().numpy(), 1.0)
    assert told.mean() >= 0.75
    got = got.double().cpu().numpy().reshape(seqs, rows, HQ, HD)
    lse = lse.double().cpu().numpy().reshape(seqs, rows, HQ)
    assert np.isfinite(got).all()
    assert np.all(np.abs(got - out)[:, told] <= (2.0 ** -8 + 2.0 ** -10) * np.abs(out)[told])
    assert np.all(np.abs(lse - want_lse)[:, told] <= bound[told])
