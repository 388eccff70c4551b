"""The limits that the 8-bit cache attention states for what it holds in fewer
than 32 bits: inside them the tolerances of test_gpu_kv8 hold."""
import numpy as np
import pytest

from helpers import need_gpu
from test_gpu_kv8 import Pool, attend
from test_gpu_kv8_many_rows import put

pytestmark = pytest.mark.gpu

HQ = 4
# rows a sequence and sequences: units of 8, 16 and, on tcgen05, 20, 48 and 128 query rows; so many that a run of
# tiles holds several of a sequence's, the loud ones and the quiet ones
BATCHES = [(1, 300), (4, 300), (5, 200), (12, 100), (45, 40)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()


@pytest.mark.parametrize("rows,seqs", BATCHES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("ratio", [0, -13, -20, -26])
def test_quiet_values_behind_loud_ones(rows, seqs, hd, ratio):
    """The weight lies on blocks whose values are 2^ratio of those before them, spread by at most 2^-2: weight times
    relative scale is 2^-28 and more.  The loud blocks' weight is below 2^-100."""
    rng = np.random.default_rng(rows + hd)
    n, loud = 512, 160
    u = rng.choice([-1.0, 1.0], hd)                  # keys of codes 1 and 1.125, exact
    k = u * (1 + 0.125 * (rng.random((n, hd)) < 0.1)) * np.where(np.arange(n) < loud, -1, 1)[:, None]
    v = rng.standard_normal((n, hd))
    v[:loud] *= 2.0 ** -ratio
    pool = Pool([n], 1, hd, 64, seed=40).fill()
    put(pool, 0, k, v)
    q = u * 36 / hd
    scores = pool.kv[0][0, :, 0] @ q
    assert scores[loud:].max() - scores[loud:].min() < 2 * np.log(2) and scores[loud:].min() - scores[:loud].max() > 70
    pool.lens, pool.kv = [n] * seqs, pool.kv * seqs
    pool.table = np.repeat(pool.table, seqs, 0)
    attend(pool, [rows] * seqs, HQ, q=np.broadcast_to(q, (rows * seqs, HQ, hd)), scale=1.0)


@pytest.mark.parametrize("rows,seqs", [(r, 1) for r, _ in BATCHES])
@pytest.mark.parametrize("top", [1.0, 1.75, 1.7578125, 1.9921875])
def test_small_elements_of_a_query(rows, seqs, top):
    """Elements of 2^-9 of the row's largest, which meets keys of zero there: the scores are the small ones' alone.
    At 1.7578125 the row's scale is the next power of two."""
    rng = np.random.default_rng(rows)
    hd, n = 64, 400
    k = rng.standard_normal((n, hd))
    k[:, 0] = 0
    q = rng.uniform(1, 2, (rows, HQ, hd)) * rng.choice([-1, 1], (rows, HQ, hd)) * top * 2.0 ** -9
    q[:, :, 0] = top
    pool = Pool([n], 1, hd, 64, seed=41).fill()
    put(pool, 0, k, rng.standard_normal((n, hd)))
    attend(pool, [rows], HQ, q=q, scale=128.0)
