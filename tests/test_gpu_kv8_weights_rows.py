"""More query rows than cached tokens in the received weights' kernel of many rows, with the additions of its own order.

That kernel takes chunks of whole tokens, up to 128 queries.  A thread adds the
64 of half a chunk in four sums of 16, joins these (2), adds the chunk's to the
run's (at most as many as there are chunks, runs included, and one), joins the
halves (1) and adds the decayed score (1): 16 + 2 + chunks + 1 + 1 + 1.
"""
import numpy as np
import pytest

from helpers import need_gpu
from oracle import kv8_evict as O
from test_gpu_kv8 import Pool
from test_gpu_kv8_weights import receive

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()


def within_the_order(pool, rows, hq, lens=None, decay=0.5, seed=1, **kw):
    """receive(), and then the same with the bound above."""
    n, G, hd = sum(rows), hq // pool.hk, pool.hd
    rng = np.random.default_rng(seed + 100)
    q = rng.standard_normal((n, hq, hd)) * 2
    lse = np.float32(rng.uniform(3.0, 6.0, (n, hq)))
    assert G * n >= 33 * len(rows)                   # the kernel of many rows
    _, qt, out = receive(pool, rows, hq, decay=decay, seed=seed, q=q, lse=lse, **kw)
    old = np.float32(np.random.default_rng(seed).exponential(1.0, (len(rows), pool.hk, pool.ld * pool.page)))
    q, got, o = qt.double().cpu().numpy(), out.double().cpu().numpy(), 0
    for s, r in enumerate(rows):
        m = pool.lens[s]
        ref, off = O.weights(q[o:o + r], pool.kv[s][0], lse[o:o + r].astype(np.float64), hd ** -0.5, r)
        o += r
        older = max(m - r, 0)
        ref[:, :older] += decay * old[s][:, :older].astype(np.float64)
        chunks = -(-r // (128 // G))
        bound = off + 2.0 ** -24 * (21 + chunks) * np.abs(ref) + r * G * 2.0 ** -125
        assert np.all(np.abs(got[s][:, :m] - ref) <= bound), s


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lens,rows", [([10, 600, 513], [100, 700, 514]), ([1], [40]), ([5, 1030], [513, 1029]),
                                       ([511, 512, 513], [1100, 1100, 1100])])
def test_rows_before_the_first_token(hd, lens, rows):
    """Chunks wholly before position 0, across it and behind it, with one and several units of 512 keys."""
    within_the_order(Pool(lens, 2, hd, 16, seed=len(lens)).fill(), rows, 8)


def test_no_tokens_and_rows_before_the_first_one():
    within_the_order(Pool([0, 30, 700], 2, 64, 32).fill(), [50, 60, 90], 6)


@pytest.mark.parametrize("group", [3, 5, 64])
def test_groups_and_rows_before_the_first_token(group):
    within_the_order(Pool([20, 530], 1, 64, 16).fill(), [90, 600], group)


def test_a_batch_of_few_rows_each_needs_no_workspace():
    """However many sequences there are; a batch of many rows each is refused one that is too small."""
    import torch

    from paper_2602_20217_gb300 import knapspec as ks
    pool = Pool([40 + 3 * s for s in range(24)], 2, 64, 16).fill()
    d = pool.device([1] * 24)
    assert d["cache"].weights_workspace(8, 24).numel() > 0       # the same rows of one sequence do
    q, lse = torch.randn(24, 8, 64, device="cuda").to(torch.bfloat16), torch.full((24, 8), 4.0, device="cuda")
    old = torch.rand(24, 2, pool.ld * 16, device="cuda")
    want = d["cache"].attention_weights(d["batch"], q, lse, old, out=torch.zeros_like(old))
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    got = d["cache"].attention_weights(d["batch"], q, lse, old, out=torch.zeros_like(old), workspace=none)
    torch.cuda.synchronize()
    assert int(d["status"]) == 0 and torch.equal(got, want)
    pool = Pool([40], 2, 64, 16).fill()
    d = pool.device([24])
    with pytest.raises(ks.KsError):
        d["cache"].attention_weights(d["batch"], q, lse, old[:1], out=torch.zeros_like(old[:1]), workspace=none)
