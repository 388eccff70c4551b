"""Token log probabilities on the GPU against the fp64 restatement (oracle/logprobs.py).

Tolerances.  With d = x - max (one rounding) and the factor log2(e) / T (two
roundings and the constant's), an exponent is off by at most 4 * 2^-24 of
itself and the exponential by 2^-22 more; a lane adds up to V / 32 terms where
one warp has the row (V / 512 with sixteen) and 5 + 16 + 8 sums follow, each
addition off by at most 2^-24.  So the sum beside the largest logit is off by
  rel = 2^-22 + 4 * 2^-24 * D + (V / 32 + 29) * 2^-24,
D the average of |d| / T under that sum; log Z by rel * tail / Z and its own
roundings (one more where several logits are the largest).  A log probability adds three roundings of its size.  The entropy adds
the second sum's relative error, twice rel, and the roundings of its terms.
Exponentials below 2^-126, the smallest normal number, are zeros: each loses at
most 2^-126 (2^-125 at its border), and 88 times that in the entropy, whose
terms are exponentials times |d| / T <= 126 log 2.
Ids are whole numbers and equal; ranks go by the logits themselves.
"""
import math

import numpy as np
import pytest

from helpers import need_gpu
from oracle import logprobs as O

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()


def bounds(x, T):
    """(bound of log Z, of the entropy) of a finite row."""
    z = (x - x.max()) / T
    e = np.exp(z)
    n = int((x == x.max()).sum())
    e[x == x.max()] = 0.0                            # not by a difference: the tail may be far below 1
    tail = e.sum()
    D = (e * np.where(e > 0, -z, 0.0)).sum() / max(tail, 1e-300)
    lost = int(((e > 0) & (e < 2.0 ** -125)).sum()) * 2.0 ** -125
    rel = 2.0 ** -22 + 4 * EPS * D + (len(x) / 32 + 29) * EPS
    Z = tail + n
    log_1 = math.log1p(tail) if n == 1 else math.log(Z)
    log_z = rel * tail / Z + 2 * EPS * (log_1 + (n > 1)) + lost + 1e-37
    mean = D * tail / Z
    return log_z, log_z + 3 * rel * mean + 4 * EPS * (mean + log_1) + 90 * lost + 1e-37


def check(logits, tokens, n_top, T, got):
    lp, h, ids, top = (np.asarray(t.double().cpu() if t.is_floating_point() else t.cpu()) for t in got)
    for r in range(len(logits)):
        x = logits[r]
        ref = O.row(x, tokens[r], n_top, T)
        assert np.array_equal(ids[r], ref[2]), (r, ids[r], ref[2])
        plain = np.isfinite(x).any() and not np.isnan(x).any() and not np.isposinf(x).any()
        bz, bh = bounds(x[np.isfinite(x)], T) if plain else (0.0, 0.0)
        for mine, want in ((lp[r], ref[0]), (top[r], ref[3])):
            assert np.array_equal(np.isnan(mine), np.isnan(want)), r
            assert np.array_equal(np.isneginf(mine), np.isneginf(want)), r
            ok = np.isfinite(want)
            assert np.all(np.abs(mine[ok] - want[ok]) <= bz + 3 * EPS * np.abs(want[ok])), (r, mine[ok] - want[ok], bz)
        assert (math.isnan(h[r]) and math.isnan(ref[1])) or abs(h[r] - ref[1]) <= bh, (r, h[r], ref[1], bh)


def run(x, tokens, n_top=5, T=1.0, dtype="f32", ld=None, shift=0, stream=None):
    """Runs the operator on logits x [rows, vocab], rows ld apart, the first one `shift` elements into its storage."""
    import torch

    from paper_2602_20217_gb300 import logprobs as lp
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    rows, V = x.shape
    ld = V if ld is None else ld
    flat = torch.full((rows * ld + shift + 8,), float("nan"), dtype=dt, device="cuda")
    dev = flat[shift:].as_strided((rows, V), (ld, 1))
    dev.copy_(torch.as_tensor(x, device="cuda"))
    t = torch.as_tensor(np.asarray(tokens, np.int32), device="cuda")
    got = lp.token_logprobs(dev, t, n_top=n_top, temperature=T, stream=stream)
    torch.cuda.synchronize()
    check(dev.double().cpu().numpy(), np.asarray(tokens, np.int32).reshape(rows, -1), n_top, float(np.float32(T)), got)
    return dev, t, got


def normal(rows, V, seed=0, std=3.0):
    return np.random.default_rng(seed).standard_normal((rows, V)) * std


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 7, 64, 511, 512, 513, 1024, 1031, 8191, 32003, 128256, 151936])
def test_vocabularies(V, dtype):
    rng = np.random.default_rng(V)
    for rows in (1, 3):
        run(normal(rows, V, V), rng.integers(0, V, (rows, 2)), min(20, V), dtype=dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1, 3, 4, 7])
def test_strides(dtype, shift):
    for V, ld in ((1000, 1003), (1021, 1021), (4096, 4097), (33, 50)):
        run(normal(5, V, shift), np.zeros((5, 1)), 4, dtype=dtype, ld=ld, shift=shift)


@pytest.mark.parametrize("rows", [2, 37, 152, 153, 700])
def test_row_counts(rows):
    run(normal(rows, 3001, rows), np.random.default_rng(1).integers(0, 3001, (rows, 1)), 3)


@pytest.mark.parametrize("n_top", [0, 1, 2, 33, 64])
@pytest.mark.parametrize("n_tokens", [0, 1, 64])
def test_counts_of_results(n_top, n_tokens):
    run(normal(4, 5000, 3), np.random.default_rng(2).integers(-1, 5001, (4, n_tokens)), n_top)


@pytest.mark.parametrize("T", [0.01, 0.7, 1.3, 1e-30, 1e30])
def test_temperatures(T):
    run(normal(3, 2000, 5), [[0], [1], [2]], 7, T)


def test_far_and_close():
    """Peaked rows keep the digits of what is next to 0; offsets do not matter; extreme logits do not overflow."""
    x = normal(6, 4000, 7)
    x[0, 123] = 60.0
    x[1] += 1e6
    x[2] = -3.4028234663852886e38
    x[3, :7] = 3.4028234663852886e38
    x[4, 5] = x[4, 3999] = 100.0
    x[5] = np.linspace(-90, 0, 4000)
    run(x.astype(np.float32), [[123], [5], [9], [6], [3999], [0]], 10)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ties_and_orders(dtype):
    """Equal logits (more than are ranked in one go), few values, rising and falling rows, both zeros."""
    V = 20011
    rng = np.random.default_rng(0)
    x = np.zeros((8, V))
    x[1] = np.round(rng.standard_normal(V))
    x[2] = np.arange(V) / 64.0
    x[3] = -np.arange(V) / 64.0
    x[4] = np.where(np.arange(V) % 2 == 0, -0.0, 0.0)
    x[5, -3:] = 1.0
    x[6, :1500] = rng.permutation(1500) * 0.25 + 100
    x[7, ::17] = 2.0
    run(x, np.full((8, 1), 17), 64, dtype=dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_and_not_finite(dtype):
    V = 2500
    x = normal(9, V, 2)
    inf, nan = math.inf, math.nan
    x[0, ::2] = -inf
    x[1] = -inf
    x[2] = -inf
    x[2, 2400] = 1.0
    x[3, 77] = nan
    x[4, 2499] = inf
    x[5, :] = nan
    x[6, 0] = -nan
    x[7, :600] = -inf
    x[7, 2000:] = -inf
    x[8, 3] = inf
    x[8, 9] = -inf
    run(x, np.tile([1, 2400, V, -1], (9, 1)), 5, dtype=dtype)
    run(x, np.tile([1], (9, 1)), 64, dtype=dtype)


def test_same_bits_again_and_on_another_stream():
    import torch
    x = normal(20, 50021, 1)
    t = np.zeros((20, 1))
    a = run(x, t, 20)[2]
    b = run(x, t, 20, stream=torch.cuda.Stream())[2]
    assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_graph_follows_its_inputs():
    import torch

    from paper_2602_20217_gb300 import logprobs as lp
    x, y = normal(6, 9001, 1), normal(6, 9001, 2)
    dev, t, _ = run(x, np.arange(6)[:, None], 8)
    out = lp.empty(6, 1, 8)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lp.token_logprobs(dev, t, n_top=8, out=out)
    dev.copy_(torch.as_tensor(y, device="cuda"))
    t.add_(3)
    g.replay()
    torch.cuda.synchronize()
    check(dev.double().cpu().numpy(), t.cpu().numpy(), 8, 1.0, out)


def test_largest_vocabulary():
    run(normal(1, 1 << 22, 4), [[5]], 64, dtype="bf16")


def test_refusals_of_the_python_face():
    import torch

    from paper_2602_20217_gb300 import logprobs as lp
    x, t = torch.zeros(4, 100, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in [(x.half(), t), (x.cpu(), t), (x[0], t), (x.t(), torch.zeros(100, dtype=torch.int32, device="cuda")),
                (x, t.long()), (x, t[:3]), (x, t.cpu())]:
        with pytest.raises(ValueError):
            lp.token_logprobs(*bad)
    with pytest.raises(ValueError):                  # no place for the results on a stream that torch cannot name
        lp.token_logprobs(x, t, stream=torch.cuda.Stream().cuda_stream)


@pytest.mark.parametrize("which", ["tiny", "bf16"])
def test_model_logprobs(which):
    """Those of the pending token after a prompt and of a verify pass's tokens, from the pass's own logits."""
    from dataclasses import replace

    from paper_2602_20217_gb300.configs import LLAMA3_8B, TINY
    from paper_2602_20217_gb300.knapspec import KsError
    from paper_2602_20217_gb300.model import Model
    shape = TINY if which == "tiny" else replace(LLAMA3_8B, n_layers=1, d_model=512, d_ff=1024, n_q_heads=8,
                                                 n_kv_heads=2, vocab=5008, name="small-bf16")
    m = Model(shape, max_seq=256)
    with pytest.raises(KsError):
        m.logprobs([0])
    pending = m.prefill(np.arange(40, dtype=np.int32))
    last = 8 if which == "bf16" else None
    rows = next(r for r in range(16, 0, -1) if _has(m, r))
    assert last is None or rows >= 1
    got = m.logprobs(np.full(1, pending), 4, first_row=rows - 1)
    x = m.logits(rows).astype(np.float64)
    check_np(x[rows - 1:], [[pending]], 4, got)
    assert got.top_ids[0, 0] == pending
    m.draft(np.ones(shape.n_sublayers, np.uint8), 4)
    n, tokens = m.verify(None, 4)[:2]
    tokens = np.asarray(tokens, np.int32)
    before = m.launches()
    got = m.logprobs(tokens, 3, temperature=0.5)
    assert m.launches() == before + 1
    check_np(m.logits(5).astype(np.float64)[:len(tokens)], tokens[:, None], 3, got, T=0.5)
    assert np.array_equal(got.top_ids[:, 0], tokens)             # greedy
    with pytest.raises(KsError):
        m.logprobs(np.zeros(2, np.int32), first_row=4)


def _has(m, rows):
    from paper_2602_20217_gb300.knapspec import KsError
    try:
        m.logprobs(np.zeros(1, np.int32), first_row=rows - 1)
        return True
    except KsError:
        return False


def check_np(x, tokens, n_top, got, T=1.0):
    import torch
    lp = torch.as_tensor(got.logprobs)
    check(x, tokens, n_top, T, (lp.reshape(len(x), -1), *(torch.as_tensor(t) for t in got[1:])))
