"""That log probabilities add up every logit once, in rows of one CTA and of clusters.

A row is cut into segments of 2 KB (512 fp32, 1024 bf16 logits); C CTAs take
every C-th of them, eight warps of a CTA every eighth of these, and a lane 64
bytes of each: L = 16 or 32 logits.  So a warp has W = ceil(ceil(segments / C) /
8) segments, and a term of the sum passes through at most
  W L additions in the lane, 3 of each segment's end, 5 + 5 + 5 of the joins
of lanes, warps and CTAs, and W + 3 changes to a larger maximum, each of which is
a product with an exponential (2^-22, and 3 roundings).  An exponent is off by
4 * 2^-24 of itself (the factor log2(e) / T has two roundings, difference and
product one each): D is the average of |x - max| / T under the sum, and the
changes of the maximum are together no further than the largest logit is from
the least of the segments' largest, `span`.  The sum beside the largest logit is
off by
  rel = 2^-22 (W + 4) + 2^-24 (4 (D + span) + W L + 6 W + 24).
"""
import math

import numpy as np
import pytest

from helpers import need_gpu
from test_gpu_logprobs import EPS

pytestmark = pytest.mark.gpu
DT = {"f32": 4, "bf16": 2}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()


def warp_segments(rows, V, size):
    """W of a call: CTAs a row double while all rows' are resident at once and four segments are left for each."""
    import torch
    seg, sms = 2048 // size, torch.cuda.get_device_properties(0).multi_processor_count
    ctas = 1
    while ctas < 8 and rows * ctas * 2 <= 4 * sms and ctas * 2 * seg * 4 <= V:
        ctas *= 2
    segs = (V + 16 // size - 1 + seg - 1) // seg
    return ctas, -(-(-(-segs // ctas)) // 8)


def made(rows, V, dtype, shift, fill):
    """Rows of logits, V + 5 apart where shift is not 0, so that rows begin at every alignment."""
    import torch
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    ld = V + (5 if shift else 0)
    flat = torch.full((rows * ld + shift + 8,), fill, dtype=dt, device="cuda")
    return flat[shift:].as_strided((rows, V), (ld, 1))


def places(V, seg):
    """Every place of a segment inside the row and of those at its ends, and one of every segment."""
    mid = V // 2 // seg * seg
    p = list(range(mid, min(mid + seg, V))) + list(range(min(seg + 8, V))) + list(range(max(0, V - seg - 8), V))
    p += [s * seg + (37 * s) % seg for s in range(V // seg)]
    return sorted(set(p))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 3])
@pytest.mark.parametrize("rows,V", [(64, 151936), (150, 50257), (300, 20011), (700, 20011), (64, 2000)])
def test_one_logit_anywhere(dtype, shift, rows, V):
    """A logit 1 below the largest, all others 80 below: without it the sum beside the largest would be next to 0 instead
    of 1 / e, and with it twice, 2 / e.  It is the only term, and passes one addition and four changes of maximum at most
    that do not keep it: rel <= 4 * 2^-22 + (4 * 1 + 24) * 2^-24."""
    import torch

    from paper_2602_20217_gb300 import logprobs as lp
    x = made(rows, V, dtype, shift, -80.0)
    tail = math.exp(-1) + (V - 2) * math.exp(-80)
    log_z, mean = math.log1p(tail), math.exp(-1) / (1 + tail)
    rel = 4 * 2.0 ** -22 + 28 * EPS
    off = rel * tail / (1 + tail) + 2 * EPS * log_z
    every = places(V, 2048 // DT[dtype])
    for a in range(0, len(every), rows):
        p = torch.tensor((every[a:a + rows] * rows)[:rows], device="cuda")
        m, r = (p + V // 2) % V, torch.arange(rows, device="cuda")
        x.fill_(-80)
        x[r, p], x[r, m] = -1.0, 0.0
        got = lp.token_logprobs(x, torch.stack((p, m), 1).int(), n_top=2)
        assert torch.equal(got.top_ids, torch.stack((m, p), 1).int()), a
        want = torch.tensor([-1 - log_z, -log_z], dtype=torch.float64, device="cuda")
        assert float((got.logprobs.double() - want).abs().max()) <= off + 3 * EPS * (1 + log_z), a
        assert torch.equal(got.top_logprobs, got.logprobs.flip(1)), a
        assert float((got.entropy.double() - (log_z + mean)).abs().max()) <= off + 3 * rel * mean + 4 * EPS, a


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(1, 128256), (1, 151936), (40, 151936), (100, 50257), (200, 128256), (650, 100277),
                                    (3, 2000), (1, 257)])
@pytest.mark.parametrize("T", [1.0, 0.7])
def test_sums_within_the_order_of_their_additions(dtype, rows, V, T):
    import torch

    from paper_2602_20217_gb300 import logprobs as lp
    g = torch.Generator(device="cuda").manual_seed(rows + V)
    x = made(rows, V, dtype, 3, 0.0)
    for r in range(0, rows, 50):
        x[r:r + 50] = torch.randn(x[r:r + 50].shape, generator=g, device="cuda") * 3
    tokens = torch.randint(0, V, (rows, 4), generator=g, device="cuda")
    got = lp.token_logprobs(x, tokens.int(), temperature=T)
    size = DT[dtype]
    ctas, W = warp_segments(rows, V, size)
    seg, t = 2048 // size, float(np.float32(T))
    for r in range(0, rows, max(1, rows // 20)):
        z = x[r].double()
        z = (z - z.max()) / t
        n = int((z == 0).sum())
        e = torch.where(z == 0, 0.0, z.exp())
        tail = float(e.sum())
        D = float((e * -z).sum()) / tail
        # the segments begin at the 16-byte boundary before the row
        start = x[r].data_ptr() % 16 // size
        padded = torch.nn.functional.pad(z, (start, -(len(z) + start) % seg), value=-math.inf)
        span = -float(padded.view(-1, seg).amax(1).min())
        rel = 2.0 ** -22 * (W + 4) + EPS * (4 * (D + span) + W * 64 / size + 6 * W + 24)
        Z = n + tail
        log_z = math.log(Z) if n > 1 else math.log1p(tail)
        off = rel * tail / Z + 2 * EPS * (log_z + (n > 1)) + 1e-30
        want = z[tokens[r]] - log_z
        assert bool(((got.logprobs[r].double() - want).abs() <= off + 3 * EPS * want.abs()).all()), (r, ctas, W, off)
        mean = D * tail / Z
        assert abs(float(got.entropy[r]) - (log_z + mean)) <= off + 3 * rel * mean + 4 * EPS * (mean + log_z), r


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [6000, 128256])
@pytest.mark.parametrize("n_top", [1, 5, 64])
def test_every_result_of_a_row_that_is_not_finite_is_written(dtype, V, n_top):
    """Rows of NaN alone, of either sign, and of NaN in most places, with more segments than alternatives."""
    import torch

    from paper_2602_20217_gb300 import logprobs as lp
    x = made(5, V, dtype, 0, math.nan)
    x[1] = -x[1]
    x[2, 100:] = 1.0
    x[3, V - 7] = 2.0
    x[4] = math.inf
    out = lp.empty(5, 1, n_top)
    for t in out:
        t.fill_(777)
    lp.token_logprobs(x, torch.full((5,), V - 7, dtype=torch.int32, device="cuda"), n_top=n_top, out=out)
    assert bool((out.top_ids == -1).all())
    assert all(bool(t.isnan().all()) for t in (out.logprobs, out.entropy, out.top_logprobs))
