"""More groups than the preparation of common beginnings keeps in shared memory, held to what the values can be.

All values are positive, so a row's output is the average of |v| that the
tolerances of test_gpu_kv8.py speak of: 2^-8 and 2^-10 of the output itself, for
each of the two calls that are compared.  Logarithms of sums: 2e-4 each.
"""
import numpy as np
import pytest

from helpers import need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()


@pytest.mark.parametrize("n_groups", [4095, 4096, 4097, 5000])
def test_thousands_of_groups(n_groups):
    """Groups of one to three sequences with one or two pages in common, and of sequences that have less than that."""
    import torch

    from paper_2602_20217_gb300 import kv8
    rng = np.random.default_rng(n_groups)
    sizes = rng.integers(1, 4, n_groups)
    groups = np.concatenate(([0], np.cumsum(sizes)))
    n = int(groups[-1])
    cache = kv8.Cache8(2 * n_groups + n, 16, 1, 64)
    cache.data.random_(0, 100)
    cache.data.view(-1, 2080)[:, -32:-24] = torch.full((2,), 2.0 ** -5, device="cuda").view(torch.uint8)
    of = np.repeat(np.arange(n_groups), sizes)
    table = np.stack((2 * of, 2 * of + 1, 2 * n_groups + np.arange(n)), 1).astype(np.int32)
    i32 = dict(dtype=torch.int32, device="cuda")
    # a row among the first 32 tokens shortens what its group shares
    lens = torch.tensor(np.where(rng.random(n) < 0.1, rng.integers(1, 33, n), rng.integers(33, 49, n)), **i32)
    batch = kv8.Batch8(torch.tensor(table, device="cuda"), torch.arange(n + 1, **i32), lens, n, torch.zeros(1, **i32))
    shared = kv8.Shared8(torch.tensor(groups, **i32), torch.tensor(rng.integers(0, 40, n_groups), **i32))
    q = torch.randn(n, 4, 64, device="cuda").to(torch.bfloat16)
    sums, plain_sums = (torch.zeros(n, 4, device="cuda") for _ in range(2))
    a = cache.attention(batch, q, lse=sums, shared=shared).double()
    b = cache.attention(batch, q, lse=plain_sums).double()
    assert int(batch._keep[3]) == 0 and bool((b > 0).any())
    assert bool(((a - b).abs() <= (2.0 ** -8 + 2.0 ** -10) * (a + b)).all())
    assert float((sums - plain_sums).abs().max()) <= 4e-4
