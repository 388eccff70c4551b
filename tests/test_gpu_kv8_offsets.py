"""The 8-bit cache attention where row offsets decrease, so that sequences would
share rows: flagged, and nothing is written.  Such a batch can hold far more
work than its sizes allow (alternating offsets give every other sequence all
rows), past what 32 bits count in the last case."""
import pytest

from helpers import need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()


@pytest.mark.parametrize("n_seqs,n_rows,hk,length", [(2, 3, 1, 90), (300, 300, 1, 900), (40, 200, 2, 900),
                                                     (8, 400, 2, 5000), (300, 300, 8, 1 << 20)])
@pytest.mark.parametrize("kind", ["alternating", "one"])
def test_decreasing_offsets_attend_nothing(n_seqs, n_rows, hk, length, kind):
    import torch

    from paper_2602_20217_gb300 import kv8
    hd, page, hq = 64, 256, 4 * hk
    pages = -(-length // page)
    cache = kv8.Cache8(1, page, hk, hd)
    cache.data.zero_()
    cache.data.view(-1, 32 * hd + 32)[:, -32:-24] = torch.ones(2, device="cuda").view(torch.uint8)       # scales
    table = torch.zeros(n_seqs, pages, dtype=torch.int32, device="cuda")
    if kind == "alternating":
        offsets = [n_rows * (i % 2) for i in range(n_seqs + 1)]
    else:                                            # the last sequence's end falls by one
        offsets = [i * n_rows // n_seqs for i in range(n_seqs - 1)] + [n_rows, n_rows - 1]
    offsets = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    lengths = torch.full((n_seqs,), length, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    batch = kv8.Batch8(table, offsets, lengths, n_rows, status)
    q = torch.randn(n_rows, hq, hd, device="cuda").to(torch.bfloat16)
    out = torch.full((n_rows, hq, hd), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n_rows, hq), 7.0, device="cuda")
    work = cache.attention_workspace(hq, n_seqs, n_rows)
    cache.attention(batch, q, out=out, lse=lse, workspace=work)
    torch.cuda.synchronize()
    assert int(status) == 2
    assert bool((out == 7).all()) and bool((lse == 7).all())
    # the same workspace and batch, mended, are as good as new
    if length > 10000:
        return
    offsets.copy_(torch.tensor([i * n_rows // n_seqs for i in range(n_seqs + 1)], dtype=torch.int32))
    status.zero_()
    cache.attention(batch, q, out=out, lse=lse, workspace=work)
    torch.cuda.synchronize()
    assert int(status) == 0 and bool((out == 0).all())       # values of zeros
    assert bool(torch.isfinite(lse).all())
