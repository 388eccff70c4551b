"""The 8-bit cache's attention on a stream that is not the current one, with an
output and a workspace that it allocates by itself: the current stream's work
neither delays nor overwrites it, and its memory is its stream's."""
import pytest

from helpers import need_gpu
from test_gpu_kv8 import Pool

pytestmark = pytest.mark.gpu

HQ, HD, SLEEP = 8, 64, 100_000_000       # clocks: some 50 ms


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()


@pytest.fixture(params=[2, 40], ids=["few rows", "many rows"])
def case(request):
    import torch
    rows = request.param
    pool = Pool([900], 2, HD, 32, seed=30).fill()
    d = pool.device([rows], pad=3)
    q = torch.randn(rows + 3, HQ, HD, device="cuda").to(torch.bfloat16)
    want = d["cache"].attention(d["batch"], q)
    torch.cuda.synchronize()
    assert bool((want[:rows] != 0).any()) and bool((want[rows:] == 0).all())
    return d, q, want


@pytest.mark.parametrize("own", ["out", "workspace", "both"])
def test_current_stream_does_not_overwrite(case, own):
    import torch
    d, q, want = case
    s = torch.cuda.Stream()
    for _ in range(3):
        torch.cuda.synchronize()
        given = {}
        if own == "out":
            given["workspace"] = d["cache"].attention_workspace(HQ, 1, q.shape[0])
        if own == "workspace":
            given["out"] = torch.zeros_like(q)
            torch.cuda.synchronize()
        torch.cuda._sleep(SLEEP)         # the current stream is busy: what it is given now runs long after the call
        out = d["cache"].attention(d["batch"], q, stream=s, **given)
        s.synchronize()
        early = out.clone() if own == "workspace" else None
        torch.cuda.synchronize()
        assert torch.equal(out, want) and (early is None or torch.equal(early, want))


def test_memory_is_not_handed_out_while_the_call_runs(case, monkeypatch):
    import torch
    d, q, want = case
    cache, s, used = d["cache"], torch.cuda.Stream(), []
    allocate = type(cache).attention_workspace

    def noted(self, *sizes):
        w = allocate(self, *sizes)
        used.append((w.data_ptr(), w.numel()))
        return w
    monkeypatch.setattr(type(cache), "attention_workspace", noted)
    with torch.cuda.stream(s):
        torch.cuda._sleep(SLEEP)
    out = cache.attention(d["batch"], q, stream=s)
    (start, size), = used
    taken = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(3)]
    assert all(t.data_ptr() + size <= start or t.data_ptr() >= start + size for t in taken)
    for t in taken:
        t.fill_(0xff)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_streams_by_address(case):
    import torch
    d, q, want = case
    s = torch.cuda.Stream()
    for given in ({}, {"out": torch.empty_like(q)}, {"workspace": d["cache"].attention_workspace(HQ, 1, q.shape[0])}):
        with pytest.raises(ValueError, match="address of a stream"):
            d["cache"].attention(d["batch"], q, stream=s.cuda_stream, **given)
    out, work = torch.zeros_like(q), d["cache"].attention_workspace(HQ, 1, q.shape[0])
    torch.cuda.synchronize()
    d["cache"].attention(d["batch"], q, out=out, workspace=work, stream=s.cuda_stream)
    here = d["cache"].attention(d["batch"], q, stream=torch.cuda.current_stream().cuda_stream)
    same = d["cache"].attention(d["batch"], q, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(here, want) and torch.equal(same, want)
