"""The 8-bit draft cache's memory and launches."""
import numpy as np
import pytest

from helpers import need_gpu
from test_gpu_draft_cache import MAX_SEQ, _check_copy, _shape

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()


def test_memory_that_the_current_stream_still_writes():
    """The model has a stream of its own; the draft cache's memory was freed by a tensor whose fill is queued."""
    import torch

    from paper_2602_20217_gb300 import knapspec as ks
    from paper_2602_20217_gb300 import synth
    from paper_2602_20217_gb300.model import Model
    shape, mask = _shape(), np.ones(4, np.uint8)
    torch.cuda.synchronize()
    m = Model(shape, max_seq=MAX_SEQ, stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    m.prefill(synth.prompt_tokens(shape, 123, seed=1))
    late = torch.empty(ks.ks_draft_cache_bytes(m.cfg), dtype=torch.uint8, device="cuda")
    at = late.data_ptr()
    for _ in range(2):                               # the first time loads the kernels, which may wait for the device
        torch.cuda.synchronize()
        torch.cuda._sleep(100_000_000)
        late.fill_(0xff)
    del late
    m.draft_cache()
    assert m.draft_memory.data_ptr() == at           # else the allocator made the case impossible
    torch.cuda.synchronize()
    first = list(m.draft(mask, 5))                   # status words raise
    for l in range(2):
        _check_copy(m, l, 123, 5)
    assert list(m.draft(mask, 5)) == first
    m.close()


@pytest.mark.parametrize("mask", [[1, 1, 1, 1], [0, 1, 1, 1]])
def test_every_launch_is_counted(mask):
    """A draft's Attn sublayer over the copy: query prep, append, attention and its merge; the first, third and
    fourth over the bf16 cache."""
    from paper_2602_20217_gb300 import knapspec as ks
    from paper_2602_20217_gb300 import synth
    from paper_2602_20217_gb300.model import Model
    shape, mask, gamma = _shape(), np.array(mask, np.uint8), 3
    sublayers = gamma * int(mask[::2].sum())
    counts, timed = {}, {}
    for cached in (False, True):
        m = Model(shape, max_seq=MAX_SEQ)
        if cached:
            m.draft_cache()
        m.prefill(synth.prompt_tokens(shape, 123, seed=1))
        m.draft(mask, gamma)                         # the copy takes the prompt
        before = ks.ks_launch_count(m.h)
        m.draft(mask, gamma)
        counts[cached] = ks.ks_launch_count(m.h) - before
        for klass in (1, 2, 10):
            ks.ks_kernel_timing(m.h, klass, 1)
            m.draft(mask, gamma)
            timed[cached, klass] = ks.ks_kernel_time(m.h, klass)[0]
            ks.ks_kernel_timing(m.h, klass, 0)
        m.close()
    assert counts[True] - counts[False] == sublayers
    for klass, per in ((1, 1), (2, 1), (10, 1)):
        assert timed[False, klass] == per * sublayers
    for klass, per in ((1, 1), (2, 1), (10, 2)):
        assert timed[True, klass] == per * sublayers
