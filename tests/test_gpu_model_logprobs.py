"""Which rows Model.logprobs has: those of the last prompt, draft or verify pass,
and none of a layer selection's, whose passes have other rows and, where they
are few or the model is fp32, put their candidates' logits in the same place."""
import numpy as np
import pytest

from helpers import need_gpu
from test_gpu_wide_edges import shape_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()


def model(which, **kw):
    from paper_2602_20217_gb300.configs import TINY
    from paper_2602_20217_gb300.model import Model
    return Model(TINY if which == "tiny" else shape_of(vocab=2000, **kw), max_seq=256)


def same_numbers(x, y):
    return all(np.array_equal(a, b) for a, b in zip(x, y))


def has_exactly(m, rows):
    """The pass has so many rows, and is asked for no more."""
    from paper_2602_20217_gb300 import knapspec as ks
    m.logprobs(np.zeros(rows, np.int32), 1)
    m.logprobs(np.zeros(1, np.int32), 1, first_row=rows - 1)
    for first, n in ((rows, 1), (0, rows + 1), (rows - 1, 2), (16, 1)):
        with pytest.raises(ks.KsError) as e:
            m.logprobs(np.zeros(n, np.int32), 1, first_row=first)
        assert e.value.status == ks.KS_ERR_INVALID_ARG


@pytest.mark.parametrize("which", ["tiny", "bf16"])
def test_rows_of_prompts_drafts_and_verify_passes(which):
    """A prompt has its last 16 rows (the model's max_rows) or all of fewer, by passes of few rows and by wide ones; a
    draft pass one, a verify pass gamma + 1."""
    m = model(which)
    for n in (1, 5, 16, 17, 40, 200):
        pending = m.prefill(np.arange(n, dtype=np.int32))
        has_exactly(m, min(n, 16))
        assert m.logprobs([0], 1, first_row=min(n, 16) - 1).top_ids[0, 0] == pending
    m.draft(np.ones(m.shape.n_sublayers, np.uint8), 4)
    has_exactly(m, 1)
    m.verify(None, 4)
    has_exactly(m, 5)
    m.close()


def test_a_selection_adds_no_rows():
    """The DP's passes over the history have more rows than the verify pass had, and leave its logits."""
    from paper_2602_20217_gb300 import knapspec as ks
    m = model("bf16", L=1)
    m.prefill(np.arange(40, dtype=np.int32))
    for _ in range(3):
        m.draft(np.ones(2, np.uint8), 2)
        m.verify(None, 2)
    before = m.logprobs(np.arange(3), 5)
    m.select_dp(ks.latency(1, units=np.ones(2, np.int32)), 8, tau=-2.0, max_states=8, max_rows=16)
    has_exactly(m, 3)
    assert same_numbers(before, m.logprobs(np.arange(3), 5))
    m.close()


@pytest.mark.parametrize("stage", ["tpt", "dp"])
def test_replaced_logits_are_not_scored(stage):
    """In an fp32 model a selection's candidates replace the pass's logits: there is nothing to score until the next pass."""
    from paper_2602_20217_gb300 import knapspec as ks
    m = model("tiny")
    n = m.shape.n_sublayers
    m.prefill(np.arange(40, dtype=np.int32))
    m.draft(np.ones(n, np.uint8), 4)
    m.verify(None, 4)
    if stage == "tpt":
        m.select_tpt(ks.latency(0, 0.08, 2e-5, 0.05), 8, 10)
    else:
        m.select_dp(ks.latency(1, units=np.ones(n, np.int32)), 8, tau=-2.0, max_states=8, max_rows=16)
    with pytest.raises(ks.KsError) as e:
        m.logprobs([0], 1)
    assert e.value.status == ks.KS_ERR_STATE
    m.draft(np.ones(n, np.uint8), 4)
    has_exactly(m, 1)
    m.verify(None, 4)
    has_exactly(m, 5)
    m.close()
