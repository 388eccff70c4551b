"""Token log probabilities without a GPU: the restatement, the refusals of the
entry points, the checks of the Python face."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import logprobs as O


def test_restatement():
    x = np.array([0.0, math.log(3.0), -math.inf, 0.0])
    lp, h, ids, top = O.row(x, [1, 2, 3, 9], 3, 1.0)
    assert np.allclose(lp[:3], [math.log(0.6), -math.inf, math.log(0.2)]) and math.isnan(lp[3])
    assert h == pytest.approx(-(0.6 * math.log(0.6) + 0.4 * math.log(0.2)))
    assert list(ids) == [1, 0, 3] and top[0] == lp[0]
    lp, h, _, _ = O.row([5.0, 5.0 - 40.0], [0], 0, 1.0)
    assert lp[0] == pytest.approx(-math.exp(-40.0), rel=1e-12) and h == pytest.approx(41 * math.exp(-40.0), rel=1e-12)
    assert O.row([1.0, math.nan], [0], 1, 1.0)[2][0] == -1
    assert list(O.row([-math.inf] * 3, [1], 2, 1.0)[2]) == [0, 1]


@pytest.fixture(scope="module")
def lib():
    import os
    import shutil
    if shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"):
        pytest.skip("nvcc not available")
    from paper_2602_20217_gb300 import build, knapspec
    build.build()
    return knapspec.load()


A = 0x10000000      # an aligned address that is never followed


def good(ks):
    return ks.KsLogprobs(A, ks.KS_DTYPE_F32, 3, 1000, 1000, A, 2, 5, 1.0, A, A, A, A)


BAD = [("logits", None, 1), ("logits", A + 2, 1), ("dtype", 2, 1), ("rows", -1, 1), ("rows", 1 << 25, 1),
       ("vocab", 0, 1), ("vocab", (1 << 22) + 1, 6), ("row_stride", 999, 1), ("row_stride", 1 << 41, 1),
       ("tokens", None, 1), ("tokens", A + 1, 1), ("n_tokens", -1, 1), ("n_tokens", 65, 6), ("n_top", -1, 1),
       ("n_top", 65, 6), ("vocab", 4, 1), ("temperature", 0.0, 1), ("temperature", -1.0, 1),
       ("temperature", math.nan, 1), ("temperature", math.inf, 1), ("logprobs", None, 1), ("logprobs", A + 2, 1),
       ("entropy", A + 1, 1), ("top_ids", None, 1), ("top_logprobs", A + 1, 1)]


@pytest.mark.parametrize("field,value,status", BAD)
def test_refusals_touch_no_device(lib, field, value, status):
    from paper_2602_20217_gb300 import knapspec as ks
    a = good(ks)
    setattr(a, field, value)
    assert lib.ks_token_logprobs(C.byref(a), None) == status
    assert lib.ks_last_error().decode().startswith("ks_token_logprobs")


def test_empty_calls_and_null(lib):
    from paper_2602_20217_gb300 import knapspec as ks
    a = good(ks)
    a.rows, a.logits = 0, None
    assert lib.ks_token_logprobs(C.byref(a), None) == ks.KS_OK
    assert lib.ks_token_logprobs(None, None) == ks.KS_ERR_INVALID_ARG
    assert lib.ks_model_logprobs(None, 0, C.byref(a)) == ks.KS_ERR_INVALID_ARG


def test_python_face_checks_its_tensors(lib):
    torch = pytest.importorskip("torch")
    from paper_2602_20217_gb300 import logprobs as lp
    tokens = torch.zeros(3, 2, dtype=torch.int32)
    out = lp.empty(3, 2, 4, device="cpu")
    a = lp.marshal(A, 0, 10, 10, tokens, 4, 1.0, out)
    assert (a.rows, a.n_tokens, a.n_top, a.vocab) == (3, 2, 4, 10)
    for bad in [(tokens.long(), 4, out), (tokens.t(), 4, lp.empty(2, 3, 4, device="cpu")), (tokens, 3, out),
                (tokens, 4, lp.empty(2, 2, 4, device="cpu")), (tokens, 4, out._replace(entropy=torch.zeros(3).double())),
                (tokens, 4, out._replace(top_ids=torch.zeros(3, 4)))]:
        with pytest.raises(ValueError):
            lp.marshal(A, 0, 10, 10, bad[0], bad[1], 1.0, bad[2])
