"""Received weights and eviction without a GPU: the restatement, the refusals of
the entry points, the checks of the Python face."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import kv8_evict as O
from test_kv8 import A, BATCH, CACHE, good, lib  # noqa: F401


def test_what_stays():
    x = np.array([5, 1, 1, 9, math.nan, -math.inf, 1, 7, 0, 2.0])
    assert list(O.kept(x, 10, 4, 0, 0, 99)) == [0, 3, 7, 9]
    assert list(O.kept(x, 10, 5, 0, 0, 99)) == [0, 1, 3, 7, 9]            # ties: the earlier
    assert list(O.kept(x, 10, 4, 1, 2, 99)) == [0, 3, 8, 9]
    assert list(O.kept(x, 10, 3, 5, 2, 99)) == [0, 8, 9] and list(O.kept(x, 10, 1, 5, 2, 99)) == [9]
    assert list(O.kept(x, 10, 9, 0, 0, 99)) == [0, 1, 2, 3, 5, 6, 7, 8, 9]  # NaN goes first
    assert list(O.kept(x, 10, 99, 0, 0, 99)) == list(range(10))
    assert list(O.kept(x, 10, 99, 0, 0, 2)) == [3, 7] and len(O.kept(x, 10, -3, 1, 1, 9)) == 0


B = A + (1 << 24)   # another one


def weights_args(ks):
    return ks.KsKv8Weights(A, 4096, 128, 32, 0.1, 1.0, A, B, B, 256, A, 1 << 30)


def evict_args(ks):
    return ks.KsKv8Eviction(A, 256, A, 2, 3, A, 2, B, B + (1 << 16), 128, B + (1 << 20), 128)


WEIGHTS = [("q", None, 1), ("q", A + 1, 1), ("q_row", -1, 1), ("n_q_heads", 12, 1), ("n_q_heads", 0, 1),
           ("n_q_heads", 1024, 6), ("scale", math.nan, 1), ("decay", math.inf, 1), ("lse", None, 1), ("lse", A + 2, 1),
           ("scores", None, 1), ("scores", A + 1, 1), ("out", None, 1), ("out", A + 2, 1), ("score_ld", 255, 1),
           ("score_ld", 1 << 50, 1), ("workspace", None, 1), ("workspace", A + 16, 1), ("workspace_bytes", 1000, 3)]
EVICT = [("scores", None, 1), ("scores", A + 2, 1), ("score_ld", 255, 1), ("keep", None, 1), ("first", -1, 1),
         ("recent", -1, 1), ("page_table", None, 1), ("table_ld", 0, 1), ("table_ld", 1 << 28, 1), ("lengths", None, 1),
         ("kept", None, 1), ("kept", A + 1, 1), ("kept_ld", 127, 1), ("new_scores", A + 2, 1), ("new_score_ld", 127, 1)]


@pytest.mark.parametrize("part,field,value,status", [("cache", *x) for x in CACHE] + [("batch", *x) for x in BATCH] +
                         [("weights", *x) for x in WEIGHTS] + [("evict", *x) for x in EVICT])
def test_refusals_touch_no_device(lib, part, field, value, status):  # noqa: F811
    from paper_2602_20217_gb300 import knapspec as ks
    cache, batch, _, _ = good(ks)
    w, e = weights_args(ks), evict_args(ks)
    setattr({"cache": cache, "batch": batch, "weights": w, "evict": e}[part], field, value)
    if field.startswith("workspace"):
        batch.n_rows = 100                           # few rows need none
    if part != "evict":
        assert lib.ks_kv8_attention_weights(C.byref(cache), C.byref(batch), C.byref(w), None) == status
        assert lib.ks_last_error().decode().startswith("ks_kv8_attention_weights")
    if part != "weights":
        assert lib.ks_kv8_evict(C.byref(cache), C.byref(batch), C.byref(e), None) == status
        assert lib.ks_last_error().decode().startswith("ks_kv8_evict")


@pytest.mark.parametrize("field", ["lengths", "kept", "new_scores"])
@pytest.mark.parametrize("place", [A, A + 4, A - 4])
def test_results_that_overlap_what_is_read_are_refused(lib, field, place):  # noqa: F811
    """The batch's lengths among them: heads read them while one writes the new ones."""
    from paper_2602_20217_gb300 import knapspec as ks
    cache, batch, _, _ = good(ks)
    e = evict_args(ks)
    setattr(e, field, place)
    assert lib.ks_kv8_evict(C.byref(cache), C.byref(batch), C.byref(e), None) == ks.KS_ERR_INVALID_ARG
    assert "overlap" in lib.ks_last_error().decode()


@pytest.mark.parametrize("field,value", [("scores", B + 4), ("scores", B - 4), ("lse", B), ("q", B + 16), ("out", A)])
def test_weights_that_overlap_what_is_read_are_refused(lib, field, value):  # noqa: F811
    from paper_2602_20217_gb300 import knapspec as ks
    cache, batch, _, _ = good(ks)
    w = weights_args(ks)
    setattr(w, field, value)
    assert lib.ks_kv8_attention_weights(C.byref(cache), C.byref(batch), C.byref(w), None) == ks.KS_ERR_INVALID_ARG
    assert "overlap" in lib.ks_last_error().decode()


def test_null_and_empty_calls(lib):  # noqa: F811
    from paper_2602_20217_gb300 import knapspec as ks
    cache, batch, rows, _ = good(ks)
    w, e = weights_args(ks), evict_args(ks)
    assert lib.ks_kv8_attention_weights(C.byref(cache), C.byref(batch), None, None) == 1
    assert lib.ks_kv8_evict(C.byref(cache), C.byref(batch), None, None) == 1
    empty = ks.KsKv8Batch(A, A, A, 0, 4, 5, None)
    assert lib.ks_kv8_attention_weights(C.byref(cache), C.byref(empty), C.byref(w), None) == 0
    assert lib.ks_kv8_evict(C.byref(cache), C.byref(empty), C.byref(e), None) == 0
    empty = ks.KsKv8Batch(A, A, A, 2, 4, 0, None)
    assert lib.ks_kv8_attention_weights(C.byref(cache), C.byref(empty), C.byref(w), None) == 0
    rows.shift = A + 2
    assert lib.ks_kv8_append(C.byref(cache), C.byref(batch), C.byref(rows), None) == 1
    cache.page_tokens, batch.table_ld, batch.n_seqs, w.score_ld = 1 << 20, 1023, 1 << 12, 1 << 31
    assert lib.ks_kv8_attention_weights(C.byref(cache), C.byref(batch), C.byref(w), None) == ks.KS_ERR_UNSUPPORTED
