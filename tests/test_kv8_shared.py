"""Refusals of the shared-prefix attention's entry points, without a GPU."""
import ctypes as C

import pytest

from test_kv8 import A, ATTN, BATCH, CACHE, good, lib  # noqa: F401

SHARED = [("group_offsets", None, 1), ("group_offsets", A + 2, 1), ("tokens", None, 1), ("tokens", A + 1, 1),
          ("n_groups", 0, 1), ("n_groups", -1, 1), ("n_groups", 1 << 21, 1)]


@pytest.mark.parametrize("part,field,value,status", [("cache", *x) for x in CACHE] + [("batch", *x) for x in BATCH] +
                         [("attn", *x) for x in ATTN] + [("shared", *x) for x in SHARED])
def test_refusals_touch_no_device(lib, part, field, value, status):  # noqa: F811
    from paper_2602_20217_gb300 import knapspec as ks
    cache, batch, _, attn = good(ks)
    shared = ks.KsKv8Shared(A, A, 2)
    setattr({"cache": cache, "batch": batch, "attn": attn, "shared": shared}[part], field, value)
    args = (C.byref(cache), C.byref(batch), C.byref(shared), C.byref(attn), None)
    assert lib.ks_kv8_shared_attention(*args) == status
    assert lib.ks_last_error().decode().startswith("ks_kv8_shared_attention")


def test_null_empty_and_workspace(lib):  # noqa: F811
    from paper_2602_20217_gb300 import knapspec as ks
    cache, batch, _, attn = good(ks)
    shared = ks.KsKv8Shared(A, A, 2)
    assert lib.ks_kv8_shared_attention(C.byref(cache), C.byref(batch), None, C.byref(attn), None) == 1
    assert lib.ks_kv8_shared_attention(C.byref(cache), C.byref(batch), C.byref(shared), None, None) == 1
    for field in ("n_seqs", "n_rows"):
        empty = ks.KsKv8Batch(A, A, A, 2, 4, 5, None)
        setattr(empty, field, 0)
        assert lib.ks_kv8_shared_attention(C.byref(cache), C.byref(empty), C.byref(shared), C.byref(attn), None) == 0
    n = ks.ks_kv8_shared_workspace(cache, 32, 4, 9, 2)
    assert n > ks.ks_kv8_attention_workspace(cache, 32, 4, 9) + 9 * 32 * 129 * 4
    for bad in [(31, 4, 9, 2), (32, -1, 9, 2), (32, 4, -1, 2), (32, 4, 9, -1), (32, 4, 9, 1 << 21)]:
        assert ks.ks_kv8_shared_workspace(cache, *bad) == 0
    attn.workspace_bytes = ks.ks_kv8_shared_workspace(cache, 32, 2, 5, 2) - 1
    assert lib.ks_kv8_shared_attention(C.byref(cache), C.byref(batch), C.byref(shared), C.byref(attn),
                                       None) == ks.KS_ERR_WORKSPACE
