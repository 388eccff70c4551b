"""The 8-bit paged cache without a GPU: the oracle's codes, scales and record
layout, the sizes and refusals of the entry points, the checks of the Python
face."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import kv8 as O


def test_codes_against_torch():
    torch = pytest.importorskip("torch")
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t, O.VALUES, equal_nan=True)
    rng = np.random.default_rng(0)
    x = np.clip(rng.standard_normal(200000) * np.exp2(rng.uniform(-14, 6, 200000)), -448, 448).astype(np.float32)
    mid = ((O.VALUES[:126] + O.VALUES[1:127]) / 2).astype(np.float32)     # every tie
    x = np.concatenate((x, mid, -mid, [0.0, -0.0, 448.0, -448.0]))
    assert np.array_equal(torch.tensor(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy(), O.e4m3_codes(x))
    assert list(O.e4m3_codes([math.nan, math.inf, -math.inf])) == [127, 127, 127]


@pytest.mark.parametrize("amax,e", [(0.0, -126), (448.0, 0), (448.0000001, 1), (224.0, -1), (1.0, -8), (1.75, -8),
                                    (1.7500001, -7), (3e38, 120), (1e-45, -126), (2.0 ** -117, -125)])
def test_scale(amax, e):
    assert O.scale_for(amax) == 2.0 ** e


@pytest.mark.parametrize("hd", [64, 128])
def test_record_round_trip(hd):
    rng = np.random.default_rng(hd)
    k, v = (rng.integers(0, 256, (16, hd)).astype(np.uint8) for _ in range(2))
    rec = O.pack_record(k, v, 0.5, 8.0)
    assert len(rec) == 32 * hd + 32
    got = O.unpack_record(rec)
    assert np.array_equal(got[0], k) and np.array_equal(got[1], v) and got[2:] == (0.5, 8.0)
    assert rec[16 * hd + 3 * 16 + 6] == v[10, 3]        # token 10: byte 4 * 1 + 2 * 1 + 0
    assert rec[(hd // 16 + 1) * 128 + 2 * 16 + 4] == k[10, 20]


def test_block_goes_on():
    """A louder token raises the scale and halves the stored codes; tokens behind the new one are zeros."""
    rng = np.random.default_rng(1)
    one = rng.standard_normal((2, 5, 64))
    b = O.append_block(None, 0, *one)
    loud = np.full((1, 64), 4 * 448 * b[2])
    c = O.append_block(b, 5, loud, loud * 0 + 0.25 * b[3])
    assert c[2] == 4 * b[2] and c[3] == b[3]
    assert np.array_equal(O.VALUES[c[0][5]] * c[2], loud[0])
    old, new = O.VALUES[b[0][:5]] * b[2], O.VALUES[c[0][:5]] * c[2]
    assert np.all(np.abs(old - new) <= c[2] * 2.0 ** -10)
    assert not c[0][6:].any() and not c[1][6:].any()


# ------------------------------------------------------------ entry points
@pytest.fixture(scope="module")
def lib():
    import os
    import shutil
    if shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"):
        pytest.skip("nvcc not available")
    from paper_2602_20217_gb300 import build, knapspec
    build.build()
    return knapspec.load()


def test_bytes(lib):
    from paper_2602_20217_gb300 import knapspec as ks
    assert ks.ks_kv8_bytes(3, 64, 8, 128) == 3 * 8 * 4 * 4128
    assert ks.ks_kv8_bytes(1, 16, 1, 64) == 2080
    assert ks.ks_kv8_bytes(1 << 20, 256, 8, 128) == (1 << 20) * 16 * 8 * 4128
    for bad in [(0, 64, 8, 128), (1, 0, 8, 128), (1, 24, 8, 128), (1, 64, 0, 128), (1, 64, 8, 96), (1, 64, 8, 256),
                (1, -16, 8, 64), (1, 64, 5000, 64)]:
        assert ks.ks_kv8_bytes(*bad) == 0, bad


A = 0x10000000      # an aligned address that is never followed


def good(ks):
    cache = ks.KsKv8Cache(A, 4, 64, 8, 128)
    batch = ks.KsKv8Batch(A, A, A, 2, 4, 5, None)
    rows = ks.KsKv8Rows(A, A, None, ks.KS_DTYPE_BF16, 0, 1024, 128, 1024, 128)
    attn = ks.KsKv8Attn(A, 4096, 128, A, 4096, 128, None, 32, 0.1, A, 1 << 40)
    return cache, batch, rows, attn


CACHE = [("data", None, 1), ("data", A + 8, 1), ("n_pages", 0, 1), ("page_tokens", 40, 1), ("head_dim", 96, 6),
         ("n_kv_heads", -1, 1)]
BATCH = [("page_table", None, 1), ("row_offsets", A + 2, 1), ("lengths", None, 1), ("n_seqs", -1, 1),
         ("n_rows", -1, 1), ("n_rows", 1 << 30, 1), ("table_ld", 0, 1), ("table_ld", 1 << 28, 1), ("status", A + 1, 1)]
ROWS = [("k", None, 1), ("v", None, 1), ("k", A + 1, 1), ("q", A + 1, 1), ("dtype", 3, 1), ("k_row", -1, 1),
        ("v_head", 1 << 50, 1), ("rope", A, 1), ("q", A, 1)]
ATTN = [("q", None, 1), ("out", None, 1), ("q", A + 1, 1), ("out", A + 1, 1), ("lse", A + 2, 1), ("n_q_heads", 12, 1),
        ("n_q_heads", 0, 1), ("n_q_heads", 1024, 6), ("scale", math.nan, 1), ("scale", math.inf, 1),
        ("workspace", None, 1), ("workspace", A + 16, 1), ("workspace_bytes", 0, 3), ("out_row", 64, 1),
        ("out_head", 64, 1), ("q_row", -1, 1)]


@pytest.mark.parametrize("part,field,value,status", [("cache", *x) for x in CACHE] + [("batch", *x) for x in BATCH] +
                         [("rows", *x) for x in ROWS] + [("attn", *x) for x in ATTN])
def test_refusals_touch_no_device(lib, part, field, value, status):
    from paper_2602_20217_gb300 import knapspec as ks
    cache, batch, rows, attn = good(ks)
    setattr({"cache": cache, "batch": batch, "rows": rows, "attn": attn}[part], field, value)
    if part != "attn":
        assert lib.ks_kv8_append(C.byref(cache), C.byref(batch), C.byref(rows), None) == status
        assert lib.ks_last_error().decode().startswith("ks_kv8_append")
    if part != "rows":
        assert lib.ks_kv8_attention(C.byref(cache), C.byref(batch), C.byref(attn), None) == status
        assert lib.ks_last_error().decode().startswith("ks_kv8_attention")
    if part in ("cache", "batch"):
        assert lib.ks_kv8_read(C.byref(cache), C.byref(batch), A, A, 1, 1024, 128, None) == status


def test_refusals_of_null_structs_and_reads(lib):
    from paper_2602_20217_gb300 import knapspec as ks
    cache, batch, rows, attn = good(ks)
    assert lib.ks_kv8_append(None, C.byref(batch), C.byref(rows), None) == 1
    assert lib.ks_kv8_append(C.byref(cache), None, C.byref(rows), None) == 1
    assert lib.ks_kv8_append(C.byref(cache), C.byref(batch), None, None) == 1
    assert lib.ks_kv8_attention(C.byref(cache), C.byref(batch), None, None) == 1
    for bad in [(None, A, 1, 1024, 128), (A, None, 1, 1024, 128), (A, A, 5, 1024, 128), (A, A + 1, 1, 1024, 128),
                (A, A + 2, 0, 1024, 128), (A, A, 1, 64, 128), (A, A, 1, 1024, 64), (A, A, 1, -1, 128)]:
        assert lib.ks_kv8_read(C.byref(cache), C.byref(batch), *bad, None) == 1, bad
    rows.q, rows.n_q_heads, rows.q_row, rows.q_head = A, 32, 4096, 128        # no q_out
    assert lib.ks_kv8_append(C.byref(cache), C.byref(batch), C.byref(rows), None) == 1
    rows.q_out, rows.q_out_row, rows.q_out_head = A, 4096, 64
    assert lib.ks_kv8_append(C.byref(cache), C.byref(batch), C.byref(rows), None) == 1


def test_empty_calls_succeed_without_a_device(lib):
    from paper_2602_20217_gb300 import knapspec as ks
    cache, batch, rows, attn = good(ks)
    for field in ("n_seqs", "n_rows"):
        empty = ks.KsKv8Batch(A, A, A, 2, 4, 5, None)
        setattr(empty, field, 0)
        assert lib.ks_kv8_append(C.byref(cache), C.byref(empty), C.byref(rows), None) == 0
        assert lib.ks_kv8_attention(C.byref(cache), C.byref(empty), C.byref(attn), None) == 0
        assert lib.ks_kv8_read(C.byref(cache), C.byref(empty), A, A, 1, 1024, 128, None) == 0
    assert ks.ks_kv8_attention_workspace(cache, 32, 0, 0) >= 0
    assert ks.ks_kv8_attention_workspace(cache, 32, 4, 9) > 0
    for bad in [(31, 4, 9), (0, 4, 9), (32, -1, 9), (32, 4, -1), (1024, 4, 9)]:
        assert ks.ks_kv8_attention_workspace(cache, *bad) == 0


def test_python_face_checks_its_tensors(lib):
    torch = pytest.importorskip("torch")
    from paper_2602_20217_gb300 import kv8
    from paper_2602_20217_gb300.knapspec import KsError

    def i32(*v):
        return torch.tensor(v, dtype=torch.int32)
    table = torch.zeros(2, 4, dtype=torch.int32)
    b = kv8.Batch8(table, i32(0, 1, 2), i32(3, 4), 2)
    assert (b.c.n_seqs, b.c.table_ld, b.c.n_rows) == (2, 4, 2)
    for bad in [(table.long(), i32(0, 1, 2), i32(3, 4)), (table, i32(0, 1), i32(3, 4)), (table, i32(0, 1, 2), i32(3)),
                (table.t().contiguous().t(), i32(0, 1, 2), i32(3, 4)), (table[0], i32(0, 1, 2), i32(3, 4)),
                (torch.zeros(2, 8, dtype=torch.int32)[:, :4], i32(0, 1, 2), i32(3, 4)),
                (table, i32(0, 0, 1, 1, 2, 2)[::2], i32(3, 4))]:
        with pytest.raises(ValueError):
            kv8.Batch8(*bad, 2)
    with pytest.raises(KsError):
        kv8.Cache8(4, 64, 8, 96, device="cpu")
    with pytest.raises(ValueError):
        kv8.Cache8(4, 64, 8, 128, data=torch.zeros(100, dtype=torch.uint8))
    c = kv8.Cache8(4, 64, 8, 128, device="cpu")
    assert c.data.numel() == c.nbytes == 4 * 8 * 4 * 4128
    with pytest.raises(KsError):
        c.attention_workspace(12, 1, 1)


def test_more_tiles_than_a_call_counts(lib):
    """Rows times tokens past what 32 bits count are refused."""
    from paper_2602_20217_gb300 import knapspec as ks
    cache, batch, rows, attn = good(ks)
    cache.page_tokens, batch.table_ld, batch.n_rows = 1 << 20, 1023, 2000
    assert lib.ks_kv8_attention(C.byref(cache), C.byref(batch), C.byref(attn), None) == ks.KS_ERR_UNSUPPORTED
    assert "too much for one call" in lib.ks_last_error().decode()


def test_longest_sequence(lib):
    """Page tables of up to 2^30 tokens."""
    from paper_2602_20217_gb300 import knapspec as ks
    cache, batch, rows, attn = good(ks)
    batch.n_rows = 0
    batch.table_ld = 1 << 24
    assert lib.ks_kv8_append(C.byref(cache), C.byref(batch), C.byref(rows), None) == 0
    batch.table_ld += 1
    for status in (lib.ks_kv8_append(C.byref(cache), C.byref(batch), C.byref(rows), None),
                   lib.ks_kv8_attention(C.byref(cache), C.byref(batch), C.byref(attn), None),
                   lib.ks_kv8_read(C.byref(cache), C.byref(batch), A, A, 1, 1024, 128, None)):
        assert status == ks.KS_ERR_INVALID_ARG
