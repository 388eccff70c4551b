"""The 8-bit draft cache without a GPU: its size and the refusals that need no model."""
import shutil

import pytest


@pytest.fixture(scope="module")
def ks():
    import os
    if shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"):
        pytest.skip("nvcc not available")
    from paper_2602_20217_gb300 import build, knapspec
    build.build()
    knapspec.load()
    return knapspec


@pytest.mark.parametrize("max_seq", [17, 256, 4396, 65836])
def test_bytes(ks, max_seq):
    from paper_2602_20217_gb300.configs import LLAMA3_8B
    n = ks.ks_draft_cache_bytes(ks.make_config(LLAMA3_8B, max_seq))
    pages = -(-max_seq // 256)
    records = LLAMA3_8B.n_layers * ks.ks_kv8_bytes(pages, 256, LLAMA3_8B.n_kv_heads, LLAMA3_8B.head_dim)
    # the records, three words a position and a fixed workspace
    assert records < n < records + 16 * max_seq + (4 << 20)


def test_no_bytes_for_other_models(ks):
    from paper_2602_20217_gb300.configs import LLAMA3_8B, TINY
    assert ks.ks_draft_cache_bytes(ks.make_config(TINY, 512)) == 0          # fp32
    cfg = ks.make_config(LLAMA3_8B, 512)
    cfg.head_dim = 96
    assert ks.ks_draft_cache_bytes(cfg) == 0


def test_null_model(ks):
    assert ks.load().ks_draft_cache(None, None, 0) == ks.KS_ERR_INVALID_ARG
    assert "null model" in ks.load().ks_last_error().decode()
    assert ks.load().ks_draft_cache_bytes(None) == 0
