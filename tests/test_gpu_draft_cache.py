"""Drafts over the 8-bit draft cache:

* the copy holds, byte for byte, what the oracle makes of the rows in the
  model's cache, whichever call drafted, after verifies, rewinds and masks that
  skipped a layer;
* the draft's logits are the oracle's over the decoded copy, within the bf16
  logit tolerance of 2e-2;
* the target's output does not change (Sec. 2.1, lossless), nor do drafts once
  the copy is taken away."""
import numpy as np
import pytest

from helpers import need_gpu, oracle_model, rel_err
from oracle import decoder as D
from oracle import kv8 as O

pytestmark = pytest.mark.gpu

PAGE = 256
MAX_SEQ = 640


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()


def _shape(hd=128, hq=8, hk=2, L=2):
    from paper_2602_20217_gb300.configs import ModelShape
    return ModelShape("draft-cache", L, 512, hq, hk, hd, 1368, 2000, qk_norm=hd == 128, dtype="bf16",
                      rope_theta=500000.0)


def _model(shape, prompt_len, cache=True, max_seq=MAX_SEQ):
    from paper_2602_20217_gb300 import synth
    from paper_2602_20217_gb300.model import Model
    m = Model(shape, max_seq=max_seq)
    if cache:
        m.draft_cache()
    m.prefill(synth.prompt_tokens(shape, prompt_len, seed=1))
    return m


def _records(m, layer):
    """[hk][blocks][bytes] of a layer's copy, the pages in order."""
    from paper_2602_20217_gb300 import knapspec as ks
    sh, pages = m.shape, -(-m.cfg.max_seq // PAGE)
    nbytes = ks.ks_kv8_bytes(pages, PAGE, sh.n_kv_heads, sh.head_dim)
    at = layer * (-(-nbytes // 256) * 256)
    raw = m.draft_memory[at:at + nbytes].cpu().numpy().reshape(pages, sh.n_kv_heads, PAGE // 16, -1)
    return raw.transpose(1, 0, 2, 3).reshape(sh.n_kv_heads, pages * PAGE // 16, -1)


def _check_copy(m, layer, p, n):
    """Positions 0 .. p were taken with block p / 16 in one piece, the n - 1 after them one by one."""
    sh = m.shape
    K, V = (m.kv(layer, 0, p + n, w).astype(np.float64) for w in "kv")
    got = _records(m, layer)
    k8, v8 = np.zeros_like(K), np.zeros_like(V)
    for h in range(sh.n_kv_heads):
        for b in range((p + n + 15) // 16):
            lo = 16 * b
            first = min(lo + 16, max(p + 1, lo + 1))
            block = O.append_block(None, 0, K[h, lo:first], V[h, lo:first])
            for t in range(first, min(lo + 16, p + n)):
                block = O.append_block(block, t - lo, K[h, t:t + 1], V[h, t:t + 1])
            want = O.pack_record(*block)
            used = 32 * sh.head_dim + 8
            assert np.array_equal(got[h, b][:used], want[:used]), (layer, h, b)
            e = min(16, p + n - lo)
            k8[h, lo:lo + e] = (O.VALUES[block[0]] * block[2])[:e]
            v8[h, lo:lo + e] = (O.VALUES[block[1]] * block[3])[:e]
    return k8, v8


def _draft(m, how, mask, gamma):
    from paper_2602_20217_gb300 import knapspec as ks
    if how == "dynamic":
        return m.draft_dynamic(mask, gamma, 0.0)[2]
    if how == "sample":
        return m.draft_sample(mask, gamma, ks.sampling(0.7, 50, 0.95, seed=3), 5)
    return m.draft(mask, gamma)


@pytest.mark.parametrize("how", ["greedy", "dynamic", "sample"])
@pytest.mark.parametrize("hd", [64, 128])
def test_copy_follows_the_cache(hd, how):
    m = _model(_shape(hd, L=3), 250)           # the drafts cross a page
    masks = [np.array(x, np.uint8) for x in ([1, 1, 1, 1, 1, 1], [1, 0, 0, 1, 1, 1], [0, 1, 1, 1, 1, 0],
                                             [1, 1, 1, 0, 1, 1])]
    for step, mask in enumerate(masks):
        p, _ = m.position()
        drafts = _draft(m, how, mask, 6)
        assert len(drafts) == 6
        for l in range(3):
            if mask[2 * l]:
                _check_copy(m, l, p, 6)
        m.verify(np.asarray(drafts, np.int32), 6)   # as given tokens: greedy acceptance
    m.rewind()
    p, _ = m.position()
    assert p == 250
    _draft(m, how, masks[0], 3)
    for l in range(3):
        _check_copy(m, l, p, 3)
    m.close()


def _oracle_logits(cfg, w, k8, v8, token, pos, mask):
    """One row through f^(S) with attention over given caches that hold the row itself already."""
    x = w["embed"][[token]].astype(np.float64)
    at = np.array([pos])
    hq, hd = cfg.n_q_heads, cfg.head_dim
    for i in range(2 * cfg.n_layers):
        lw = w["layers"][i // 2]
        if not mask[i]:
            continue
        if i % 2:
            x = D.mlp_sublayer(cfg, lw, x)
            continue
        q = (D.rms_norm(x, lw["attn_norm"], cfg.rms_eps) @ lw["w_qkv"].T)[:, :hq * hd].reshape(1, hq, hd)
        if cfg.qk_norm:
            q = D.rms_norm(q, lw["q_norm"], cfg.rms_eps)
        o = D.gqa_attention(D.rope(q, at, cfg.rope_theta), k8[i // 2], v8[i // 2], at)
        x = x + o.reshape(1, -1) @ lw["w_o"].T
    return D.final_logits(cfg, w, x)


# head groups of both row counts that a model has
@pytest.mark.parametrize("hd,hq,hk", [(128, 8, 2), (64, 8, 2), (128, 16, 1), (64, 32, 2)])
@pytest.mark.parametrize("n", [1, 16, 300])
def test_logits_over_the_decoded_copy(hd, hq, hk, n):
    shape = _shape(hd, hq, hk)
    m = _model(shape, n)
    cfg, w = oracle_model(shape, seed=0)
    for mask in ([1, 1, 1, 1], [0, 1, 1, 0]):
        p, pending = m.position()
        m.draft(np.array(mask, np.uint8), 1)
        copies = [_check_copy(m, l, p, 1) if mask[2 * l] else (None, None) for l in range(2)]
        ref = _oracle_logits(cfg, w, [c[0] for c in copies], [c[1] for c in copies], pending, p, mask)
        assert rel_err(m.logits(1), ref) < 2e-2
        m.verify(None, 1)
    m.close()


@pytest.mark.parametrize("kind", ["full", "skips", "dynamic", "knapsack"])
def test_target_output_is_unchanged(kind):
    from paper_2602_20217_gb300 import knapspec as ks
    shape = _shape(L=4)
    m = _model(shape, 300)
    want = m.decode_greedy(60)
    m.rewind()
    args = {"full": dict(mask=np.ones(8, np.uint8)),
            "skips": dict(mask=np.array([1, 1, 0, 1, 1, 0, 1, 1], np.uint8)),
            "dynamic": dict(mask=np.ones(8, np.uint8), tau_conf=0.02),
            "knapsack": dict(latency=ks.latency(0, 0.279, 0.735e-4, 0.279), resolve_every=4)}[kind]
    out = m.generate(60, 4, **args)
    tokens = out[0] if isinstance(out, tuple) else out
    assert np.array_equal(np.asarray(tokens)[:60], want)
    m.close()


def test_same_draft_again_and_after_a_rewind():
    m = _model(_shape(), 123)
    mask = np.ones(4, np.uint8)
    first, logits = list(m.draft(mask, 5)), m.logits(1)
    assert list(m.draft(mask, 5)) == first and np.array_equal(m.logits(1), logits)
    m.verify(None, 5)
    m.draft(mask, 7)
    m.rewind()
    assert list(m.draft(mask, 5)) == first and np.array_equal(m.logits(1), logits)
    m.decode_greedy(20)                         # rewrites the positions behind the prompt
    m.rewind()
    assert list(m.draft(mask, 5)) == first and np.array_equal(m.logits(1), logits)
    m.close()


def test_stopped_passes_leave_no_gap():
    """Passes after the dynamic exit write nothing; the next draft takes their positions again."""
    m = _model(_shape(), 40)
    mask = np.ones(4, np.uint8)
    for _ in range(4):
        p, _ = m.position()
        n, _, _ = m.draft_dynamic(mask, 6, 2.0)     # stops after one token
        assert n == 1
        m.verify(None, 6)
        p, _ = m.position()
        m.draft(mask, 5)
        for l in range(2):
            _check_copy(m, l, p, 5)
    m.close()


def test_without_it_nothing_changes():
    shape, mask = _shape(), np.array([1, 1, 0, 1], np.uint8)
    plain = _model(shape, 200, cache=False)
    m = _model(shape, 200)
    want = list(plain.draft(mask, 4))
    logits = plain.logits(1)
    m.draft(mask, 4)
    assert not np.array_equal(m.logits(1), logits)  # the 8-bit copy was read
    m.draft_cache(False)
    assert list(m.draft(mask, 4)) == want and np.array_equal(m.logits(1), logits)
    m.draft_cache()                                  # and back, in the middle of a sequence
    m.draft(mask, 4)
    _check_copy(m, 0, 200, 4)
    plain.close()
    m.close()


def test_refusals():
    import torch
    from paper_2602_20217_gb300 import knapspec as ks
    from paper_2602_20217_gb300.configs import TINY
    from paper_2602_20217_gb300.model import Model
    lib = ks.load()
    m = _model(_shape(), 20, cache=False)
    n = ks.ks_draft_cache_bytes(m.cfg)
    mem = torch.empty(n + 256, dtype=torch.uint8, device="cuda")
    assert lib.ks_draft_cache(m.h, mem.data_ptr(), n - 1) == ks.KS_ERR_WORKSPACE
    assert lib.ks_draft_cache(m.h, mem.data_ptr() + 16, n) == ks.KS_ERR_INVALID_ARG
    m.close()
    tiny = Model(TINY, max_seq=64)
    assert lib.ks_draft_cache(tiny.h, mem.data_ptr(), n) == ks.KS_ERR_UNSUPPORTED
    with pytest.raises(ks.KsError):
        tiny.draft_cache()
    tiny.close()


@pytest.mark.parametrize("kind", ["tpt", "dp"])
def test_target_output_under_the_selection_stages(kind):
    """The selection stages run between drafts; the DP one writes over the history's rows and puts them back."""
    from paper_2602_20217_gb300 import knapspec as ks
    m = _model(_shape(L=4), 300)
    want = m.decode_greedy(40)
    m.rewind()
    args = {"tpt": dict(latency=ks.latency(0, 0.279, 0.735e-4, 0.279), resolve_every=2, tpt=(4, 5)),
            "dp": dict(latency=ks.latency(1, units=[2, 1] * 4), resolve_every=2, dp=(5, 0.5, 16, 8))}[kind]
    out, stats, _ = m.generate(40, 4, **args)
    assert np.array_equal(np.asarray(out)[:40], want)
    m.close()


def test_sampled_jobs_repeat():
    """The same seed gives the same sampled tokens again; drafts are taken from the copy."""
    from paper_2602_20217_gb300 import knapspec as ks
    m = _model(_shape(), 100)
    samp = ks.sampling(0.7, 50, 0.95, seed=9)
    first, _, _ = m.generate(40, 4, mask=np.ones(4, np.uint8), sampling=samp)
    m.rewind()
    again, _, _ = m.generate(40, 4, mask=np.ones(4, np.uint8), sampling=samp)
    assert np.array_equal(first, again)
    assert first.min() >= 0 and first.max() < 2000
    m.close()
