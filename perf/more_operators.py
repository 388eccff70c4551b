"""Operators around several samples of one prompt and a cache that is kept small, as measurable cases.

A case names an operator (``op``) and its sizes:

``logprobs``  log probabilities of given tokens under rows of logits, with the
              rows' entropies and their top alternatives;
``shared``    causal attention over the 8-bit paged cache for sequences that
              come in groups with a common beginning, read once for a group;
``weights``   the attention weight that every cached token receives from the
              batch's rows, added to what it received before;
``evict``     keep a sequence's first, most recent and heaviest tokens, head
              by head, in fresh pages of the cache, and read them back.

Heads are the configured decoders' (Llama-3-8B, Qwen3-32B, the tiny decoder)
and the tests' small ones, vocabularies the configured ones and odd ones, and
contexts those of the configured workloads and ragged ones below.

The cache is ``[page][KV head][block of 16 tokens]`` records of 32 head_dim +
32 bytes: key codes ``[2][head_dim / 16][8 tokens][16]``, value codes
``[head_dim][16]`` with token t at byte ``4 ((t % 8) / 2) + 2 (t / 8) + t % 2``,
then the key scale and the value scale as fp32 powers of two.  Codes are e4m3.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BLOCK = 16
HEADS = {"llama8b": (32, 8, 128), "qwen32b": (64, 8, 128), "tiny": (4, 2, 64), "small64": (8, 2, 64),
         "small128": (8, 2, 128), "wide": (12, 4, 128)}


# ------------------------------------------------------------------ cases
def listed():
    return [
        # The token that a decode step of the 8B decoder chose, with twenty alternatives: all latency.
        {"name": "logprobs_token_8b", "op": "logprobs", "rows": 1, "vocab": 128256, "ld": 128256, "dtype": "f32",
         "tokens": 1, "top": 20, "temperature": 1.0, "banned": False},
        # A serving batch in bf16 with an odd vocabulary out of a padded matrix, sampled at 0.7, some words banned.
        {"name": "logprobs_batch_bf16", "op": "logprobs", "rows": 251, "vocab": 100277, "ld": 100352,
         "dtype": "bf16", "tokens": 2, "top": 5, "temperature": 0.7, "banned": True},
        # A prompt that is scored: the tokens' own probabilities and the best alternative.
        {"name": "logprobs_prompt_32b", "op": "logprobs", "rows": 1500, "vocab": 151936, "ld": 151936,
         "dtype": "f32", "tokens": 1, "top": 1, "temperature": 1.0, "banned": False},
        # Four samples of a short prompt.
        {"name": "shared_few", "op": "shared", "heads": "llama8b", "page": 64, "groups": 1, "seqs": 4,
         "shared_lo": 4096, "shared_hi": 4096, "tail_lo": 40, "tail_hi": 300, "rows_lo": 1, "rows_hi": 1},
        # Sixty-four samples behind a 16k prompt.
        {"name": "shared_64", "op": "shared", "heads": "llama8b", "page": 64, "groups": 1, "seqs": 64,
         "shared_lo": 16384, "shared_hi": 16384, "tail_lo": 100, "tail_hi": 1000, "rows_lo": 1, "rows_hi": 1},
        # Several prompts, each with drafts of its samples to verify; ragged beginnings, small pages.
        {"name": "shared_groups", "op": "shared", "heads": "qwen32b", "page": 16, "groups": 5, "seqs": 12,
         "shared_lo": 700, "shared_hi": 9000, "tail_lo": 20, "tail_hi": 900, "rows_lo": 1, "rows_hi": 6},
        # The tokens of a serving batch's decode step add to what the cache's tokens have received.
        {"name": "weights_batch", "op": "weights", "heads": "llama8b", "page": 64, "seqs": 24, "len_lo": 500,
         "len_hi": 16000, "rows_lo": 1, "rows_hi": 1, "decay": 1.0},
        # The last 64 rows of a 32k prompt decide what it may forget.
        {"name": "weights_window", "op": "weights", "heads": "qwen32b", "page": 128, "seqs": 1, "len_lo": 32768,
         "len_hi": 32768, "rows_lo": 64, "rows_hi": 64, "decay": 0.0},
        # A prompt's chunk behind 6k cached tokens, every row counted, older weight fading.
        {"name": "weights_chunk", "op": "weights", "heads": "llama8b", "page": 64, "seqs": 1, "len_lo": 8150,
         "len_hi": 8150, "rows_lo": 2001, "rows_hi": 2001, "decay": 0.9},
        # A cache of the tiny decoder is cut to 200 tokens.
        {"name": "evict_tiny", "op": "evict", "heads": "tiny", "page": 16, "seqs": 1, "len_lo": 251, "len_hi": 251,
         "keep": 0.8, "first": 4, "recent": 32},
        # A 64k prompt of the 32B decoder is cut to a tenth.
        {"name": "evict_64k", "op": "evict", "heads": "qwen32b", "page": 64, "seqs": 1, "len_lo": 65537,
         "len_hi": 65537, "keep": 0.1, "first": 4, "recent": 512},
        # A ragged batch is cut to half.
        {"name": "evict_batch", "op": "evict", "heads": "llama8b", "page": 32, "seqs": 24, "len_lo": 300,
         "len_hi": 12000, "keep": 0.5, "first": 0, "recent": 100},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "shared", "weights", "evict"])
    if op == "logprobs":
        vocab = _log_int(rng, 200, 262144)
        dtype = rng.choice(["f32", "bf16"])
        rows = _log_int(rng, 1, max(1, min(4000, 200_000_000 // vocab)))
        return {"op": op, "rows": rows, "vocab": vocab, "ld": vocab + rng.choice([0, 0, 1, 7, 64]), "dtype": dtype,
                "tokens": rng.randint(1, 4), "top": rng.choice([0, 1, 2, 5, 20, 33, 64]),
                "temperature": rng.choice([1.0, 1.0, 0.7, 1.3]), "banned": rng.random() < 0.3}
    case = {"op": op, "heads": rng.choice(sorted(HEADS)), "page": rng.choice([16, 32, 48, 64, 128, 256])}
    if op == "shared":
        groups = _log_int(rng, 1, 8)
        seqs = _log_int(rng, 1, 96 // groups)
        shared = _log_int(rng, case["page"], 20000 // groups)
        tail = _log_int(rng, 8, max(8, min(4000, 30000 // (groups * seqs))))
        case.update(groups=groups, seqs=seqs, shared_lo=max(case["page"], int(shared * rng.uniform(0.2, 1.0))),
                    shared_hi=shared, tail_lo=max(8, int(tail * rng.uniform(0.1, 1.0))), tail_hi=tail, rows_lo=1,
                    rows_hi=1 if rng.random() < 0.5 else rng.randint(2, 8))
        return case
    if op == "weights":
        case["decay"] = rng.choice([0.0, 0.9, 1.0])
        if rng.random() < 0.3:                       # a prompt's window or chunk
            seqs = rng.randint(1, 4)
            rows = _log_int(rng, 16, 1600 // seqs)
            hi = rows + _log_int(rng, 1, 5000)
            case.update(seqs=seqs, len_lo=max(1, int(hi * rng.uniform(0.6, 1.0))), len_hi=hi,
                        rows_lo=max(1, int(rows * rng.uniform(0.3, 1.0))), rows_hi=rows)
            return case
        seqs = _log_int(rng, 1, 64)
        hi = min(_log_int(rng, 40, 65536), 200000 // seqs)
        case.update(seqs=seqs, len_lo=max(1, int(hi * rng.uniform(0.1, 1.0))), len_hi=hi, rows_lo=1,
                    rows_hi=1 if rng.random() < 0.5 else rng.randint(2, 16))
        return case
    seqs, keep = _log_int(rng, 1, 64), rng.uniform(0.05, 1.0)
    hi = min(_log_int(rng, 40, 65536), int(40000 / keep) // seqs)
    case.update(seqs=seqs, len_lo=max(1, int(hi * rng.uniform(0.1, 1.0))), len_hi=hi, keep=keep,
                first=rng.choice([0, 1, 4, 16]), recent=rng.choice([0, 1, 32, 100, 500]))
    return case


def _offsets(counts):
    o = [0]
    for c in counts:
        o.append(o[-1] + c)
    return o


class _Sizes:
    """Lengths, row counts and pages of a case's sequences, from the case alone."""

    def __init__(self, case):
        r = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
        page = case["page"]
        if case["op"] == "shared":
            n = case["groups"] * case["seqs"]
            common = [_log_int(r, case["shared_lo"], case["shared_hi"]) for _ in range(case["groups"])]
            common[r.randrange(len(common))] = case["shared_hi"]
            self.shared = [c // page * page for c in common]
            tails = [_log_int(r, case["tail_lo"], case["tail_hi"]) for _ in range(n)]
            tails[r.randrange(n)] = case["tail_hi"]
            self.lens = [self.shared[s // case["seqs"]] + t for s, t in enumerate(tails)]
            self.rows = [min(t, r.randint(case["rows_lo"], case["rows_hi"])) for t in tails]
        else:
            n = case["seqs"]
            self.lens = [_log_int(r, case["len_lo"], case["len_hi"]) for _ in range(n)]
            self.lens[r.randrange(n)] = case["len_hi"]
            if case["op"] == "weights":
                self.rows = [min(x, r.randint(case["rows_lo"], case["rows_hi"])) for x in self.lens]
            else:
                self.keep = [max(1, int(x * case["keep"])) for x in self.lens]
                self.kept = [min(x, k) for x, k in zip(self.lens, self.keep)]
                self.rows = [1] * n
        self.n = n
        self.pages = [-(-x // page) for x in self.lens]


# ----------------------------------------------------------------- inputs
def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _logits(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, vocab, ld = case["rows"], case["vocab"], case["ld"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    full = torch.empty(rows, ld, dtype=dt, device="cuda")
    step = max(1, (1 << 26) // ld)
    for a in range(0, rows, step):                   # a broad floor of scores and a few words that stand out
        x = torch.randn(min(step, rows - a), ld, generator=g, device="cuda") * 2.2
        at = torch.randint(0, vocab, (x.shape[0], 12), generator=g, device="cuda")
        x.scatter_add_(1, at, torch.rand(at.shape, generator=g, device="cuda") * 14)
        if case["banned"]:
            x.masked_fill_(torch.rand(ld, generator=g, device="cuda") < 0.02, -math.inf)
        full[a:a + step] = x
    logits = full[:, :vocab]
    tokens = torch.randint(0, vocab, (rows, case["tokens"]), generator=g, device="cuda")
    likely = torch.rand(rows, generator=g, device="cuda") < 0.7
    tokens[:, 0] = torch.where(likely, logits.max(1).indices, tokens[:, 0])
    return {"case": dict(case), "logits": logits, "tokens": tokens.int()}


def prepare(case, seed):
    if case["op"] == "logprobs":
        st = _logits(case, seed)
        if own:                                      # where a serving loop has the results
            from paper_2602_20217_gb300 import logprobs
            st["out"] = logprobs.empty(case["rows"], case["tokens"], case["top"])
        return st
    z = _Sizes(case)
    hq, hk, hd = HEADS[case["heads"]]
    page, n, op = case["page"], z.n, case["op"]
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    fresh = [-(-k // page) for k in z.kept] if op == "evict" else []
    n_pages, bpp = sum(z.pages) + sum(fresh) + 3, page // BLOCK
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    at = 0

    def take(counts):
        nonlocal at
        table = torch.zeros(len(counts), max(counts), dtype=torch.int32, device="cuda")
        for s, c in enumerate(counts):
            table[s, :c] = order[at:at + c]
            at += c
        return table

    table = take(z.pages)
    if op == "shared":                               # a group's sequences begin on the same pages
        for s in range(n):
            common = z.shared[s // case["seqs"]] // page
            table[s, :common] = table[s // case["seqs"] * case["seqs"], :common]
    rec = 2 * BLOCK * hd + 32
    data = torch.zeros(n_pages, hk, bpp, rec, dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 28) // (hk * bpp * rec * 4))
    for a in range(0, n_pages, step):                # codes of a block fill the type's upper binades
        d = data[a:a + step]
        x = randn(*d.shape[:3], 2 * BLOCK * hd) * 96
        d[..., :-32] = x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    e = torch.randint(-8, -5, (n_pages, hk, bpp, 2), generator=g, device="cuda")
    data[..., -32:-24] = (e.int() + 127 << 23).view(torch.uint8)
    st = {"case": dict(case), "sizes": z, "heads": (hq, hk, hd), "data": data, "table": table,
          "lengths": _i32(z.lens), "offsets": _i32(_offsets(z.rows)), "n_rows": sum(z.rows), "scale": hd ** -0.5}
    most = table.shape[1] * page
    if op == "evict":
        # weight gathers on few tokens; some have never received any, some the same
        score = torch.exp(randn(n, hk, most) * 2.5 - 4)
        odd = torch.rand(n, hk, most, generator=g, device="cuda")
        score = torch.where(odd < 0.05, torch.zeros_like(score), torch.where(odd < 0.1, score.round(decimals=2), score))
        st["scores"], st["keep"] = score, _i32(z.keep)
        st["new_table"] = take(fresh)
        room = st["new_table"].shape[1] * page
        st["kept"] = torch.full((n, hk, room), -1, dtype=torch.int32, device="cuda")
        st["new_scores"] = torch.zeros(n, hk, room, device="cuda")
        st["new_lengths"] = torch.zeros(n, dtype=torch.int32, device="cuda")
        rows = sum(z.kept)
        st["k"] = torch.empty(rows, hk, hd, dtype=torch.bfloat16, device="cuda")
        st["v"] = torch.empty_like(st["k"])
        st["kept_offsets"] = _i32(_offsets(z.kept))
    else:
        st["q"] = (randn(st["n_rows"], hq, hd) * 2).to(torch.bfloat16)
    if op == "shared":
        st["group_offsets"] = _i32([i * case["seqs"] for i in range(case["groups"] + 1)])
        st["shared"] = _i32(z.shared)
        st["out"] = torch.empty(st["n_rows"], hq, hd, dtype=torch.bfloat16, device="cuda")
    if op == "weights":
        st["scores"] = torch.exp(randn(n, hk, most) - 5)
        st["out"] = torch.zeros(n, hk, most, device="cuda")
        st["lse"] = _lse(st)
    if own:                                          # the handles that a serving loop keeps
        from paper_2602_20217_gb300 import kv8
        st["cache"] = kv8.Cache8(n_pages, page, hk, hd, data=data)
        st["batch"] = kv8.Batch8(table, st["offsets"], st["lengths"], st["n_rows"])
        if op == "shared":
            st["groups"] = kv8.Shared8(st["group_offsets"], st["shared"])
            st["work"] = st["cache"].attention_workspace(hq, n, st["n_rows"], shared=st["groups"])
        if op == "evict":
            st["new_batch"] = kv8.Batch8(st["new_table"], st["kept_offsets"], st["new_lengths"], sum(z.kept))
    return st


def _lse(st):
    """What the attention of the same rows returns beside its output: the logarithm of each row's sum."""
    hq, hk, _ = st["heads"]
    z, got, at = st["sizes"], [], 0
    for s, (length, r) in enumerate(zip(z.lens, z.rows)):
        k = _dense(st, torch.tensor([s], device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda"),
                   -(-length // BLOCK))[0][0, :, :length]
        seen = torch.arange(length, device="cuda") <= torch.arange(length - r, length, device="cuda")[:, None]
        q = st["q"][at:at + r].float()
        got.append(torch.stack([(q[:, h] @ k[h * hk // hq].T * st["scale"]).masked_fill_(~seen, -math.inf)
                                .double().logsumexp(-1).float() for h in range(hq)], 1))
        at += r
    return torch.cat(got)


# ------------------------------------------------------------ plain forms
def _token_at(t):
    """Byte of token t in a row of value codes."""
    return 4 * ((t % 8) // 2) + 2 * (t // 8) + t % 2


def _dense(st, seqs, start, blocks):
    """Keys and values [sequence][KV head][token][hd] of so many blocks of sequences seqs from blocks start on; those
    behind a sequence's pages are some page's."""
    _, hk, hd = st["heads"]
    bpp = st["case"]["page"] // BLOCK
    b = (start[:, None] + torch.arange(blocks, device="cuda")).clamp(max=st["table"].shape[1] * bpp - 1)
    rec = st["data"][st["table"][seqs[:, None], b // bpp].long(), :, b % bpp]    # [sequence][block][head][bytes]
    sc = rec[..., -32:-24].contiguous().view(torch.float32)
    x = rec[..., :-32].view(torch.float8_e4m3fn).float()
    k = x[..., :BLOCK * hd].unflatten(-1, (2, hd // 16, 8, 16)).transpose(-3, -2).flatten(-5, -4)
    k = k.reshape(*rec.shape[:3], BLOCK, hd) * sc[..., :1, None]
    v = x[..., BLOCK * hd:].unflatten(-1, (hd, BLOCK))[..., _token_at(torch.arange(BLOCK, device="cuda"))]
    v = v.transpose(-1, -2) * sc[..., 1:, None]
    return [y.transpose(1, 2).reshape(len(seqs), hk, blocks * BLOCK, hd) for y in (k, v)]


def _padded(x, offsets, most):
    """Rows offsets[i] .. offsets[i + 1] of x as [i][row], and which of them there are."""
    i = offsets.long()[:-1, None] + torch.arange(most, device="cuda")
    return x[i.clamp(max=len(x) - 1)], i < offsets.long()[1:, None]


def _logprobs(st):
    case, x = st["case"], st["logits"].float()
    top = x.amax(1, keepdim=True)
    d = (x - top) / case["temperature"]
    p = d.exp()
    total = p.sum(1, keepdim=True, dtype=torch.float64)           # a likely token's logarithm is next to 0
    mean = torch.where(p > 0, p * d, 0.0).sum(1, keepdim=True, dtype=torch.float64) / total
    log_total = total.log()
    got = {"logprobs": (d.gather(1, st["tokens"].long()) - log_total).float(),
           "entropy": (log_total - mean)[:, 0].float()}
    if case["top"]:
        n = min(case["top"], case["vocab"])
        order = x.sort(dim=1, descending=True, stable=True).indices[:, :n]
        got["top_ids"] = order.int()
        got["top_logprobs"] = (d.gather(1, order) - log_total).float()
    return got


def _shared(st):
    case, z = st["case"], st["sizes"]
    hq, hk, hd = st["heads"]
    per, G, page = case["seqs"], hq // hk, case["page"]
    first, seqs = torch.arange(0, z.n, per, device="cuda"), torch.arange(z.n, device="cuda")
    common = torch.tensor(z.shared, device="cuda")
    row_seq = torch.repeat_interleave(seqs, torch.tensor(z.rows, device="cuda"))
    group_rows = st["offsets"][::per]                                            # the groups' first rows
    q = (st["q"].float() * st["scale"]).view(-1, hk, G, hd)

    def part(k, v, q, unseen):
        """(maximum, sum, weighted values) of rows q [i][row][hk][G][hd] over their keys."""
        p = torch.einsum("irhgd,ihtd->irhgt", q, k).masked_fill_(unseen[:, :, None, None], -math.inf)
        m = p.amax(-1, keepdim=True).clamp(min=-1e30)
        p = p.sub_(m).exp_()
        return m, p.sum(-1, keepdim=True), torch.einsum("irhgt,ihtd->irhgd", p, v)

    # what a group has in common, for all of its rows
    k, v = _dense(st, first, torch.zeros_like(first), max(1, max(z.shared) // BLOCK))
    x, there0 = _padded(q, group_rows, int(max(sum(z.rows[i:i + per]) for i in range(0, z.n, per))))
    unseen = (torch.arange(k.shape[2], device="cuda") >= common[:, None])[:, None].expand(-1, x.shape[1], -1)
    m0, l0, o0 = (y[there0] for y in part(k, v, x, unseen))
    # what a sequence has by itself
    own_len = st["lengths"].long() - common[seqs // per]
    k, v = _dense(st, seqs, common[seqs // per] // BLOCK, -(-int(max(x - z.shared[s // per] for s, x in enumerate(z.lens))) // BLOCK))
    x, there = _padded(q, st["offsets"], max(z.rows))
    pos = (own_len - st["offsets"].diff())[:, None] + torch.arange(max(z.rows), device="cuda")
    m1, l1, o1 = (y[there] for y in part(k, v, x, torch.arange(k.shape[2], device="cuda") > pos[..., None]))
    m = torch.maximum(m0, m1)
    f0, f1 = (m0 - m).exp(), (m1 - m).exp()
    st["out"].copy_(((o0 * f0 + o1 * f1) / (l0 * f0 + l1 * f1)).view(-1, hq, hd))
    return {"out": st["out"]}


def _weights(st):
    case, z = st["case"], st["sizes"]
    hq, hk, hd = st["heads"]
    seqs, most = torch.arange(z.n, device="cuda"), max(z.lens)
    k, _ = _dense(st, seqs, torch.zeros_like(seqs), -(-most // BLOCK))
    q, there = _padded(st["q"].float().view(-1, hk, hq // hk, hd), st["offsets"], max(z.rows))
    lse, _ = _padded(st["lse"].view(-1, hk, hq // hk, 1), st["offsets"], max(z.rows))
    start = (st["lengths"] - st["offsets"].diff())[:, None, None]
    t = torch.arange(k.shape[2], device="cuda")
    seen = there[..., None] & (t <= start + torch.arange(max(z.rows), device="cuda")[:, None])
    p = torch.einsum("irhgd,ihtd->irhgt", q, k).mul_(st["scale"]).sub_(lse).exp_()
    got = p.masked_fill_(~seen[:, :, None, None], 0.0).sum((1, 3))[..., :most]
    if case["decay"] != 0:
        got = got + torch.where(t[:most] < start, case["decay"] * st["scores"][..., :most], 0.0)
    inside = t[:most] < st["lengths"][:, None, None]
    st["out"][..., :most] = torch.where(inside, got, st["out"][..., :most])
    return {"scores": st["out"]}


def _scale_of(amax):
    """Smallest power of two with amax <= 448 times it (2^-126 at least)."""
    m, e = torch.frexp(amax)                         # amax = m 2^e, 0.5 <= m < 1
    e = e - 9 + (m > 0.875)
    return (torch.where(amax > 0, e.clamp(min=-126), -126).int() + 127 << 23).view(torch.float32)


def _evict(st):
    case, z = st["case"], st["sizes"]
    _, hk, hd = st["heads"]
    bpp, most, room = case["page"] // BLOCK, max(z.lens), max(z.kept)
    seqs, length = torch.arange(z.n, device="cuda"), st["lengths"].long()[:, None, None]
    n = torch.minimum(st["keep"].long()[:, None, None], length)
    recent = n.clamp(max=case["recent"])
    first = (n - recent).clamp(max=case["first"])
    t = torch.arange(most, device="cuda")
    score = torch.where((t < first) | (t >= length - recent), math.inf, st["scores"][..., :most])
    kept = score.masked_fill_(t >= length, -math.inf).sort(dim=2, descending=True, stable=True).indices[..., :room]
    there = torch.arange(room, device="cuda") < n                                # [sequence][1][place]
    kept = torch.where(there, kept, most).sort(2).values
    at = kept.clamp(max=most - 1)
    st["kept"][..., :room] = torch.where(there, kept.int(), st["kept"][..., :room])
    st["new_scores"][..., :room] = torch.where(there, st["scores"].gather(2, at), st["new_scores"][..., :room])
    st["new_lengths"].copy_(n[:, 0, 0])
    # blocks of 16 kept tokens
    nb = -(-room // BLOCK)
    b = torch.arange(nb, device="cuda")
    s, b = (b * BLOCK < n[:, 0]).nonzero().unbind(1)
    page, blk = st["new_table"][s, b // bpp].long(), b % bpp
    at = torch.nn.functional.pad(at, (0, nb * BLOCK - room))[..., None].expand(-1, -1, -1, hd)
    valid = torch.nn.functional.pad(there, (0, nb * BLOCK - room))[..., None]
    for i, (x, out) in enumerate(zip(_dense(st, seqs, torch.zeros_like(seqs), -(-most // BLOCK)), (st["k"], st["v"]))):
        x = x.gather(2, at).masked_fill_(~valid, 0.0).view(z.n, hk, nb, BLOCK, hd)
        scale = _scale_of(x.abs().amax((3, 4)))
        code = (x / scale[..., None, None]).to(torch.float8_e4m3fn)
        x = (code.float() * scale[..., None, None]).view(z.n, hk, nb * BLOCK, hd)[:, :, :room].transpose(1, 2)
        out.copy_(x[there[:, 0]])
        c = code.view(torch.uint8)[s, :, b]                                      # [block][head][16][hd]
        if i == 0:
            c = c.unflatten(2, (2, 8)).unflatten(4, (hd // 16, 16)).transpose(3, 4)
        else:                                                                    # byte of a row -> its token
            order = _token_at(torch.arange(BLOCK, device="cuda")).argsort()
            c = c[:, :, order].transpose(2, 3)
        st["data"][page, :, blk, i * BLOCK * hd:(i + 1) * BLOCK * hd] = c.flatten(2)
        c = scale[s, :, b][..., None].view(torch.uint8)
        st["data"][page, :, blk, 2 * BLOCK * hd + 4 * i:2 * BLOCK * hd + 4 * i + 4] = c
    return {n: st[n] for n in ("kept", "new_scores", "new_lengths", "k", "v")}


def run(state):
    st = state
    op, case = st["case"]["op"], st["case"]
    if not own:
        return {"logprobs": _logprobs, "shared": _shared, "weights": _weights, "evict": _evict}[op](st)
    if op == "logprobs":
        from paper_2602_20217_gb300 import logprobs
        got = logprobs.token_logprobs(st["logits"], st["tokens"], n_top=case["top"], temperature=case["temperature"],
                                      out=st["out"])
        return {n: x for n, x in got._asdict().items() if x is not None and (case["top"] or not n.startswith("top"))}
    if op == "shared":
        st["cache"].attention(st["batch"], st["q"], scale=st["scale"], out=st["out"], workspace=st["work"],
                              shared=st["groups"])
        return {"out": st["out"]}
    if op == "weights":
        st["cache"].attention_weights(st["batch"], st["q"], st["lse"], st["scores"], scale=st["scale"],
                                      decay=case["decay"], out=st["out"])
        return {"scores": st["out"]}
    st["cache"].evict(st["batch"], st["scores"], st["keep"], st["new_table"], st["new_lengths"], st["kept"],
                      new_scores=st["new_scores"], first=case["first"], recent=case["recent"])
    st["cache"].read(st["new_batch"], st["k"], st["v"])
    return {n: st[n] for n in ("kept", "new_scores", "new_lengths", "k", "v")}


# ------------------------------------------------------------------- work
def work(case):
    if case["op"] == "logprobs":
        n = case["rows"] * case["vocab"]
        top = min(case["top"], case["vocab"])
        return {"bytes": n * (2 if case["dtype"] == "bf16" else 4) + case["rows"] * (8 * case["tokens"] + 4 + 8 * top),
                "flops": 5 * n}
    z = _Sizes(case)
    hq, hk, hd = HEADS[case["heads"]]
    n = sum(z.rows)
    pairs = sum(r * (x - r) + r * (r + 1) // 2 for x, r in zip(z.lens, z.rows))
    if case["op"] == "shared":
        cached = sum(z.shared) + sum(x - z.shared[s // case["seqs"]] for s, x in enumerate(z.lens))
        return {"bytes": cached * hk * (2 * hd + 8 / BLOCK) + 2 * n * hq * hd * 2, "flops": 4 * hd * hq * pairs}
    if case["op"] == "weights":
        old = sum(x - r for x, r in zip(z.lens, z.rows)) if case["decay"] != 0 else 0
        return {"bytes": sum(z.lens) * hk * (hd + 4 / BLOCK + 4) + old * hk * 4 + n * hq * (2 * hd + 4),
                "flops": (2 * hd + 2) * hq * pairs}
    # scores and the kept tokens in; indexes, scores and codes out; codes in and values out once more
    kept = sum(z.kept)
    return {"bytes": sum(z.lens) * hk * 4 + kept * hk * (3 * 2 * hd + 2 * 2 * hd + 8), "flops": 0}


# --------------------------------------------------- the definition, 64 bits
def _e4m3_values():
    """The 256 values of the code: sign, four exponent bits (bias 7), three fraction bits."""
    out = []
    for c in range(256):
        e, f = c >> 3 & 15, c & 7
        v = math.nan if c & 127 == 127 else (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
        out.append(-v if c & 128 else v)
    return torch.tensor(out, dtype=torch.float64, device="cuda")


def _pow2(e):
    """2^e in 64 bits, from its bits."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _to_e4m3(x):
    """Nearest value of the code, ties to the even fraction."""
    e = torch.frexp(x.abs().clamp(min=2.0 ** -6)).exponent - 1
    ulp = _pow2(e - 3)
    return torch.round(x / ulp) * ulp


def _sequence(st, s, values):
    """[K, V][head][token][hd] of sequence s."""
    _, hk, hd = st["heads"]
    length, bpp = st["sizes"].lens[s], st["case"]["page"] // BLOCK
    t = torch.arange(length, device="cuda")
    rec = st["data"][st["table"][s, t // BLOCK // bpp].long(), :, t // BLOCK % bpp]      # [token][head][bytes]
    scale = rec[..., -32:-24].contiguous().view(torch.float32).double()
    d, i = torch.arange(hd, device="cuda"), t % BLOCK
    kb = (i[:, None] // 8 * (hd // 16) + d // 16) * 128 + i[:, None] % 8 * 16 + d % 16
    vb = BLOCK * hd + d * 16 + 4 * (i[:, None] % 8 // 2) + 2 * (i[:, None] // 8) + i[:, None] % 2
    kv = [values[rec.gather(2, b[:, None].expand(-1, hk, -1)).int()] * scale[..., j, None]
          for j, b in enumerate((kb, vb))]
    return torch.stack(kv).transpose(1, 2)


def exact(case, seed):
    if case["op"] == "logprobs":
        st = _logits(case, seed)
        got = {"logprobs": [], "entropy": [], "top_ids": [], "top_logprobs": []}
        n = min(case["top"], case["vocab"])
        for x, token in zip(st["logits"].split(64), st["tokens"].long().split(64)):
            lp = torch.log_softmax(x.double() / case["temperature"], 1)
            got["logprobs"].append(lp.gather(1, token))
            got["entropy"].append(torch.special.entr(lp.exp()).sum(1))
            if n:
                # whole numbers from the values themselves: larger first, then the lower place
                order = torch.argsort(x.double(), dim=1, descending=True, stable=True)[:, :n]
                got["top_ids"].append(order.int())
                got["top_logprobs"].append(lp.gather(1, order))
        return {k: torch.cat(v) for k, v in got.items() if v}
    st = prepare(case, seed)
    z = st["sizes"]
    hq, hk, hd = st["heads"]
    values = _e4m3_values()
    off = _offsets(z.rows)
    if case["op"] == "evict":
        got = {"kept": st["kept"].clone(), "new_scores": st["new_scores"].double(), "new_lengths": _i32(z.kept), "k": [], "v": []}
        for s, (length, n) in enumerate(zip(z.lens, z.kept)):
            recent = min(case["recent"], n)
            first = min(case["first"], n - recent)
            kv = _sequence(st, s, values)
            middle = st["scores"][s, :, first:length - recent]
            heavy = torch.argsort(-middle.double(), dim=1, stable=True)[:, :n - first - recent] + first
            ends = [i for i in range(length) if i < first or i >= length - recent]
            ends = torch.tensor(ends, dtype=torch.int64, device="cuda").expand(hk, -1)
            places = torch.cat((heavy, ends), 1).sort(1).values
            got["kept"][s, :, :n] = places.int()
            for h in range(hk):
                got["new_scores"][s, h, :n] = st["scores"][s, h, places[h]].double()
            x = torch.stack([kv[:, h, places[h]] for h in range(hk)], 1)         # [K, V][head][kept][hd]
            full = torch.zeros(2, hk, -(-n // BLOCK) * BLOCK, hd, dtype=torch.float64, device="cuda")
            full[:, :, :n] = x
            full = full.view(2, hk, -1, BLOCK * hd)
            m, e = torch.frexp(full.abs().amax(-1, keepdim=True) / 448)          # a power of two has m = 1 / 2
            sc = _pow2(torch.where(m > 0, e - (m == 0.5).int(), -126).clamp(min=-126))
            full = (_to_e4m3(full / sc) * sc).view(2, hk, -1, hd)[:, :, :n].transpose(1, 2)
            got["k"].append(full[0])
            got["v"].append(full[1])
        return {k: torch.cat(v) if isinstance(v, list) else v for k, v in got.items()}
    out, scores = [], st["out"].double() if case["op"] == "weights" else None
    for s, (length, r) in enumerate(zip(z.lens, z.rows)):
        kv = _sequence(st, s, values)
        q = st["q"][off[s]:off[s + 1]].double()
        seen = torch.arange(length, device="cuda") <= torch.arange(length - r, length, device="cuda")[:, None]
        o = []
        for h in range(hq):
            g = h * hk // hq
            x = (q[:, h] @ kv[0, g].T * st["scale"]).masked_fill_(~seen, -math.inf)
            if case["op"] == "shared":
                o.append(torch.softmax(x, -1) @ kv[1, g])
            else:
                scores[s, g, :length] += torch.exp(x - st["lse"][off[s]:off[s + 1], h, None].double()).sum(0)
        if case["op"] == "shared":
            out.append(torch.stack(o, 1))
        elif case["decay"] != 0:
            scores[s, :, :length - r] += case["decay"] * st["scores"][s, :, :length - r].double()
    return {"out": torch.cat(out)} if case["op"] == "shared" else {"scores": scores}
