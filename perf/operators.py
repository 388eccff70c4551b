"""The operators of the 8-bit paged key/value cache, as measurable cases.

A case names an operator (``op``) and its sizes:

``append``     rotate the new rows' keys (and queries), quantise keys and values
               to 8 bits with a scale per block of 16 tokens and head, write them
               into the sequences' pages, and read the touched blocks back;
``attention``  causal attention of the sequences' last rows over their pages;
``step``       what a decoder layer does with them: append, then attend with the
               rotated queries.

Shapes are the configured decoders' heads (Llama-3-8B, Qwen3-32B, the tiny
decoder) and the tests' small ones; contexts are those of the configured
workloads (4k, 32k, 64k, 128k) and ragged ones below.

The cache is ``[page][KV head][block of 16 tokens]`` records of 32 head_dim +
32 bytes: key codes ``[2][head_dim / 16][8 tokens][16]``, value codes
``[head_dim][16]`` with token t at byte ``4 ((t % 8) / 2) + 2 (t / 8) + t % 2``,
then the key scale and the value scale as fp32 powers of two.  Codes are e4m3.

Cached keys and values are drawn as normal values with a magnitude per block;
queries are scaled so that the attention is peaked, as a trained decoder's is.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BLOCK = 16
HEADS = {"llama8b": (32, 8, 128), "qwen32b": (64, 8, 128), "tiny": (4, 2, 64), "small64": (8, 2, 64),
         "small128": (8, 2, 128), "wide": (12, 4, 128)}
THETA = 500000.0


# ------------------------------------------------------------------ cases
def listed():
    return [
        # One decoded token of the 8B decoder goes into its cache: all latency.
        {"name": "append_one_8b", "op": "append", "heads": "llama8b", "page": 64, "seqs": 1, "len_lo": 4097,
         "len_hi": 4097, "rows_lo": 1, "rows_hi": 1, "dtype": "bf16"},
        # A serving batch after its verify passes: one to eleven accepted rows each, fp32 projections.
        {"name": "append_batch", "op": "append", "heads": "qwen32b", "page": 128, "seqs": 96, "len_lo": 300,
         "len_hi": 9000, "rows_lo": 1, "rows_hi": 11, "dtype": "f32"},
        # The 4k workload's prompt, whole.
        {"name": "append_prompt_4k", "op": "append", "heads": "llama8b", "page": 64, "seqs": 1, "len_lo": 4096,
         "len_hi": 4096, "rows_lo": 4096, "rows_hi": 4096, "dtype": "bf16"},
        # Several ragged prompts at once.
        {"name": "append_prompts", "op": "append", "heads": "qwen32b", "page": 32, "seqs": 9, "len_lo": 700,
         "len_hi": 9001, "rows_lo": 700, "rows_hi": 9001, "dtype": "bf16"},
        # The tiny decoder's token at a short context.
        {"name": "attn_tiny", "op": "attention", "heads": "tiny", "page": 16, "seqs": 1, "len_lo": 251,
         "len_hi": 251, "rows_lo": 1, "rows_hi": 1},
        # One token of the 8B decoder at the 4k workload.
        {"name": "attn_8b_4k", "op": "attention", "heads": "llama8b", "page": 64, "seqs": 1, "len_lo": 4099,
         "len_hi": 4099, "rows_lo": 1, "rows_hi": 1},
        # A draft token of the 32B decoder at 64k.
        {"name": "attn_32b_64k", "op": "attention", "heads": "qwen32b", "page": 128, "seqs": 1, "len_lo": 65537,
         "len_hi": 65537, "rows_lo": 1, "rows_hi": 1},
        # Five verify rows (gamma 4) of the 8B decoder at 128k.
        {"name": "attn_8b_128k_r5", "op": "attention", "heads": "llama8b", "page": 64, "seqs": 1,
         "len_lo": 131077, "len_hi": 131077, "rows_lo": 5, "rows_hi": 5},
        # A serving batch of single tokens over ragged contexts, small pages.
        {"name": "attn_batch", "op": "attention", "heads": "llama8b", "page": 16, "seqs": 64, "len_lo": 60,
         "len_hi": 16000, "rows_lo": 1, "rows_hi": 1},
        # A batch of verify passes of the paper's longest drafts (11 rows, eight query heads a KV head).
        {"name": "attn_verify_batch", "op": "attention", "heads": "qwen32b", "page": 128, "seqs": 24,
         "len_lo": 900, "len_hi": 16000, "rows_lo": 2, "rows_hi": 11},
        # A prompt's chunk behind 6k cached tokens: compute, not bytes.
        {"name": "attn_prompt_32b", "op": "attention", "heads": "qwen32b", "page": 64, "seqs": 1, "len_lo": 8150,
         "len_hi": 8150, "rows_lo": 2001, "rows_hi": 2001},
        # One layer's decode step of eight sequences around 32k.
        {"name": "step_32b_32k", "op": "step", "heads": "qwen32b", "page": 64, "seqs": 8, "len_lo": 30000,
         "len_hi": 32768, "rows_lo": 1, "rows_hi": 1, "dtype": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append", "attention", "attention", "attention", "attention", "step"])
    case = {"op": op, "heads": rng.choice(sorted(HEADS)), "page": rng.choice([16, 32, 48, 64, 128, 256])}
    seqs = _log_int(rng, 1, 128)
    if op == "append":
        rows = _log_int(rng, 1, 24000 // seqs)
        hi = rows + (0 if rng.random() < 0.5 else _log_int(rng, 1, 4000))
        case.update(seqs=seqs, len_lo=max(1, int(hi * rng.uniform(0.3, 1.0))), len_hi=hi,
                    rows_lo=max(1, int(rows * rng.uniform(0.1, 1.0))), rows_hi=rows,
                    dtype=rng.choice(["bf16", "f32"]))
        return case
    if op == "attention" and rng.random() < 0.2:      # a prompt's chunk
        seqs = rng.randint(1, 4)
        rows = _log_int(rng, 64, 2000 // seqs)
        hi = rows + _log_int(rng, 1, 6000)
        case.update(seqs=seqs, len_lo=max(1, int(hi * rng.uniform(0.6, 1.0))), len_hi=hi,
                    rows_lo=max(1, int(rows * rng.uniform(0.3, 1.0))), rows_hi=rows)
        return case
    hi = min(_log_int(rng, 40, 131072), 240000 // seqs)
    rows = 1 if rng.random() < 0.5 else rng.randint(2, 16)
    case.update(seqs=seqs, len_lo=max(1, int(hi * rng.uniform(0.1, 1.0))), len_hi=hi, rows_lo=1, rows_hi=rows)
    if op == "step":
        case["dtype"] = rng.choice(["bf16", "f32"])
    return case


def _lengths(case):
    """Lengths and row counts of the sequences, from the case alone."""
    r = random.Random("%d %d %d %d" % (case["seqs"], case["len_lo"], case["len_hi"], case["rows_hi"]))
    n = case["seqs"]
    lens = [_log_int(r, case["len_lo"], case["len_hi"]) for _ in range(n)]
    lens[r.randrange(n)] = case["len_hi"]
    rows = [min(x, r.randint(case["rows_lo"], case["rows_hi"])) for x in lens]
    if case["rows_lo"] == case["len_lo"] and case["rows_hi"] == case["len_hi"]:
        rows = list(lens)                            # whole prompts
    return lens, rows


# ----------------------------------------------------------------- inputs
def _table(positions, hd):
    j = torch.arange(hd // 2, dtype=torch.float64, device="cuda")
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * THETA ** (-2 * j / hd)
    return torch.stack((a.cos(), a.sin()), -1).float().contiguous()


def _offsets(counts):
    o = [0]
    for c in counts:
        o.append(o[-1] + c)
    return o


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    hq, hk, hd = HEADS[case["heads"]]
    lens, rows = _lengths(case)
    n, page = case["seqs"], case["page"]
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    per = [-(-x // page) for x in lens]
    n_pages, bpp = sum(per) + 3, page // BLOCK
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros(n, max(per), dtype=torch.int32, device="cuda")
    at = 0
    for s, c in enumerate(per):
        table[s, :c] = order[at:at + c]
        at += c
    rec = 2 * BLOCK * hd + 32
    data = torch.zeros(n_pages, hk, bpp, rec, dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 28) // (hk * bpp * rec * 4))
    for a in range(0, n_pages, step):                # codes of a block fill the type's upper binades
        d = data[a:a + step]
        x = randn(*d.shape[:3], 2 * BLOCK * hd) * 96
        d[..., :-32] = x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    e = torch.randint(-8, -5, (n_pages, hk, bpp, 2), generator=g, device="cuda")
    data[..., -32:-24] = torch.exp2(e.float()).view(torch.uint8)
    n_rows = sum(rows)
    st = {"case": dict(case), "data": data, "table": table, "lengths": _i32(lens),
          "offsets": _i32(_offsets(rows)), "n_rows": n_rows, "scale": hd ** -0.5}
    # rows as (sequence, place) for the plain form
    st["row_seq"] = torch.repeat_interleave(torch.arange(n, device="cuda"), torch.tensor(rows, device="cuda"))
    st["row_at"] = torch.arange(n_rows, device="cuda") - st["offsets"].long()[st["row_seq"]]
    if case["op"] != "attention":
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        qkv = randn(n_rows, hq + 2 * hk, hd)         # one row of projections, as a QKV product leaves it
        qkv[:, :hq] *= 2
        st["qkv"] = qkv.to(dt)
        st["rope"] = _table(max(lens), hd)
        st["q_out"] = torch.empty(n_rows, hq, hd, dtype=torch.bfloat16, device="cuda")
        # the touched blocks' tokens, old ones among them
        back = [x - (x - r) // BLOCK * BLOCK for x, r in zip(lens, rows)]
        st["back_offsets"], st["n_back"] = _i32(_offsets(back)), sum(back)
        st["back_seq"] = torch.repeat_interleave(torch.arange(n, device="cuda"), torch.tensor(back, device="cuda"))
        st["back_at"] = torch.arange(sum(back), device="cuda") - st["back_offsets"].long()[st["back_seq"]]
        st["k_back"] = torch.empty(sum(back), hk, hd, dtype=torch.bfloat16, device="cuda")
        st["v_back"] = torch.empty_like(st["k_back"])
    else:
        st["q"] = (randn(n_rows, hq, hd) * 2).to(torch.bfloat16)
    st["out"] = torch.empty(n_rows, hq, hd, dtype=torch.bfloat16, device="cuda")
    st["heads"], st["page"], st["max_rows"], st["max_len"] = (hq, hk, hd), page, max(rows), max(lens)
    if own:                                          # the handles that a serving loop keeps
        from paper_2602_20217_gb300 import kv8
        st["cache"] = kv8.Cache8(n_pages, page, hk, hd, data=data)
        st["batch"] = kv8.Batch8(table, st["offsets"], st["lengths"], n_rows)
        if "n_back" in st:
            st["back"] = kv8.Batch8(table, st["back_offsets"], st["lengths"], st["n_back"])
        st["work"] = st["cache"].attention_workspace(hq, n, n_rows)
    return st


# ------------------------------------------------------------ plain forms
def _token_at(t):
    """Byte of token t in a row of value codes."""
    return 4 * ((t % 8) // 2) + 2 * (t // 8) + t % 2


def _rotate(x, c, s):
    a, b = x.chunk(2, -1)
    return torch.cat((a * c - b * s, b * c + a * s), -1)


def _place(st, seq, pos):
    """(page, block of the page, token of the block) of tokens pos of sequences seq."""
    page = st["table"][seq, pos // st["page"]].long()
    return page, pos % st["page"] // BLOCK, pos % BLOCK


def _scale_of(amax):
    """Smallest power of two with amax <= 448 times it (2^-126 at least)."""
    m, e = torch.frexp(amax)                         # amax = m 2^e, 0.5 <= m < 1
    e = e - 9 + (m > 0.875)
    return torch.exp2(torch.where(amax > 0, e.clamp(min=-126), -126).float())


def _parts(st):
    """Views of the cache: key codes, value codes, scales."""
    hd, d = st["heads"][2], st["data"]
    keys = d[..., :BLOCK * hd].unflatten(-1, (2, hd // 16, 8, 16))
    values = d[..., BLOCK * hd:2 * BLOCK * hd].unflatten(-1, (hd, BLOCK))
    return keys, values, d[..., -32:-24].view(torch.float32)


def _append(st):
    hq, hk, hd = st["heads"]
    keys, values, scales = _parts(st)
    x = st["qkv"].float()
    lens, counts = st["lengths"].long(), st["offsets"].long().diff()
    seq = st["row_seq"]
    pos = lens[seq] - counts[seq] + st["row_at"]
    c, s = st["rope"][pos].unbind(-1)
    c, s = c[:, None], s[:, None]
    st["q_out"].copy_(_rotate(x[:, :hq], c, s))
    new = torch.stack((_rotate(x[:, hq:hq + hk], c, s), x[:, hq + hk:]), 2)      # [row][head][K, V][hd]
    page, blk, tok = _place(st, seq, pos)
    # the block's scale: of its new tokens, and of the stored ones where the block goes on
    block = page * scales.shape[2] + blk
    amax = torch.zeros(scales.shape[0] * scales.shape[2], hk, 2, device="cuda")
    amax.scatter_reduce_(0, block[:, None, None].expand(-1, hk, 2), new.abs().amax(-1), "amax")
    bseq = st["back_seq"]
    bpos = (lens[bseq] - counts[bseq]) // BLOCK * BLOCK + st["back_at"]
    bpage, bblk, btok = _place(st, bseq, bpos)
    start = lens[bseq] - counts[bseq]
    stored = scales[bpage, :, bblk]                                              # [row][head][K, V]
    goes_on = (bpos // BLOCK * BLOCK < start)[:, None, None]
    scale = _scale_of(amax[bpage * scales.shape[2] + bblk])
    scale = torch.where(goes_on, torch.maximum(scale, stored), scale)
    k_code = keys[bpage, :, bblk][torch.arange(len(bpos), device="cuda"), :, btok // 8, :, btok % 8].flatten(2)
    v_code = values[bpage, :, bblk][torch.arange(len(bpos), device="cuda"), :, :, _token_at(btok)]
    old = torch.stack((k_code, v_code), 2).view(torch.float8_e4m3fn).float() * stored[..., None]
    row = st["offsets"].long()[bseq] + (bpos - start).clamp(min=0)
    value = torch.where((bpos >= start)[:, None, None, None], new[row], old)
    code = (value / scale[..., None]).to(torch.float8_e4m3fn)
    bytes_ = code.view(torch.uint8)
    h = torch.arange(hk, device="cuda")[None]
    keys[bpage[:, None], h, bblk[:, None], (btok // 8)[:, None], :, (btok % 8)[:, None]] = \
        bytes_[:, :, 0].unflatten(-1, (hd // 16, 16))
    values[bpage[:, None], h, bblk[:, None], :, _token_at(btok)[:, None]] = bytes_[:, :, 1]
    scales[bpage[:, None], h, bblk[:, None]] = scale
    got = (code.float() * scale[..., None]).to(torch.bfloat16)
    return {"q": st["q_out"], "k": got[:, :, 0].contiguous(), "v": got[:, :, 1].contiguous()}


def _attention(st, q):
    hq, hk, hd = st["heads"]
    keys, values, scales = _parts(st)
    lens, counts, n = st["lengths"].long(), st["offsets"].long().diff(), st["lengths"].numel()
    nb = -(-st["max_len"] // BLOCK)
    b = torch.arange(nb, device="cuda")
    page = st["table"][:, b // (st["page"] // BLOCK)].long()
    blk = (b % (st["page"] // BLOCK)).expand(n, -1)
    sc = scales[page, :, blk]                                                    # [seq][block][head][K, V]
    k = keys[page, :, blk].view(torch.float8_e4m3fn).float()                     # [s][b][h][2][hd/16][8][16]
    k = k.permute(0, 2, 1, 3, 5, 4, 6).reshape(n, hk, nb, BLOCK, hd) * sc[..., 0].permute(0, 2, 1)[..., None, None]
    v = values[page, :, blk].view(torch.float8_e4m3fn).float()[..., _token_at(torch.arange(BLOCK, device="cuda"))]
    v = v.permute(0, 2, 1, 4, 3) * sc[..., 1].permute(0, 2, 1)[..., None, None]  # [s][h][b][16][hd]
    k, v = k.reshape(n, hk, nb * BLOCK, hd), v.reshape(n, hk, nb * BLOCK, hd)
    r = torch.arange(st["max_rows"], device="cuda")
    row = (st["offsets"].long()[:-1, None] + r).clamp(max=st["n_rows"] - 1)      # [seq][row], padded
    qs = q.float()[row].view(n, -1, hk, hq // hk, hd).permute(0, 2, 1, 3, 4).reshape(n, hk, -1, hd)
    p = (qs * st["scale"]) @ k.transpose(-1, -2)
    pos = (lens - counts)[:, None] + r                                           # of each row
    seen = torch.arange(nb * BLOCK, device="cuda") <= pos[..., None]             # [seq][row][key]
    seen = seen.repeat_interleave(hq // hk, 1)[:, None]
    p.masked_fill_(~seen, -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.where(total > 0, p @ v / total, 0.0)
    o = o.view(n, hk, -1, hq // hk, hd).permute(0, 2, 1, 3, 4).reshape(n, -1, hq, hd)
    return {"out": st["out"].copy_(o[st["row_seq"], st["row_at"]])}


def run(state):
    st = state
    op = st["case"]["op"]
    if own:
        hq, hk, _ = st["heads"]
        got, q = {}, st.get("q")
        if op != "attention":
            x = st["qkv"]
            st["cache"].append(st["batch"], x[:, hq:hq + hk], x[:, hq + hk:], rope=st["rope"], q=x[:, :hq],
                               q_out=st["q_out"])
            st["cache"].read(st["back"], st["k_back"], st["v_back"])
            got, q = {"q": st["q_out"], "k": st["k_back"], "v": st["v_back"]}, st["q_out"]
        if op != "append":
            got["out"] = st["cache"].attention(st["batch"], q, scale=st["scale"], out=st["out"],
                                               workspace=st["work"])
        return got
    got, q = {}, st.get("q")
    if op != "attention":
        got = _append(st)
        q = got["q"]
    if op != "append":
        got.update(_attention(st, q))
    return got


# ------------------------------------------------------------------- work
def work(case):
    hq, hk, hd = HEADS[case["heads"]]
    lens, rows = _lengths(case)
    n = sum(rows)
    got = {"bytes": 0, "flops": 0}
    if case["op"] != "attention":
        # projections and angles in; rotated queries, codes and the blocks' values out
        es = 2 if case["dtype"] == "bf16" else 4
        back = sum(x - (x - r) // BLOCK * BLOCK for x, r in zip(lens, rows))
        angles = min(n, max(lens)) * hd * 4
        got["bytes"] += n * (hq + 2 * hk) * hd * es + angles + n * hq * hd * 2 + 2 * n * hk * hd + back * 2 * hk * hd * 2
        got["flops"] += n * (hq + hk) * hd * 3
    if case["op"] != "append":
        pairs = sum(r * (x - r) + r * (r + 1) // 2 for x, r in zip(lens, rows))
        got["bytes"] += sum(lens) * hk * 2 * hd + sum(-(-x // BLOCK) for x in lens) * hk * 8 + 2 * n * hq * hd * 2
        got["flops"] += 4 * hd * hq * pairs
    return got


# --------------------------------------------------- the definition, 64 bits
def _e4m3_values():
    """The 256 values of the code: sign, four exponent bits (bias 7), three fraction bits."""
    out = []
    for c in range(256):
        e, f = c >> 3 & 15, c & 7
        v = math.nan if c & 127 == 127 else (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
        out.append(-v if c & 128 else v)
    return torch.tensor(out, dtype=torch.float64, device="cuda")


def _to_e4m3(x):
    """Nearest value of the code, ties to the even fraction."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    ulp = torch.exp2(e - 3)
    return torch.round(x / ulp) * ulp


def _dense(st, s, values):
    """Sequence s's cached tokens as [K, V][head][token][hd], and the scales of its blocks."""
    _, hk, hd = st["heads"]
    length = int(st["lengths"][s])
    nb, bpp = -(-length // BLOCK), st["page"] // BLOCK
    b = torch.arange(nb, device="cuda")
    rec = st["data"][st["table"][s, b // bpp].long(), :, b % bpp]                # [block][head][bytes]
    scale = rec[..., -32:-24].contiguous().view(torch.float32).double()          # [block][head][2]
    code = values[rec[..., :-32].int()]
    k = code[..., :BLOCK * hd].view(nb, hk, 2, hd // 16, 8, 16).transpose(3, 4).reshape(nb, hk, BLOCK, hd)
    order = [4 * (t % 8 // 2) + 2 * (t // 8) + t % 2 for t in range(BLOCK)]
    v = code[..., BLOCK * hd:].view(nb, hk, hd, BLOCK)[..., order].transpose(2, 3)
    kv = torch.stack((k, v)) * scale.permute(2, 0, 1)[..., None, None]
    return kv.transpose(1, 2).reshape(2, hk, nb * BLOCK, hd), scale.permute(2, 1, 0)


def exact(case, seed):
    st = prepare(case, seed)
    hq, hk, hd = st["heads"]
    lens, rows = _lengths(case)
    values = _e4m3_values()
    offs = _offsets(rows)
    got = {"q": [], "k": [], "v": [], "out": []}
    for s, (length, r) in enumerate(zip(lens, rows)):
        start = length - r
        kv, scale = _dense(st, s, values)
        if case["op"] == "attention":
            q = st["q"][offs[s]:offs[s + 1]].double()
        else:
            x = st["qkv"][offs[s]:offs[s + 1]].double()
            cs = st["rope"][start:length].double()[:, None]
            z = torch.complex(x[:, :hq + hk, :hd // 2].contiguous(), x[:, :hq + hk, hd // 2:].contiguous())
            z = z * torch.complex(cs[..., 0].contiguous(), cs[..., 1].contiguous())
            turned = torch.cat((z.real, z.imag), -1)
            q = turned[:, :hq].to(torch.bfloat16).double()
            got["q"].append(turned[:, :hq])
            first = start // BLOCK * BLOCK
            new = torch.stack((turned[:, hq:], x[:, hq + hk:])).transpose(1, 2)  # [K, V][head][row][hd]
            nb = -(-length // BLOCK) - first // BLOCK
            amax = torch.zeros(2, hk, nb * BLOCK, dtype=torch.float64, device="cuda")
            amax[..., start - first:length - first] = new.abs().amax(-1)
            amax = amax.view(2, hk, nb, BLOCK).amax(-1)
            sc = torch.exp2(torch.ceil(torch.log2(amax / 448)).clamp(min=-126))
            if start > first:
                sc[..., 0] = torch.maximum(sc[..., 0], scale[..., first // BLOCK])
            kv[:, :, start:length] = new
            tail = torch.zeros(2, hk, nb * BLOCK, hd, dtype=torch.float64, device="cuda")
            tail[:, :, :length - first] = kv[:, :, first:length]
            sc = sc.repeat_interleave(BLOCK, -1)[..., None]
            kv[:, :, first:length] = (_to_e4m3(tail / sc) * sc)[:, :, :length - first]
            got["k"].append(kv[0, :, first:length].transpose(0, 1))
            got["v"].append(kv[1, :, first:length].transpose(0, 1))
        if case["op"] != "append":
            seen = torch.arange(length, device="cuda") <= torch.arange(start, length, device="cuda")[:, None]
            o = []
            for h in range(hq):
                k, v = kv[:, h * hk // hq, :length]
                p = (q[:, h] @ k.T * st["scale"]).masked_fill_(~seen, -math.inf)
                o.append(torch.softmax(p, -1) @ v)
            got["out"].append(torch.stack(o, 1))
    return {name: torch.cat(x) for name, x in got.items() if x}
