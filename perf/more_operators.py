"""What a step of a served batch needs beside its attention: the operators whose speed counts, and their plain forms.

A program that serves several sequences from a paged cache (`operators.py`) draws the next token of each from the logits
of its rows (`sample`), or verifies the drafts of all of them in one call (`verify`), both with temperature, top-k, top-p
and min-p of each row or sequence.  Models whose layers look at the last `window` positions and at the first `sinks` only
attend so (`step` for the few new tokens of a step, `prompt` for whole prompts), and the pages that no such layer will look at again are
given back (`trim`).  Models with other rotary positions - neighbouring elements as pairs, a part of the head,
frequencies scaled for long contexts - append so (`rotary`).

Random numbers are inputs.  Filters, in this order: the `top_k` largest logits; of these, in falling order, as many as it
takes to reach `top_p` of their mass; of these those with at least `min_p` times the largest probability.  Equal logits count in the
order of the vocabulary.  A draw is the first token, in the order of the vocabulary, whose running mass exceeds u times the whole.

Sizes of a case follow from the case alone (`_lengths`, `_news`), what the tensors hold from the seed.  `run` computes
the plain forms (elementary torch) where `own` is false and calls `paper_2603_01399_amd.binding` where it is true; `exact` is
the definition once more in 64 bits.
"""
import math

import torch

own = False

D = 128
BLOCK = 32
EPS = 1e-6
E4M3_MOST = 448.0
OPS = ("sample", "verify", "step", "prompt", "rotary", "trim")
FILTERS = ("plain", "k", "p", "min_p", "k_p", "greedy", "all")


def listed():
    return [
        # the next token of one sequence, from bf16 logits as a linear writes them
        {"name": "sample_1_k_p_bf16", "op": "sample", "rows": 1, "vocab": 151936, "pad": 0, "type": "bf16", "filters": "k_p"},
        # a batch whose sequences ask for different things
        {"name": "sample_64_mixed_fp32", "op": "sample", "rows": 64, "vocab": 151936, "pad": 0, "type": "fp32", "filters": "mixed"},
        # the draft of one sequence, an odd vocabulary in padded rows
        {"name": "verify_1x8_p_bf16", "op": "verify", "seqs": 1, "new": 8, "vocab": 50257, "pad": 15, "type": "bf16", "filters": "p"},
        # drafts of a batch
        {"name": "verify_16x8_mixed_fp32", "op": "verify", "seqs": 16, "new": 8, "vocab": 151936, "pad": 0, "type": "fp32", "filters": "mixed"},
        # one token of each of a few sequences, a short window
        {"name": "step_4x1_ctx5000_w1024_bf16", "op": "step", "seqs": 4, "new": 1, "ctx": 5000, "window": 1024, "sinks": 4, "trimmed": False,
         "heads": 32, "kv_heads": 8, "page": 64, "kv": "bf16"},
        # a full batch of long contexts whose old pages are given back
        {"name": "step_64x1_ctx16000_w4096_e4m3", "op": "step", "seqs": 64, "new": 1, "ctx": 16000, "window": 4096, "sinks": 0, "trimmed": True,
         "heads": 64, "kv_heads": 8, "page": 128, "kv": "e4m3"},
        # a packed batch of prompts into 8-bit pages, windows of odd length, first tokens that stay visible
        {"name": "prompt_9x1531_w333_s4_e4m3", "op": "prompt", "seqs": 9, "new": 1531, "ctx": 0, "window": 333, "sinks": 4, "trimmed": False,
         "heads": 32, "kv_heads": 8, "page": 64, "kv": "e4m3"},
        # one long prompt
        {"name": "prompt_1x8192_w1024_bf16", "op": "prompt", "seqs": 1, "new": 8192, "ctx": 0, "window": 1024, "sinks": 0, "trimmed": False,
         "heads": 64, "kv_heads": 8, "page": 64, "kv": "bf16"},
        # one token, neighbouring elements as pairs, no norms: a launch and one trip to memory
        {"name": "rotary_1x1_pairs_bf16", "op": "rotary", "seqs": 1, "new": 1, "ctx": 1000, "layout": "interleaved", "dims": 128, "scaling": "none",
         "norm": False, "heads": 32, "kv_heads": 8, "page": 64, "kv": "bf16"},
        # the packed rows of prompts behind long contexts, three quarters of the head, frequencies scaled by parts
        {"name": "rotary_11x1531_part_e4m3", "op": "rotary", "seqs": 11, "new": 1531, "ctx": 40000, "layout": "half", "dims": 96, "scaling": "by_parts",
         "norm": True, "heads": 32, "kv_heads": 8, "page": 64, "kv": "e4m3"},
        # a step of a small batch: hardly a page is given back
        {"name": "trim_8_sequences", "op": "trim", "seqs": 8, "ctx": 3000, "window": 1024, "sinks": 4, "page": 64, "forked": False},
        # long prompts after their first pass, shared by continuations
        {"name": "trim_200_long_forked", "op": "trim", "seqs": 200, "ctx": 100000, "window": 4096, "sinks": 64, "page": 32, "forked": True},
    ]


def _log_int(rng, lo, hi):
    """An integer in lo .. hi, spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(OPS)
    c = {"op": op}
    if op in ("sample", "verify"):
        c["vocab"] = _log_int(rng, 1000, 200000)
        most = max(1, min(256, 128 * 151936 // c["vocab"]))
        if op == "sample":
            c["rows"] = _log_int(rng, 1, most)
        else:
            c["new"] = rng.randint(1, min(16, most))
            c["seqs"] = _log_int(rng, 1, most // c["new"])
        c["pad"] = rng.choice([0, 0, 1, 7, 64])
        c["type"] = rng.choice(["bf16", "fp32"])
        c["filters"] = rng.choice(FILTERS + ("mixed", "mixed"))
        return c
    c["page"] = rng.choice([32, 64, 128])
    c["window"] = _log_int(rng, 1, 6000)
    c["sinks"] = rng.choice([0, 4, rng.randint(1, 200)])
    if op == "trim":
        c["seqs"], c["ctx"], c["forked"] = _log_int(rng, 1, 200), _log_int(rng, 1, 100000), rng.choice([False, True])
        return c
    c["kv"], c["kv_heads"] = rng.choice(["bf16", "e4m3"]), rng.choice([1, 2, 4, 8])
    c["heads"] = c["kv_heads"] * rng.choice([1, 2, 4, 5, 8])
    if op == "rotary":
        del c["window"], c["sinks"]
        c["seqs"] = _log_int(rng, 1, 64)
        c["new"] = _log_int(rng, 1, max(1, 12000 // c["seqs"]))
        c["ctx"] = rng.choice([0, _log_int(rng, 1, max(1, 400000 // c["seqs"]))])
        c["layout"], c["dims"] = rng.choice(["half", "interleaved"]), rng.choice([128, 128, 96, 64, 32, 16])
        c["scaling"], c["norm"] = rng.choice(["none", "linear", "ntk", "by_parts"]), rng.choice([False, True])
        return c
    c["trimmed"] = rng.choice([False, True])
    if op == "step":
        c["seqs"] = _log_int(rng, 1, 128)
        c["new"] = rng.choice([1, 1, _log_int(rng, 1, 32)])
        # what the plain form reads, and its scores
        most = 64 * 4096 * 8 // (c["seqs"] * c["kv_heads"] * (1 + c["new"] * c["heads"] // c["kv_heads"] // 32))
        c["window"] = min(c["window"], max(1, most))
        c["ctx"] = _log_int(rng, 1, max(1, min(100000, 1000000 // c["seqs"])))
    else:
        c["seqs"] = _log_int(rng, 1, 32)
        c["new"] = _log_int(rng, 1, max(1, int((0.8 * 64 * 8192 ** 2 / (c["seqs"] * c["heads"])) ** 0.5)) if c["seqs"] > 1 else 8000)
        c["new"] = min(c["new"], 8000)
        room = int(0.8 * 64 * 8192 ** 2 / (c["seqs"] * c["heads"] * c["new"])) - c["new"]
        c["ctx"] = rng.choice([0, _log_int(rng, 1, max(1, min(room, 65536 // c["seqs"])))])
    return c


# ------------------------------------------------------------------------------------------------- what a case means

def _spread(i, most, least):
    """most for i = 0, else values between the two that look ragged and do not repeat soon."""
    return most - int((most - least) * ((i * 0.6180339887498949) % 1.0))


def _news(c):
    """New rows of each sequence: a draft's or a token's are alike, prompts are not."""
    if c["op"] in ("verify", "step"):
        return [c["new"]] * c["seqs"]
    return [_spread(i, c["new"], min(c["new"], 1 + c["new"] // 8)) for i in range(c["seqs"])]


def _lengths(c):
    """Cached positions of each sequence ahead of the new rows."""
    return [_spread(i, c["ctx"], c["ctx"] // 8) for i in range(c["seqs"])]


def _elem(c):
    return 1 if c["kv"] == "e4m3" else 2


def _trimmed_columns(c, length):
    """Columns of the table whose every position is behind the first tokens and ahead of the next token's window: first, last + 1."""
    return -(-c["sinks"] // c["page"]), max(0, length - c["window"] + 1) // c["page"]


def _seen(c, length, n):
    """Positions that some of n rows behind `length` cached ones see, and pairs of a row and a position that it sees."""
    w, s = c["window"], c["sinks"]
    low = max(0, length - w + 1)
    pairs = 0
    for i in range(n):
        p = length + i
        first = max(0, p - w + 1)
        pairs += p - first + 1 + min(s, first)
    return min(s, low) + length + n - low, pairs


def work(case):
    c = case
    if c["op"] in ("sample", "verify"):
        rows = c["rows"] if c["op"] == "sample" else c["seqs"] * c["new"]
        # the logits and a few numbers of each row; of each logit a comparison and its part of a sum
        return {"bytes": rows * (c["vocab"] * (2 if c["type"] == "bf16" else 4) + 32), "flops": 2 * rows * c["vocab"]}
    lengths = _lengths(c)
    if c["op"] == "trim":
        held = sum(-(-n // c["page"]) for n in lengths)
        gone = sum(max(0, b - a) for a, b in (_trimmed_columns(c, n) for n in lengths))
        return {"bytes": 4 * (held + 3 * gone + c["seqs"]), "flops": 0}
    news = _news(c)
    rows = sum(news)
    hq, hk = c["heads"], c["kv_heads"]
    if c["op"] == "rotary":
        return {"bytes": rows * D * (2 * (hq + 2 * hk) + 2 * hq + 2 * hk * _elem(c)), "flops": rows * (hq + hk) * (6 * c["dims"] // 2 + (3 * D if c["norm"] else 0))}
    seen = [_seen(c, l, n) for l, n in zip(lengths, news)]
    return {"bytes": sum(s for s, _ in seen) * hk * D * 2 * _elem(c) + 2 * rows * hq * D * 2, "flops": 4 * hq * D * sum(p for _, p in seen)}


# ----------------------------------------------------------------------------------------------------------- inputs

class _Inputs:
    """Draws a case's inputs on the GPU in a fixed order; prepare() and exact() see the same values."""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(int(seed))

    def normal(self, *shape, dtype=torch.float32):
        return torch.randn(shape, generator=self.gen, device="cuda", dtype=dtype)

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.gen, device="cuda", dtype=torch.float32)

    def permutation(self, n):
        return torch.randperm(n, generator=self.gen, device="cuda")


def _logits(c, inp, rows):
    """A broad body and a few hundred tokens that stand out, more in some rows than in others, as a language model's: from rows that
    are nearly sure of one token to rows that leave thousands open."""
    shape = (rows, c["vocab"] + c["pad"])
    z = inp.normal(*shape).mul_(1.7)
    z += torch.where(inp.uniform(*shape) < 0.002, inp.uniform(*shape), 0.0) * (4.0 + 16.0 * inp.uniform(rows, 1))
    return z.to(torch.bfloat16 if c["type"] == "bf16" else torch.float32)[:, :c["vocab"]]


def _parameters(c, inp, n):
    """temperature, top_k, top_p, min_p of n rows or sequences: of one kind, or all kinds in turn."""
    kind = torch.arange(n, device="cuda") % len(FILTERS) if c["filters"] == "mixed" else torch.full((n,), FILTERS.index(c["filters"]), device="cuda")
    of = {name: kind == i for i, name in enumerate(FILTERS)}
    temperature = torch.where(of["greedy"], 0.0, 0.6 + 0.7 * inp.uniform(n))
    top_k = torch.where(of["k"] | of["k_p"] | of["all"], torch.exp(inp.uniform(n) * math.log(1000.0)).round(), 0.0).to(torch.int32)
    top_p = torch.where(of["p"] | of["k_p"] | of["all"], 0.5 + 0.49 * inp.uniform(n), 1.0)
    min_p = torch.where(of["min_p"] | of["all"], 0.01 + 0.2 * inp.uniform(n), 0.0)
    return {"temperature": temperature, "top_k": top_k, "top_p": top_p, "min_p": min_p}


def _offsets():
    """Place of (position in the block, d) in a block of keys and of values, for 16- and for 8-bit pages: [32, 128] each."""
    p, d = torch.arange(BLOCK, device="cuda")[:, None], torch.arange(D, device="cuda")[None, :]
    sub, p16, step, g4, e = p // 16, p % 16, d // 32, d % 32 // 8, d % 8
    o, dt, dd = p % 16, d // 16, d % 16
    slot = o % 4 + 4 * (p // 16)
    return {"bf16": ((((sub * 4 + step) * 4 + g4) * 16 + p16) * 8 + e, ((dt * 4 + o // 4) * 16 + dd) * 8 + slot),
            "e4m3": (((((sub * 2 + step // 2) * 4 + g4) * 16 + p16) * 2 + step % 2) * 8 + e,
                     (((dt // 2 * 4 + o // 4) * 16 + dd) * 2 + dt % 2) * 8 + slot)}


def _pool(c, inp, pages):
    """One layer's pages as they lie in memory; whatever earlier sequences left there in those that nobody holds."""
    x = inp.normal(1, pages, c["kv_heads"], c["page"] // BLOCK, 2, BLOCK * D, dtype=torch.bfloat16)
    return x if c["kv"] == "bf16" else (x * 16.0).to(torch.float8_e4m3fn)


def _books(inp, held, columns, pages, gone=None):
    """One buffer of refs | lengths | table, and the three as views: pages scattered over the pool.  gone: columns of each sequence that
    have been given back."""
    seqs = len(held)
    meta = torch.zeros(pages + seqs + seqs * columns, dtype=torch.int32, device="cuda")
    refs, length, table = meta[:pages], meta[pages:pages + seqs], meta[pages + seqs:].view(seqs, columns)
    col = torch.arange(columns, device="cuda")[None, :]
    here = col < torch.tensor(held, device="cuda")[:, None]
    if gone is not None:
        first, end = torch.tensor(gone, device="cuda").unbind(1)
        here &= (col < first[:, None]) | (col >= end[:, None])
    ids = inp.permutation(pages)[:int(here.sum())].to(torch.int32)
    table.fill_(-1)
    table[here] = ids
    refs[ids.long()] = 1
    return {"meta": meta, "refs": refs, "lengths": length, "table": table}


def _starts(news):
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    return starts


def prepare(case, seed):
    c, inp = dict(case), _Inputs(seed)
    op = c["op"]
    s = {"c": c, "op": op}
    if op == "sample":
        s["logits"] = _logits(c, inp, c["rows"])
        s["filters"] = _parameters(c, inp, c["rows"])
        s["u"] = inp.uniform(c["rows"])
        return s
    if op == "verify":
        rows = c["seqs"] * c["new"]
        s["logits"] = _logits(c, inp, rows)
        s["filters"] = _parameters(c, inp, c["seqs"])
        s["u_accept"], s["u_sample"] = inp.uniform(rows), inp.uniform(rows)
        s["row_start"] = torch.tensor(_starts(_news(c)), dtype=torch.int32, device="cuda")
        # a draft that agrees with the model now and then: a token of its own distribution, made sharper
        noise = -torch.log(-torch.log(inp.uniform(rows, c["vocab"]).clamp_(1e-7, 1.0 - 1e-7)))
        s["draft"] = (2.0 * s["logits"].float() + noise).argmax(1).to(torch.int32)
        return s
    lengths = _lengths(c)
    if op == "trim":
        held = [-(-n // c["page"]) for n in lengths]
        columns, pages = max(held) + 1, sum(held) + 3
        s.update(_books(inp, held, columns, pages))
        if c["forked"]:                                   # every second sequence goes on from the one before it
            pairs = c["seqs"] // 2
            for i in range(pairs):
                n = min(lengths[2 * i], lengths[2 * i + 1])
                lengths[2 * i + 1] = n
            held = torch.tensor([-(-n // c["page"]) for n in lengths], device="cuda")
            table = s["table"]
            here = torch.arange(columns, device="cuda")[None, :] < held[:, None]
            table[1:2 * pairs:2] = table[0:2 * pairs:2]
            table.masked_fill_(~here, -1)
            s["refs"].copy_(torch.bincount(table[table >= 0].long(), minlength=pages))
        s["lengths"].copy_(torch.tensor(lengths, dtype=torch.int32))
        s["pool"] = torch.zeros(1, pages, 1, c["page"] // BLOCK, 2, BLOCK * D, dtype=torch.bfloat16, device="cuda")
        s["before"] = s["meta"].clone()
        return s
    news = _news(c)
    held = [-(-(l + n) // c["page"]) for l, n in zip(lengths, news)]
    gone = [_trimmed_columns(c, n) for n in lengths] if c.get("trimmed") else None
    pages = sum(held) + 3 - (sum(max(0, b - a) for a, b in gone) if gone else 0)
    s.update(_books(inp, held, max(held), pages, gone))
    s["lengths"].copy_(torch.tensor(lengths, dtype=torch.int32))
    s["pool"] = _pool(c, inp, pages)
    s["k_scale"] = s["v_scale"] = None
    if c["kv"] == "e4m3":
        s["k_scale"], s["v_scale"] = ((inp.uniform(1, c["kv_heads"]) * 0.5 + 0.75) / 16.0 for _ in range(2))
    starts = _starts(news)
    s["row_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    s["most"] = max(news)
    s["longest"] = max(l + n for l, n in zip(lengths, news))
    s["places"] = _offsets()[c["kv"]]
    if op == "rotary":
        s["qkv"] = inp.normal(starts[-1], (c["heads"] + 2 * c["kv_heads"]) * D, dtype=torch.bfloat16)
        s["qg"] = s["kg"] = None
        if c["norm"]:
            s["qg"], s["kg"] = ((1.0 + 0.2 * inp.normal(D)).to(torch.bfloat16) for _ in range(2))
    else:
        s["q"] = inp.normal(starts[-1], c["heads"] * D, dtype=torch.bfloat16)
    return s


def _scaling(c):
    """How a case's frequencies follow from theta: (theta, scaling, factor, trained length, turns that are slow, that are fast)."""
    return {"none": (1.0e6, None, 1.0, None, 1.0, 32.0), "linear": (1.0e4, "linear", 4.0, None, 1.0, 32.0), "ntk": (1.0e4, "ntk", 8.0, None, 1.0, 32.0),
            "by_parts": (1.0e6, "by_parts", 4.0, 32768, 1.0, 32.0)}[c["scaling"]]


# ------------------------------------------------------------------------------------------------------ plain forms

def _masses(logits, f):
    """The mass of every token that the filters leave, [rows, vocab] in 64 bits, relative to the row's largest."""
    z = logits.float()
    greedy = f["temperature"] <= 0.0
    t = torch.where(greedy, 1.0, f["temperature"]).double()[:, None]
    k = torch.where(greedy, 1, f["top_k"])[:, None]
    k = torch.where(k <= 0, z.shape[1], k)
    z, order = torch.sort(z, dim=1, descending=True, stable=True)
    z = z.double()
    w = ((z - z[:, :1]) / t).exp()
    rank = torch.arange(z.shape[1], device="cuda")
    w_k = torch.where(rank < k, w, 0.0)
    before = w_k.cumsum(1) - w_k
    keep = (before < f["top_p"].double()[:, None] * w_k.sum(1, keepdim=True)) | (rank == 0)
    keep &= w >= f["min_p"].double()[:, None]
    return torch.zeros_like(w).scatter_(1, order, torch.where(keep, w_k, 0.0))


def _drawn(masses, u):
    """The first token whose running mass exceeds u times the whole."""
    c = masses.cumsum(1)
    return torch.searchsorted(c, u.double()[:, None] * c[:, -1:], right=True).clamp(max=c.shape[1] - 1)


def _plain_sample(s):
    m = _masses(s["logits"], s["filters"])
    token = _drawn(m, s["u"])
    return {"token": token[:, 0].to(torch.int32), "p": (m.gather(1, token) / m.sum(1, keepdim=True))[:, 0].float()}


def _plain_verify(s):
    start = s["row_start"].long()
    rows = s["logits"].shape[0]
    row = torch.arange(rows, device="cuda")
    seq = torch.searchsorted(start, row, right=True) - 1
    m = _masses(s["logits"], {k: v[seq] for k, v in s["filters"].items()})
    draft = s["draft"].long()[:, None]
    p = (m.gather(1, draft) / m.sum(1, keepdim=True))[:, 0]
    last = row == start[seq + 1] - 1
    refused = (s["u_accept"].double() >= p) | last
    # rows ahead of a sequence's first refusal; its last row, the token behind the whole draft, ends every sequence
    first = torch.full((start.numel() - 1,), rows, device="cuda").scatter_reduce_(0, seq, torch.where(refused, row, rows), "amin")
    m = m.scatter(1, torch.where(last[:, None], 0, draft), torch.where(last[:, None], m[:, :1], 0.0))
    token = _drawn(m[first], s["u_sample"][first])
    return {"accepted": (first - start[:-1]).to(torch.int32), "token": token[:, 0].to(torch.int32), "p": p.float()}


def _rows(s, rows):
    """Sequence and position of every new row."""
    row = torch.arange(rows, device="cuda")
    seq = torch.searchsorted(s["row_start"].long(), row, right=True) - 1
    return seq, s["lengths"].long()[seq] + row - s["row_start"].long()[seq]


def _blocks(s):
    """Blocks of 32 positions that a sequence's rows see something of, [seqs, blocks], -1 where there are fewer."""
    c, length = s["c"], s["lengths"].long()[:, None]
    if c["op"] == "prompt":
        return torch.arange(-(-s["longest"] // BLOCK), device="cuda").expand(length.shape[0], -1)
    first = -(-c["sinks"] // BLOCK)
    low = ((length - c["window"] + 1).clamp(min=0) // BLOCK).clamp(min=first)
    i = torch.arange(first + (c["window"] + c["new"] - 2) // BLOCK + 2, device="cuda")[None, :]
    b = torch.where(i < first, i, low + i - first)
    return torch.where(b * BLOCK < length + c["new"], b, -1)


def _gathered(s, half, blocks):
    """Keys or values of the blocks: [seqs, kv heads, positions, 128] fp32."""
    c = s["c"]
    per = c["page"] // BLOCK
    b = blocks.clamp(min=0)
    page = s["table"].long().gather(1, (b // per).clamp(max=s["table"].shape[1] - 1)).clamp(min=0)
    raw = s["pool"][0].view(torch.int16 if c["kv"] == "bf16" else torch.uint8)
    x = raw[page, :, b % per, half]                                                # [seqs, blocks, heads, 4096]
    x = x[..., s["places"][half].reshape(-1)].view(s["pool"].dtype).float()
    scale = s["k_scale"] if half == 0 else s["v_scale"]
    seqs, nb, hk, _ = x.shape
    x = x.view(seqs, nb, hk, BLOCK, D).permute(0, 2, 1, 3, 4).reshape(seqs, hk, nb * BLOCK, D)
    return x if scale is None else x * scale[0][:, None, None]


def _plain_attention(s):
    c = s["c"]
    hq, hk, most = c["heads"], c["kv_heads"], s["most"]
    start, lengths = s["row_start"].long(), s["lengths"].long()
    rows, seqs = s["q"].shape[0], lengths.numel()
    i = torch.arange(most, device="cuda")
    at = (start[:-1, None] + i).clamp(max=rows - 1)
    q = s["q"].view(rows, hk, hq // hk, D)[at].float()                             # [seqs, most, kv heads, group, 128]
    q = q.permute(0, 2, 3, 1, 4).reshape(seqs, hk, hq // hk * most, D)
    blocks = _blocks(s)
    score = torch.matmul(q, _gathered(s, 0, blocks).transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(D))
    pos = torch.where(blocks[..., None] < 0, 1 << 30, blocks[..., None] * BLOCK + torch.arange(BLOCK, device="cuda")).view(seqs, 1, -1)
    here = (lengths[:, None] + i)[..., None]
    seen = (pos <= here) & ((pos > here - c["window"]) | (pos < c["sinks"]))
    score = score.view(seqs, hk, hq // hk, most, -1).masked_fill_(~seen[:, None, None], -math.inf)
    score = score.sub_(score.amax(-1, keepdim=True)).exp_()
    score = score.div_(score.sum(-1, keepdim=True)).view(seqs, hk, hq // hk * most, -1)
    out = torch.matmul(score, _gathered(s, 1, blocks)).view(seqs, hk, hq // hk, most, D)
    seq, p = _rows(s, rows)
    out = out.permute(0, 3, 1, 2, 4)[seq, p - lengths[seq]]                        # [rows, kv heads, group, 128]
    return out.reshape(rows, hq * D).to(torch.bfloat16)


def _frequencies(c):
    """Radians a position of every pair, and what cosines and sines are multiplied by."""
    theta, scaling, factor, trained, slow, fast = _scaling(c)
    n = c["dims"]
    i = torch.arange(n // 2, device="cuda", dtype=torch.float64)
    if scaling == "ntk":
        theta = theta * factor ** (n / (n - 2.0))
    f = theta ** (-2.0 * i / n)
    if scaling == "linear":
        f = f / factor
    if scaling == "by_parts":                             # pairs that turn often in the trained length as they are, those that hardly turn slowed down
        keep = ((trained * f / (2.0 * math.pi) - slow) / (fast - slow)).clamp(0.0, 1.0)
        f = keep * f + (1.0 - keep) * f / factor
        return f, 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _rotated(x, gamma, angle, magnitude, c):
    """x [rows, heads, 128] fp32: a norm of each head, rounded as bf16 code does, then the first dims rotated."""
    if gamma is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        x = (x.to(torch.bfloat16).float() * gamma.float()).to(torch.bfloat16).float()
    n = c["dims"]
    cos, sin = (angle.cos() * magnitude).float()[:, None], (angle.sin() * magnitude).float()[:, None]
    turned, rest = x[..., :n], x[..., n:]
    if c["layout"] == "half":
        a, b = turned[..., :n // 2], turned[..., n // 2:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, rest], -1).to(torch.bfloat16)


def _plain_rotary(s):
    c, pool = s["c"], s["pool"]
    hq, hk = c["heads"], c["kv_heads"]
    rows = s["qkv"].shape[0]
    seq, pos = _rows(s, rows)
    f, magnitude = _frequencies(c)
    angle = pos.double()[:, None] * f
    x = s["qkv"].view(rows, hq + 2 * hk, D).float()
    q = _rotated(x[:, :hq], s["qg"], angle, magnitude, c)
    k = _rotated(x[:, hq:hq + hk], s["kg"], angle, magnitude, c)
    v = x[:, hq + hk:].to(torch.bfloat16)
    page = s["table"].long()[seq, pos // c["page"]]
    flat = pool.view(torch.int16 if c["kv"] == "bf16" else torch.uint8).view(-1)
    block = ((page[:, None] * hk + torch.arange(hk, device="cuda")) * (c["page"] // BLOCK) + (pos % c["page"] // BLOCK)[:, None]) * 2
    for half, (x, scale) in enumerate(((k, s["k_scale"]), (v, s["v_scale"]))):
        if scale is not None:
            x = (x.float() / scale[0][:, None]).clamp(-E4M3_MOST, E4M3_MOST).to(torch.float8_e4m3fn)
        at = (block + half)[..., None] * (BLOCK * D) + s["places"][half][pos % BLOCK][:, None]
        flat[at] = x.view(flat.dtype)
    return {"q": q.reshape(rows, hq * D), "pool": pool}


def _plain_trim(s):
    """Pages of positions that are none of the first `sinks` and ahead of the next token's window are given back."""
    c, table, refs = s["c"], s["table"], s["refs"]
    begin = torch.arange(table.shape[1], device="cuda")[None, :] * c["page"]
    gone = (begin >= c["sinks"]) & (begin + c["page"] <= s["lengths"][:, None] - c["window"] + 1) & (table >= 0)
    ids = table[gone].long()
    refs.index_add_(0, ids, torch.full_like(ids, -1, dtype=torch.int32))
    table.masked_fill_(gone, -1)


# -------------------------------------------------------------------------------------------------------------- run

def _own(s):
    """The binding, and the handles that a program keeps: a cache over its own tensors, its rotary positions."""
    from paper_2603_01399_amd import binding as qb
    c = s["c"]
    if "pool" in s and "cache" not in s:
        pool = s["pool"]
        s["cache"] = qb.PagedKvCache(1, pool.shape[2], pool.shape[1], page_len=c["page"], max_seqs=s["table"].shape[0], max_pages=s["table"].shape[1],
                                     dtype=pool.dtype, k_scale=s.get("k_scale"), v_scale=s.get("v_scale"), pool=pool, books=s["meta"])
    if c["op"] == "rotary" and "rope" not in s:
        theta, scaling, factor, trained, slow, fast = _scaling(c)
        s["rope"] = qb.Rope(c["dims"], theta, layout=c["layout"], scaling=scaling, factor=factor, trained_len=trained, slow=slow, fast=fast)
    return qb


def run(state):
    s = state
    op, c = s["op"], s["c"]
    if op == "trim":
        s["meta"].copy_(s["before"])                      # (the books as they were: a pass can be repeated)
    if not own:
        if op == "trim":
            _plain_trim(s)
            return {"table": s["table"], "refs": s["refs"]}
        return {"sample": _plain_sample, "verify": _plain_verify, "step": _plain_attention, "prompt": _plain_attention, "rotary": _plain_rotary}[op](s)
    qb = _own(s)
    if op == "sample":
        token, p = qb.sample_tokens(s["logits"], s["u"], **s["filters"])
        return {"token": token, "p": p}
    if op == "verify":
        accepted, token, p = qb.verify_tokens(s["logits"], s["row_start"], s["draft"], s["u_accept"], s["u_sample"], **s["filters"])
        return {"accepted": accepted, "token": token, "p": p}
    if op == "step":
        return qb.paged_attention(s["q"], c["heads"], s["cache"], 0, s["row_start"], s["most"], window=c["window"], sinks=c["sinks"])
    if op == "prompt":
        return qb.prompt_attention(s["q"], c["heads"], s["cache"], 0, s["row_start"], window=c["window"], sinks=c["sinks"])
    if op == "rotary":
        q = qb.paged_prepare(s["qkv"], c["heads"], s["cache"], 0, s["row_start"], s["qg"], s["kg"], eps=EPS, rope=s["rope"])
        return {"q": q, "pool": s["pool"]}
    s["cache"].trim(c["window"], c["sinks"])
    return {"table": s["table"], "refs": s["refs"]}


# ------------------------------------------------------------------------------------------------------------ exact

def _exact_row(z, temperature, top_k, top_p, min_p):
    """Tokens that one row's filters leave, in the order of the vocabulary, and their probabilities."""
    if temperature <= 0.0:
        temperature, top_k = 1.0, 1
    z = z.double()
    # falling logits, equal ones by their place: places from the back in a rising sort of the reversed row
    order = (z.numel() - 1 - torch.sort(z.flip(0), stable=True)[1]).flip(0)
    if 0 < top_k < z.numel():
        order = order[:top_k]
    p = torch.softmax(z[order] / temperature, 0)
    most = p[0].clone()
    reached = int((p.cumsum(0) < top_p).sum()) + 1        # as many as it takes
    order = order[:reached]
    p = p[:reached]
    inside = p >= min_p * most
    order, p = order[inside], p[inside]
    order, by_place = order.sort()
    return order, p[by_place] / p.sum()


def _exact_draw(token, p, u):
    c = p.cumsum(0)
    return min(int((c <= u * c[-1]).sum()), token.numel() - 1)


def _exact_sampling(s):
    z, f = s["logits"], {k: v.tolist() for k, v in s["filters"].items()}
    if s["op"] == "sample":
        tokens, ps = [], []
        for r, u in enumerate(s["u"].tolist()):
            token, p = _exact_row(z[r], *(f[k][r] for k in ("temperature", "top_k", "top_p", "min_p")))
            at = _exact_draw(token, p, u)
            tokens.append(int(token[at]))
            ps.append(float(p[at]))
        return {"token": torch.tensor(tokens, dtype=torch.int32, device="cuda"), "p": torch.tensor(ps, dtype=torch.float64, device="cuda")}
    start, draft, ua, us = (s[k].tolist() for k in ("row_start", "draft", "u_accept", "u_sample"))
    accepted, tokens, ps = [], [], []
    for b in range(len(start) - 1):
        going, count = True, 0
        for r in range(start[b], start[b + 1]):
            token, p = _exact_row(z[r], *(f[k][b] for k in ("temperature", "top_k", "top_p", "min_p")))
            is_draft = token == draft[r]
            ps.append(float(p[is_draft].sum()))
            last = r == start[b + 1] - 1
            if going and not last and ua[r] < ps[-1]:
                count += 1
            elif going:
                going = False
                if not last:
                    token, p = token[~is_draft], p[~is_draft]
                tokens.append(int(token[_exact_draw(token, p, us[r])]))
        accepted.append(count)
    return {"accepted": torch.tensor(accepted, dtype=torch.int32, device="cuda"), "token": torch.tensor(tokens, dtype=torch.int32, device="cuda"),
            "p": torch.tensor(ps, dtype=torch.float64, device="cuda")}


def _exact_places(kv):
    """Position and d of every element of a block of keys and of values, read off the stored order."""
    if kv == "bf16":
        sub, step, g4, p, e = torch.meshgrid(*(torch.arange(n) for n in (2, 4, 4, 16, 8)), indexing="ij")
        keys = 16 * sub + p, 32 * step + 8 * g4 + e
        dt, g4, dd, hi, lo = torch.meshgrid(*(torch.arange(n) for n in (8, 4, 16, 2, 4)), indexing="ij")
        values = 16 * hi + 4 * g4 + lo, 16 * dt + dd
    else:
        sub, pair, g4, p, one, e = torch.meshgrid(*(torch.arange(n) for n in (2, 2, 4, 16, 2, 8)), indexing="ij")
        keys = 16 * sub + p, 32 * (2 * pair + one) + 8 * g4 + e
        pair, g4, dd, one, hi, lo = torch.meshgrid(*(torch.arange(n) for n in (4, 4, 16, 2, 2, 4)), indexing="ij")
        values = 16 * hi + 4 * g4 + lo, 16 * (2 * pair + one) + dd
    return [(p.reshape(-1).cuda(), d.reshape(-1).cuda()) for p, d in (keys, values)]


def _exact_rotary(s, places, scales):
    c = s["c"]
    hq, hk, page = c["heads"], c["kv_heads"], c["page"]
    table, lengths, start = s["table"].tolist(), s["lengths"].tolist(), s["row_start"].tolist()
    rows, n = s["qkv"].shape[0], c["dims"]
    pos = torch.cat([torch.arange(lengths[b], lengths[b] + start[b + 1] - start[b], device="cuda") for b in range(c["seqs"])])
    x = s["qkv"].view(rows, hq + 2 * hk, D).double()
    theta, scaling, factor, trained, slow, fast = _scaling(c)
    freq, magnitude = [], 1.0
    for i in range(n // 2):
        f = (theta * factor ** (n / (n - 2.0)) if scaling == "ntk" else theta) ** (-2.0 * i / n)
        if scaling == "linear":
            f /= factor
        if scaling == "by_parts":
            magnitude = 1.0 + 0.1 * math.log(factor)
            part = min(1.0, max(0.0, (trained / (2.0 * math.pi / f) - slow) / (fast - slow)))
            f = (1.0 - part) * f / factor + part * f
        freq.append(f)
    turn = torch.polar(torch.tensor(magnitude, dtype=torch.float64, device="cuda"),
                       pos.double()[:, None] * torch.tensor(freq, dtype=torch.float64, device="cuda"))[:, None]
    done = []
    for y, gamma in ((x[:, :hq], s["qg"]), (x[:, hq:hq + hk], s["kg"])):
        if gamma is not None:
            y = y / (y.square().mean(-1, keepdim=True) + EPS).sqrt() * gamma.double()
        pairs = y[..., :n].unflatten(-1, (2, n // 2)).transpose(-1, -2) if c["layout"] == "half" else y[..., :n].unflatten(-1, (n // 2, 2))
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        done.append(torch.cat([(z.transpose(-1, -2) if c["layout"] == "half" else z).flatten(-2), y[..., n:]], -1))
    pool = s["pool"].double()
    stored = [done[1] / scales[0][:, None], x[:, hq + hk:] / scales[1][:, None]]
    if c["kv"] == "e4m3":
        stored = [t.clamp(-E4M3_MOST, E4M3_MOST) for t in stored]
    for half in range(2):
        p, d = places[half]
        where = torch.empty((BLOCK, D), dtype=torch.long, device="cuda")
        where[p, d] = torch.arange(BLOCK * D, device="cuda")
        for b in range(c["seqs"]):
            j = torch.arange(lengths[b], lengths[b] + start[b + 1] - start[b], device="cuda")
            ids = torch.tensor(table[b], device="cuda")[j // page]
            for h in range(hk):
                pool[0, ids[:, None], h, (j % page // BLOCK)[:, None], half, where[j % BLOCK]] = stored[half][start[b]:start[b + 1], h]
    return {"q": done[0].reshape(rows, hq * D), "pool": pool}


def _exact_attention(s, places, scales):
    c = s["c"]
    hq, hk, page = c["heads"], c["kv_heads"], c["page"]
    table, lengths, start = s["table"].tolist(), s["lengths"].tolist(), s["row_start"].tolist()
    out = torch.zeros(s["q"].shape[0], hq, D, dtype=torch.float64, device="cuda")
    group = hq // hk
    for b in range(c["seqs"]):
        n, length = start[b + 1] - start[b], lengths[b]
        if n == 0:
            continue
        low = max(0, length - c["window"] + 1)            # positions that some row may see: the first ones, and from here on
        pos = torch.cat([torch.arange(min(c["sinks"], low), device="cuda"), torch.arange(low, length + n, device="cuda")])
        ids = torch.tensor(table[b], device="cuda")[pos // page]
        behind = length + torch.arange(n, device="cuda")[:, None] - pos[None, :]
        hidden = (behind < 0) | ((behind >= c["window"]) & (pos[None, :] >= c["sinks"]))
        for h in range(hk):
            kv = []
            for half in range(2):
                p, d = places[half]
                where = torch.empty((BLOCK, D), dtype=torch.long, device="cuda")
                where[p, d] = torch.arange(BLOCK * D, device="cuda")
                block = s["pool"][0, :, h, :, half].view(torch.int16 if c["kv"] == "bf16" else torch.uint8)[ids, pos % page // BLOCK]
                kv.append(block.gather(1, where[pos % BLOCK]).view(s["pool"].dtype).double() * scales[half][h])
            for g in range(group):
                q = s["q"].view(-1, hq, D)[start[b]:start[b] + n, h * group + g].double()
                w = (q @ kv[0].t() / math.sqrt(D)).masked_fill(hidden, -math.inf).softmax(-1)
                out[start[b]:start[b] + n, h * group + g] = w @ kv[1]
    return out.reshape(-1, hq * D)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if s["op"] == "trim":
        return None                                       # books: nothing is computed
    if s["op"] in ("sample", "verify"):
        return _exact_sampling(s)
    places = _exact_places(c["kv"])
    scales = [torch.ones(c["kv_heads"], dtype=torch.float64, device="cuda") if x is None else x[0].double() for x in (s["k_scale"], s["v_scale"])]
    return (_exact_rotary if s["op"] == "rotary" else _exact_attention)(s, places, scales)
