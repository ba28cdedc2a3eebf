"""Serving a batch of sequences from a paged key/value cache: the operators whose speed counts, and their plain forms.

A program that serves several sequences keeps the keys and values of all of them in pages of `page` positions (a
multiple of 32) that are handed out as sequences grow.  Per step it makes room (`reserve`), normalises, rotates and
appends the new tokens (`prepare`), and attends: `paged` for the few new tokens of a step (one, or a draft), `prompt`
for a whole prompt or a chunk of one.  Between steps it shares a prompt's pages with several continuations (`fork`)
and moves the pages that are in use together (`compact`).  Head dimension 128; pages hold bf16, or e4m3 codes with a
scale for each key/value head.

Pages are stored as [layer, page, kv head, block of 32 positions, keys | values, 4096] with the block in the order in
which the matrix cores take it (`_offsets`).  Lengths and new rows of a case follow from the case alone (`_lengths`,
`_news`), what the tensors hold from the seed.

`run` computes the plain forms (elementary torch, 32 bits) where `own` is false and calls
`paper_2603_01399_amd.binding` where it is true; `exact` is the definition once more in 64 bits.
"""
import math

import torch

own = False

D = 128
BLOCK = 32
EPS = 1e-6
THETA = 1.0e6
E4M3_MOST = 448.0
OPS = ("prepare", "paged", "prompt", "reserve", "fork", "compact")


def listed():
    return [
        # one token of one sequence, where launch and latency are everything
        {"name": "prepare_1x1_bf16", "op": "prepare", "seqs": 1, "new": 1, "ctx": 1000, "heads": 32, "kv_heads": 8, "page": 64, "kv": "bf16"},
        # the packed rows of eleven prompts of different lengths into 8-bit pages
        {"name": "prepare_11_prompts_e4m3", "op": "prepare", "seqs": 11, "new": 1531, "ctx": 0, "heads": 32, "kv_heads": 8, "page": 64, "kv": "e4m3"},
        # a small batch of short contexts, one token each
        {"name": "paged_4x1_ctx1000_bf16", "op": "paged", "seqs": 4, "new": 1, "ctx": 1000, "heads": 32, "kv_heads": 8, "page": 64, "kv": "bf16"},
        # a full batch of ragged contexts, one token each
        {"name": "paged_64x1_ctx8192_bf16", "op": "paged", "seqs": 64, "new": 1, "ctx": 8191, "heads": 32, "kv_heads": 8, "page": 64, "kv": "bf16"},
        # drafts of seven tokens over two long contexts in 8-bit pages: few rows, a long axis
        {"name": "paged_2x8_ctx100000_e4m3", "op": "paged", "seqs": 2, "new": 8, "ctx": 100003, "heads": 64, "kv_heads": 8, "page": 128, "kv": "e4m3"},
        # one short prompt
        {"name": "prompt_1x61_bf16", "op": "prompt", "seqs": 1, "new": 61, "ctx": 0, "heads": 32, "kv_heads": 8, "page": 64, "kv": "bf16"},
        # a packed batch of prompts of different lengths
        {"name": "prompt_9x1531_bf16", "op": "prompt", "seqs": 9, "new": 1531, "ctx": 0, "heads": 32, "kv_heads": 8, "page": 64, "kv": "bf16"},
        # a chunk of a prompt behind a long cached prefix in 8-bit pages
        {"name": "prompt_1x512_ctx16000_e4m3", "op": "prompt", "seqs": 1, "new": 512, "ctx": 16000, "heads": 40, "kv_heads": 8, "page": 128, "kv": "e4m3"},
        # one long prompt
        {"name": "prompt_1x8192_bf16", "op": "prompt", "seqs": 1, "new": 8192, "ctx": 0, "heads": 64, "kv_heads": 8, "page": 64, "kv": "bf16"},
        # room for the next draft of every sequence: bookkeeping alone
        {"name": "reserve_48_sequences", "op": "reserve", "seqs": 48, "new": 8, "ctx": 4000, "layers": 1, "kv_heads": 2, "page": 64, "kv": "bf16", "slack": 100},
        # eight prompts with eight continuations each: shared pages, and a copy of the last page of all but one of each
        {"name": "fork_8_to_64", "op": "fork", "seqs": 64, "from": 8, "new": 1, "ctx": 500, "layers": 36, "kv_heads": 8, "page": 64, "kv": "bf16", "slack": 30},
        # half of the pages in use, scattered: moved together
        {"name": "compact_1024_of_2048", "op": "compact", "seqs": 40, "pages": 2048, "live": 1024, "moves": 512, "layers": 4, "kv_heads": 8, "page": 64, "kv": "bf16"},
    ]


def _log_int(rng, lo, hi):
    """An integer in lo .. hi, spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(OPS)
    c = {"op": op, "kv": rng.choice(["bf16", "e4m3"]), "page": rng.choice([32, 64, 128])}
    if op in ("prepare", "paged", "prompt"):
        c["kv_heads"] = rng.choice([1, 2, 4, 8])
        c["heads"] = c["kv_heads"] * rng.choice([1, 2, 4, 5, 8])
    if op == "prepare":
        c["seqs"] = _log_int(rng, 1, 64)
        c["new"] = _log_int(rng, 1, max(1, 12000 // c["seqs"]))
        c["ctx"] = rng.choice([0, _log_int(rng, 1, 60000 // c["seqs"])])
    elif op == "paged":
        c["seqs"] = _log_int(rng, 1, 128)
        c["new"] = rng.choice([1, 1, _log_int(rng, 1, 32)])
        # cost of the plain form: positions x heads it reads, and scores
        most = 64 * 8192 * 8 // (c["seqs"] * c["kv_heads"] * (1 + c["new"] * c["heads"] // c["kv_heads"] // 32))
        c["ctx"] = _log_int(rng, 1, max(1, min(120000, most)))
    elif op == "prompt":
        c["seqs"] = _log_int(rng, 1, 32)
        c["new"] = _log_int(rng, 1, max(1, int((0.8 * 64 * 8192 ** 2 / (c["seqs"] * c["heads"])) ** 0.5)) if c["seqs"] > 1 else 8000)
        c["new"] = min(c["new"], 8000)
        room = int(0.8 * 64 * 8192 ** 2 / (c["seqs"] * c["heads"] * c["new"])) - c["new"]
        c["ctx"] = rng.choice([0, _log_int(rng, 1, max(1, min(room, 65536 // c["seqs"])))])
    else:
        c["kv_heads"], c["layers"] = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 8])
        if op == "reserve":
            c["seqs"], c["new"], c["ctx"] = _log_int(rng, 1, 200), _log_int(rng, 1, 600), _log_int(rng, 1, 6000)
            c["layers"], c["kv_heads"] = 1, 1
            c["slack"] = rng.randint(-40, 200)
        elif op == "fork":
            c["from"] = _log_int(rng, 1, 16)
            c["seqs"] = c["from"] * _log_int(rng, 1, 8)
            c["new"], c["ctx"] = _log_int(rng, 1, 200), _log_int(rng, 1, 2000)
            c["slack"] = rng.randint(-20, 60)
        else:
            c["pages"] = _log_int(rng, 16, 2048)
            c["live"] = max(2, int(c["pages"] * rng.uniform(0.1, 0.9)))
            c["moves"] = int(min(c["live"], c["pages"] - c["live"]) * rng.uniform(0.0, 1.0))
            c["seqs"] = _log_int(rng, 1, min(100, c["live"]))
            c["layers"] = rng.choice([1, 2, 4])
    return c


# ------------------------------------------------------------------------------------------------- what a case means

def _spread(i, most, least):
    """most for i = 0, else values between the two that look ragged and do not repeat soon."""
    return most - int((most - least) * ((i * 0.6180339887498949) % 1.0))


def _news(c):
    """New rows of each sequence: a draft's or a token's are alike, prompts are not."""
    if c["op"] in ("paged", "reserve", "fork"):
        return [c["new"]] * c["seqs"]
    return [_spread(i, c["new"], min(c["new"], 1 + c["new"] // 8)) for i in range(c["seqs"])]


def _lengths(c):
    """Cached positions of each sequence ahead of the new rows."""
    return [_spread(i, c["ctx"], c["ctx"] // 8) for i in range(c["seqs"])]


def _columns(c, lengths, news):
    return max(1, max(-(-(l + n) // c["page"]) for l, n in zip(lengths, news)))


def _elem(c):
    return 1 if c["kv"] == "e4m3" else 2


def work(case):
    c = case
    if c["op"] == "compact":
        page = c["layers"] * c["kv_heads"] * c["page"] * D * 2 * _elem(c)
        return {"bytes": 2 * c["moves"] * page + 4 * (3 * c["pages"] + 2 * c["live"]), "flops": 0}
    news, lengths = _news(c), _lengths(c)
    if c["op"] in ("reserve", "fork"):
        page, of = c["page"], c.get("from", c["seqs"])
        lengths = [lengths[i % of] for i in range(c["seqs"])]
        # the books once in and once out; a copy of the blocks in use of the last page of every continuation but one
        books = 4 * (2 * sum(-(-(l + n) // page) for l, n in zip(lengths, news)) + 2 * c["seqs"])
        copies = 0
        if c["op"] == "fork" and c["slack"] >= 0:
            copies = sum(-(-(lengths[i] % page) // BLOCK) for i in range(of)) * (c["seqs"] // of - 1)
        return {"bytes": books + 2 * copies * BLOCK * c["layers"] * c["kv_heads"] * D * 2 * _elem(c), "flops": 0}
    rows = sum(news)
    hq, hk = c["heads"], c["kv_heads"]
    if c["op"] == "prepare":
        return {"bytes": rows * D * (2 * (hq + 2 * hk) + 2 * hq + 2 * hk * _elem(c)), "flops": rows * D * (hq + hk) * 9}
    pairs = sum(n * l + n * (n + 1) // 2 for l, n in zip(lengths, news))
    cached = sum(l + n for l, n in zip(lengths, news) if n)
    return {"bytes": cached * hk * D * 2 * _elem(c) + 2 * rows * hq * D * 2, "flops": 4 * hq * D * pairs}


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


def _offsets():
    """Place of (position in the block, d) in a block of keys and of values, for 16- and for 8-bit pages: [32, 128] each."""
    p, d = torch.arange(BLOCK, device="cuda")[:, None], torch.arange(D, device="cuda")[None, :]
    sub, p16, step, g4, e = p // 16, p % 16, d // 32, d % 32 // 8, d % 8
    o, dt, dd = p % 16, d // 16, d % 16
    slot = o % 4 + 4 * (p // 16)
    return {"bf16": ((((sub * 4 + step) * 4 + g4) * 16 + p16) * 8 + e, ((dt * 4 + o // 4) * 16 + dd) * 8 + slot),
            "e4m3": (((((sub * 2 + step // 2) * 4 + g4) * 16 + p16) * 2 + step % 2) * 8 + e,
                     (((dt // 2 * 4 + o // 4) * 16 + dd) * 2 + dt % 2) * 8 + slot)}


def _pool(c, inp, layers, pages):
    """Pages as they lie in memory; whatever earlier sequences left there in those that nobody holds."""
    shape = (layers, pages, c["kv_heads"], c["page"] // BLOCK, 2, BLOCK * D)
    x = inp.normal(*shape, dtype=torch.bfloat16)
    return x if c["kv"] == "bf16" else (x * 16.0).to(torch.float8_e4m3fn)


def _books(c, inp, lengths, columns, pages, rows=None):
    """One buffer of refs | lengths | table, and the three as views: the sequences' pages scattered over the pool."""
    seqs = len(lengths)
    held = [-(-l // c["page"]) for l in lengths]
    meta = torch.zeros(pages + seqs + seqs * columns, dtype=torch.int32, device="cuda")
    refs, length, table = meta[:pages], meta[pages:pages + seqs], meta[pages + seqs:].view(seqs, columns)
    length.copy_(torch.tensor(lengths, dtype=torch.int32))
    ids = inp.permutation(pages)[:sum(held)].to(torch.int32) if rows is None else rows
    here = torch.arange(columns, device="cuda")[None, :] < torch.tensor(held, device="cuda")[:, None]
    table.fill_(-1)
    table[here] = ids
    refs[ids.long()] = 1
    return {"meta": meta, "refs": refs, "lengths": length, "table": table}


def _scales(c, inp):
    if c["kv"] == "bf16":
        return None, None
    return tuple((inp.uniform(1, c["kv_heads"]) * 0.5 + 0.75) / 16.0 for _ in range(2))


def prepare(case, seed):
    c, inp = dict(case), _Inputs(seed)
    op = c["op"]
    s = {"c": c, "op": op}
    if op == "compact":
        live, moves, pages = c["live"], c["moves"], c["pages"]
        ids = torch.cat([inp.permutation(live)[:live - moves], live + inp.permutation(pages - live)[:moves]])
        ids = ids[inp.permutation(live)].to(torch.int32)
        each = [live // c["seqs"] + (i < live % c["seqs"]) for i in range(c["seqs"])]
        s.update(_books(c, inp, [n * c["page"] - 7 for n in each], max(each), pages, ids))
        s["pool"] = _pool(c, inp, c["layers"], pages)
        s["before"] = s["meta"].clone()
        return s
    news, lengths = _news(c), _lengths(c)
    columns = _columns(c, lengths, news)
    if op in ("reserve", "fork"):
        at = lengths
        if op == "fork":                                  # the prompts' rows are in use, the others are not yet
            at = [l if i < c["from"] else 0 for i, l in enumerate(lengths)]
            s["parent"] = torch.arange(c["seqs"], device="cuda", dtype=torch.int32) % c["from"]
            lengths = [lengths[i % c["from"]] for i in range(c["seqs"])]
            columns = _columns(c, lengths, news)
        grown = sum(-(-(l + n) // c["page"]) for l, n in zip(lengths, news))
        pages = max(1 + sum(-(-l // c["page"]) for l in at), grown + c["slack"])
        s.update(_books(c, inp, at, columns, pages))
        s["pool"] = _pool(c, inp, c["layers"], pages)
        s["news"] = torch.tensor(news, dtype=torch.int32, device="cuda")
        s["before"] = s["meta"].clone()
        return s
    total = [l + n for l, n in zip(lengths, news)]
    pages = sum(-(-t // c["page"]) for t in total) + 3
    s.update(_books(c, inp, total, columns, pages))       # (room for the new rows is there)
    s["lengths"].copy_(torch.tensor(lengths, dtype=torch.int32))
    s["pool"] = _pool(c, inp, 1, pages)
    s["k_scale"], s["v_scale"] = _scales(c, inp)
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    s["row_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    s["most"] = max(news)
    s["places"] = _offsets()[c["kv"]]
    if op == "prepare":
        s["qkv"] = inp.normal(starts[-1], (c["heads"] + 2 * c["kv_heads"]) * D, dtype=torch.bfloat16)
        s["qg"], s["kg"] = ((1.0 + 0.2 * inp.normal(D)).to(torch.bfloat16) for _ in range(2))
    else:
        s["q"] = inp.normal(starts[-1], c["heads"] * D, dtype=torch.bfloat16)
    return s


# ------------------------------------------------------------------------------------------------------ plain forms

def _rows(s, rows):
    """Sequence and position of every new row."""
    row = torch.arange(rows, device="cuda")
    seq = torch.searchsorted(s["row_start"].long(), row, right=True) - 1
    return seq, s["lengths"].long()[seq] + row - s["row_start"].long()[seq]


def _norm_rope(x, gamma, pos):
    """x [rows, heads, 128] fp32: a norm of each head, rounded as bf16 code does, then rotated by its position."""
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    x = (x.to(torch.bfloat16).float() * gamma.float()).to(torch.bfloat16).float()
    inv = THETA ** (-2.0 * torch.arange(D // 2, device="cuda", dtype=torch.float64) / D)
    a = pos.double()[:, None] * inv
    cos, sin = a.cos().float()[:, None], a.sin().float()[:, None]
    x1, x2 = x[..., :D // 2], x[..., D // 2:]
    return torch.cat([x1 * cos - x2 * sin, x2 * cos + x1 * sin], -1).to(torch.bfloat16)


def _plain_prepare(s):
    c, pool = s["c"], s["pool"]
    hq, hk = c["heads"], c["kv_heads"]
    rows = s["qkv"].shape[0]
    seq, pos = _rows(s, rows)
    x = s["qkv"].view(rows, hq + 2 * hk, D).float()
    q = _norm_rope(x[:, :hq], s["qg"], pos)
    k = _norm_rope(x[:, hq:hq + hk], s["kg"], pos)
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


def _gathered(s, half, columns):
    """Keys or values of every sequence by position: [seqs, kv heads, columns * page, 128] fp32."""
    c = s["c"]
    ids = s["table"][:, :columns].long().clamp(min=0)
    x = s["pool"][0].view(torch.int16 if c["kv"] == "bf16" else torch.uint8)[:, :, :, half][ids]     # [seqs, columns, heads, blocks, 4096]
    x = x[..., s["places"][half].reshape(-1)].view(s["pool"].dtype).float()
    scale = s["k_scale"] if half == 0 else s["v_scale"]
    seqs, cols, hk, nb, _ = x.shape
    x = x.view(seqs, cols, hk, nb, BLOCK, D).permute(0, 2, 1, 3, 4, 5).reshape(seqs, hk, cols * nb * BLOCK, D)
    return x if scale is None else x * scale[0][:, None, None]


def _plain_attention(s):
    c = s["c"]
    hq, hk, most = c["heads"], c["kv_heads"], s["most"]
    start, lengths = s["row_start"].long(), s["lengths"].long()
    news = start[1:] - start[:-1]
    rows = s["q"].shape[0]
    i = torch.arange(most, device="cuda")
    at = (start[:-1, None] + i).clamp(max=rows - 1)
    q = s["q"].view(rows, hk, hq // hk, D)[at].float()                             # [seqs, most, kv heads, group, 128]
    q = q.permute(0, 2, 3, 1, 4).reshape(len(news), hk, hq // hk * most, D)
    columns = s["table"].shape[1]
    score = torch.matmul(q, _gathered(s, 0, columns).transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(D))
    seen = torch.arange(columns * c["page"], device="cuda") <= (lengths[:, None] + i)[..., None]
    score = score.view(len(news), hk, hq // hk, most, -1).masked_fill_(~seen[:, None, None], -math.inf)
    score = score.sub_(score.amax(-1, keepdim=True)).exp_()
    score = score.div_(score.sum(-1, keepdim=True)).view(len(news), hk, hq // hk * most, -1)
    out = torch.matmul(score, _gathered(s, 1, columns)).view(len(news), hk, hq // hk, most, D)
    seq, pos = _rows(s, rows)
    out = out.permute(0, 3, 1, 2, 4)[seq, pos - lengths[seq]]                      # [rows, kv heads, group, 128]
    return out.reshape(rows, hq * D).to(torch.bfloat16)


def _plain_fork(s):
    """Row s of the table becomes row parent[s]; the pages count their new holders."""
    table, refs, lengths, page = s["table"], s["refs"], s["lengths"], s["c"]["page"]
    old = table.clone()
    lengths.copy_(lengths[s["parent"].long()])
    held = torch.arange(table.shape[1], device="cuda") < (lengths[:, None] + page - 1) // page
    table.copy_(torch.where(held, old[s["parent"].long()], -1))
    one = torch.ones_like(old)
    spare = torch.zeros(refs.numel() + 1, dtype=torch.int32, device="cuda")        # (the last entry counts what is no page)
    spare.index_add_(0, torch.where(table < 0, refs.numel(), table).flatten().long(), one.flatten())
    spare.index_add_(0, torch.where(old < 0, refs.numel(), old).flatten().long(), -one.flatten())
    refs.add_(spare[:-1])


def _plain_reserve(s):
    """Pages for the new rows of every sequence, lowest free ones first; a shared last page is replaced by a copy."""
    table, refs, lengths, page, news = s["table"], s["refs"], s["lengths"], s["c"]["page"], s["news"]
    first, need = lengths // page, (lengths + news + page - 1) // page
    col = torch.arange(table.shape[1], device="cuda")[None, :]
    asks = (news > 0) & (need <= table.shape[1])
    span = (col >= first[:, None]) & (col < need[:, None]) & asks[:, None]
    last = table.gather(1, first.long().clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    writes = asks & (lengths % page != 0) & (last >= 0)
    same = (last[:, None] == last[None, :]) & writes[:, None] & writes[None, :]
    earlier = same.tril(-1).sum(1)
    copied = writes & (refs[last.clamp(min=0).long()] - earlier > 1)
    wanted = span & ((table < 0) | (copied[:, None] & (col == first[:, None])))
    free = torch.nonzero(refs == 0).flatten()
    ok = (wanted.sum(1).cumsum(0) <= free.numel()) & asks
    wanted &= ok[:, None]
    copied &= ok
    got = free[:int(wanted.sum())].to(torch.int32)
    table[wanted] = got
    refs[got.long()] = 1
    refs.index_add_(0, last[copied].long(), -torch.ones_like(last[copied]))
    new = table.gather(1, first.long().clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    blocks = (lengths % page + BLOCK - 1) // BLOCK
    pair = copied[:, None] & (torch.arange(page // BLOCK, device="cuda")[None, :] < blocks[:, None])
    seq, block = torch.nonzero(pair).unbind(1)
    raw = s["pool"].view(torch.int16 if s["c"]["kv"] == "bf16" else torch.uint8)
    raw[:, new[seq].long(), :, block] = raw[:, last[seq].long(), :, block]
    return (ok | (news <= 0)).to(torch.int32)


def _plain_compact(s):
    """The pages in use become the first of the pool: those beyond move to the free ones below, in order."""
    table, refs = s["table"], s["refs"]
    live = refs > 0
    n = int(live.sum())
    moved, holes = torch.nonzero(live[n:]).flatten() + n, torch.nonzero(~live[:n]).flatten()
    to = torch.arange(refs.numel(), dtype=torch.int32, device="cuda")
    to[moved] = holes.to(torch.int32)
    table.copy_(torch.where(table < 0, table, to[table.clamp(min=0).long()]))
    refs[holes] = refs[moved]
    refs[moved] = 0
    raw = s["pool"].view(torch.int16 if s["c"]["kv"] == "bf16" else torch.uint8)
    raw[:, holes] = raw[:, moved]
    return to


# -------------------------------------------------------------------------------------------------------------- run

def _cache(s):
    """The handle that a program keeps: made once, over the program's own tensors."""
    if "cache" not in s:
        from paper_2603_01399_amd import binding as qb
        pool, c = s["pool"], s["c"]
        s["cache"] = qb.PagedKvCache(pool.shape[0], pool.shape[2], pool.shape[1], page_len=c["page"], max_seqs=s["table"].shape[0],
                                     max_pages=s["table"].shape[1], dtype=pool.dtype, k_scale=s.get("k_scale"), v_scale=s.get("v_scale"),
                                     pool=pool, books=s["meta"])
        s["qb"] = qb
    return s["qb"], s["cache"]


def run(state):
    s = state
    op, c = s["op"], s["c"]
    if op in ("reserve", "fork", "compact"):
        s["meta"].copy_(s["before"])                      # (the books as they were: a pass can be repeated)
    if own:
        qb, cache = _cache(s)
        if op == "prepare":
            q = qb.paged_prepare(s["qkv"], c["heads"], cache, 0, s["row_start"], s["qg"], s["kg"], eps=EPS, rope_theta=THETA)
            return {"q": q, "pool": s["pool"]}
        if op == "paged":
            return qb.paged_attention(s["q"], c["heads"], cache, 0, s["row_start"], s["most"])
        if op == "prompt":
            return qb.prompt_attention(s["q"], c["heads"], cache, 0, s["row_start"])
        if op == "compact":
            to = cache.compact()
            return {"to": to, "table": s["table"], "refs": s["refs"], "pool": s["pool"]}
        if op == "fork":
            cache.fork(s["parent"])
        status = cache.reserve(s["news"])
    else:
        if op == "prepare":
            return _plain_prepare(s)
        if op in ("paged", "prompt"):
            return _plain_attention(s)
        if op == "compact":
            to = _plain_compact(s)
            return {"to": to, "table": s["table"], "refs": s["refs"], "pool": s["pool"]}
        if op == "fork":
            _plain_fork(s)
        status = _plain_reserve(s)
    out = {"status": status, "table": s["table"], "refs": s["refs"], "lengths": s["lengths"]}
    return dict(out, pool=s["pool"]) if op == "fork" else out


# ------------------------------------------------------------------------------------------------------------ exact

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


def exact(case, seed):
    s = prepare(case, seed)
    c, places = s["c"], _exact_places(case["kv"])
    if s["op"] not in ("prepare", "paged", "prompt"):
        return None                                       # books and copies: nothing is computed
    hq, hk, page = c["heads"], c["kv_heads"], c["page"]
    table, lengths, start = s["table"].tolist(), s["lengths"].tolist(), s["row_start"].tolist()
    scales = [torch.ones(hk, dtype=torch.float64, device="cuda") if x is None else x[0].double() for x in (s["k_scale"], s["v_scale"])]
    if s["op"] == "prepare":
        rows = s["qkv"].shape[0]
        pos = torch.cat([torch.arange(lengths[b], lengths[b] + start[b + 1] - start[b], device="cuda") for b in range(c["seqs"])])
        x = s["qkv"].view(rows, hq + 2 * hk, D).double()
        n = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt()
        freq = torch.tensor([THETA ** (-i / 64.0) for i in range(64)], dtype=torch.float64, device="cuda")
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), pos.double()[:, None] * freq)[:, None]
        done = []
        for part, gamma in ((n[:, :hq], s["qg"]), (n[:, hq:hq + hk], s["kg"])):
            y = part * gamma.double()
            z = torch.complex(y[..., :64].contiguous(), y[..., 64:].contiguous()) * turn
            done.append(torch.cat([z.real, z.imag], -1))
        pool = s["pool"].double()
        stored = [done[1] / scales[0][:, None], x[:, hq + hk:] / scales[1][:, None]]
        if c["kv"] == "e4m3":
            stored = [t.clamp(-E4M3_MOST, E4M3_MOST) for t in stored]
        for half in range(2):
            p, d = places[half]
            where = torch.empty((BLOCK, D), dtype=torch.long, device="cuda")
            where[p, d] = torch.arange(BLOCK * D, device="cuda")
            r = 0
            for b in range(c["seqs"]):
                n_b, j = start[b + 1] - start[b], torch.arange(lengths[b], lengths[b] + start[b + 1] - start[b], device="cuda")
                ids = torch.tensor(table[b], device="cuda")[j // page]
                for h in range(hk):
                    pool[0, ids[:, None], h, (j % page // BLOCK)[:, None], half, where[j % BLOCK]] = stored[half][r:r + n_b, h]
                r += n_b
        return {"q": done[0].reshape(rows, hq * D), "pool": pool}
    out = torch.zeros(s["q"].shape[0], hq, D, dtype=torch.float64, device="cuda")
    group = hq // hk
    for b in range(c["seqs"]):
        n, l = start[b + 1] - start[b], lengths[b]
        if n == 0:
            continue
        ids = torch.tensor(table[b], device="cuda")[:-(-(l + n) // page)]
        for h in range(hk):
            kv = []
            for half in range(2):
                block = s["pool"][0, :, h, :, half].view(torch.int16 if c["kv"] == "bf16" else torch.uint8)[ids]
                block = block.view(s["pool"].dtype).reshape(-1, BLOCK * D).double() * scales[half][h]
                p, d = places[half]
                plain = torch.empty(block.shape[0], BLOCK, D, dtype=torch.float64, device="cuda")
                plain[:, p, d] = block
                kv.append(plain.reshape(-1, D)[:l + n])
            hidden = torch.arange(l + n, device="cuda")[None, :] > l + torch.arange(n, device="cuda")[:, None]
            for g in range(group):
                q = s["q"].view(-1, hq, D)[start[b]:start[b] + n, h * group + g].double()
                w = (q @ kv[0].t() / math.sqrt(D)).masked_fill(hidden, -math.inf).softmax(-1)
                out[start[b]:start[b] + n, h * group + g] = w @ kv[1]
    return out.reshape(-1, hq * D)
