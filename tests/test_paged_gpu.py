"""GPU parity of the paged cache's operators through the C ABI against the CPU oracle: append, attention of a step and of prompts, the
books.  Attention is held element by element to a tolerance counted from its roundings (paged_util.Batch.expected); pages that no
position lies in hold NaN patterns throughout."""
import numpy as np
import pytest
import torch

from oracle import quasar_attention_ref as at
from oracle import quasar_paged_ref as pg
from oracle import quasar_ref as ref
from paged_marks import attention_and_bound, block_values
from paged_util import Batch, rnd_bits
from gpu_util import bf16_to_dev, bf16_to_host, i32_to_dev

pytestmark = pytest.mark.gpu
D = 128


@pytest.fixture(scope="module")
def qb():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2603_01399_amd import binding
    return binding


def say(*a):
    print(*a, flush=True)


def close(got_bits, b):
    got = ref.bf16_bits_to_f64(got_bits).reshape(b.rows, b.hq, D)
    want, tol = b.expected()
    over = np.abs(got - want) / tol
    say("   worst of tolerance", float(over.max()))
    assert np.isfinite(got).all() and (over <= 1.0).all()


# kv, page, Hq, Hkv, cached, new
STEP = [("bf16", 64, 8, 2, [0], [1]), ("bf16", 32, 4, 4, [31], [1]), ("bf16", 32, 4, 1, [32], [1]), ("bf16", 64, 32, 8, [1000, 0, 77, 4095], [1, 1, 1, 1]),
        ("bf16", 64, 32, 8, [63, 64, 65], [8, 8, 8]), ("bf16", 128, 40, 8, [500, 3], [3, 7]), ("bf16", 64, 8, 1, [100, 5000, 20], [5, 0, 2]),
        ("bf16", 1024, 8, 8, [2000, 10], [2, 1]), ("bf16", 64, 16, 2, [700], [32]), ("bf16", 32, 64, 8, [90, 1], [16, 13]),
        ("e4m3", 64, 8, 2, [0], [1]), ("e4m3", 32, 32, 8, [1000, 0, 77, 4095], [1, 1, 1, 1]), ("e4m3", 128, 64, 8, [9000, 130], [8, 8]),
        ("e4m3", 64, 16, 2, [700, 64], [32, 1]), ("e4m3", 256, 5, 1, [3000], [10]), ("bf16", 64, 4, 2, [200] * 70, [1] * 70),
        ("e4m3", 32, 4, 2, list(range(0, 280, 7)), [1, 2, 0, 3] * 10), ("bf16", 64, 2, 1, [30000, 5, 12000], [4, 4, 4]), ("bf16", 32, 24, 1, [33], [32])]


@pytest.mark.parametrize("kv,page,hq,hk,lengths,news", STEP)
def test_attention_of_a_step(qb, kv, page, hq, hk, lengths, news):
    say("paged attention", kv, page, hq, hk, lengths[:5], news[:5])
    b = Batch(qb, kv, page, hq, hk, lengths, news, seed=len(lengths) + hq)
    close(bf16_to_host(qb.paged_attention(b.q(), hq, b.cache, 0, b.row_start, max(news))), b)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("group,new", [(1, 1), (1, 16), (1, 17), (1, 32), (3, 5), (3, 11), (5, 7), (8, 8), (8, 9), (2, 32), (7, 10), (8, 16), (8, 17), (16, 32), (32, 32)])
def test_attention_of_any_number_of_rows(qb, kv, group, new):
    """Rows of a sequence and kv head around every form's border, over lengths that one worker and that many take."""
    say("rows", kv, group, new)
    b = Batch(qb, kv, 64, 2 * group, 2, [1500, 31, 4, 0, 700], [new, 1, max(new - 1, 0), new, 0], seed=200 + group + new)
    close(bf16_to_host(qb.paged_attention(b.q(), 2 * group, b.cache, 0, b.row_start, new)), b)


PROMPT = STEP[:9] + STEP[10:16] + [
    ("bf16", 64, 4, 1, [0], [64]), ("bf16", 64, 4, 4, [0], [1]), ("bf16", 64, 8, 2, [0], [65]), ("bf16", 32, 8, 2, [0, 0, 0], [130, 0, 257]),
    ("bf16", 64, 5, 1, [0, 40], [300, 77]), ("bf16", 128, 2, 2, [1000, 0], [200, 700]), ("e4m3", 64, 8, 2, [0, 100], [129, 311]),
    ("e4m3", 32, 3, 1, [37], [500]), ("bf16", 64, 8, 1, [0], [1100]), ("e4m3", 1024, 8, 4, [1500], [40])]


@pytest.mark.parametrize("kv,page,hq,hk,lengths,news", PROMPT)
def test_attention_of_prompts(qb, kv, page, hq, hk, lengths, news):
    say("prompt attention", kv, page, hq, hk, lengths[:5], news[:5])
    b = Batch(qb, kv, page, hq, hk, lengths, news, seed=len(lengths) + hq + 50)
    close(bf16_to_host(qb.prompt_attention(b.q(), hq, b.cache, 0, b.row_start)), b)


@pytest.mark.parametrize("call", ["paged", "prompt"])
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_strides_other_layers_and_rows_of_nobody(qb, call, kv):
    """q and out as column blocks of wider tensors, the second of three layers, rows ahead of the first and behind the last sequence."""
    say("strides", call, kv)
    b = Batch(qb, kv, 64, 8, 2, [70, 0, 300], [3, 0, 5], layers=3, layer=1, seed=9, empty_rows=2)
    wide = torch.full((b.rows + 7, 8 * D + 48), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[2:2 + b.rows, 16:16 + 8 * D] = b.q()
    out = torch.full((b.rows + 7, 8 * D + 12), 7.0, dtype=torch.bfloat16, device="cuda")
    q, o, starts = wide[:, 16:16 + 8 * D], out[:, 4:4 + 8 * D], b.row_start + 2
    if call == "paged":
        qb.paged_attention(q, 8, b.cache, 1, starts, 5, out=o)
    else:
        qb.prompt_attention(q, 8, b.cache, 1, starts, out=o)
    close(bf16_to_host(o[2:2 + b.rows]), b)
    assert (out[:2] == 7).all() and (out[2 + b.rows:] == 7).all() and (out[:, :4] == 7).all() and (out[:, 4 + 8 * D:] == 7).all()


@pytest.mark.parametrize("call", ["paged", "prompt"])
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_positions_without_a_page_are_not_visible(qb, call, kv):
    """Ids below 0 or beyond the pool read nothing; a row that is left with nothing gives zeros."""
    say("missing pages", call, kv)
    b = Batch(qb, kv, 32, 4, 2, [100, 20, 64], [4, 4, 2], seed=21)
    table = b.cache.table.clone()
    table[0, 1] = -1                                   # positions 32 .. 63 of the first sequence
    table[0, 2] = b.cache.n_pages
    table[1, 0] = 2 ** 31 - 1                          # the whole second one
    b.cache.table.copy_(table)
    fn = (lambda: qb.paged_attention(b.q(), 4, b.cache, 0, b.row_start, 4)) if call == "paged" else (lambda: qb.prompt_attention(b.q(), 4, b.cache, 0, b.row_start))
    got = ref.bf16_bits_to_f64(bf16_to_host(fn())).reshape(b.rows, 4, D)
    assert (got[4:8] == 0).all()
    # the first sequence by hand: what is left of it, in order
    kept = np.r_[0:32, 96:104]
    b.keys[0], b.values[0], b.lengths[0] = b.keys[0][kept], b.values[0][kept], 36
    want, tol = b.expected()
    assert (np.abs(got - want) <= tol)[np.r_[0:4, 8:10]].all()


@pytest.mark.parametrize("kv,bad", [("bf16", np.inf), ("bf16", -np.inf), ("bf16", np.nan), ("e4m3", np.nan)])
@pytest.mark.parametrize("call,hq,news", [(c, *x) for c in ("paged", "prompt") for x in ((2, [6, 1]), (8, [5, 3]), (20, [8, 2]))] + [("prompt", 8, [40, 7])])
def test_what_is_not_finite_reaches_the_rows_that_see_it_alone(qb, call, kv, bad, hq, news):
    """A key and a value that are not finite, at new positions: rows behind them get no finite value for the head; rows before them and
    other sequences and heads are as near the oracle as ever.  (Not their bits: 32 rows move the maximum that their weights are taken
    against together, and another one rounds the weights elsewhere.)"""
    say("not finite", call, kv, bad, hq, news)
    b = Batch(qb, kv, 64, hq, 2, [90, 33], news, seed=300 + hq)
    fn = lambda: (qb.paged_attention(b.q(), hq, b.cache, 0, b.row_start, max(news)) if call == "paged" else qb.prompt_attention(b.q(), hq, b.cache, 0, b.row_start))
    want, tol = b.expected()
    places, raw = pg.block_places(kv), b.cache.pool[0].view(torch.int16 if kv == "bf16" else torch.uint8)
    bits = int(ref.f32_to_bf16_bits(np.array([bad], np.float32)).view(np.int16)[0]) if kv == "bf16" else 0x7F
    for half in (0, 1):
        keep = raw.clone()
        pos = 90 + 3                                       # row 3 of the first sequence
        raw[int(b.table[0, pos // 64]), 1, pos % 64 // 32, half, int(places[half][pos % 32, 17])] = bits
        got = fn().view(b.rows, hq, D)
        raw.copy_(keep)
        same = torch.ones((b.rows, hq), dtype=torch.bool, device="cuda")
        same[3:news[0], hq // 2:] = False
        same = same.cpu().numpy()
        assert (np.abs(got.double().cpu().numpy() - want)[same] <= tol[same]).all()
        seen = got[3:news[0], hq // 2:].float()
        if half == 1:                                      # (a score of -inf is a weight of 0: no fault of the output)
            assert not torch.isfinite(seen).all(dim=2).any()
        elif not np.isinf(bad):
            assert not torch.isfinite(seen).all(dim=2).any()


@pytest.mark.parametrize("call", ["paged", "prompt"])
def test_books_that_do_not_fit(qb, call):
    """Lengths beyond the table end with it, rows beyond the tensor or below 0 are nobody's, more than max_new rows are left."""
    say("odd books", call)
    b = Batch(qb, "bf16", 32, 4, 2, [60, 40, 30, 20], [2, 2, 2, 6], seed=22, more_columns=0)
    fn = lambda starts, out: (qb.paged_attention(b.q(), 4, b.cache, 0, starts, 4, out=out) if call == "paged" else qb.prompt_attention(b.q(), 4, b.cache, 0, starts, out=out))
    good = torch.full((b.rows, 4 * D), 5.0, dtype=torch.bfloat16, device="cuda")
    fn(b.row_start, good)
    torch.cuda.synchronize()
    assert (good[:10] != 5).any(dim=1).all() and ((good[10:] == 5).all() if call == "paged" else (good != 5).any(dim=1).all())
    for starts in ([0, 2, 4, 6, 99], [-3, 2, 4, 6, 12], [0, 2, 1, 6, 12], [2 ** 31 - 1] * 5, [-2 ** 31] * 5):
        out = torch.full((b.rows, 4 * D), 5.0, dtype=torch.bfloat16, device="cuda")
        fn(i32_to_dev(starts), out)
        torch.cuda.synchronize()
        if starts[:4] == [0, 2, 4, 6]:
            assert torch.equal(out[:6], good[:6]) and (out[6:] == 5).all()
        if abs(starts[0]) > 99:
            assert (out == 5).all()
    for length in (-1, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31):
        b.cache.lengths[0] = length
        out = torch.full((b.rows, 4 * D), 5.0, dtype=torch.bfloat16, device="cuda")
        fn(b.row_start, out)
        assert torch.equal(out[2:], good[2:]) and (out[:2] == 5).all()
    b.cache.lengths[0] = 2 ** 24                       # (a length that is allowed, of which the table holds the first 64)
    out = fn(b.row_start, torch.empty_like(good))
    assert torch.equal(out[2:10], good[2:10])


@pytest.mark.parametrize("call", ["paged", "prompt"])
def test_peaked_and_even_scores(qb, call):
    """Scores that grow along the positions move the running maximum at every step; equal keys give the mean; one key dominates."""
    say("peaked", call)
    b = Batch(qb, "bf16", 64, 4, 2, [400], [3], seed=23)
    fn = lambda: bf16_to_host(qb.paged_attention(b.q(), 4, b.cache, 0, b.row_start, 3) if call == "paged" else qb.prompt_attention(b.q(), 4, b.cache, 0, b.row_start))
    kp, vp = pg.block_places("bf16")
    for kind in ("growing", "falling", "equal", "one"):
        j = np.arange(403)
        keys = np.zeros((403, 2, D))
        if kind in ("growing", "falling"):
            keys[..., 0] = (j if kind == "growing" else 402 - j)[:, None] * 2.0
        if kind == "one":
            keys[137] = 8.0
        bits = ref.f32_to_bf16_bits(keys.astype(np.float32))
        b.q_bits = ref.f32_to_bf16_bits(np.full((3, 4, D), 2.0, np.float32))
        raw = b.cache.pool[0].view(torch.int16).cpu().numpy()
        for h in range(2):
            raw[b.table[0, j // 64][:, None], h, (j % 64 // 32)[:, None], 0, kp[j % 32]] = bits[:, h].view(np.int16)
        b.cache.pool[0].view(torch.int16).copy_(torch.from_numpy(raw))
        b.keys[0] = ref.bf16_bits_to_f64(bits)
        close(fn(), b)


PREPARE = [("bf16", 64, 32, 8, [0], [1]), ("bf16", 32, 4, 2, [31, 0, 64], [2, 0, 3]), ("e4m3", 64, 32, 8, [1000, 5], [1, 1]), ("bf16", 64, 6, 2, [0, 100, 31], [70, 33, 2]),
           ("e4m3", 128, 8, 8, [0, 17, 95], [200, 40, 161]), ("bf16", 64, 5, 5, [30000, 3], [4, 300]), ("e4m3", 32, 8, 1, [0], [1]), ("bf16", 64, 8, 2, [20] * 40, [1] * 40)]


@pytest.mark.parametrize("kv,page,hq,hk,lengths,news", PREPARE)
def test_prepare(qb, kv, page, hq, hk, lengths, news):
    """Values the given bits (or their rounding); queries and keys near the fp64 oracle; every other byte of the pool as it was.

    How near: the two roundings of the norm go either way where fp32 and fp64 lie on two sides of a border.  The first moves the
    normalised value by one bf16 step, 2^-7 of it at most; times gamma and rounded again, by another step: n is off by at most 2^-6 |n|.  The
    rotation takes that over from both halves of a pair, 2^-6 (|n_i| + |n_j|), and its own rounding may go the other way too, 2^-7 of the
    result.  All of that is rare: 98 % are the oracle's bits.  An 8-bit code adds half a step, 2^-4 of the value or 2^-10 scales."""
    say("paged prepare", kv, page, hq, hk, lengths[:4], news[:4])
    b = Batch(qb, kv, page, hq, hk, lengths, news, layers=2, layer=1, seed=31 + hq)
    T, heads = b.rows, hq + 2 * hk
    qkv = rnd_bits((T, heads, D), 41, 2.0)
    gq, gk = (ref.f32_to_bf16_bits((1.0 + 0.2 * np.random.Generator(np.random.Philox(s)).standard_normal(D)).astype(np.float32)) for s in (5, 6))
    before = b.cache.pool.view(torch.uint8).clone()
    wide = torch.zeros((T, heads * D + 24), dtype=torch.bfloat16, device="cuda")
    wide[:, 8:8 + heads * D] = bf16_to_dev(qkv.reshape(T, -1))
    q_out = torch.full((T + 2, hq * D + 8), 3.0, dtype=torch.bfloat16, device="cuda")
    qb.paged_prepare(wide[:, 8:8 + heads * D], hq, b.cache, 1, b.row_start, bf16_to_dev(gq), bf16_to_dev(gk), eps=1e-6, rope_theta=1e6, q_out=q_out[1:T + 1, :hq * D])
    torch.cuda.synchronize()
    assert (q_out[0] == 3).all() and (q_out[T + 1] == 3).all() and (q_out[:, hq * D:] == 3).all()
    pos = np.concatenate([np.arange(l, l + n) for l, n in zip(lengths, news)])
    want_q, want_k = at.head_norm_rope(qkv[:, :hq], gq, 1e-6, pos, 1e6), at.head_norm_rope(qkv[:, hq:hq + hk], gk, 1e-6, pos, 1e6)
    f64, none = ref.bf16_bits_to_f64, np.zeros(T)

    def slack(bits, x, gamma):
        n = np.abs(f64(at.head_norm_rope(x, gamma, 1e-6, none, 1e6)))                     # (position 0 is not rotated)
        return 2.0 ** -6 * (n + np.roll(n, D // 2, axis=2)) + 2.0 ** -7 * np.abs(f64(bits))

    got_q = bf16_to_host(q_out[1:T + 1, :hq * D]).reshape(T, hq, D)
    assert (np.abs(f64(got_q) - f64(want_q)) <= slack(want_q, qkv[:, :hq], gq)).all() and np.mean(got_q != want_q) < 0.02
    k_slack = slack(want_k, qkv[:, hq:hq + hk], gk)
    row = 0
    for s, (l, n) in enumerate(zip(lengths, news)):
        got_k, got_v = b.read(s, l + n, 0)[l:], b.read(s, l + n, 1)[l:]
        k, v, near = want_k[row:row + n], qkv[row:row + n, hq + hk:], k_slack[row:row + n]
        row += n
        if kv == "bf16":
            assert np.array_equal(got_v, v) and (np.abs(f64(got_k) - f64(k)) <= near).all() and (n == 0 or np.mean(got_k != k) < 0.02)
            continue
        ks, vs = b.scales[0][1][:, None], b.scales[1][1][:, None]
        code = lambda x, scale: pg.f64_to_e4m3((ref.bf16_bits_to_f64(x).astype(np.float32) / scale).astype(np.float32))
        assert np.array_equal(got_v, code(v, vs))
        assert (np.abs(pg.e4m3_to_f64(got_k) * ks - f64(k)) <= near + 2.0 ** -4 * (np.abs(f64(k)) + near) + 2.0 ** -10 * ks).all()
        assert n == 0 or np.mean(got_k != code(k, ks)) < 0.02
    # nothing else has changed
    mine = torch.zeros_like(before, dtype=torch.bool)
    e = 2 if kv == "bf16" else 1
    flat = mine.view(2, b.cache.n_pages, hk, page // 32, 2, 4096, e)
    for half, places in enumerate(pg.block_places(kv)):
        for s, (l, n) in enumerate(zip(lengths, news)):
            j = np.arange(l, l + n)
            for h in range(hk):
                ix = [torch.from_numpy(np.ascontiguousarray(a)).cuda().long() for a in (b.table[s, j // page][:, None], (j % page // 32)[:, None], places[j % 32])]
                flat[1][ix[0], h, ix[1], half, ix[2]] = True
    after = b.cache.pool.view(torch.uint8)
    assert torch.equal(after[~mine], before[~mine])


def test_prepare_writes_nothing_without_a_page(qb):
    say("prepare without pages")
    b = Batch(qb, "bf16", 32, 4, 2, [30, 10, 5], [4, 3, 2], seed=33)
    b.cache.table[0, 1] = -1
    b.cache.table[1, 0] = b.cache.n_pages
    b.cache.lengths[2] = 2 ** 24                         # beyond the table
    before = b.cache.pool.clone()
    qkv = bf16_to_dev(rnd_bits((b.rows, 8 * D), 42))
    g = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    q = qb.paged_prepare(qkv, 4, b.cache, 0, b.row_start, g, g)
    changed = (before.view(torch.int16) != b.cache.pool.view(torch.int16)).flatten(2).any(2)[0]
    page = int(b.cache.table[0, 0])
    assert changed.nonzero().flatten().tolist() == [page] and torch.isfinite(q).all()
    other = torch.full_like(q, 9.0)                      # rows behind the last sequence
    qb.paged_prepare(qkv, 4, b.cache, 0, b.row_start[:2], g, g, q_out=other)
    assert torch.equal(other[:4], q[:4]) and (other[4:] == 9).all()


def test_saturating_codes(qb):
    """Values beyond the 8-bit range are stored as its largest."""
    say("saturation")
    b = Batch(qb, "e4m3", 32, 2, 1, [0], [2], seed=34, scaled=False)
    qkv = torch.zeros((2, 4 * D), dtype=torch.bfloat16, device="cuda")
    qkv[0, 3 * D:] = 1000.0
    qkv[1, 3 * D:] = -464.0
    g = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    qb.paged_prepare(qkv, 2, b.cache, 0, b.row_start, g, g)
    got = pg.e4m3_to_f64(b.read(0, 2, 1))
    assert (got[0] == 448).all() and (got[1] == -448).all()


# -------------------------------------------------------------------------------------------------------------- books

def books_of(cache):
    return cache.refs.tolist(), cache.lengths.tolist(), cache.table.tolist()


def random_cache(qb, r, *, seqs, columns, page, pages, layers=2, hk=2, kv="bf16", shared=0.5):
    """A cache whose sequences hold random lengths, some of them prefixes of others' pages, every byte of the pool random."""
    cache = qb.PagedKvCache(layers, hk, pages, page_len=page, max_seqs=seqs, max_pages=columns, dtype=torch.bfloat16 if kv == "bf16" else torch.float8_e4m3fn)
    refs, lengths, table = np.zeros(pages, int), np.zeros(seqs, int), np.full((seqs, columns), -1)
    for s in range(seqs):
        if s and r.random() < shared:
            p = int(r.integers(0, s))
            lengths[s] = int(r.integers(0, lengths[p] + 1))
            held = -(-lengths[s] // page)
            table[s, :held] = table[p, :held]
            refs[table[s, :held]] += 1
        else:
            free = np.flatnonzero(refs == 0)
            most = min(columns, len(free), 1 + 2 * pages // max(seqs, 1))
            lengths[s] = int(r.integers(0, most * page + 1))
            held = -(-lengths[s] // page)
            table[s, :held] = r.permutation(free)[:held]
            refs[table[s, :held]] = 1
            if held < min(columns, most) and r.random() < 0.3:            # a page without positions yet
                table[s, held] = np.flatnonzero(refs == 0)[0]
                refs[table[s, held]] = 1
    cache.refs.copy_(i32_to_dev(refs)); cache.lengths.copy_(i32_to_dev(lengths)); cache.table.copy_(i32_to_dev(table))
    raw = torch.from_numpy(r.integers(0, 256, cache.pool.nbytes, dtype=np.uint8)).cuda()
    cache.pool.view(torch.uint8).view(-1).copy_(raw)
    return cache, pg.Books(refs, lengths, table, page)


def check(cache, books, pool):
    """Books equal to the oracle's, and the pool to `pool` with the oracle's copies done in order."""
    refs, lengths, table = books_of(cache)
    assert refs == books.refs and lengths == books.lengths and table == books.table
    want = pool.clone()
    for src, dst, blocks in books.copies:
        want[:, dst, :, :blocks] = pool[:, src, :, :blocks]
    books.copies = []
    assert torch.equal(cache.pool.view(torch.uint8), want)


@pytest.mark.parametrize("seed", range(12))
def test_books_over_many_steps(qb, seed):
    """Reserve, fork, cut, free and compact in turn, in odd sizes, with too few pages now and then."""
    r = np.random.Generator(np.random.Philox(1000 + seed))
    seqs, columns, page = int(r.integers(1, 40)), int(r.integers(1, 30)), int(r.choice([32, 64, 128]))
    pages = int(r.integers(4, 300))
    say("books", seed, seqs, columns, page, pages)
    cache, books = random_cache(qb, r, seqs=seqs, columns=columns, page=page, pages=pages, kv=["bf16", "e4m3"][seed % 2], hk=1 + seed % 3, layers=1 + seed % 2)
    for step in range(6):
        pool = cache.pool.view(torch.uint8).clone()
        n_new = r.integers(-1, [3, 40, 700][step % 3], seqs)
        status = cache.reserve(i32_to_dev(n_new))
        assert status.tolist() == books.reserve(n_new)
        check(cache, books, pool)
        grown = np.where(np.array(status.tolist()) == 1, np.maximum(n_new, 0) * r.random(seqs), 0).astype(int)   # (some of it accepted)
        books.lengths = [int(a + b) for a, b in zip(books.lengths, grown)]
        cache.lengths += i32_to_dev(grown)
        pool = cache.pool.view(torch.uint8).clone()
        parent = np.where(r.random(seqs) < 0.5, np.arange(seqs), r.integers(-1, seqs + 1, seqs))
        keep = None if step % 2 else np.where(r.random(seqs) < 0.5, 1 << 25, r.integers(-2, 2000, seqs))
        cache.fork(i32_to_dev(parent), None if keep is None else i32_to_dev(keep))
        books.copies = []
        books.fork(parent, keep)
        check(cache, books, pool)
        if step % 2:
            to = cache.compact()
            assert to.tolist() == books.compact()
            check(cache, books, pool)
            live = sum(x > 0 for x in books.refs)
            assert all(x > 0 for x in books.refs[:live])


@pytest.mark.parametrize("seqs,pages", [(1, 1), (1024, 5000), (3, 70000)])
def test_books_at_the_largest_sizes(qb, seqs, pages):
    say("books", seqs, pages)
    r = np.random.Generator(np.random.Philox(seqs))
    cache, books = random_cache(qb, r, seqs=seqs, columns=9, page=32, pages=pages, layers=1, hk=1, shared=0.2)
    pool = cache.pool.view(torch.uint8).clone()
    n_new = r.integers(0, 70, seqs)
    assert cache.reserve(i32_to_dev(n_new)).tolist() == books.reserve(n_new)
    check(cache, books, pool)
    parent = r.integers(0, seqs, seqs)
    cache.fork(i32_to_dev(parent))
    books.fork(parent)
    pool = cache.pool.view(torch.uint8).clone()
    check(cache, books, pool)
    assert cache.compact().tolist() == books.compact()
    check(cache, books, pool)


def test_all_forks_of_one_sequence_write(qb):
    """One last page held by every row: all but the last take copies, in order."""
    say("all forks write")
    cache = qb.PagedKvCache(3, 2, 40, page_len=64, max_seqs=20, max_pages=4)
    cache.reserve(i32_to_dev([100] + [0] * 19))
    cache.lengths[0] = 100
    cache.pool.view(torch.int16).random_(-9999, 9999)
    cache.fork(torch.zeros(20, dtype=torch.int32, device="cuda"))
    books = pg.Books(*books_of(cache), 64)
    pool = cache.pool.view(torch.uint8).clone()
    assert books.refs[:2] == [20, 20]
    assert cache.reserve(torch.ones(20, dtype=torch.int32, device="cuda")).tolist() == books.reserve([1] * 20) == [1] * 20
    assert len(books.copies) == 19 and books.refs[1] == 1 and books.table[19][1] == 1
    check(cache, books, pool)


# ------------------------------------------------------------------------------------- streams, graphs, the whole path

def test_a_step_replayed_as_a_graph(qb):
    """Room, append, both attentions, acceptance and cut in one graph: every replay equals the eager step."""
    say("graph")
    hq, hk, seqs = 4, 2, 3
    g = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    starts = i32_to_dev([0, 5, 7, 13])
    n_new, parent = i32_to_dev([5, 2, 6]), i32_to_dev([0, 1, 1])
    rows = bf16_to_dev(rnd_bits((13, 8 * D), 51))

    def step(c, out_q, out_a, out_b, ws):
        c.reserve(n_new)
        qb.paged_prepare(rows, hq, c, 0, starts, g, g, q_out=out_q)
        qb.paged_attention(out_q, hq, c, 0, starts, 6, workspace=ws, out=out_a)
        qb.prompt_attention(out_q, hq, c, 0, starts, out=out_b)
        c.lengths += n_new - 1
        c.fork(parent)

    def fresh():
        c = qb.PagedKvCache(1, hk, 60, page_len=32, max_seqs=seqs, max_pages=12)
        c.pool.zero_()
        return c, *(torch.empty((13, hq * D), dtype=torch.bfloat16, device="cuda") for _ in range(3)), \
            torch.empty(qb.lib().quasar_paged_attention_workspace_bytes(6, hq, hk), dtype=torch.uint8, device="cuda")

    eager, graph = fresh(), fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*graph)                                     # (allocations of the first call)
    torch.cuda.synchronize()
    graph[0].books[:60 + seqs].zero_()
    graph[0].table.fill_(-1)
    graph[0].pool.zero_()
    torch.cuda.synchronize()
    captured = torch.cuda.CUDAGraph()
    with torch.cuda.graph(captured):
        step(*graph)
    for i in range(6):
        captured.replay()
        step(*eager)
        torch.cuda.synchronize()
        assert torch.equal(graph[0].books, eager[0].books), i
        assert torch.equal(graph[0].pool.view(torch.int16), eager[0].pool.view(torch.int16)), i
        for a, b in zip(graph[1:4], eager[1:4]):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16)), i
    assert int(eager[0].lengths[0]) == 24


def test_calls_on_two_streams_at_once(qb):
    say("two streams")
    batches = [Batch(qb, "bf16", 64, 8, 2, [3000 + 50 * s, 17, 900], [4, 4, 4], seed=60 + s) for s in range(2)]
    want = [[qb.paged_attention(b.q(), 8, b.cache, 0, b.row_start, 4), qb.prompt_attention(b.q(), 8, b.cache, 0, b.row_start)] for b in batches]
    qs = [b.q() for b in batches]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in batches]
    got = [[], []]
    for _ in range(20):
        for i, b in enumerate(batches):
            with torch.cuda.stream(streams[i]):
                got[i].append([qb.paged_attention(qs[i], 8, b.cache, 0, b.row_start, 4), qb.prompt_attention(qs[i], 8, b.cache, 0, b.row_start)])
    torch.cuda.synchronize()
    for i in range(2):
        for pair in got[i]:
            for a, b in zip(pair, want[i]):
                assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    close(bf16_to_host(want[0][0]), batches[0])
    close(bf16_to_host(want[1][1]), batches[1])


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_prompts_forks_and_drafts_as_they_are_served(qb, kv):
    """Two prompts, forked, continued by drafts of which parts are accepted, compacted on the way: at every step both attentions equal the
    oracle over the history of each sequence."""
    say("served", kv)
    hq, hk, seqs, page = 6, 2, 5, 32
    r = np.random.Generator(np.random.Philox(71))
    scale = None if kv == "bf16" else torch.full((2, hk), 0.05, device="cuda")
    cache = qb.PagedKvCache(2, hk, 64, page_len=page, max_seqs=seqs, max_pages=10, dtype=torch.bfloat16 if kv == "bf16" else torch.float8_e4m3fn, k_scale=scale, v_scale=scale)
    cache.pool.view(torch.uint8).fill_(0xFF)
    gq, gk = rnd_bits((D,), 72, 0.1), rnd_bits((D,), 73, 0.1)
    gq, gk = (ref.f32_to_bf16_bits(1.0 + ref.bf16_bits_to_f64(x).astype(np.float32)) for x in (gq, gk))
    history = [(np.zeros((0, hk, D)), np.zeros((0, hk, D))) for _ in range(seqs)]
    plans = [([45, 0, 70, 0, 0], None), ([3, 3, 1, 8, 2], [0, 0, 2, 2, 2]), ([8, 1, 0, 4, 8], [0, 1, 2, 3, 4]), ([1, 1, 1, 1, 1], [4, 1, 2, 0, -1]), ([6, 6, 6, 6, 6], [0, 1, 2, 3, 4])]
    for step, (news, parent) in enumerate(plans):
        if parent is not None:
            cache.fork(i32_to_dev(parent))
            history = [history[p] if p >= 0 else (np.zeros((0, hk, D)), np.zeros((0, hk, D))) for p in parent]
        assert cache.reserve(i32_to_dev(news)).tolist() == [1] * seqs
        if step == 2:
            cache.compact()
        T = sum(news)
        starts = i32_to_dev(np.concatenate([[0], np.cumsum(news)]))
        qkv = rnd_bits((T, hq + 2 * hk, D), 80 + step)
        q = qb.paged_prepare(bf16_to_dev(qkv.reshape(T, -1)), hq, cache, 1, starts, bf16_to_dev(gq), bf16_to_dev(gk))
        outs = [qb.prompt_attention(q, hq, cache, 1, starts)]
        if max(news) <= 32:
            outs.append(qb.paged_attention(q, hq, cache, 1, starts, max(news)))
        outs = [ref.bf16_bits_to_f64(bf16_to_host(o)).reshape(T, hq, D) for o in outs]
        # what the pages hold of the new rows is read back (test_prepare holds it to the oracle)
        b = Batch.__new__(Batch)
        b.kv, b.page_len, b.hk, b.layer, b.cache = kv, page, hk, 1, cache
        b.scales = [None, None] if kv == "bf16" else [np.full((2, hk), 0.05, np.float32)] * 2
        q_host, at_ = ref.bf16_bits_to_f64(bf16_to_host(q)).reshape(T, hq, D), 0
        lengths = cache.lengths.tolist()
        for s, n in enumerate(news):
            k, v = (b.decoded(b.read(s, lengths[s] + n, half), half) for half in range(2))
            assert lengths[s] == len(history[s][0])
            assert np.array_equal(k[:lengths[s]], history[s][0]) and np.array_equal(v[:lengths[s]], history[s][1])
            if n:
                want, size = pg.attention(q_host[at_:at_ + n], k, v, lengths[s])
                most = np.linalg.norm(q_host[at_:at_ + n], axis=2).max() * np.linalg.norm(k, axis=2).max() / np.sqrt(D)
                tol = 1.01 * (2.0 ** -8 * np.abs(want) + (2.0 ** -7 + 4 * 132 * 2.0 ** -24 * most) * size)
                for o in outs:
                    assert (np.abs(o[at_:at_ + n] - want) <= tol).all()
            at_ += n
            kept = n if step == 0 else int(r.integers(0, n + 1))               # accepted
            history[s] = (k[:lengths[s] + kept], v[:lengths[s] + kept])
        cache.lengths.copy_(i32_to_dev([len(h[0]) for h in history]))
    cache.fork(i32_to_dev([-1] * seqs))
    assert int(cache.refs.abs().sum()) == 0 and int((cache.table != -1).sum()) == 0 and int(cache.lengths.sum()) == 0


def test_another_device_is_refused(qb, monkeypatch):
    """Launches go to the current device: tensors of another one are refused (here: another device is made current in name)."""
    say("other device")
    b = Batch(qb, "bf16", 32, 4, 2, [30], [2], seed=90)
    q, n, g, qkv = b.q(), i32_to_dev([1]), torch.ones(D, dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 8 * D), dtype=torch.bfloat16, device="cuda")
    addresses = qb._native_addresses(qb.lib())
    monkeypatch.setattr(qb, "_current_device", lambda: 1)
    qb._fast.bind(addresses, lambda: 1, qb._current_raw_stream)
    try:
        for call in (lambda: qb.paged_attention(q, 4, b.cache, 0, b.row_start, 2), lambda: qb.prompt_attention(q, 4, b.cache, 0, b.row_start),
                     lambda: qb.paged_prepare(qkv, 4, b.cache, 0, b.row_start, g, g), lambda: b.cache.reserve(n), lambda: b.cache.fork(n), lambda: b.cache.compact()):
            with pytest.raises(ValueError, match="current device"):
                call()
    finally:
        monkeypatch.undo()
        qb._fast.bind(addresses, qb._current_device, qb._current_raw_stream)


def test_native_and_python_marshalling_give_the_same(qb, monkeypatch):
    """Every call on a handle answers as the Python path does: same bits, same output tensors, the same errors of the library."""
    say("marshalling")
    b = Batch(qb, "e4m3", 32, 4, 2, [30, 3, 100], [2, 1, 2], seed=92, layers=2, layer=1)
    g = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    qkv = bf16_to_dev(rnd_bits((5, 8 * D), 93))
    out, ws = torch.empty((5, 4 * D), dtype=torch.bfloat16, device="cuda"), torch.empty(qb.lib().quasar_paged_attention_workspace_bytes(2, 4, 2), dtype=torch.uint8, device="cuda")
    n_new, parent, keep = i32_to_dev([2, 40, 0]), i32_to_dev([1, 1, -1]), i32_to_dev([2, 9, 9])
    saved, pool = b.cache.books.clone(), b.cache.pool.view(torch.uint8).clone()

    def calls():
        b.cache.books.copy_(saved)
        b.cache.pool.view(torch.uint8).copy_(pool)
        q = qb.paged_prepare(qkv, 4, b.cache, 1, b.row_start, g, g, eps=1e-5, rope_theta=1e4)
        assert qb.paged_prepare(qkv, 4, b.cache, 1, b.row_start, g, g, q_out=out) is out
        got = [q, out.clone(), qb.paged_attention(q, 4, b.cache, 1, b.row_start, 2), qb.prompt_attention(q, 4, b.cache, 1, b.row_start)]
        assert qb.paged_attention(q, 4, b.cache, 1, b.row_start, 2, workspace=ws, out=out) is out
        got.append(out.clone())
        assert qb.prompt_attention(q[:1], 4, b.cache, 0, i32_to_dev([0, 1]), out=out[:1]).shape == (1, 4 * D)
        got += [out.clone(), b.cache.reserve(n_new), b.cache.books.clone()]
        assert b.cache.fork(parent, keep) is None
        got += [b.cache.books.clone(), b.cache.compact(), b.cache.books.clone(), b.cache.pool.view(torch.uint8).clone()]
        for bad in (lambda: qb.paged_attention(q, 4, b.cache, 1, b.row_start, 33), lambda: qb.paged_prepare(qkv, 4, b.cache, 1, b.row_start, g, g, eps=2.0),
                    lambda: qb.paged_attention(q, 4, b.cache, 1, b.row_start, 2, workspace=ws[:64])):
            with pytest.raises(qb.QuasarError):
                bad()
        return [t.view(torch.int16) if t.dtype == torch.bfloat16 else t for t in got]

    native = calls()
    for name in ("paged_prepare", "paged_attention", "prompt_attention", "pages_reserve", "pages_fork", "pages_compact"):
        monkeypatch.setattr(qb._fast, name, lambda *a: -1)
    for x, y in zip(native, calls()):
        assert torch.equal(x, y)


def test_refusals_of_the_binding(qb):
    say("refusals")
    b = Batch(qb, "bf16", 32, 4, 2, [30, 3], [2, 2], seed=91)
    q = b.q()
    for bad in (lambda: qb.paged_attention(q, 8, b.cache, 0, b.row_start, 2), lambda: qb.paged_attention(q, 4, b.cache, 1, b.row_start, 2),
                lambda: qb.prompt_attention(q, 4, b.cache, -1, b.row_start), lambda: qb.prompt_attention(q, 4, b.cache, 0, b.row_start[::2]),
                lambda: qb.prompt_attention(q, 4, b.cache, 0, i32_to_dev([0, 1, 2, 3])), lambda: qb.prompt_attention(q.t(), 4, b.cache, 0, b.row_start),
                lambda: qb.paged_attention(q, 4, b.cache, 0, b.row_start, 2, out=torch.empty((3, 512), dtype=torch.bfloat16, device="cuda")),
                lambda: b.cache.reserve(i32_to_dev([1, 1, 1])), lambda: b.cache.fork(i32_to_dev([[0, 1]]))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: qb.prompt_attention(q.float(), 4, b.cache, 0, b.row_start), lambda: qb.prompt_attention(q, 4, b.cache, 0, b.row_start.long()),
                lambda: qb.prompt_attention(q.cpu(), 4, b.cache, 0, b.row_start), lambda: b.cache.reserve(torch.ones(2, device="cuda"))):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: qb.paged_attention(q, 4, b.cache, 0, b.row_start, 0), lambda: qb.paged_attention(q, 4, b.cache, 0, b.row_start, 33),
                lambda: qb.paged_attention(q, 4, b.cache, 0, b.row_start, 2, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(qb.QuasarError):
            bad()
    empty = qb.prompt_attention(q[:0], 4, b.cache, 0, i32_to_dev([0, 0, 0]))
    assert empty.shape == (0, 512)


def test_an_expanded_workspace_is_refused(qb):
    """Its nbytes count elements that share memory."""
    say("expanded workspace")
    b = Batch(qb, "bf16", 32, 4, 2, [30, 3], [2, 2], seed=92)
    need = qb._lib.quasar_paged_attention_workspace_bytes(2, 4, 2)
    with pytest.raises(ValueError):
        qb.paged_attention(b.q(), 4, b.cache, 0, b.row_start, 2, workspace=torch.empty(1, dtype=torch.uint8, device="cuda").expand(need))
    close(bf16_to_host(qb.paged_attention(b.q(), 4, b.cache, 0, b.row_start, 2, workspace=torch.empty(need, dtype=torch.uint8, device="cuda"))), b)


def test_a_cache_keeps_its_buffers(qb):
    """Calls go to the buffers that the cache was made with: another tensor in their place is refused, writing into them is not."""
    say("buffers")
    b = Batch(qb, "e4m3", 32, 4, 2, [30, 3], [2, 2], seed=93)
    c = b.cache
    for name in ("pool", "books", "refs", "lengths", "table", "k_scale", "v_scale"):
        with pytest.raises(AttributeError):
            setattr(c, name, getattr(c, name).clone())
    for name in ("n_pages", "page_len", "max_pages"):
        with pytest.raises(AttributeError):
            setattr(c, name, getattr(c, name) + 32)
    c.lengths += 1
    c.lengths -= 1
    c.table[0, 0] = c.table[0, 0]
    c.note = "the caller's own"
    close(bf16_to_host(qb.paged_attention(b.q(), 4, c, 0, b.row_start, 2)), b)


def test_offsets_beyond_32_bits(qb):
    """The pages of a small pool's layer in the second layer of one of 10 GB, counted from its end: the same bits, page for page."""
    say("large pool")
    hq, hk, page, n_big = 16, 8, 256, 5000
    b = Batch(qb, "bf16", page, hq, hk, [700, 255, 0], [8, 3, 0], seed=94)
    small = b.cache
    big = qb.PagedKvCache(2, hk, n_big, page_len=page, max_seqs=small.max_seqs, max_pages=small.max_pages)
    assert big.pool[1].nbytes > 1 << 32
    away = lambda ids: torch.where(ids >= 0, n_big - 1 - ids, ids)
    at = torch.arange(n_big - 1, n_big - 1 - small.n_pages, -1, device="cuda")
    big.pool[1, at] = small.pool[0]
    big.table.copy_(away(small.table)); big.lengths.copy_(small.lengths)
    big.refs.fill_(1)                                    # (room at the end alone)
    big.refs[at] = small.refs
    calls = (lambda c, l: qb.paged_attention(b.q(), hq, c, l, b.row_start, 8), lambda c, l: qb.prompt_attention(b.q(), hq, c, l, b.row_start))
    for call in calls:
        got = bf16_to_host(call(big, 1))
        assert np.array_equal(got, bf16_to_host(call(small, 0)))
        close(got, b)
    qkv = bf16_to_dev(rnd_bits((b.rows, (hq + 2 * hk) * D), 95))
    g = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    assert torch.equal(qb.paged_prepare(qkv, hq, big, 1, b.row_start, g, g), qb.paged_prepare(qkv, hq, small, 0, b.row_start, g, g))
    same = lambda: torch.equal(big.pool[1, at].view(torch.int16), small.pool[0].view(torch.int16))
    assert same()
    # a fork that writes: its copy goes to the one page that is free, which lies at the end too
    parent, news = i32_to_dev([0, 1, 0]), i32_to_dev([0, 0, 1])
    free = int(torch.nonzero(small.refs == 0)[0])
    for c, end in ((small, False), (big, True)):
        c.fork(parent)                                   # (which frees the second sequence's page without positions, too)
        c.refs[c.refs == 0] = 1
        c.refs[n_big - 1 - free if end else free] = 0
        assert c.reserve(news).tolist() == [1, 1, 1]
    assert torch.equal(away(small.table), big.table) and int(small.table[2, 2]) == free
    assert same()
    # and back to the beginning: with nothing else in use every page moves, as it is
    for c in (small, big):
        c.refs.zero_()
        c.refs[c.table[c.table >= 0].long()] = 1
    was = big.pool[1, big.table[0, :3].long()].clone()
    to = big.compact()
    live = int((big.refs > 0).sum())
    assert int(big.table.max()) == live - 1 and (to[at[small.refs > 0]] < live).all()
    assert torch.equal(big.pool[1, big.table[0, :3].long()].view(torch.int16), was.view(torch.int16))


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("group", [1, 8, 16])
def test_rows_beyond_max_new_are_left_as_they_were(qb, kv, group):
    say("max_new", kv, group)
    hq, lengths, news, most = 2 * group, [70, 5, 300], [8, 2, 5], 3
    b = Batch(qb, kv, 32, hq, 2, lengths, news, seed=300 + group, scaled=False)
    out = torch.full((b.rows, hq * D), 5.0, dtype=torch.bfloat16, device="cuda")
    qb.paged_attention(b.q(), hq, b.cache, 0, b.row_start, most, out=out)
    want, tol = b.expected()
    got = ref.bf16_bits_to_f64(bf16_to_host(out)).reshape(b.rows, hq, D)
    row = 0
    for n in news:
        kept = min(n, most)
        assert (np.abs(got - want)[row:row + kept] <= tol[row:row + kept]).all() and (got[row + kept:row + n] == 5.0).all()
        row += n


# kv, Hq, sequences, tokens of one at most, max_new
MANY = [("bf16", 2, 1024, 1, 1), ("e4m3", 3, 1024, 3, 3), ("bf16", 12, 1000, 2, 2), ("bf16", 24, 1024, 2, 2), ("e4m3", 40, 1024, 1, 2), ("bf16", 32, 700, 1, 9),
        ("bf16", 4, 1024, 0, 1), ("e4m3", 16, 257, 4, 4)]


@pytest.mark.parametrize("kv,hq,seqs,new,most", MANY)
def test_as_many_sequences_as_there_may_be(qb, kv, hq, seqs, new, most):
    """Every form over a thousand sequences, many of them empty, one of them long."""
    say("many sequences", kv, hq, seqs, new, most)
    r = np.random.Generator(np.random.Philox(400 + hq))
    lengths, news = r.integers(0, 90, seqs), r.integers(0, new + 1, seqs)
    lengths[seqs // 3], news[seqs // 3], news[-1] = 2500, max(new, 1), 1
    lengths[::5] = 0
    b = Batch(qb, kv, 64, hq, 1, lengths.tolist(), news.tolist(), seed=401 + hq)
    close(bf16_to_host(qb.paged_attention(b.q(), hq, b.cache, 0, b.row_start, most)), b)
    close(bf16_to_host(qb.prompt_attention(b.q(), hq, b.cache, 0, b.row_start)), b)


@pytest.mark.parametrize("group", [1, 5, 8])
def test_the_last_positions_there_may_be(qb, group):
    """A sequence that ends at position 2^24 - 1, of which only the last page exists: append, and both attentions over what exists."""
    say("last positions", group)
    hq, page, n, total = group, 1024, 8, 1 << 24
    cache = qb.PagedKvCache(1, 1, 2, page_len=page, max_seqs=1, max_pages=total // page)
    cache.pool.view(torch.uint8).fill_(0xFF)
    cache.table[0, -1] = 1
    cache.lengths[0] = total - page
    g = rnd_bits((D,), 501, 0.1)
    g = ref.f32_to_bf16_bits(1.0 + ref.bf16_bits_to_f64(g).astype(np.float32))
    chunks, pos = [page - n, n], total - page
    for i, rows in enumerate(chunks):
        qkv = rnd_bits((rows, hq + 2, D), 502 + i)
        starts = i32_to_dev([0, rows])
        q = qb.paged_prepare(bf16_to_dev(qkv.reshape(rows, -1)), hq, cache, 0, starts, bf16_to_dev(g), bf16_to_dev(g))
        want = at.head_norm_rope(qkv[:, :hq], g, 1e-6, np.arange(pos, pos + rows), 1e6)
        got = bf16_to_host(q).reshape(rows, hq, D)
        f64 = ref.bf16_bits_to_f64
        size = np.abs(f64(at.head_norm_rope(qkv[:, :hq], g, 1e-6, np.zeros(rows), 1e6)))
        # (as in test_prepare)
        assert (np.abs(f64(got) - f64(want)) <= 2.0 ** -6 * (size + np.roll(size, D // 2, axis=2)) + 2.0 ** -7 * np.abs(f64(want))).all()
        assert np.mean(got != want) < 0.02
        pos += rows
        if i == 0:
            cache.lengths += rows
    b = Batch.__new__(Batch)
    b.kv, b.page_len, b.hk, b.hq, b.layer, b.cache, b.scales, b.rows, b.news, b.lengths = "bf16", page, 1, hq, 0, cache, [None, None], n, [n], [page - n]
    raw = cache.pool[0, 1, 0].view(torch.int16).cpu().numpy().view(np.uint16)              # [block][half][4096]
    j = np.arange(page)
    b.keys, b.values = ([ref.bf16_bits_to_f64(raw[(j // 32)[:, None], half, pg.block_places("bf16")[half][j % 32]])[:, None]] for half in range(2))
    b.q_bits = bf16_to_host(q).reshape(n, hq, D)
    close(bf16_to_host(qb.paged_attention(q, hq, cache, 0, starts, n)), b)
    close(bf16_to_host(qb.prompt_attention(q, hq, cache, 0, starts)), b)
    assert int(cache.lengths[0]) == total - n


@pytest.mark.parametrize("rows", [512, 16])
def test_every_value_over_many_scales(qb, rows):
    """All bf16 values but NaN, over scales of every kind: the codes of the fp32 quotient.  512 rows go block by block, 16 row by row."""
    say("every value", rows)
    r = np.random.Generator(np.random.Philox(601))
    near = lambda x, steps: (np.float32(x).view(np.int32) + np.asarray(steps, np.int32)).view(np.float32)
    scales = np.concatenate([near(1.0, [0, 1, -1, 2, -2, 1 << 22]), near(2.0 ** -60, [-1, 0, 1]), near(2.0 ** 60, [-1, 0, 1]), np.float32([1e-44, 1e-38, 3e38, 1 / 448, 448, 1 / 3, 0.05]),
                             (2.0 ** r.uniform(-59, 59, 18)).astype(np.float32), (2.0 ** r.uniform(-9, 3, 27)).astype(np.float32)])
    hk, hq = len(scales), len(scales)
    cache = qb.PagedKvCache(1, hk, 16, page_len=32, max_seqs=1, max_pages=16, dtype=torch.float8_e4m3fn, k_scale=torch.from_numpy(scales)[None].cuda(),
                            v_scale=torch.from_numpy(scales)[None].cuda())
    cache.table[0] = torch.arange(16, device="cuda")
    g = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    values = np.arange(1 << 16, dtype=np.uint32).astype(np.uint16).reshape(512, D)
    b = Batch.__new__(Batch)
    b.kv, b.page_len, b.hk, b.layer, b.cache = "e4m3", 32, hk, 0, cache
    for at_ in range(0, 512, rows):
        qkv = np.zeros((rows, hq + 2 * hk, D), np.uint16)
        qkv[:, hq + hk:] = values[at_:at_ + rows, None]
        qb.paged_prepare(bf16_to_dev(qkv.reshape(rows, -1)), hq, cache, 0, i32_to_dev([0, rows]), g, g)
        cache.lengths += rows
    got = b.read(0, 512, 1)
    bits = (values.astype(np.uint32) << 16).view(np.float32)
    with np.errstate(all="ignore"):
        want = np.stack([pg.f64_to_e4m3(np.nan_to_num((bits / s).astype(np.float32), nan=0.0, posinf=np.inf, neginf=-np.inf)) for s in scales], 1)
    number = ~np.isnan(bits)
    assert scales.min() > 0 and number.sum() > 65000
    wrong = (got != want) & number[:, None]
    assert not wrong.any(), (scales[np.nonzero(wrong)[1][:5]], bits[np.nonzero(wrong)[0][:5], np.nonzero(wrong)[2][:5]])
    assert ((got[~number[:, None].repeat(hk, 1)] & 0x7F) == 0x7F).all()


# kv, Hq, Hkv, cached, new: tiles that stay whole and tiles that are shared, on both sides of the rule
WIDE = [("bf16", 32, 8, [0], [61]), ("bf16", 32, 8, [0], [512]), ("e4m3", 32, 8, [0], [512]), ("bf16", 32, 8, [300], [512]), ("bf16", 32, 8, [900], [61]),
        ("e4m3", 32, 8, [400, 0, 77, 0], [61, 0, 130, 5]), ("bf16", 8, 1, [0], [700]), ("bf16", 8, 2, [0, 30], [1100, 65]), ("e4m3", 5, 1, [2000], [40])]


@pytest.mark.parametrize("kv,hq,hk,lengths,news", WIDE)
def test_prompts_do_not_depend_on_the_width_of_the_table(qb, kv, hq, hk, lengths, news):
    """A table of 32768 positions, as a cache with room to grow has, gives the bits of one that just holds the sequences."""
    say("wide table", kv, hq, hk, lengths, news)
    a, b = (Batch(qb, kv, 64, hq, hk, lengths, news, seed=700 + hq, more_columns=0), Batch(qb, kv, 64, hq, hk, lengths, news, seed=700 + hq, more_columns=512))
    assert np.array_equal(a.q_bits, b.q_bits) and b.cache.max_pages >= 512
    got = [bf16_to_host(qb.prompt_attention(x.q(), hq, x.cache, 0, x.row_start)) for x in (a, b)]
    assert np.array_equal(*got)
    close(got[1], b)


def test_other_memory_in_a_buffer_is_refused(qb):
    """A cache's tensor that is given other memory (by `.data`, a resize) is refused by every call before anything is launched."""
    say("other memory")
    b = Batch(qb, "e4m3", 32, 4, 2, [30, 3], [2, 2], seed=96, layers=2)
    c, q, n = b.cache, b.q(), i32_to_dev([1, 1])
    g, qkv = torch.ones(D, dtype=torch.bfloat16, device="cuda"), torch.zeros((4, 8 * D), dtype=torch.bfloat16, device="cuda")
    calls = (lambda: qb.paged_attention(q, 4, c, 0, b.row_start, 2), lambda: qb.prompt_attention(q, 4, c, 0, b.row_start),
             lambda: qb.paged_prepare(qkv, 4, c, 0, b.row_start, g, g), lambda: c.reserve(n), lambda: c.fork(n), lambda: c.compact())
    for name in ("pool", "books", "refs", "lengths", "table", "k_scale", "v_scale"):
        t = getattr(c, name)
        was = t.data
        for other in (was.clone(), was[:1].clone(), was[:1]):
            t.data = other
            for call in calls:
                with pytest.raises(ValueError, match="other memory"):
                    call()
        t.data = was
        with pytest.raises(AttributeError):
            delattr(c, name)
    close(bf16_to_host(qb.paged_attention(q, 4, c, 0, b.row_start, 2)), b)


@pytest.mark.parametrize("page", [32, 1024])
def test_a_pool_larger_than_a_sequence_may_be(qb, page):
    """Without max_pages a row of the table holds what a sequence may have, 2^24 positions, also where the pool holds more."""
    say("large pool by default", page)
    c = qb.PagedKvCache(1, 1, (1 << 24) // page + 3, page_len=page, max_seqs=2, dtype=torch.float8_e4m3fn)
    assert c.max_pages * page == 1 << 24 and tuple(c.table.shape) == (2, c.max_pages)
    assert c.reserve(i32_to_dev([1 << 24, 3 * page])).tolist() == [1, 1]
    assert int(c.table[0, -1]) == c.max_pages - 1 and c.table[1, :4].tolist() == [c.max_pages, c.max_pages + 1, c.max_pages + 2, -1]
    assert c.reserve(i32_to_dev([0, 3 * page + 1])).tolist() == [1, 0]
    assert qb.PagedKvCache(1, 1, 5, page_len=page).max_pages == 5
    for bad in (0, (1 << 24) // page + 1):
        with pytest.raises(ValueError):
            qb.PagedKvCache(1, 1, 5, page_len=page, max_pages=bad)


def near(got_bits, b, kv):
    """Every row of every sequence within attention_and_bound."""
    got, q, at_ = ref.bf16_bits_to_f64(got_bits).reshape(b.rows, b.hq, D), ref.bf16_bits_to_f64(b.q_bits), 0
    worst = 0.0
    for s, n in enumerate(b.news):
        if n:
            want, tol = attention_and_bound(q[at_:at_ + n], b.keys[s], b.values[s], b.lengths[s], kv)
            worst = max(worst, float((np.abs(got[at_:at_ + n] - want) / tol).max()))
            at_ += n
    say("   worst of tolerance", worst)
    assert np.isfinite(got).all() and worst <= 1.0


def mark_blocks(b):
    """The batch with block_values in its pages (times the head's scale, in 8-bit pages), and smaller queries: no position outweighs the others."""
    places, c = pg.block_places(b.kv)[1], b.cache
    raw = c.pool[b.layer].view(torch.int16 if b.kv == "bf16" else torch.uint8).cpu().numpy()
    for s, (length, n) in enumerate(zip(b.lengths, b.news)):
        v = block_values(length + n)
        bits = ref.f32_to_bf16_bits(v.astype(np.float32)).view(np.int16) if b.kv == "bf16" else pg.f64_to_e4m3(v)
        j = np.arange(length + n)
        for h in range(b.hk):
            raw[b.table[s, j // b.page_len][:, None], h, (j % b.page_len // 32)[:, None], 1, places[j % 32]] = bits
        b.values[s] = b.decoded(np.repeat((bits.view(np.uint16) if b.kv == "bf16" else bits)[:, None], b.hk, 1), 1)
    c.pool[b.layer].view(torch.int16 if b.kv == "bf16" else torch.uint8).copy_(torch.from_numpy(raw))
    b.q_bits = rnd_bits((b.rows, b.hq, D), 778, 0.4)


# call, page, Hq, Hkv, cached, new: every form, over contexts that many workers share
BLOCKS = [("paged", 64, 8, 1, [30000, 5, 12000], [1, 1, 1]), ("paged", 32, 4, 2, [20000, 12000], [8, 3]), ("paged", 128, 8, 1, [30000, 7000], [4, 4]),
          ("paged", 64, 8, 1, [33000, 100, 9000], [8, 8, 5]), ("paged", 1024, 16, 1, [20000, 3000], [16, 9]), ("paged", 64, 1, 1, [100003], [1]),
          ("paged", 64, 2, 2, [2500] * 30, [1] * 30), ("prompt", 64, 8, 1, [0], [4000]), ("prompt", 64, 8, 1, [20000, 0], [300, 500]), ("prompt", 128, 4, 2, [16000], [512]),
          ("prompt", 32, 8, 1, [50000], [20]), ("prompt", 64, 16, 8, [0, 3000, 64], [2100, 900, 700]), ("prompt", 64, 32, 8, [0], [512])]


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("call,page,hq,hk,lengths,news", BLOCKS)
def test_every_block_of_a_long_context_counts(qb, kv, call, page, hq, hk, lengths, news):
    say("blocks", kv, call, page, hq, hk, lengths[:5], news[:5])
    b = Batch(qb, kv, page, hq, hk, lengths, news, seed=800 + hq)
    mark_blocks(b)
    got = qb.paged_attention(b.q(), hq, b.cache, 0, b.row_start, max(news)) if call == "paged" else qb.prompt_attention(b.q(), hq, b.cache, 0, b.row_start)
    near(bf16_to_host(got), b, kv)


@pytest.mark.parametrize("page,hq,hk,lengths,news", [s[1:] for s in STEP if s[0] == "e4m3"] + [(64, 8, 2, [0, 100], [129, 311]), (32, 3, 1, [37], [500]), (64, 16, 1, [1500, 30], [32, 7])])
def test_weights_over_8_bit_pages_have_11_bits(qb, page, hq, hk, lengths, news):
    say("fp16 weights", page, hq, hk, lengths[:5], news[:5])
    b = Batch(qb, "e4m3", page, hq, hk, lengths, news, seed=850 + hq)
    if max(news) <= 32:
        near(bf16_to_host(qb.paged_attention(b.q(), hq, b.cache, 0, b.row_start, max(news))), b, "e4m3")
    near(bf16_to_host(qb.prompt_attention(b.q(), hq, b.cache, 0, b.row_start)), b, "e4m3")


# kv, page, Hq, Hkv, cached, new, heads that a workgroup of the block form takes on 256 compute units
HEADS = [("bf16", 64, 32, 8, [0, 100], [1400, 133], 2), ("e4m3", 128, 32, 8, [31], [1520], 2), ("bf16", 32, 32, 8, [0, 7, 0], [2000, 0, 1500], 5), ("e4m3", 64, 32, 8, [5], [3500], 5),
         ("bf16", 64, 32, 8, [40, 0], [2400, 2400], 7), ("e4m3", 64, 32, 8, [0, 1000], [4000, 810], 7), ("bf16", 64, 40, 8, [3], [5000], 8), ("e4m3", 32, 40, 8, [0, 64], [5000, 999], 8),
         ("e4m3", 64, 6, 3, [0, 1], [9000, 9500], 6)]


@pytest.mark.parametrize("kv,page,hq,hk,lengths,news,parts", HEADS)
def test_prepare_with_several_heads_a_workgroup(qb, kv, page, hq, hk, lengths, news, parts):
    """Heads one after another in a workgroup, from queries to keys and from keys to values, groups that the heads do not fill among them."""
    heads = hq + 2 * hk
    units = torch.cuda.get_device_properties(0).multi_processor_count
    assert sum(news) >= 64 * len(news) and (units != 256 or min(8, sum(news) // 32 * heads // 1024) == parts)
    test_prepare(qb, kv, page, hq, hk, lengths, news)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("rows", [80, 700])
def test_prepare_by_blocks_writes_nothing_without_a_page(qb, kv, rows):
    """As test_prepare_writes_nothing_without_a_page, block by block: no id, an id beyond the pool, a length beyond the table, a length that is none.
    Queries are written where there is a position, and nothing of a sequence whose length is none."""
    say("prepare by blocks without pages", kv, rows)
    b = Batch(qb, kv, 32, 8, 4, [30, 10, 5, 40], [rows] * 4, seed=97, scaled=False)
    b.cache.table[0, 1] = -1
    b.cache.table[1, 0] = b.cache.n_pages
    b.cache.table[1, 2] = 2 ** 31 - 1
    b.cache.lengths[2] = 2 ** 24                         # beyond the table
    b.cache.lengths[3] = -1
    raw = b.cache.pool.view(torch.uint8)
    before = raw.clone()
    qkv = bf16_to_dev(rnd_bits((b.rows, 16 * D), 98))
    g = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    q = torch.full((b.rows, 8 * D), 9.0, dtype=torch.bfloat16, device="cuda")
    qb.paged_prepare(qkv, 8, b.cache, 0, b.row_start, g, g, q_out=q)
    torch.cuda.synchronize()
    assert torch.isfinite(q).all() and (q[3 * rows:] == 9).all() and (q[:3 * rows] != 9).any(dim=1).all()
    changed = sorted((before != raw).flatten(2).any(2)[0].nonzero().flatten().tolist())
    last = lambda s: -(-(b.lengths[s] + rows) // 32)
    assert changed == sorted([int(b.table[0, c]) for c in range(last(0)) if c != 1] + [int(b.table[1, c]) for c in range(last(1)) if c not in (0, 2)])
    # what is written is what a cache with all of its pages gets
    whole = Batch(qb, kv, 32, 8, 4, [30, 10, 5, 40], [rows] * 4, seed=97, scaled=False)
    q2 = qb.paged_prepare(qkv, 8, whole.cache, 0, whole.row_start, g, g)
    assert torch.equal(q2[:2 * rows], q[:2 * rows]) and torch.equal(whole.cache.pool.view(torch.uint8)[0, changed], raw[0, changed])


# call, Hq, Hkv, cached, new: the forms of both attentions, and of the append
IN_PLACE = [("paged", 8, 2, [3000, 0, 77], [1, 1, 1]), ("paged", 8, 2, [3000, 20], [8, 5]), ("paged", 16, 2, [3000, 20, 9000], [8, 5, 8]), ("paged", 16, 1, [2000, 20], [32, 7]),
            ("prompt", 8, 2, [0, 30], [61, 200]), ("prompt", 8, 2, [4000], [100]), ("prompt", 32, 8, [0, 64], [2100, 77])]


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("call,hq,hk,lengths,news", IN_PLACE)
def test_queries_and_outputs_in_place(qb, kv, call, hq, hk, lengths, news):
    """The queries' part of the projection, rotated and then replaced by the attention's output where it lies, gives what tensors of their own give."""
    say("in place", kv, call, hq, hk, lengths, news)
    b = Batch(qb, kv, 64, hq, hk, lengths, news, seed=860 + hq)
    g = bf16_to_dev(ref.f32_to_bf16_bits((1.0 + 0.2 * np.random.Generator(np.random.Philox(7)).standard_normal(D)).astype(np.float32)))
    qkv = bf16_to_dev(rnd_bits((b.rows, (hq + 2 * hk) * D), 861))
    attend = lambda q, out: (qb.paged_attention(q, hq, b.cache, 0, b.row_start, max(news), out=out) if call == "paged" else qb.prompt_attention(q, hq, b.cache, 0, b.row_start, out=out))
    q = qb.paged_prepare(qkv, hq, b.cache, 0, b.row_start, g, g)
    pool = b.cache.pool.view(torch.uint8).clone()
    want = attend(q, None)
    rest, part = qkv[:, hq * D:].clone(), qkv[:, :hq * D]
    qb.paged_prepare(qkv, hq, b.cache, 0, b.row_start, g, g, q_out=part)
    assert torch.equal(part, q) and torch.equal(b.cache.pool.view(torch.uint8), pool)
    attend(part, part)
    assert torch.equal(part, want) and torch.equal(qkv[:, hq * D:], rest)
