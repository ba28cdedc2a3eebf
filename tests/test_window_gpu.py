"""GPU parity of windows over a paged cache - attention of a step and of prompts, trim - through the binding against the CPU oracle.  Attention is
held element by element to the tolerance of the full one (paged_util.Batch.expected: its count of roundings has no length in it); pages that no
position lies in hold NaN patterns."""
import numpy as np
import pytest
import torch

from oracle import quasar_paged_ref as pg
from oracle import quasar_ref as ref
from oracle import quasar_window_ref as win
from paged_util import Batch
from gpu_util import bf16_to_host, i32_to_dev

pytestmark = pytest.mark.gpu
D = 128
CALLS = ["paged", "prompt"]


@pytest.fixture(scope="module")
def qb():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2603_01399_amd import binding
    return binding


def say(*a):
    print(*a, flush=True)


def attend(qb, call, b, window, sinks, q=None, starts=None, layer=0, out=None):
    q, starts = b.q() if q is None else q, b.row_start if starts is None else starts
    if call == "paged":
        return qb.paged_attention(q, b.hq, b.cache, layer, starts, max(b.news), out=out, window=window, sinks=sinks)
    return qb.prompt_attention(q, b.hq, b.cache, layer, starts, out=out, window=window, sinks=sinks)


def expected(b, window, sinks):
    """As Batch.expected, of what the rows see."""
    out, tol = [], []
    q, at = ref.bf16_bits_to_f64(b.q_bits), 0
    for s, n in enumerate(b.news):
        rows = q[at:at + n]
        at += n
        if n:
            o, size = win.attention(rows, b.keys[s], b.values[s], b.lengths[s], window, sinks)
            most = np.linalg.norm(rows, axis=2).max() * np.linalg.norm(b.keys[s], axis=2).max() / np.sqrt(D)
            out.append(o)
            tol.append(1.01 * (2.0 ** -8 * np.abs(o) + (2.0 ** -7 + 4 * 132 * 2.0 ** -24 * most) * size) + 1e-30)
    return np.concatenate(out), np.concatenate(tol)


def close(got_bits, b, window, sinks):
    got = ref.bf16_bits_to_f64(got_bits).reshape(b.rows, b.hq, D)
    want, tol = expected(b, window, sinks)
    over = np.abs(got - want) / tol
    say("   worst of tolerance", float(over.max()))
    assert np.isfinite(got).all() and (over <= 1.0).all()


# kv, page, Hq, Hkv, cached, new, window, sinks
SHAPES = [("bf16", 64, 8, 2, [0], [1], 1, 0), ("bf16", 32, 4, 4, [31], [1], 1, 1), ("bf16", 32, 4, 1, [100], [1], 32, 0), ("bf16", 64, 32, 8, [1000, 0, 77, 4095], [1, 1, 1, 1], 100, 4),
          ("bf16", 64, 32, 8, [63, 64, 65], [8, 8, 8], 33, 1), ("bf16", 128, 40, 8, [500, 3], [3, 7], 64, 65), ("bf16", 64, 8, 1, [100, 5000, 20], [5, 0, 2], 1000, 0),
          ("bf16", 1024, 8, 8, [2000, 10], [2, 1], 5, 700), ("bf16", 64, 16, 2, [700], [32], 16, 3), ("bf16", 32, 64, 8, [90, 1], [16, 13], 7, 2),
          ("e4m3", 64, 8, 2, [300], [1], 31, 33), ("e4m3", 32, 32, 8, [1000, 0, 77, 4095], [1, 1, 1, 1], 500, 4), ("e4m3", 128, 64, 8, [9000, 130], [8, 8], 2000, 0),
          ("e4m3", 64, 16, 2, [700, 64], [32, 1], 129, 128), ("e4m3", 256, 5, 1, [3000], [10], 3001, 4), ("bf16", 64, 4, 2, [200] * 70, [1] * 70, 40, 4),
          ("e4m3", 32, 4, 2, list(range(0, 280, 7)), [1, 2, 0, 3] * 10, 50, 10), ("bf16", 64, 2, 1, [30000, 5, 12000], [4, 4, 4], 9000, 64), ("bf16", 32, 24, 1, [33], [32], 8, 0),
          ("bf16", 64, 16, 1, [300, 40], [32, 32], 50, 4), ("e4m3", 64, 64, 8, [2000], [16], 1 << 30, 0), ("bf16", 64, 8, 2, [2000], [2], 1, 1 << 40)]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("kv,page,hq,hk,lengths,news,window,sinks", SHAPES)
def test_windows(qb, call, kv, page, hq, hk, lengths, news, window, sinks):
    say("window", call, kv, page, hq, hk, lengths[:4], news[:4], window, sinks)
    b = Batch(qb, kv, page, hq, hk, lengths, news, seed=len(lengths) + hq + window % 97)
    close(bf16_to_host(attend(qb, call, b, window, sinks)), b, window, sinks)


PROMPTS = [("bf16", 64, 4, 1, [0], [64], 20, 0), ("bf16", 64, 8, 2, [0], [400], 64, 4), ("bf16", 32, 8, 2, [0, 0, 0], [130, 0, 257], 31, 0), ("bf16", 64, 5, 1, [0, 40], [300, 77], 100, 70),
           ("bf16", 128, 2, 2, [1000, 0], [200, 700], 128, 0), ("e4m3", 64, 8, 2, [0, 100], [129, 311], 65, 64), ("e4m3", 32, 3, 1, [37], [500], 200, 1),
           ("bf16", 64, 8, 1, [0], [1100], 513, 0), ("e4m3", 1024, 8, 4, [1500], [40], 700, 300), ("bf16", 64, 8, 2, [0], [700], 1, 0), ("e4m3", 64, 8, 2, [0, 50], [300, 200], 1, 2),
           ("bf16", 64, 16, 2, [3000, 0], [500, 90], 1024, 4), ("bf16", 64, 1, 1, [20], [600], 300, 0), ("e4m3", 64, 32, 1, [600], [50], 77, 9)]


@pytest.mark.parametrize("kv,page,hq,hk,lengths,news,window,sinks", PROMPTS)
def test_windows_of_prompts(qb, kv, page, hq, hk, lengths, news, window, sinks):
    say("windows of prompts", kv, page, hq, hk, lengths, news, window, sinks)
    b = Batch(qb, kv, page, hq, hk, lengths, news, seed=hq + window)
    close(bf16_to_host(attend(qb, "prompt", b, window, sinks)), b, window, sinks)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("group,new", [(1, 1), (1, 17), (3, 5), (3, 11), (5, 7), (8, 8), (8, 9), (2, 32), (16, 32)])
def test_windows_of_any_number_of_rows(qb, kv, group, new):
    say("rows", kv, group, new)
    b = Batch(qb, kv, 64, 2 * group, 2, [1500, 31, 4, 0, 700], [new, 1, max(new - 1, 0), new, 0], seed=200 + group + new)
    close(bf16_to_host(attend(qb, "paged", b, 90, 5)), b, 90, 5)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("group,new", [(1, 1), (4, 4), (4, 7), (8, 8), (16, 8)])
def test_windows_that_workers_share(qb, kv, group, new):
    """Windows so long beside the number of sequences that several workers have parts of one, with pieces that end anywhere."""
    say("shared", kv, group, new)
    b = Batch(qb, kv, 64, 2 * group, 2, [3000, 31, 1400, 0, 5000], [new, 1, max(new - 1, 0), new, new], seed=300 + group + new)
    for window, sinks in ((1300, 40), (2500, 0)):
        close(bf16_to_host(attend(qb, "paged", b, window, sinks)), b, window, sinks)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("group,new,heads", [(1, 1, 2), (4, 4, 2), (4, 7, 2), (16, 2, 1), (8, 1, 1)])
def test_windows_of_few_sequences(qb, kv, group, new, heads):
    """A sequence a workgroup of eight waves, of fewer blocks than waves, and of many more."""
    say("few sequences", kv, group, new, heads)
    b = Batch(qb, kv, 64, heads * group, heads, [3000, 31, 1400, 0, 400], [new, 1, max(new - 1, 0), new, new], seed=500 + group + new)
    for window, sinks in ((1, 0), (200, 3), (600, 40), (700, 0)):
        close(bf16_to_host(attend(qb, "paged", b, window, sinks)), b, window, sinks)
    one = Batch(qb, kv, 64, heads * group, heads, [2000], [new], seed=600 + group + new)
    for window, sinks in ((300, 1), (600, 0), (900, 0)):
        close(bf16_to_host(attend(qb, "paged", one, window, sinks)), one, window, sinks)


@pytest.mark.parametrize("group,new,seqs", [(2, 1, 1000), (2, 4, 1000), (16, 2, 600), (16, 2, 500), (32, 2, 300)])
def test_windows_of_many_sequences(qb, group, new, seqs):
    say("many sequences", group, new, seqs)
    r = np.random.Generator(np.random.Philox(group + seqs))
    b = Batch(qb, "bf16", 32, 2 * group, 2, r.integers(0, 90, seqs).tolist(), r.integers(0, new + 1, seqs).tolist(), seed=400 + group)
    close(bf16_to_host(attend(qb, "paged", b, 33, 3)), b, 33, 3)


@pytest.mark.parametrize("call", CALLS)
def test_a_window_of_everything_gives_the_same_bits(qb, call):
    """Windows and first tokens that hide nothing: the kernels without a window where the table says so, and the same sums where it does not (one
    worker: nothing is joined in another order)."""
    say("everything", call)
    b = Batch(qb, "bf16", 64, 8, 2, [100, 37], [3, 2], seed=5)
    full = qb.paged_attention(b.q(), 8, b.cache, 0, b.row_start, 3) if call == "paged" else qb.prompt_attention(b.q(), 8, b.cache, 0, b.row_start)
    for window, sinks in ((10 ** 6, 0), (1, 10 ** 6), (b.cache.max_pages * 64, 3)):
        assert torch.equal(attend(qb, call, b, window, sinks), full)
    for window, sinks in ((103, 0), (50, 60)):
        close(bf16_to_host(attend(qb, call, b, window, sinks)), b, 200, 0)


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_pages_outside_are_not_needed_and_strides(qb, call, kv):
    """trim takes the pages that nobody sees and the result keeps its bits; q and out as column blocks of wider tensors, the second of three layers,
    rows ahead of the first and behind the last sequence."""
    say("trimmed", call, kv)
    window, sinks = 70, 33
    b = Batch(qb, kv, 32, 8, 2, [1000, 0, 300, 64], [3, 0, 5, 1], layers=3, layer=1, seed=9, empty_rows=2)
    wide = torch.full((b.rows + 7, 8 * D + 48), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[2:2 + b.rows, 16:16 + 8 * D] = b.q()
    out = torch.full((b.rows + 7, 8 * D + 12), 7.0, dtype=torch.bfloat16, device="cuda")
    q, o, starts = wide[:, 16:16 + 8 * D], out[:, 4:4 + 8 * D], b.row_start + 2
    attend(qb, call, b, window, sinks, q, starts, 1, o)
    close(bf16_to_host(o[2:2 + b.rows]), b, window, sinks)
    assert (out[:2] == 7).all() and (out[2 + b.rows:] == 7).all() and (out[:, :4] == 7).all() and (out[:, 4 + 8 * D:] == 7).all()
    before = o.clone()
    pages = int((b.cache.table >= 0).sum())
    b.cache.trim(window, sinks)
    assert int((b.cache.table >= 0).sum()) < pages - 25
    free = (b.cache.refs == 0).nonzero().flatten()
    b.cache.pool.view(torch.uint8)[:, free] = 0xFF                        # whatever comes to lie there
    attend(qb, call, b, window, sinks, q, starts, 1, o)
    assert torch.equal(o, before)


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_a_missing_page_inside_is_not_visible(qb, call, kv):
    say("missing pages", call, kv)
    b = Batch(qb, kv, 32, 4, 2, [100, 20], [4, 4], seed=21)
    b.cache.table[0, 2] = -1                           # positions 64 .. 95 of the first sequence
    b.cache.table[1, 0] = b.cache.n_pages              # the whole second one
    got = ref.bf16_bits_to_f64(bf16_to_host(attend(qb, call, b, 50, 3))).reshape(b.rows, 4, D)
    assert (got[4:8] == 0).all()
    # what the first sequence's rows still see: 0 .. 2, of the window 54 + i .. 63, and 96 .. 100 + i
    for i in range(4):
        kept = np.r_[0:3, 51 + i:64, 96:101 + i]
        rows = ref.bf16_bits_to_f64(b.q_bits)[i:i + 1]
        want, size = pg.attention(rows, b.keys[0][kept], b.values[0][kept], len(kept) - 1)
        most = np.linalg.norm(rows, axis=2).max() * np.linalg.norm(b.keys[0][kept], axis=2).max() / np.sqrt(D)
        assert (np.abs(got[i] - want[0]) <= 1.01 * (2.0 ** -8 * np.abs(want[0]) + (2.0 ** -7 + 4 * 132 * 2.0 ** -24 * most) * size[0])).all()


@pytest.mark.parametrize("kv,bad", [("bf16", np.inf), ("bf16", np.nan), ("e4m3", np.nan)])
@pytest.mark.parametrize("call,hq,news", [(c, *x) for c in CALLS for x in ((2, [6, 1]), (8, [5, 3]), (20, [8, 2]), (2, [1, 1]))] + [("prompt", 8, [40, 7])])
def test_what_is_not_finite_reaches_the_rows_that_see_it_alone(qb, call, kv, bad, hq, news):
    """Two of them in a head: one that the first rows' windows still hold and the later ones' have passed, and one at a new position; and one among
    the first tokens.  Rows that see none are as near the oracle as ever."""
    say("not finite", call, kv, bad, hq, news)
    window, sinks = 60, 4
    b = Batch(qb, kv, 64, hq, 2, [130, 33], news, seed=300 + hq)
    want, tol = expected(b, window, sinks)
    places, raw = pg.block_places(kv), b.cache.pool[0].view(torch.int16 if kv == "bf16" else torch.uint8)
    bits = int(ref.f32_to_bf16_bits(np.array([bad], np.float32)).view(np.int16)[0]) if kv == "bf16" else 0x7F
    for where in ([130 - window + 1 + 1, 130 + 4], [130 - window - 1], [2], [5], [130 - window + 1]):
        for half in (0, 1):
            keep = raw.clone()
            for pos in where:
                if pos < 130 + news[0]:
                    raw[int(b.table[0, pos // 64]), 1, pos % 64 // 32, half, int(places[half][pos % 32, 17])] = bits
            got = attend(qb, call, b, window, sinks).view(b.rows, hq, D).double().cpu().numpy()
            raw.copy_(keep)
            hit = np.zeros((b.rows, hq), bool)
            for i in range(news[0]):
                hit[i, hq // 2:] = any(win.sees(130 + i, p, window, sinks) for p in where)
            assert (np.abs(got - want)[~hit] <= tol[~hit]).all(), (where, half)
            if half == 1 or not np.isinf(bad):
                assert not np.isfinite(got[hit]).all(axis=-1).any(), (where, half)


@pytest.mark.parametrize("call", CALLS)
def test_books_that_do_not_fit(qb, call):
    say("odd books", call)
    b = Batch(qb, "bf16", 32, 4, 2, [60, 40, 30, 20], [2, 2, 2, 4], seed=22, more_columns=0)
    good = attend(qb, call, b, 25, 2)
    for starts in ([0, 2, 4, 6, 99], [-3, 2, 4, 6, 10], [0, 2, 1, 6, 10], [2 ** 31 - 1] * 5, [-2 ** 31] * 5):
        out = torch.full_like(good, 5.0)
        attend(qb, call, b, 25, 2, starts=i32_to_dev(starts), out=out)
        torch.cuda.synchronize()
        if starts[:4] == [0, 2, 4, 6]:
            assert torch.equal(out[:6], good[:6]) and (out[6:] == 5).all()
        if abs(starts[0]) > 99:
            assert (out == 5).all()
    for length in (-1, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31):
        b.cache.lengths[0] = length
        out = attend(qb, call, b, 25, 2, out=torch.full_like(good, 5.0))
        assert torch.equal(out[2:], good[2:]) and (out[:2] == 5).all()
    b.cache.lengths[0] = 2 ** 24                       # (allowed, and nothing of its window has a place in the table)
    out = attend(qb, call, b, 25, 0, out=torch.empty_like(good))
    assert (out[:2] == 0).all()


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("hq,hk,lengths,news,window", [(8, 2, [3000, 40, 0, 700], [2, 1, 3, 0], 60), (8, 2, [3000, 40, 0, 700], [2, 1, 3, 0], 1500), (16, 2, [900, 2500], [8, 7], 100),
                                                       (16, 2, [900, 2500], [8, 7], 1500), (16, 1, [300, 64], [30, 32], 200)])
def test_in_place(qb, call, hq, hk, lengths, news, window):
    """The output over the queries: the same bits as beside them, also in rows of a wider tensor."""
    say("in place", call, hq, window)
    b = Batch(qb, "bf16", 64, hq, hk, lengths, news, seed=50 + window)
    want = attend(qb, call, b, window, 4)
    q = b.q().clone()
    assert torch.equal(attend(qb, call, b, window, 4, q=q, out=q), want)
    wide = torch.zeros(q.shape[0], q.shape[1] + 64, dtype=q.dtype, device="cuda")
    wide[:, :q.shape[1]] = b.q()
    view = wide[:, :q.shape[1]]
    assert torch.equal(attend(qb, call, b, window, 4, q=view, out=view), want) and not wide[:, q.shape[1]:].any()


@pytest.mark.parametrize("call", CALLS)
def test_a_captured_call_follows_the_lengths(qb, call):
    """One graph over lengths and row counts that change, with eager calls on the same cache between the replays."""
    say("captured", call)
    b = Batch(qb, "bf16", 64, 8, 2, [500, 200, 3000], [2, 2, 2], seed=31)
    q, out = b.q(), torch.empty(b.rows, 8 * D, dtype=torch.bfloat16, device="cuda")
    attend(qb, call, b, 200, 4, q=q, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        attend(qb, call, b, 200, 4, q=q, out=out)
    for lengths in ([500, 200, 3000], [10, 100, 2998], [499, 0, 1]):
        b.cache.lengths.copy_(i32_to_dev(lengths))
        eager = attend(qb, call, b, 200, 4, q=q)
        out.fill_(9.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        attend(qb, call, b, 7, 0, q=q)


def test_refusals_of_the_binding(qb):
    say("refusals")
    b = Batch(qb, "bf16", 64, 4, 2, [100], [2], seed=41)
    for fn in (lambda **k: qb.paged_attention(b.q(), 4, b.cache, 0, b.row_start, 2, **k), lambda **k: qb.prompt_attention(b.q(), 4, b.cache, 0, b.row_start, **k)):
        for bad in (dict(window=0), dict(window=-5), dict(window=5, sinks=-1), dict(sinks=3)):
            with pytest.raises(ValueError):
                fn(**bad)
        for bad in (dict(window=2.0), dict(window=True), dict(window=5, sinks="4")):
            with pytest.raises(TypeError):
                fn(**bad)
        fn(window=2 ** 70, sinks=2 ** 70)
    for bad in ((0, 0), (-1, 0), (4, -1)):
        with pytest.raises(ValueError):
            b.cache.trim(*bad)
    with pytest.raises(TypeError):
        b.cache.trim(4.0)


# --------------------------------------------------------------------------------------------------------------- trim

@pytest.mark.parametrize("page,seqs,columns,window,sinks", [(32, 1, 5, 1, 0), (32, 7, 40, 100, 4), (64, 64, 30, 333, 65), (128, 33, 9, 1, 1), (1024, 3, 4, 1500, 0), (32, 200, 60, 32, 32),
                                                            (32, 3, 3000, 40, 64), (64, 5, 20, 1 << 40, 0), (64, 5, 20, 1, 1 << 40)])
def test_trim(qb, page, seqs, columns, window, sinks):
    """Books of every kind, shared pages, missing ones and pages without positions among them, against the oracle position by position; twice gives the same."""
    say("trim", page, seqs, columns, window, sinks)
    r = np.random.Generator(np.random.Philox(page + seqs))
    pages = seqs * columns
    lengths = r.integers(0, columns * page + 1, seqs)
    table = np.where(r.random((seqs, columns)) < 0.9, r.integers(0, pages, (seqs, columns)), -1)
    refs = np.bincount(table[table >= 0], minlength=pages)
    c = qb.PagedKvCache(1, 1, pages, page_len=page, max_seqs=seqs, max_pages=columns)
    c.refs.copy_(i32_to_dev(refs)); c.lengths.copy_(i32_to_dev(lengths)); c.table.copy_(i32_to_dev(table))
    want_refs, want_table = win.trim(refs.tolist(), lengths.tolist(), table.tolist(), page, min(window, 1 << 25), min(sinks, 1 << 25))
    for _ in range(2):
        c.trim(window, sinks)
        assert c.refs.tolist() == want_refs and c.table.tolist() == want_table and c.lengths.tolist() == lengths.tolist()


@pytest.mark.parametrize("seqs,parents", [(2, 1), (9, 1), (29, 2), (64, 5), (1024, 3)])
def test_trim_of_forks(qb, seqs, parents):
    """Pages that many sequences share, in neighbouring rows and others, of different lengths."""
    say("trim, forks", seqs, parents)
    r = np.random.Generator(np.random.Philox(seqs))
    columns, page = 300, 32
    table = r.permutation(parents * columns).reshape(parents, columns)[np.sort(r.integers(0, parents, seqs)) if seqs < 64 else r.integers(0, parents, seqs)]
    lengths = r.integers(columns * page // 2, columns * page + 1, seqs)
    table = np.where(np.arange(columns) * page < lengths[:, None], table, -1)
    refs = np.bincount(table[table >= 0], minlength=parents * columns)
    c = qb.PagedKvCache(1, 1, parents * columns, page_len=page, max_seqs=seqs, max_pages=columns)
    c.refs.copy_(i32_to_dev(refs)); c.lengths.copy_(i32_to_dev(lengths)); c.table.copy_(i32_to_dev(table))
    want_refs, want_table = win.trim(refs.tolist(), lengths.tolist(), table.tolist(), page, 700, 40)
    c.trim(700, 40)
    assert c.refs.tolist() == want_refs and c.table.tolist() == want_table


def test_trim_leaves_odd_books(qb):
    """Lengths that are none leave their rows; ids beyond the pool go without touching a count."""
    say("trim, odd books")
    c = qb.PagedKvCache(1, 1, 6, page_len=32, max_seqs=5, max_pages=4)
    c.refs.fill_(3)
    c.lengths.copy_(i32_to_dev([-1, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31, 128]))
    c.table.copy_(i32_to_dev([[0, 1, 2, 3]] * 4 + [[6, 2 ** 31 - 1, 5, -7]]))
    c.trim(1)
    assert c.table.tolist() == [[0, 1, 2, 3]] * 4 + [[-1, -1, -1, -7]] and c.refs.tolist() == [3, 3, 3, 3, 3, 2]


def test_a_windowed_run_of_steps_in_few_pages(qb):
    """Prompts, then steps: reserve, append, attention of a window, trim.  The pool holds the windows, not the contexts; every step's output is that of a
    cache which keeps everything."""
    say("a run of steps")
    hq, hk, page, window, sinks, seqs = 4, 2, 32, 50, 5, 3
    r = np.random.Generator(np.random.Philox(77))
    small = qb.PagedKvCache(2, hk, seqs * 5, page_len=page, max_seqs=seqs, max_pages=40)
    large = qb.PagedKvCache(2, hk, seqs * 40, page_len=page, max_seqs=seqs, max_pages=40)
    rope = qb.Rope(64, 1e4, layout="interleaved")
    peak = 0
    for step in range(60):
        news = [70, 33, 90] if step == 0 else [int(n) for n in r.integers(0, 9, seqs)]
        rows = sum(news)
        starts, new = i32_to_dev(np.concatenate([[0], np.cumsum(news)])), i32_to_dev(news)
        qkv = torch.randn(rows, (hq + 2 * hk) * D, device="cuda", generator=torch.Generator("cuda").manual_seed(step)).bfloat16()
        out = []
        for cache in (small, large):
            assert cache.reserve(new).tolist() == [1] * seqs
            for layer in range(2):
                q = qb.paged_prepare(qkv, hq, cache, layer, starts, None, None, rope=rope)
                if step:
                    out.append(qb.paged_attention(q, hq, cache, layer, starts, 8, window=window, sinks=sinks))
                else:
                    out.append(qb.prompt_attention(q, hq, cache, layer, starts, window=window, sinks=sinks))
            cache.lengths.add_(new)
        small.trim(window, sinks)
        assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3]) and torch.isfinite(out[0]).all()
        peak = max(peak, int((small.refs > 0).sum()))
    assert int(large.lengths.min()) > 200 and peak <= seqs * 4


class _Sub(torch.Tensor):
    pass


def test_calls_that_are_not_ordinary(qb):
    """What the native side leaves to the Python path has the same bits."""
    say("not ordinary")
    b = Batch(qb, "bf16", 64, 8, 2, [100, 700], [2, 5], seed=42)
    q, sub = b.q(), b.q().as_subclass(_Sub)
    assert qb._fast.paged_attention_window(b.cache._handle, sub, 8, 0, b.row_start, 5, 90, 3, None, None) == -1
    assert qb._fast.prompt_attention_window(b.cache._handle, sub, 8, 0, b.row_start, 90, 3, None) == -1
    for args in ((5, 0, 0), (5, 90, -1), (5, 90.0, 3), (5, True, 3)):
        assert qb._fast.paged_attention_window(b.cache._handle, q, 8, 0, b.row_start, *args, None, None) == -1
        assert qb._fast.prompt_attention_window(b.cache._handle, q, 8, 0, b.row_start, *args[1:], None) == -1
    w = dict(window=90, sinks=3)
    assert torch.equal(qb.paged_attention(sub, 8, b.cache, 0, b.row_start, 5, **w), qb.paged_attention(q, 8, b.cache, 0, b.row_start, 5, **w))
    assert torch.equal(qb.prompt_attention(sub, 8, b.cache, 0, b.row_start, **w), qb.prompt_attention(q, 8, b.cache, 0, b.row_start, **w))
    qkv = torch.randn(7, 12 * D, device="cuda").bfloat16()
    rope = qb.Rope(32, 1e4)
    append = lambda x: qb.paged_prepare(x, 8, b.cache, 0, b.row_start, None, None, rope=rope)
    assert torch.equal(append(qkv.as_subclass(_Sub)), append(qkv))
    before = b.cache.table.clone()
    assert qb._fast.pages_trim(b.cache._handle, 0, 0) == -1 and qb._fast.pages_trim(b.cache._handle, 90, -1) == -1 and torch.equal(before, b.cache.table)


def test_forks_and_moves_of_trimmed_sequences(qb):
    """A trimmed sequence is forked, steps on twice over, and its pages move: every output is that of a cache which keeps everything."""
    say("forks of trimmed")
    hq, hk, page, window, sinks = 4, 1, 32, 40, 2
    small, large = (qb.PagedKvCache(1, hk, n, page_len=page, max_seqs=3, max_pages=30) for n in (24, 90))
    rope = qb.Rope(128, 1e4)

    def step(news, seed):
        starts, new = i32_to_dev(np.concatenate([[0], np.cumsum(news)])), i32_to_dev(news)
        qkv = torch.randn(sum(news), (hq + 2 * hk) * D, device="cuda", generator=torch.Generator("cuda").manual_seed(seed)).bfloat16()
        outs = []
        for cache in (small, large):
            assert cache.reserve(new).tolist() == [1] * 3
            q = qb.paged_prepare(qkv, hq, cache, 0, starts, None, None, rope=rope)
            outs.append(qb.prompt_attention(q, hq, cache, 0, starts, window=window, sinks=sinks))
            cache.lengths.add_(new)
        small.trim(window, sinks)
        assert torch.equal(*outs) and torch.isfinite(outs[0]).all()
    step([200, 0, 250], 1)
    for turn, parent in enumerate(([0, 0, 2], [2, 1, 2], [1, 0, 0])):
        for cache in (small, large):
            cache.fork(i32_to_dev(parent))
        for i in range(4):
            step([7, 20, 1], 10 * turn + i + 2)
        small.compact()
        held = np.bincount(small.table.cpu().numpy()[small.table.cpu().numpy() >= 0], minlength=24)
        assert (small.refs.cpu().numpy() == held).all()
    assert int(large.lengths.max()) > 300 and (small.table[:, 1:4] == -1).all()
