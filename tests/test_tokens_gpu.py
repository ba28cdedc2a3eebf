"""GPU parity of drawing and verifying tokens through the binding against the CPU oracle.

How near.  The kernels take weights as whole multiples of 2^-48 of the largest of a part of the vocabulary, each off by half of one, and leave out what
weighs less than 2^-46 of the largest, or some of it (the buckets end 32 units below it; 2^-46.17): together off by less than V 2^-46 of the whole.  fp64 sums of V terms and the
exponentials (2^-46 relatively) add less than V 2^-52 and 2^-46.  A running mass, and a point u C, are therefore off by at most TOL = V 2^-45 + 2^-44 of the whole:
the token has to be one that covers the point within that, and THE oracle's where its own interval is clear of the point by more.  The same holds
for the cuts; the inputs here are continuous (no border lies that near) or exact (equal weights, whole shares: nothing rounds).  A probability is
rounded to fp32 once (2^-24 of it)."""
import numpy as np
import pytest
import torch

from oracle import quasar_tokens_ref as tok

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qb():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2603_01399_amd import binding
    return binding


def say(*a):
    print(*a, flush=True)


def tol_of(V):
    return V * 2.0 ** -45 + 2.0 ** -44


def dev(a, dtype):
    return torch.as_tensor(np.asarray(a)).to(dtype).cuda()


def logits_of(r, T, V, kind="broad"):
    z = r.standard_normal((T, V)) * 1.7
    if kind == "broad":
        z += (r.random((T, V)) < 0.01) * r.random((T, V)) * (4 + 12 * r.random((T, 1)))
    return z


def check_draw(z, u, token, p, V, **filters):
    """The token and its probability, of a row that is what the GPU saw (fp64)."""
    tokens, q = tok.left(z, **filters)
    tol = tol_of(V)
    at = np.flatnonzero(tokens == token)
    assert len(at) == 1, ("not one of those left", token, len(tokens), filters)
    through = np.cumsum(q)
    lo, hi = through[at[0]] - q[at[0]], through[at[0]]
    point = min(float(u), 1 - 2.0 ** -24)
    assert lo - tol <= point < hi + tol, (token, lo, hi, u)
    want = tok.draw(tokens, q, point)
    edge = np.abs(through - point).min()
    assert token == want or edge <= tol
    if p is not None:
        assert abs(float(p) - q[at[0]]) <= 2.0 ** -24 * q[at[0]] + 2 * tol


def seen(t):
    return t.double().cpu().numpy()


FILTERS = [dict(), dict(temperature=0.7), dict(top_k=1), dict(top_k=5), dict(top_k=50, temperature=1.3), dict(top_p=0.9), dict(top_p=0.3, temperature=0.8), dict(top_p=1e-6),
           dict(min_p=0.05), dict(min_p=0.5), dict(min_p=1.0), dict(top_k=40, top_p=0.95), dict(top_k=200, top_p=0.7, min_p=0.02, temperature=0.9), dict(temperature=0.0),
           dict(top_p=0.99, min_p=1e-4), dict(top_p=0.0), dict(temperature=30.0, top_p=0.6), dict(temperature=0.02)]


def params(rows):
    """Filters of rows -> the tensors of a call."""
    get = lambda k, d: [f.get(k, d) for f in rows]
    return dict(temperature=dev(get("temperature", 1.0), torch.float32), top_k=dev(get("top_k", 0), torch.int32), top_p=dev(get("top_p", 1.0), torch.float32),
                min_p=dev(get("min_p", 0.0), torch.float32))


def as_seen(f):
    """As fp32 parameters."""
    return {k: v if k == "top_k" else float(np.float32(v)) for k, v in f.items()}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,pad,off", [(1, 0, 0), (2, 3, 1), (3, 0, 0), (7, 1, 2), (16, 0, 0), (255, 2, 3), (257, 0, 1), (1000, 24, 0), (8191, 0, 0), (8192, 0, 0), (8193, 1, 5),
                                       (8199, 0, 7), (16381, 0, 3), (20011, 13, 1)])
def test_sample(qb, dtype, V, pad, off):
    """Every kind of filter, each its row; rows that begin anywhere, in wider tensors whose other columns must not be read as logits."""
    say("sample", dtype, V, pad, off)
    r = np.random.Generator(np.random.Philox(V))
    T = len(FILTERS) * 2
    wide = torch.full((T, V + pad + off), float("nan"), dtype=dtype, device="cuda")
    wide[:, ::2] = 1e30
    z = wide[:, off:off + V]
    z.copy_(dev(logits_of(r, T, V), torch.float32))
    rows = [FILTERS[i % len(FILTERS)] for i in range(T)]
    u = r.random(T).astype(np.float32)
    token, p = qb.sample_tokens(z, dev(u, torch.float32), **params(rows))
    for i in range(T):
        check_draw(seen(z[i]), u[i], int(token[i]), p[i], V, **as_seen(rows[i]))


@pytest.mark.parametrize("dtype,V", [(torch.float32, 151936), (torch.bfloat16, 151936), (torch.bfloat16, 1 << 20), (torch.float32, (1 << 20) - 3)])
def test_sample_of_large_vocabularies(qb, dtype, V):
    say("large", dtype, V)
    r = np.random.Generator(np.random.Philox(7))
    rows = [FILTERS[i] for i in (0, 4, 5, 8, 12, 13)]
    z = dev(logits_of(r, len(rows), V), torch.float32).to(dtype)
    u = r.random(len(rows)).astype(np.float32)
    token, p = qb.sample_tokens(z, dev(u, torch.float32), **params(rows))
    for i, f in enumerate(rows):
        check_draw(seen(z[i]), u[i], int(token[i]), p[i], V, **as_seen(f))


@pytest.mark.parametrize("V", [5, 3000, 9000, 50257])
def test_equal_logits(qb, V):
    """Nothing rounds: the cut and the draw are the first ones, exactly; more equal tokens than are kept in LDS."""
    say("equal", V)
    us = [0.0, 0.25, 0.5, 0.75, 1 - 2.0 ** -24]
    for dtype in (torch.float32, torch.bfloat16):
        z = torch.full((len(us), V), -3.5, dtype=dtype, device="cuda")
        u = dev(us, torch.float32)
        for left, filters in ((V, {}), (min(V, 4000), dict(top_k=4000)), (-(-V // 2), dict(top_p=0.5)), (-(-min(V, 4000) // 4), dict(top_k=4000, top_p=0.25)), (V, dict(min_p=1.0)), (1, dict(top_k=1)),
                              (1, dict(temperature=0.0)), (1, dict(top_p=1e-30))):
            token, p = qb.sample_tokens(z, u, **params([filters] * len(us)))
            assert token.tolist() == [min(left - 1, int(x * left)) for x in us], filters
            assert np.allclose(p.cpu(), 1 / left, rtol=2.0 ** -23)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,off", [(1, 0), (5, 3), (130, 1), (8190, 7), (30000, 2), (151936, 5), (1 << 20, 0)])
def test_the_first_of_equal_ones_wherever_it_is(qb, dtype, V, off):
    """Temperature 0, top_k 1, top_p 0: the largest logit's first place, of ties at the row's ends and at borders of what is read together, among what is no number."""
    say("first", dtype, V, off)
    r = np.random.Generator(np.random.Philox(V))
    ends = sorted({v for v in (0, 1, 6, 7, 8, 63, 64, 127, 128, 8185, 8191, 8192, 16383, V // 2, V - 2, V - 1) if 0 <= v < V})
    wide = torch.full((len(ends), V + off), float("nan"), dtype=dtype, device="cuda")
    z = wide[:, off:]
    z.copy_(dev(np.where(r.random(V) < 0.02, np.nan, np.where(r.random(V) < 0.02, -np.inf, -np.abs(r.standard_normal(V)) - 1)), torch.float32))
    top = (0.0, 3.5, np.inf, -0.5)
    for i, v in enumerate(ends):
        z[i, v] = -0.0 if top[i % 4] == 0 else top[i % 4]
        for w in ends[i + 1:]:
            z[i, w] = top[i % 4]
    n = len(ends)
    u = dev(r.random(n), torch.float32)
    for f in (dict(temperature=dev([0.0] * n, torch.float32)), dict(top_k=dev([1] * n, torch.int32), top_p=dev([0.5] * n, torch.float32)), dict(top_p=dev([0.0] * n, torch.float32))):
        token, p = qb.sample_tokens(z, u, **f)
        assert token.tolist() == ends and (p == 1).all()
    starts, one = dev([0, n], torch.int32), dev([1], torch.int32)
    accepted, token, p = qb.verify_tokens(z, starts, dev(ends, torch.int32), u * 0 + 0.999, u, top_k=one)
    assert (accepted.tolist(), token.tolist()) == ([n - 1], [ends[-1]]) and (p == 1).all()
    if n > 1:
        wrong = dev([ends[0], *[v + 1 for v in ends[1:]]], torch.int32)
        accepted, token, p = qb.verify_tokens(z, starts, wrong, u * 0, u, top_k=one)
        assert (accepted.tolist(), token.tolist()) == ([min(1, n - 1)], [ends[1]]) and p.tolist() == [1.0] + [0.0] * (n - 1)


@pytest.mark.parametrize("spread", [1e-6, 1e-3, 0.05])
def test_a_bucket_of_more_than_fit(qb, spread):
    """Continuous logits so near that they share a bucket or a few: the cut is found in tokens that are read again."""
    say("crowded", spread)
    r = np.random.Generator(np.random.Philox(8))
    V = 30000
    rows = [dict(top_k=1), dict(top_k=17), dict(top_k=20000), dict(top_p=0.5), dict(top_p=0.999), dict(min_p=0.9999), dict(min_p=float(np.exp(-spread))), dict(top_k=9000, top_p=0.3, min_p=0.01), {}]
    z = dev(5 + r.standard_normal((len(rows), V)) * spread, torch.float32)
    u = r.random(len(rows)).astype(np.float32)
    token, p = qb.sample_tokens(z, dev(u, torch.float32), **params(rows))
    for i, f in enumerate(rows):
        check_draw(seen(z[i]), u[i], int(token[i]), p[i], V, **as_seen(f))


def test_odd_logits(qb):
    """Rows without a finite logit, with one, infinities and what is not a number, both zeros, the largest numbers, sorted rows."""
    say("odd logits")
    inf, nan, V = float("inf"), float("nan"), 10007
    r = np.random.Generator(np.random.Philox(9))
    base = logits_of(r, 1, V)[0]
    rows = [np.full(V, -inf), np.full(V, nan), np.where(np.arange(V) == 9000, 1.0, -inf), np.where(np.arange(V) % 7 == 0, base, -inf), np.where(np.arange(V) % 3 == 0, nan, base),
            np.where((np.arange(V) == 5) | (np.arange(V) == 9999), inf, base), np.where(np.arange(V) % 2, 0.0, -0.0), base * 1e37, np.sort(base), -np.sort(-base), base - 3e38, base * 1e-40,
            np.where(np.arange(V) == 77, 40.0, base), np.where(np.arange(V) < 20, 3e38, -3e38)]
    z = dev(np.stack(rows), torch.float32)
    for filters in ({}, dict(top_k=100), dict(top_p=0.8), dict(min_p=0.1), dict(top_k=6000, top_p=0.9, min_p=1e-3), dict(temperature=0.0), dict(temperature=1e-30, top_p=0.9), dict(temperature=3e38),
                    dict(temperature=inf, top_p=0.5), dict(temperature=1e-45)):
        u = r.random(len(rows)).astype(np.float32)
        token, p = qb.sample_tokens(z, dev(u, torch.float32), **params([filters] * len(rows)))
        assert token[:2].tolist() == [-1, -1] and p[:2].tolist() == [0.0, 0.0] and int(token[2]) == 9000 and float(p[2]) == 1.0
        for i in range(2, len(rows)):
            check_draw(seen(z[i]), u[i], int(token[i]), p[i], V, **as_seen(filters))
    for u, want in ((-1.0, 5), (nan, 5), (0.0, 5), (0.49, 5), (0.51, 9999), (1.0, 9999), (7.0, 9999), (inf, 9999)):
        assert int(qb.sample_tokens(z[5:6], dev([u], torch.float32))[0]) == want


def test_odd_parameters(qb):
    """What is not a number or beyond its range counts as documented; None is the default of each."""
    say("odd parameters")
    nan, inf, V = float("nan"), float("inf"), 5000
    r = np.random.Generator(np.random.Philox(10))
    z = dev(np.repeat(logits_of(r, 1, V), 12, axis=0), torch.float32)
    u = dev(np.full(12, 0.6), torch.float32)
    def draw(**k):
        return [int(t) for t in qb.sample_tokens(z, u, **{n: dev([v] * 12, torch.int32 if n == "top_k" else torch.float32) for n, v in k.items()})[0].unique()]
    first = [int(z[0].argmax())]
    plain = draw()
    assert draw(temperature=0.0) == draw(temperature=-2.0) == draw(temperature=nan) == draw(top_k=1) == draw(top_p=0.0) == draw(top_p=-1.0) == draw(min_p=1.0) == draw(min_p=9.0) == first
    assert draw(temperature=1.0) == draw(top_k=0) == draw(top_k=-5) == draw(top_k=V) == draw(top_k=2 ** 31 - 1) == draw(top_p=1.0) == draw(top_p=nan) == draw(top_p=inf) == draw(min_p=0.0) \
        == draw(min_p=nan) == draw(min_p=-1.0) == plain


def test_many_rows(qb):
    """More rows than are in the workspace at a time."""
    say("many rows")
    r = np.random.Generator(np.random.Philox(11))
    T, V = 1300, 300
    z = dev(logits_of(r, T, V), torch.float32).bfloat16()
    rows = [FILTERS[i % len(FILTERS)] for i in range(T)]
    u = r.random(T).astype(np.float32)
    token, p = qb.sample_tokens(z, dev(u, torch.float32), **params(rows))
    host = seen(z)
    for i in range(T):
        check_draw(host[i], u[i], int(token[i]), p[i], V, **as_seen(rows[i]))


def test_logits_of_more_than_4_gb(qb):
    """Rows behind the 2^32nd byte and the 2^31st logit; equal logits of 2^k tokens have equal shares, exactly."""
    say("4 GB of logits")
    V, T = 131072, 17000
    z = torch.zeros(T, V, dtype=torch.bfloat16, device="cuda")
    r = np.random.Generator(np.random.Philox(17))
    z[-3:] = dev(logits_of(r, 3, V), torch.float32).bfloat16()
    u = (torch.arange(T, device="cuda") % 4096 + 0.5) / 4096
    token, p = qb.sample_tokens(z, u)
    assert torch.equal(token[:-3], (u[:-3] * V).int()) and (p[:-3] == 1 / V).all()
    for i in range(T - 3, T):
        check_draw(seen(z[i]), float(u[i]), int(token[i]), p[i], V)


def test_the_draw_follows_the_distribution(qb):
    """Numbers on a grid give every token its share: the inverse CDF, through all steps of a draw."""
    say("shares")
    r = np.random.Generator(np.random.Philox(12))
    V, n = 20000, 4000
    z = np.concatenate([r.standard_normal(V - 40) - 6, r.standard_normal(40) * 2])[r.permutation(V)]
    f = dict(top_k=60, top_p=0.97, temperature=0.9)
    zt = dev(z, torch.float32)[None].expand(n, V)
    token, _ = qb.sample_tokens(zt, dev((np.arange(n) + 0.5) / n, torch.float32), **params([f] * n))
    tokens, q = tok.left(seen(zt[0]), **as_seen(f))
    assert (np.diff(token.cpu().numpy()) >= 0).all()                              # in vocabulary order
    share = np.bincount(token.cpu().numpy(), minlength=V)[tokens]
    assert np.abs(share / n - q).max() <= 1.01 / n and share.sum() == n            # (whole numbers: quotients by n would each be rounded)


# -------------------------------------------------------------------------------------------------------------- drafts

def check_verify(qb, z, starts, drafts, ua, us, seq_filters, kwargs):
    T, V = z.shape
    accepted, token, p = qb.verify_tokens(z, dev(starts, torch.int32), dev(drafts, torch.int32), dev(ua, torch.float32), dev(us, torch.float32), **kwargs)
    host, tol = seen(z), tol_of(V)
    accepted, token, p = accepted.tolist(), token.tolist(), p.double().cpu().numpy()
    for s, f in enumerate(seq_filters):
        a, b = starts[s], starts[s + 1]
        if a == b:
            assert (accepted[s], token[s]) == (0, -1)
            continue
        n, last = 0, b - a - 1
        for i in range(a, b):
            tokens, q = tok.left(host[i], **f)
            want = float(q[tokens == drafts[i]].sum())
            assert abs(p[i] - want) <= 2.0 ** -24 * want + 2 * tol
            if n == i - a and n < last and ua[i] < want:
                assert accepted[s] > n or want - ua[i] <= 2 * tol
                n += 1
            elif n == i - a:
                assert accepted[s] == n or abs(want - ua[i]) <= 2 * tol
                if accepted[s] == n:
                    if n < last:
                        stays = tokens != drafts[i]
                        tokens, q = tokens[stays], q[stays] / max(q[stays].sum(), 1e-300)
                    if len(tokens) == 0:
                        assert token[s] == -1
                    else:
                        through, at = np.cumsum(q), np.flatnonzero(tokens == token[s])
                        assert len(at) == 1 and through[at[0]] - q[at[0]] - 1e-9 <= us[i] < through[at[0]] + 1e-9       # (what is left may be a small part of the whole)
                        assert token[s] == tok.draw(tokens, q, us[i]) or np.abs(through - us[i]).min() <= 1e-9
                n = -1
    return accepted


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,news", [(50, [1]), (257, [4, 1, 0, 7]), (8193, [8, 8, 3]), (30011, [1, 2, 5, 0, 0, 9]), (1000, [33, 1, 70])])
def test_verify(qb, dtype, V, news):
    say("verify", dtype, V, news)
    r = np.random.Generator(np.random.Philox(V + len(news)))
    starts = np.concatenate([[0], np.cumsum(news)])
    T = int(starts[-1])
    some = []
    for trial in range(4):
        z = dev(logits_of(r, T, V), torch.float32).to(dtype)
        z = torch.cat([z, z], 1)[:, :V] if trial == 1 else z                    # (a row stride of twice the vocabulary)
        seqs = [FILTERS[int(i)] for i in r.integers(0, len(FILTERS), len(news))]
        host = seen(z)
        drafts = []
        for i in range(T):
            s = int(np.searchsorted(starts, i, side="right")) - 1
            tokens, q = tok.left(host[i], **as_seen(seqs[s]))
            drafts.append(int(tokens[np.argmax(q)]) if r.random() < 0.8 else int(r.integers(0, V)))
        ua, us = r.random(T).astype(np.float32) * np.float32(0.5), r.random(T).astype(np.float32)
        some += check_verify(qb, z, starts, drafts, ua, us, [as_seen(f) for f in seqs], params(seqs))
    assert V < 200 or max(some) > 0


def test_verify_of_more_rows_than_are_in_the_workspace_at_a_time(qb):
    """Sequences whose rows lie in one launch's rows, in two, in three."""
    say("many rows of drafts")
    r = np.random.Generator(np.random.Philox(16))
    V, news = 300, [300, 0, 400, 1, 1100, 7]
    starts = np.concatenate([[0], np.cumsum(news)])
    T = int(starts[-1])
    z = dev(logits_of(r, T, V), torch.float32)
    seqs = [FILTERS[i] for i in (0, 4, 13, 8, 13, 12)]
    drafts = seen(z).argmax(1)
    ua, us = np.zeros(T, np.float32), r.random(T).astype(np.float32)
    ua[[150, 1700]] = 1.0
    assert check_verify(qb, z, starts, drafts, ua, us, [as_seen(f) for f in seqs], params(seqs)) == [150, 0, 399, 0, 999, 6]


def test_verify_of_odd_drafts_and_rows(qb):
    """Ids outside the vocabulary are never accepted and take nothing away; a draft that has all the mass is accepted, and refused (a number of 1 or more)
    leaves nothing; rows of nobody are left; starts that do not fit have no rows."""
    say("odd drafts")
    V = 9001
    r = np.random.Generator(np.random.Philox(13))
    z = dev(logits_of(r, 8, V), torch.float32)
    z[2] = float("-inf")
    z[2, 8200] = 1.0
    host = seen(z)
    top = host.argmax(1)
    ones, zeros, half = np.full(8, 1.0), np.zeros(8), np.full(8, 0.5)
    f = [dict()]
    for d in (-1, V, 2 ** 31 - 1, -2 ** 31):
        assert check_verify(qb, z, [0, 3], np.where(np.arange(8) == 1, d, top), zeros, half, f, {}) == [1]
    run = lambda ua, starts=(0, 8): [t.tolist() for t in qb.verify_tokens(z, dev(starts, torch.int32), dev(top, torch.int32), dev(ua, torch.float32), dev(half, torch.float32))[:2]]
    assert run(zeros)[0] == [7] and run(np.where(np.arange(8) == 2, 0.999999, 0.0))[0] == [7]
    assert run(np.where(np.arange(8) == 2, 1.0, 0.0)) == [[2], [-1]] and run(np.full(8, np.nan))[0] == [0]
    for starts in ((-1, 8), (0, 9), (5, 3), (2 ** 31 - 1, -2 ** 31)):
        assert run(zeros, starts) == [[0], [-1]]
    assert run(zeros, (3, 5, 4, 8))[0][1] == 0                                   # (starts that fall: whose row is whose is not said)
    # rows ahead of, behind and between sequences
    lib, p = qb.lib(), torch.full((8,), 5.0, device="cuda")
    acc, token = (torch.empty(1, dtype=torch.int32, device="cuda") for _ in range(2))
    ws = torch.empty(lib.quasar_verify_tokens_workspace_bytes(8, V), dtype=torch.uint8, device="cuda")
    starts, ids, ua = dev([2, 5], torch.int32), dev(top, torch.int32), dev(zeros, torch.float32)
    assert lib.quasar_verify_tokens(z.data_ptr(), 0, 8, V, V, starts.data_ptr(), 1, ids.data_ptr(), None, None, None, None, ua.data_ptr(), ua.data_ptr(), acc.data_ptr(), token.data_ptr(),
                                    p.data_ptr(), ws.data_ptr(), ws.nbytes, torch.cuda.current_stream().cuda_stream) == 0
    assert int(acc) == 2 and (p[:2] == 5).all() and (p[5:] == 5).all() and (p[2:5] < 5).all()


@pytest.mark.parametrize("others", [-20.0, -19.0, -18.5, -10.0, -3.0])
def test_a_refused_draft_that_was_nearly_all_of_its_part(qb, others):
    """The mass that is left is the others', not what rounding leaves of a difference.  (-20 is 32 below the largest: e^-32 is 2^-46.2, which may be left out.)
    Each weight is off by at most 2^-49 of the largest, 1, so the running masses of what is left, R in all, by V 2^-49 / R of R each, twice that between
    a running mass and the point: 10 % at -19, where a weight is ten units of 2^-48, 2^-19 at -3."""
    say("nearly all", others)
    V = 20000
    z = torch.full((2, V), others, device="cuda")
    z[0, 100], z[0, 15000] = 12.0, -18.0
    for u in np.linspace(0, 0.9999, 30).astype(np.float32):
        us = dev([u, u], torch.float32)
        accepted, token, _ = qb.verify_tokens(z, dev([0, 2], torch.int32), dev([100, 0], torch.int32), dev([1.0, 0.0], torch.float32), us)
        rest = seen(z[0])
        rest[100] = -np.inf
        assert int(accepted) == 0 and int(token) in range(V) and int(token) != 100
        if others == -20.0:
            continue
        tokens, q = tok.left(rest)
        slack = 2 * V * 2.0 ** -49 / np.exp(rest - 12.0).sum()
        through, at = np.cumsum(q), np.flatnonzero(tokens == int(token))
        assert len(at) == 1
        assert through[at[0]] - q[at[0]] - slack <= u < through[at[0]] + slack


# ---------------------------------------------------------------------------------------------------- as it is used

def test_captured_and_on_another_stream(qb):
    """One graph, replayed over new logits, numbers and parameters with eager calls between; every result the eager one's bits.  A second graph beside it."""
    say("captured")
    r = np.random.Generator(np.random.Philox(14))
    T, V = 6, 20001
    z = torch.empty(T, V, device="cuda")
    u, f = torch.empty(T, device="cuda"), params([FILTERS[12]] * T)
    starts, ids = dev([0, 4, 6], torch.int32), torch.empty(T, dtype=torch.int32, device="cuda")
    pair = {k: v[:2].clone() for k, v in f.items()}

    def fill(seed):
        r = np.random.Generator(np.random.Philox(seed))
        z.copy_(dev(logits_of(r, T, V), torch.float32))
        u.copy_(dev(r.random(T), torch.float32))
        ids.copy_(z.argmax(1).int())
        f["top_k"].fill_(10 * seed + 1)
    fill(1)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        qb.sample_tokens(z, u, **f)
        qb.verify_tokens(z, starts, ids, u, u, **pair)
    torch.cuda.synchronize()
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        a = qb.sample_tokens(z, u, **f)
    with torch.cuda.graph(g2):
        b = qb.verify_tokens(z, starts, ids, u, u, **pair)
    for seed in (2, 3, 4):
        fill(seed)
        want = (*qb.sample_tokens(z, u, **f), *qb.verify_tokens(z, starts, ids, u, u, **pair))
        for t in (*a, *b):
            t.fill_(-7)
        g1.replay()
        g2.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((*a, *b), want))


def test_calls_on_two_streams_at_once(qb):
    """Each with scratch of its own; the results are those of calls one after another."""
    say("two streams")
    r = np.random.Generator(np.random.Philox(19))
    T, V = 40, 30000
    z = [dev(logits_of(r, T, V), torch.float32) for _ in range(2)]
    u, f = dev(r.random(T), torch.float32), params([FILTERS[i % len(FILTERS)] for i in range(T)])
    starts, seqs = dev(np.arange(0, T + 1, 8), torch.int32), params([FILTERS[i] for i in (0, 5, 11, 8, 4)])
    ids = [x.argmax(1).int() for x in z]
    call = lambda i: (*qb.sample_tokens(z[i], u, **f), *qb.verify_tokens(z[i], starts, ids[i], u, u, **seqs))
    want = [call(0), call(1)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(call(i))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i in range(2) for g in got[i] for a, b in zip(g, want[i]))


def test_a_step_of_a_batch(qb):
    """Logits as a linear writes them, drafts, the cache's lengths: a step goes on from what verify_tokens says, without the host."""
    say("a step")
    V, K, seqs, gamma = 4096, 256, 3, 3
    gen = torch.Generator("cuda").manual_seed(3)
    w, s = qb.quantize_weights(torch.randn(V, K, generator=gen, device="cuda"))
    cache = qb.PagedKvCache(1, 1, 12, page_len=32, max_seqs=seqs)
    cache.lengths.copy_(dev([5, 31, 0], torch.int32))
    starts = dev([0, 4, 8, 12], torch.int32)
    hidden = (torch.randn(seqs * (gamma + 1), K, generator=gen, device="cuda") * 0.2).bfloat16()
    logits = qb.w8_linear(hidden, w, s, V)
    ids = logits.float().argmax(1).int()
    ids[5] = (ids[5] + 1) % V
    u = torch.rand(12, generator=gen, device="cuda")
    accepted, token, p = qb.verify_tokens(logits, starts, ids, u * 0, u, temperature=dev([0.0, 0.0, 1.0], torch.float32))
    cache.lengths.add_(accepted + 1)
    assert accepted.tolist()[:2] == [3, 1] and token.tolist()[:2] == [int(logits[3].float().argmax()), int(logits[5].float().argmax())]
    assert cache.lengths.tolist() == [9, 33, int(accepted[2]) + 1]


def test_refusals_of_the_binding(qb):
    say("refusals")
    z, u = torch.zeros(3, 100, device="cuda"), torch.zeros(3, device="cuda")
    ids, starts = torch.zeros(3, dtype=torch.int32, device="cuda"), dev([0, 3], torch.int32)
    assert qb.sample_tokens(z[:0], u[:0])[0].numel() == 0
    assert [t.tolist() for t in qb.verify_tokens(z[:0], dev([0, 0], torch.int32), ids[:0], u[:0], u[:0])] == [[0], [-1], []]
    qb.sample_tokens(z[:, :1].t().contiguous().t(), u)
    for bad, error in ((dict(u=u[:2]), ValueError), (dict(u=u.double()), TypeError), (dict(u=torch.zeros(6, device="cuda")[::2]), ValueError), (dict(logits=z.half()), TypeError), (dict(logits=z[0]), ValueError),
                       (dict(logits=z.t().contiguous().t()), ValueError), (dict(logits=z.cpu()), TypeError), (dict(top_k=u), TypeError), (dict(top_k=ids[:1]), ValueError), (dict(top_p=ids), TypeError),
                       (dict(temperature=1.0), TypeError), (dict(min_p=u[None]), ValueError), (dict(logits=z[:, :0]), ValueError), (dict(u=None), TypeError)):
        with pytest.raises(error):
            qb.sample_tokens(**(dict(logits=z, u=u) | bad))
    for bad, error in ((dict(row_start=starts.long()), TypeError), (dict(row_start=starts[:1]), ValueError), (dict(row_start=torch.zeros(1026, dtype=torch.int32, device="cuda")), ValueError),
                       (dict(draft_ids=ids.long()), TypeError), (dict(draft_ids=ids[:2]), ValueError), (dict(u_accept=u[:2]), ValueError), (dict(u_sample=None), TypeError),
                       (dict(temperature=u), ValueError)):
        with pytest.raises(error):
            qb.verify_tokens(**(dict(logits=z, row_start=starts, draft_ids=ids, u_accept=u, u_sample=u) | bad))
    with pytest.raises(qb.QuasarError):
        qb.sample_tokens(torch.zeros(1, (1 << 20) + 1, device="cuda"), u[:1])


class _Sub(torch.Tensor):
    pass


def test_calls_that_are_not_ordinary(qb):
    """What the native side leaves to the Python path has the same bits; what it takes is what the public functions give."""
    say("not ordinary")
    r = np.random.Generator(np.random.Philox(18))
    T, V = 4, 5000
    z, u = dev(logits_of(r, T, V), torch.float32), dev(r.random(T), torch.float32)
    f, pair = params([FILTERS[12]] * T), params([FILTERS[12]] * 2)
    starts, ids = dev([0, 3, 4], torch.int32), z.argmax(1).int()
    sample, verify = (z, u, *f.values()), (z, starts, ids, u, u, *pair.values())
    for native, args, public in ((qb._fast.sample_tokens, sample, qb.sample_tokens(z, u, **f)), (qb._fast.verify_tokens, verify, qb.verify_tokens(z, starts, ids, u, u, **pair))):
        assert all(torch.equal(a, b) for a, b in zip(native(*args), public))
        assert native(*args[:-1]) == -1 and native(*args, None) == -1
        for i in range(len(args)):
            assert native(*args[:i], args[i].cpu(), *args[i + 1:]) == -1 and native(*args[:i], "x", *args[i + 1:]) == -1
    sub = z.as_subclass(_Sub)
    assert qb._fast.sample_tokens(sub, *sample[1:]) == -1 and qb._fast.verify_tokens(sub, *verify[1:]) == -1
    assert all(torch.equal(a, b) for a, b in zip(qb.sample_tokens(sub, u, **f), qb.sample_tokens(z, u, **f)))
    assert all(torch.equal(a, b) for a, b in zip(qb.verify_tokens(sub, starts, ids, u, u, **pair), qb.verify_tokens(z, starts, ids, u, u, **pair)))
