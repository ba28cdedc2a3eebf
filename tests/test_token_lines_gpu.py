"""GPU parity of drawing tokens where logits are many times the temperature, so that a place on the line of buckets is far from 0.  Tolerances as derived in
test_tokens_gpu.py; weights are of a few values here, whose running masses do not meet a share of the whole."""
import numpy as np
import pytest
import torch

import test_tokens_gpu as base

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qb():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2603_01399_amd import binding
    return binding


NEAR = [dict(top_k=3), dict(top_k=100), dict(top_k=2500), dict(top_p=0.5), dict(top_p=0.9), dict(top_p=0.999), dict(min_p=0.1654), dict(min_p=1.95e-5), dict(top_k=100, top_p=0.8),
        dict(top_k=4000, top_p=0.7, min_p=1e-3), dict()]


def check(qb, z, filters, us=(0.0, 0.37, 0.8, 0.999, 1 - 2.0 ** -24)):
    """Every row with every one of the filters, at every one of the numbers."""
    T, V = z.shape
    rows = [f for _ in range(T) for f in filters for _ in us]
    many = z.repeat_interleave(len(filters) * len(us), 0)
    u = np.array(list(us) * (T * len(filters)), np.float32)
    token, p = qb.sample_tokens(many, base.dev(u, torch.float32), **base.params(rows))
    token, p, host = token.tolist(), p.tolist(), base.seen(z)
    for i, f in enumerate(rows):
        base.check_draw(host[i // (len(filters) * len(us))], u[i], token[i], p[i], V, **base.as_seen(f))


def test_ten_equal_ones_a_bucket_below_the_largest(qb):
    """exp(-1/4) each: of 1 + 7.788 the first six hold a half."""
    base.say("ten equal ones")
    z = torch.full((1, 3000), 2.0 ** 21 - 40, device="cuda")
    z[0, 700], z[0, 1000:2000:100] = 2.0 ** 21 + 0.25, 2.0 ** 21
    check(qb, z, [dict(top_p=0.5), dict(top_k=4), dict(min_p=0.5), dict(top_k=6, top_p=0.6)])
    u = torch.ones(1, device="cuda")
    assert int(qb.sample_tokens(z, u, top_p=u * 0.5)[0]) == 1400 and int(qb.sample_tokens(z, u, top_k=u.int() * 4)[0]) == 1200


@pytest.mark.parametrize("most,t", [(2097152.25, 1.0), (200.000015, 1e-4), (20.0000019, 1e-5), (413.573486, 3.93e-5), (30.7390366, 8.96e-7), (3.9999998, 1.4901161e-8), (1e9, 100.0), (-2097152.25, 1.0),
                                    (-20.0000019, 1e-5), (-3.9999998, 1.4901161e-8), (1e30, 1e22), (7.5, 1.0)])
def test_logits_of_many_temperatures(qb, most, t):
    """Logits a few temperatures below the largest, on what grid fp32 has there: within a part, in several, in a row that is not aligned."""
    base.say("many temperatures", most, t)
    r = np.random.Generator(np.random.Philox(3))
    for V, off in ((1000, 0), (20011, 1)):
        z = torch.full((3, V + off), float(most), device="cuda")[:, off:]
        away = np.stack([r.exponential(2.0, V), r.exponential(6.0, V), r.random(V) * 40])
        away[0, V // 2:] += 3                                     # (a part's largest is not the row's)
        z.copy_(base.dev(np.minimum(np.float64(np.float32(most)) - away * t, most), torch.float32))
        check(qb, z, [f | dict(temperature=t) for f in NEAR], us=(0.0, 0.37, 0.999))


def test_min_p_alone_far_from_zero(qb):
    """Logits, temperatures and bounds of every size: what min_p keeps is counted, in whatever bucket it lies."""
    base.say("min_p far from zero")
    r = np.random.Generator(np.random.Philox(4))
    for _ in range(60):
        most, t, m = np.float32(16 * 64 ** r.random()), float(np.float32(10 ** r.uniform(-8, -2))), float(np.float32(10 ** r.uniform(-6, -0.3)))
        V = 2000
        steps = np.floor(r.exponential(2.0 + 8 * r.random(), V))
        step = max(float(np.spacing(most)), t / 3)
        z = base.dev(np.float64(most) - steps * step, torch.float32)[None]
        check(qb, z, [dict(min_p=m, temperature=t)], us=(0.0, 0.5, 0.9, 0.999))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_zeros_that_are_the_largest(qb, dtype):
    """Of either sign, alone or with others below them: both count as the same number, also where all have the sign."""
    base.say("zeros", dtype)
    r = np.random.Generator(np.random.Philox(5))
    for V in (100, 5000, 20011):
        z = torch.full((6, V), -0.0, dtype=dtype, device="cuda")
        z[1] = 0.0
        z[2, 1::2] = 0.0
        z[3] = base.dev(-np.abs(r.standard_normal(V)) * 0.05, torch.float32).to(dtype)
        z[3, r.permutation(V)[:40]] = -0.0
        z[4] = base.dev(-np.abs(r.standard_normal(V)) - 0.2, torch.float32).to(dtype)
        z[4, r.permutation(V)[:40]] = -0.0
        z[5, V // 2:] = -1.0
        assert bool((torch.signbit(z[0])).all()) and bool(torch.signbit(z[3]).all())
        us = (0.0, 0.4, 0.999)
        check(qb, z, [dict(top_k=5), dict(top_k=30), dict(top_k=V // 2), dict(min_p=1.0), dict(min_p=0.97), dict(top_k=7, top_p=0.5), dict(top_k=3000, top_p=0.3), dict(temperature=0.0), dict()], us)
        # (a half of V equal ones is the first V / 2 of them, or one more)
        u = torch.full((6,), 1.0, device="cuda")
        token, _ = qb.sample_tokens(z, u, top_k=u.int() * 5)
        assert token.tolist()[:3] == [4, 4, 4]
        token, _ = qb.sample_tokens(z[:3].contiguous(), u[:3], top_p=u[:3] * 0.5)
        assert token.tolist() == [-(-V // 2) - 1] * 3


# One token of weight 1, n equal ones of about 2^-30, whose units are no whole numbers; the last one left (a number of 1 draws it) says where top-p cuts.  Running masses and the
# share of the whole are off by at most V 2^-45 + 2^-44 of the whole each (test_tokens_gpu.py), which is less than the weight of a token, or of two.
@pytest.mark.parametrize("V,k,steps", [(1900, 1899, 14), (1900, 1899, 25), (60000, 50000, 300), (60000, 50000, 9), (2049, 2048, 20)])
def test_where_top_p_cuts_among_small_equal_weights(qb, V, k, steps):
    base.say("small equal weights", V, k, steps)
    T = 400
    small = -20.7944 - np.arange(T) * 2.0 ** -17
    z = torch.full((T, V), float("-inf"), device="cuda")
    z[:, 1:] = base.dev(small, torch.float32)[:, None]
    z[:, 0] = 0.0
    p = 1 - steps * 2.0 ** -24
    ones = torch.ones(T, device="cuda")
    token, _ = qb.sample_tokens(z, ones, top_k=ones.int() * k, top_p=base.dev([p] * T, torch.float32))
    w = np.exp(base.seen(z[:, 1]))
    whole, n = 1 + (k - 1) * w, token.cpu().numpy()               # (tokens behind the first one that are left)
    tol = base.tol_of(V) * whole
    assert (1 + (n - 1) * w < p * whole + 2 * tol).all() and (1 + n * w >= p * whole - 2 * tol).all()
    assert (n > 0).all() and (n < k - 1).all()


@pytest.mark.parametrize("most,t", [(2097152.25, 1.0), (20.0000019, 1e-5), (-0.0, 0.3)])
def test_drafts_far_from_zero(qb, most, t):
    """Candidates that are kept, cut, or nobody's, of rows as above."""
    base.say("drafts far from zero", most, t)
    r = np.random.Generator(np.random.Philox(6))
    V, news = 9001, [4, 1, 7, 3, 5, 2, 6]
    starts = np.concatenate([[0], np.cumsum(news)])
    T = int(starts[-1])
    away = r.exponential(4.0, (T, V)) * t
    away[:, 77] = 0.0
    z = base.dev(np.float64(np.float32(most)) - away, torch.float32)
    z[:, 77] = most
    seqs = [NEAR[i] | dict(temperature=t) for i in (1, 3, 4, 6, 8, 9, 10)]
    drafts = np.where(r.random(T) < 0.6, 77, np.argsort(away, 1)[:, 3])
    ua, us = r.random(T).astype(np.float32) * np.float32(1e-3), r.random(T).astype(np.float32)
    some = base.check_verify(qb, z, starts, drafts, ua, us, [base.as_seen(f) for f in seqs], base.params(seqs))
    assert max(some) > 0
