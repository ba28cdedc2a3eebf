"""GPU parity of the append with other rotary positions (layouts, part of the head, scaled frequencies, with and without norms) through the binding
against the fp64 oracle: queries, keys and values, and every other byte of the pool as it was."""
import numpy as np
import pytest
import torch

from oracle import quasar_attention_ref as at
from oracle import quasar_paged_ref as pg
from oracle import quasar_ref as ref
from oracle import quasar_window_ref as win
from paged_util import Batch, rnd_bits
from gpu_util import bf16_to_dev, bf16_to_host, i32_to_dev

pytestmark = pytest.mark.gpu
D = 128
f64 = ref.bf16_bits_to_f64


@pytest.fixture(scope="module")
def qb():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2603_01399_amd import binding
    return binding


def say(*a):
    print(*a, flush=True)


SHAPES = [("bf16", 64, 32, 8, [0], [1]), ("bf16", 32, 4, 2, [31, 0, 64], [2, 0, 3]), ("e4m3", 64, 32, 8, [1000, 5], [1, 1]), ("bf16", 64, 6, 2, [0, 100, 31], [70, 133, 2]),
          ("e4m3", 128, 8, 8, [0, 17, 95], [200, 40, 161]), ("bf16", 64, 5, 5, [300, 3], [4, 300])]
FORMS = [("half", 128), ("interleaved", 128), ("half", 96), ("interleaved", 48), ("half", 16), ("interleaved", 16), ("half", 64), ("interleaved", 112)]


def partner(n, layout, dims):
    """|n| of the other element of every pair, 0 where none is."""
    other = np.zeros_like(n)
    h = dims // 2
    if layout == "half":
        other[..., :h], other[..., h:dims] = n[..., h:dims], n[..., :h]
    else:
        other[..., 0:dims:2], other[..., 1:dims:2] = n[..., 1:dims:2], n[..., 0:dims:2]
    return other


def want_and_slack(x_bits, gamma, pos, freq, layout, magnitude):
    """Oracle bits [rows, heads, 128] and how far a value may be off.

    Without a norm the input is exact: cosines and sines are off by 2^-24 of 1 each from their own rounding, 2^-24 from the reduced angle's (at most pi, so
    pi 2^-24) and 2^-22 from the functions, so by less than 2^-20; a product and a sum add 2^-23: together below 2^-19 magnitude (|a| + |b|).  The rounding to
    bf16 may go the other way: one step, 2^-7 of the result.  With a norm: its two roundings may go either way, 2^-6 (|a| + |b|) magnitude more
    (test_paged_gpu.test_prepare)."""
    x = f64(x_bits)
    dims = 2 * len(freq)
    if gamma is not None:
        x = f64(at.head_norm_rope(x_bits, gamma, 1e-6, np.zeros(x.shape[0]), 1e6))       # (position 0 is not rotated)
    y = win.rotate(x, pos, freq, layout, magnitude)
    size = np.abs(x) + partner(np.abs(x), layout, dims)
    mag = np.where(np.arange(D) < dims, magnitude, 1.0)
    slack = (2.0 ** -19 + (2.0 ** -6 if gamma is not None else 0.0)) * mag * size + 2.0 ** -7 * np.abs(y) + 1e-37
    if gamma is None:
        slack[..., dims:] = 0.0
    return ref.f64_to_bf16_bits(y), slack


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("kv,page,hq,hk,lengths,news", SHAPES)
@pytest.mark.parametrize("layout,dims", FORMS)
def test_rotary_append(qb, layout, dims, kv, page, hq, hk, lengths, news, norm):
    say("rotary", layout, dims, kv, page, hq, hk, lengths, news, norm)
    b = Batch(qb, kv, page, hq, hk, lengths, news, layers=2, layer=1, seed=31 + hq)
    T, heads = b.rows, hq + 2 * hk
    qkv = rnd_bits((T, heads, D), 41, 2.0)
    gq, gk = (ref.f32_to_bf16_bits((1.0 + 0.2 * np.random.Generator(np.random.Philox(s)).standard_normal(D)).astype(np.float32)) for s in (5, 6))
    if not norm:
        gq = gk = None
    rope = qb.Rope(dims, 1e4, layout=layout, scaling="by_parts", factor=4.0, trained_len=256) if dims == 64 else qb.Rope(dims, 1e5, layout=layout)
    freq = rope.inv_freq.cpu().numpy()
    before = b.cache.pool.view(torch.uint8).clone()
    wide = torch.zeros((T, heads * D + 24), dtype=torch.bfloat16, device="cuda")
    wide[:, 8:8 + heads * D] = bf16_to_dev(qkv.reshape(T, -1))
    q_out = torch.full((T + 2, hq * D + 8), 3.0, dtype=torch.bfloat16, device="cuda")
    dev = lambda g: None if g is None else bf16_to_dev(g)
    qb.paged_prepare(wide[:, 8:8 + heads * D], hq, b.cache, 1, b.row_start, dev(gq), dev(gk), eps=1e-6, q_out=q_out[1:T + 1, :hq * D], rope=rope)
    torch.cuda.synchronize()
    assert (q_out[0] == 3).all() and (q_out[T + 1] == 3).all() and (q_out[:, hq * D:] == 3).all()
    pos = np.concatenate([np.arange(l, l + n) for l, n in zip(lengths, news)])
    want_q, q_slack = want_and_slack(qkv[:, :hq], gq, pos, freq, layout, rope.magnitude)
    want_k, k_slack = want_and_slack(qkv[:, hq:hq + hk], gk, pos, freq, layout, rope.magnitude)
    got_q = bf16_to_host(q_out[1:T + 1, :hq * D]).reshape(T, hq, D)
    assert (np.abs(f64(got_q) - f64(want_q)) <= q_slack).all() and np.mean(got_q != want_q) < 0.02
    row = 0
    for s, (l, n) in enumerate(zip(lengths, news)):
        got_k, got_v = b.read(s, l + n, 0)[l:], b.read(s, l + n, 1)[l:]
        k, v, near = want_k[row:row + n], qkv[row:row + n, hq + hk:], k_slack[row:row + n]
        row += n
        if kv == "bf16":
            assert np.array_equal(got_v, v) and (np.abs(f64(got_k) - f64(k)) <= near).all()
            continue
        ks, vs = b.scales[0][1][:, None], b.scales[1][1][:, None]
        assert np.array_equal(got_v, pg.f64_to_e4m3((f64(v).astype(np.float32) / vs).astype(np.float32)))
        # a code is off by half a step, 2^-4 of the value or 2^-10 scales, and saturates at 448
        k = np.clip(f64(k), -448 * ks, 448 * ks)
        assert (np.abs(pg.e4m3_to_f64(got_k) * ks - k) <= near + 2.0 ** -4 * (np.abs(k) + near) + 2.0 ** -10 * ks).all()
    mine = torch.zeros_like(before, dtype=torch.bool)
    flat = mine.view(2, b.cache.n_pages, hk, page // 32, 2, 4096, 2 if kv == "bf16" else 1)
    for half, places in enumerate(pg.block_places(kv)):
        for s, (l, n) in enumerate(zip(lengths, news)):
            j = np.arange(l, l + n)
            for h in range(hk):
                ix = [torch.from_numpy(np.ascontiguousarray(a)).cuda().long() for a in (b.table[s, j // page][:, None], (j % page // 32)[:, None], places[j % 32])]
                flat[1][ix[0], h, ix[1], half, ix[2]] = True
    assert torch.equal(b.cache.pool.view(torch.uint8)[~mine], before[~mine])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("n", [1, 200])
def test_far_positions(qb, layout, n):
    """Positions of millions, where an angle in fp32 would be off by a radian."""
    say("far", layout, n)
    b = Batch(qb, "bf16", 1024, 2, 1, [0], [n], seed=3, more_columns=0)
    far = 3_000_000 if n == 1 else 9_999_999
    b.cache.lengths.fill_(far)                              # (beyond the table: nothing is stored, queries are)
    qkv = rnd_bits((n, 4, D), 43)
    rope = qb.Rope(128, 1e6, layout=layout, scaling="ntk", factor=3.0)
    got = bf16_to_host(qb.paged_prepare(bf16_to_dev(qkv.reshape(n, -1)), 2, b.cache, 0, b.row_start, None, None, rope=rope)).reshape(n, 2, D)
    want, slack = want_and_slack(qkv[:, :2], None, far + np.arange(n), rope.inv_freq.cpu().numpy(), layout, 1.0)
    assert (np.abs(f64(got) - f64(want)) <= slack).all() and np.mean(got != want) < 0.02


@pytest.mark.parametrize("n", [3, 300])
def test_near_the_append_by_theta(qb, n):
    """The half layout over the whole head with norms is the older form, but for a few roundings; queries in place of the input's give the same bits; what is not
    finite in the elements that are not rotated stays where it is."""
    say("older form", n)
    b = Batch(qb, "bf16", 64, 4, 2, [77], [n], seed=4)
    x = bf16_to_dev(rnd_bits((n, 8 * D), 44))
    g = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    old = qb.paged_prepare(x, 4, b.cache, 0, b.row_start, g, g, rope_theta=1e6)
    rope = qb.Rope(128, 1e6)
    new = qb.paged_prepare(x, 4, b.cache, 0, b.row_start, g, g, rope=rope)
    assert (old != new).float().mean() < 1e-3 and (old - new).abs().max() <= 2.0 ** -7 * old.abs().max()
    own = x.clone()
    assert torch.equal(qb.paged_prepare(own, 4, b.cache, 0, b.row_start, g, g, rope=rope, q_out=own[:, :4 * D])[:, :4 * D], new)
    part = qb.Rope(32, 1e4, layout="interleaved")
    x[0, 40], x[0, 41] = float("inf"), float("nan")
    got = qb.paged_prepare(x, 4, b.cache, 0, b.row_start, None, None, rope=part)
    assert torch.equal(got[0, :D].isfinite(), x[0, :D].isfinite()) and got[0, 40] == float("inf") and torch.equal(got[:, 32:40], x[:, 32:40])


def test_refusals_of_the_binding(qb):
    say("refusals")
    b = Batch(qb, "bf16", 64, 4, 2, [100], [2], seed=41)
    x = torch.zeros(2, 8 * D, dtype=torch.bfloat16, device="cuda")
    g = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    rope = qb.Rope(64)
    call = lambda *a, **k: qb.paged_prepare(x, 4, b.cache, 0, b.row_start, *a, **k)
    call(None, None, rope=rope)
    for a in ((g, None), (None, g)):
        with pytest.raises(ValueError):
            call(*a, rope=rope)
    with pytest.raises(TypeError):
        call(None, None)
    with pytest.raises(TypeError):
        call(None, None, rope=qb.Rope(64, device="cpu"))
    with pytest.raises(ValueError):
        call(g[:64], g[:64], rope=rope)
    rope.inv_freq = rope.inv_freq[:16]
    with pytest.raises(ValueError):
        call(g, g, rope=rope)
    with pytest.raises(qb.QuasarError):
        call(g, g, eps=-1.0, rope=qb.Rope(64))
