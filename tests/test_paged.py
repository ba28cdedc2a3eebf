"""Paged cache without a GPU: its oracle, the bounds that the kernels put on what they read from the books (the library's own
functions, csrc/books.hpp), how a step's blocks are shared, and the calls that are refused before anything is launched."""
import ctypes
import subprocess
from pathlib import Path

import numpy as np
import pytest
import torch

from oracle import quasar_attention_ref as at
from oracle import quasar_paged_ref as pg
from oracle import quasar_ref as ref

HERE = Path(__file__).resolve().parent
INT_MIN, INT_MAX = -2 ** 31, 2 ** 31 - 1


@pytest.fixture(scope="module")
def model(tmp_path_factory):
    out = tmp_path_factory.mktemp("books") / "libbooks_model.so"
    subprocess.run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fsanitize=undefined", "-fno-sanitize-recover", "-o", str(out),
                    str(HERE / "books_model.cpp")], check=True)
    return ctypes.CDLL(str(out))


@pytest.fixture(scope="module")
def lib():
    from paper_2603_01399_amd import binding
    return binding.lib()


# ------------------------------------------------------------------------------------------------------------ oracle

@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_places_are_a_permutation(kv):
    for places in pg.block_places(kv):
        assert sorted(places.reshape(-1)) == list(range(32 * 128))


def test_e4m3_against_torch():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).to(torch.float64).numpy()
    assert np.array_equal(pg.e4m3_to_f64(codes), want, equal_nan=True)
    r = np.random.Generator(np.random.Philox(3))
    x = np.concatenate([r.standard_normal(20000) * np.exp2(r.integers(-12, 9, 20000)), pg.e4m3_to_f64(codes[:0x7F]), [448, -448, 464, 1e9, 0.0]])
    mid = (pg.e4m3_to_f64(codes[:0x7E]) + pg.e4m3_to_f64(codes[1:0x7F])) / 2                # ties
    x = np.concatenate([x, mid, -mid]).astype(np.float32)
    want = torch.from_numpy(x).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(pg.f64_to_e4m3(x), want)


def test_attention_oracle_is_the_verification_oracle():
    r = np.random.Generator(np.random.Philox(4))
    q, k, v = (ref.f32_to_bf16_bits(r.standard_normal(s).astype(np.float32)) for s in ((3, 4, 128), (11, 2, 128), (11, 2, 128)))
    out, size = pg.attention(*(ref.bf16_bits_to_f64(t) for t in (q, k, v)), 8)
    assert np.array_equal(ref.f64_to_bf16_bits(out), at.verify_attention(q, k, v)) and (np.abs(out) <= size + 1e-12).all()


def test_books_oracle_by_hand():
    b = pg.Books([1, 2, 0, 0, 0], [40, 40, 0], [[1, -1], [1, -1], [-1, -1]], 64)
    assert b.reserve([1, 1, 65]) == [1, 1, 1]                 # the first writer copies page 1, the second is its last holder
    assert b.copies == [(1, 2, 2)] and b.table == [[2, -1], [1, -1], [3, 4]] and b.refs == [1, 1, 1, 1, 1]
    b.fork([0, 0, 5], [64, 10, 9])
    assert b.table == [[2, -1], [2, -1], [-1, -1]] and b.lengths == [40, 10, 0] and b.refs == [1, 0, 2, 0, 0]
    assert b.compact() == [0, 1, 1, 3, 4] and b.table == [[1, -1], [1, -1], [-1, -1]] and b.refs == [1, 2, 0, 0, 0]
    assert b.reserve([0, 25, 200]) == [1, 1, 0] and b.copies == [(1, 2, 1)]


# ------------------------------------------------------------------------------------- bounds on what the books say

ODD = [INT_MIN, -5, -1, 0, 1, 7, 8, 9, 31, 32, 33, 1 << 24, (1 << 24) + 1, INT_MAX]


def test_spans_stay_within_the_rows(model):
    out = (ctypes.c_int * 3)()
    for T in (1, 8, 1 << 24):
        for begin in ODD:
            for end in ODD:
                for length in ODD:
                    model.span_model(begin, end, length, T, out)
                    row0, n, kept = out
                    assert 0 <= row0 and n >= 0 and row0 + n <= T and 0 <= kept <= 1 << 24
                    if 0 <= begin <= end <= T and 0 <= length <= 1 << 24:
                        assert (row0, n, kept) == (begin, end - begin, length)
                    else:
                        assert n == 0


def test_blocks_and_pages_stay_within_table_and_pool(model):
    for columns, shift in ((1, 0), (1, 5), (7, 1), (1 << 19, 0), (1 << 14, 5)):
        for total in (0, 1, 31, 32, 33, 1000, 1 << 24, (1 << 24) + 32):
            nb = model.blocks_model(total, columns, shift)
            assert 0 <= nb <= columns << shift and nb == min(-(-total // 32), columns << shift)
            if nb:
                assert (nb - 1) >> shift < columns
    for n_pages in (1, 8, 1 << 20):
        for page in ODD:
            assert bool(model.page_model(page, n_pages)) == (0 <= page < n_pages)


@pytest.mark.parametrize("workers", [1, 2, 5, 32, 256])
def test_every_block_is_taken_once_and_every_part_is_joined(model, workers):
    """Sequences of random lengths as one line: pieces cover it; the parts of a shared sequence lie in slots of their own, and the
    merge looks for them there."""
    r = np.random.Generator(np.random.Philox(workers))
    out = (ctypes.c_int * 3)()
    for trial in range(60):
        blocks = r.integers(0, [2, 9, 300][trial % 3], r.integers(1, 40)) * (r.random() < 0.9)
        prefix = np.concatenate([[0], np.cumsum(blocks)]).astype(int)
        total, at_, slots = int(prefix[-1]), 0, {}
        for w in range(workers):
            model.share_model(total, workers, 4, w, out)
            share, begin, end = out
            assert begin == at_ and begin <= end <= total
            at_ = end
            goes_on = 0
            for s in range(len(blocks)):
                lo, hi = max(begin, prefix[s]), min(end, prefix[s + 1])
                if lo >= hi:
                    continue
                whole = (lo, hi) == (prefix[s], prefix[s + 1])
                if not whole:
                    slot = model.slot_model(total, workers, 4, w, int(prefix[s]))
                    assert 0 <= slot < 2 * workers and slot not in slots
                    slots[slot] = (s, lo, hi)
                    if lo == prefix[s]:
                        goes_on += 1
                        last = (int(prefix[s + 1]) - 1) // share
                        assert last < workers
                        first, here = slot, w
                        parts = [model.part_slot_model(here, first, k) for k in range(last - here + 1)]
                        slots[("parts", s)] = parts
            assert goes_on <= 1                               # what a worker has one record for
        assert at_ == total
        for key in [k for k in slots if isinstance(k, tuple)]:
            s = key[1]
            found = [slots[p] for p in slots[key]]
            assert all(f[0] == s for f in found) and found[0][1] == prefix[s] and found[-1][2] == prefix[s + 1]
            assert all(a[2] == b[1] for a, b in zip(found, found[1:]))
        assert {v[0] for k, v in slots.items() if not isinstance(k, tuple)} == {k[1] for k in slots if isinstance(k, tuple)}


# ---------------------------------------------------------------------------------------------------------- refusals

def test_sizes(lib):
    assert lib.quasar_paged_cache_bytes(2, 8, 10, 64, 1) == 2 * 10 * 8 * 64 * 128 * 2 * 2
    assert lib.quasar_paged_cache_bytes(2, 8, 10, 64, 2) == 2 * 10 * 8 * 64 * 128 * 2
    for bad in ((0, 8, 10, 64, 1), (1, 0, 10, 64, 1), (1, 8, 0, 64, 1), (1, 8, 10, 48, 1), (1, 8, 10, 16, 1), (1, 8, 10, 2048, 1), (1, 8, 10, 64, 0),
                (1, 8, 10, 64, 3), (1, 8, (1 << 20) + 1, 64, 1)):
        assert lib.quasar_paged_cache_bytes(*bad) == 0, bad
    assert lib.quasar_paged_attention_workspace_bytes(1, 32, 8) > 0 and lib.quasar_paged_attention_workspace_bytes(32, 32, 1) > 0
    for bad in ((0, 32, 8), (33, 32, 8), (1, 30, 8), (32, 64, 1), (1, 8, 0), (1, 8192, 8)):
        assert lib.quasar_paged_attention_workspace_bytes(*bad) == 0, bad
    assert lib.quasar_pages_workspace_bytes(4, 100) > 0
    for bad in ((0, 100), (1025, 100), (4, 0), (4, (1 << 20) + 1)):
        assert lib.quasar_pages_workspace_bytes(*bad) == 0


NULL, SHAPE, ALIGN, WORKSPACE, DTYPE = 1, 2, 3, 4, 5
A, ODD_ADDRESS = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1002)      # never dereferenced on the host
PAGED = dict(pages=A, n_pages=10, page_len=64, kv=1, k_scale=None, v_scale=None, table=A, table_ld=4, max_pages=4, lengths=A)
BAD_PAGED = [(dict(pages=None), NULL), (dict(table=None), NULL), (dict(lengths=None), NULL), (dict(row_start=None), NULL), (dict(kv=0), DTYPE),
             (dict(kv=7), DTYPE), (dict(k_scale=A), DTYPE), (dict(n_pages=0), SHAPE), (dict(n_pages=(1 << 20) + 1), SHAPE), (dict(page_len=40), SHAPE),
             (dict(max_pages=0), SHAPE), (dict(table_ld=3), SHAPE), (dict(max_pages=1 << 19, table_ld=1 << 19), SHAPE), (dict(T=0), SHAPE),
             (dict(T=(1 << 24) + 1), SHAPE), (dict(hq=9), SHAPE), (dict(hk=0), SHAPE), (dict(n_seqs=0), SHAPE), (dict(n_seqs=1025), SHAPE),
             (dict(pages=ODD_ADDRESS), ALIGN), (dict(table=ODD_ADDRESS), ALIGN), (dict(row_start=ODD_ADDRESS), ALIGN)]


def paged_args(c):
    return [c[n] for n in PAGED]


@pytest.mark.parametrize("change,status", BAD_PAGED + [(dict(x=None), NULL), (dict(q=None), NULL), (dict(g=None), NULL), (dict(ld=32 * 128), SHAPE), (dict(ld=6148), SHAPE),
                                                       (dict(ldq=4090), SHAPE), (dict(eps=-1.0), SHAPE), (dict(theta=1.0), SHAPE), (dict(x=ODD_ADDRESS), ALIGN), (dict(g=ODD_ADDRESS), ALIGN)])
def test_prepare_refuses(lib, change, status):
    c = dict(PAGED, x=A, T=5, ld=48 * 128, hq=32, hk=8, row_start=A, n_seqs=2, g=A, eps=1e-6, theta=1e6, q=A, ldq=4096, **{}) | change
    assert lib.quasar_paged_prepare(c["x"], c["T"], c["ld"], c["hq"], c["hk"], c["row_start"], c["n_seqs"], c["g"], c["g"], c["eps"], c["theta"], c["q"],
                                    c["ldq"], *paged_args(c), None) == status


@pytest.mark.parametrize("change,status", BAD_PAGED + [(dict(x=None), NULL), (dict(out=None), NULL), (dict(ldq=4088), SHAPE), (dict(ldq=4100), SHAPE), (dict(ldo=4098), SHAPE),
                                                       (dict(new=0), SHAPE), (dict(new=33), SHAPE), (dict(hq=512, hk=8, new=32, ldq=65536, ldo=65536), SHAPE),
                                                       (dict(x=ODD_ADDRESS), ALIGN), (dict(out=ODD_ADDRESS), ALIGN), (dict(ws=None), WORKSPACE), (dict(room=1000), WORKSPACE),
                                                       (dict(ws=ODD_ADDRESS), ALIGN)])
def test_paged_attention_refuses(lib, change, status):
    c = dict(PAGED, x=A, T=5, ldq=4096, hq=32, hk=8, row_start=A, n_seqs=2, new=4, out=A, ldo=4096, ws=A, room=1 << 30) | change
    assert lib.quasar_paged_attention(c["x"], c["T"], c["ldq"], c["hq"], c["hk"], c["row_start"], c["n_seqs"], c["new"], *paged_args(c), c["out"], c["ldo"],
                                      c["ws"], c["room"], None) == status


@pytest.mark.parametrize("change,status", BAD_PAGED + [(dict(x=None), NULL), (dict(out=None), NULL), (dict(ldq=4088), SHAPE), (dict(ldo=4098), SHAPE),
                                                       (dict(T=1 << 24, hq=64), SHAPE), (dict(x=ODD_ADDRESS), ALIGN), (dict(out=ODD_ADDRESS), ALIGN), (dict(ws=ODD_ADDRESS), ALIGN)])
def test_prompt_attention_refuses(lib, change, status):
    c = dict(PAGED, x=A, T=5, ldq=8192, hq=32, hk=8, row_start=A, n_seqs=2, out=A, ldo=8192, ws=None) | change
    if status == SHAPE and "ldq" in change:
        c["hq"] = 64
    assert lib.quasar_prompt_attention(c["x"], c["T"], c["ldq"], c["hq"], c["hk"], c["row_start"], c["n_seqs"], *paged_args(c), c["out"], c["ldo"], c["ws"], 1 << 30, None) == status


BOOKS = dict(table=A, table_ld=4, n_seqs=2, max_pages=4, lengths=A, other=A, refs=A, n_pages=10, page_len=64, out=A, pool=A, layers=2, hk=8, kv=1, ws=A, room=1 << 30)
BAD_BOOKS = [(dict(table=None), NULL), (dict(refs=None), NULL), (dict(table_ld=3), SHAPE), (dict(n_seqs=0), SHAPE), (dict(n_seqs=1025), SHAPE),
             (dict(max_pages=0), SHAPE), (dict(n_pages=0), SHAPE), (dict(page_len=0), SHAPE), (dict(page_len=96), SHAPE), (dict(table=ODD_ADDRESS), ALIGN), (dict(refs=ODD_ADDRESS), ALIGN)]
BAD_POOL = [(dict(pool=None), NULL), (dict(kv=0), DTYPE), (dict(layers=0), SHAPE), (dict(hk=0), SHAPE), (dict(pool=ODD_ADDRESS), ALIGN), (dict(ws=None), WORKSPACE),
            (dict(room=100), WORKSPACE), (dict(ws=ODD_ADDRESS), ALIGN), (dict(out=None), NULL), (dict(out=ODD_ADDRESS), ALIGN)]


@pytest.mark.parametrize("change,status", BAD_BOOKS + BAD_POOL + [(dict(lengths=None), NULL), (dict(other=None), NULL), (dict(other=ODD_ADDRESS), ALIGN)])
def test_reserve_refuses(lib, change, status):
    c = BOOKS | change
    assert lib.quasar_pages_reserve(c["table"], c["table_ld"], c["n_seqs"], c["max_pages"], c["lengths"], c["other"], c["refs"], c["n_pages"], c["page_len"], c["out"],
                                    c["pool"], c["layers"], c["hk"], c["kv"], c["ws"], c["room"], None) == status


@pytest.mark.parametrize("change,status", BAD_BOOKS + [(dict(lengths=None), NULL), (dict(other=None), NULL), (dict(other=ODD_ADDRESS), ALIGN), (dict(lengths=ODD_ADDRESS), ALIGN)])
def test_fork_refuses(lib, change, status):
    c = BOOKS | change
    assert lib.quasar_pages_fork(c["table"], c["table_ld"], c["n_seqs"], c["max_pages"], c["lengths"], c["other"], None, c["refs"], c["n_pages"], c["page_len"], None) == status


@pytest.mark.parametrize("change,status", BAD_BOOKS + BAD_POOL)
def test_compact_refuses(lib, change, status):
    c = BOOKS | change
    assert lib.quasar_pages_compact(c["table"], c["table_ld"], c["n_seqs"], c["max_pages"], c["refs"], c["n_pages"], c["page_len"], c["out"], c["pool"], c["layers"],
                                    c["hk"], c["kv"], c["ws"], c["room"], None) == status


def test_binding_refuses_host_tensors_and_odd_shapes():
    from paper_2603_01399_amd import binding as qb
    with pytest.raises(TypeError):
        qb.PagedKvCache(1, 8, 4, dtype=torch.float16)
    for bad in (dict(page_len=48), dict(max_seqs=0), dict(max_seqs=1025), dict(max_pages=0)):
        with pytest.raises(ValueError):
            qb.PagedKvCache(1, 8, 4, **bad)
    with pytest.raises(TypeError):
        qb.PagedKvCache(1, 8, 4, pool=torch.empty((1, 4, 8, 2, 2, 4096), dtype=torch.bfloat16))


def test_a_cache_holds_its_buffers_and_knows_them():
    """The handle keeps the tensors that calls go to, and says when one of them has other memory; the cache's own names stay (host tensors:
    nothing is launched)."""
    from paper_2603_01399_amd import binding as qb
    pool, books, scale = torch.zeros(4, 8), torch.zeros(12, dtype=torch.int32), torch.ones(2)
    views = [books[:4], books[4:6], books[6:].view(2, 3)]
    handle = qb._fast.paged_cache(1, 1, 4, 32, 2, 3, 1, 128, 64, pool, books, *views, scale, None)
    intact = lambda: qb._fast.paged_cache_as_made(handle)
    assert intact()
    pool[1], books[5] = 3.0, 7                            # (writing into them is what they are for)
    assert intact()
    for t in (pool, books, *views, scale):
        was = t.data
        t.data = t.data.clone()
        assert not intact()
        t.data = was
        assert intact()
        t.data = was[:1]
        assert not intact()
        t.data = was
    at_ = pool.data_ptr()
    del pool, t, was
    fresh = [torch.zeros(4, 8) for _ in range(64)]        # (memory that had been freed would come again)
    assert intact() and all(f.data_ptr() != at_ for f in fresh)
    for bad in ((1, 1, 4, 32, 2, 3, 1, 128, 64, 17, books, *views, None, None), (1,) * 9):
        with pytest.raises(TypeError):
            qb._fast.paged_cache(*bad)
    c = qb.PagedKvCache.__new__(qb.PagedKvCache)
    c.pool, c._handle = books, handle
    object.__setattr__(c, "_own", frozenset(("pool", "_handle", "_own")))
    for name in ("pool", "_handle", "_own"):
        with pytest.raises(AttributeError):
            delattr(c, name)
        with pytest.raises(AttributeError):
            setattr(c, name, 0)
    c.pool += 0
    c.note = 1
    c.note = 2
    del c.note


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("length,n", [(30000, 4), (100003, 1), (3000, 40), (0, 2100)])
def test_a_block_more_or_less_shows(kv, length, n):
    """The values of paged_marks with a mistake in the oracle: a block left out, or taken twice, wherever it lies, is beyond the tolerance that
    the kernels are held to, for every row that sees it whole."""
    from paged_marks import attention_and_bound, block_values
    r = np.random.Generator(np.random.Philox(900 + n))
    total = length + n
    q, k = r.standard_normal((n, 1, 128)) * 0.4, r.standard_normal((total, 1, 128))
    v = block_values(total)
    want, tol = attention_and_bound(q, k, v[:, None], length, kv)
    s = q[:, 0] @ k[:, 0].T / np.sqrt(128)
    s[np.arange(total)[None, :] > length + np.arange(n)[:, None]] = -np.inf
    w = np.exp(s - s.max(axis=1, keepdims=True))
    for b in np.unique(np.r_[0, 1, 2, 3, total // 64, r.integers(0, total // 32, 40), total // 32 - 1]):
        rows = length + np.arange(n) >= 32 * b + 31
        assert rows.any()
        for times in (0.0, 2.0):
            wrong = w.copy()
            wrong[:, 32 * b:32 * b + 32] *= times
            with np.errstate(invalid="ignore"):
                got = wrong @ v / wrong.sum(axis=1, keepdims=True)               # (a row that sees that block alone: not a number)
            off = ~(np.abs(got - want[:, 0]) <= tol[:, 0]).all(axis=1)
            alone = (32 * b == 0) & (length + np.arange(n) < 32)                 # (twice the only block: the same weights)
            assert (off | ~rows | alone).all(), (b, times)
