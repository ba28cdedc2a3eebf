"""Windows, trim and rotary positions without a GPU: the oracle, what the kernels read of a sequence (the library's own functions,
csrc/books.hpp) against the definition asked position by position, and the calls that are refused before anything is launched."""
import ctypes
import math
import subprocess
from pathlib import Path

import numpy as np
import pytest
import torch

from oracle import quasar_attention_ref as at
from oracle import quasar_paged_ref as pg
from oracle import quasar_ref as ref
from oracle import quasar_window_ref as win
from test_paged import A, ALIGN, BAD_BOOKS, BAD_PAGED, BOOKS, DTYPE, NULL, ODD_ADDRESS, PAGED, SHAPE, WORKSPACE, paged_args

HERE = Path(__file__).resolve().parent
MOST = 1 << 25


@pytest.fixture(scope="module")
def model(tmp_path_factory):
    out = tmp_path_factory.mktemp("window") / "libwindow_model.so"
    subprocess.run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fsanitize=undefined", "-fno-sanitize-recover", "-o", str(out),
                    str(HERE / "window_model.cpp")], check=True)
    lib = ctypes.CDLL(str(out))
    lib.seen_model.restype = ctypes.c_uint
    return lib


@pytest.fixture(scope="module")
def lib():
    from paper_2603_01399_amd import binding
    return binding.lib()


# ------------------------------------------------------------------------------------------------------------ oracle

def test_oracle_without_a_window_is_the_causal_one():
    r = np.random.Generator(np.random.Philox(1))
    q, k, v = r.standard_normal((5, 4, 128)), r.standard_normal((23, 2, 128)), r.standard_normal((23, 2, 128))
    want = pg.attention(q, k, v, 18)
    for window, sinks in ((23, 0), (1000, 3), (1, 23), (7, 100)):
        for a, b in zip(win.attention(q, k, v, 18, window, sinks), want):
            assert np.allclose(a, b, rtol=1e-13, atol=1e-15)


def test_oracle_by_hand():
    """A window of one sees its own value; with one first token and equal keys, the mean of both."""
    v = np.arange(6.0)[:, None, None] * np.ones((6, 1, 128))
    q, k = np.zeros((2, 1, 128)), np.zeros((6, 1, 128))
    assert np.array_equal(win.attention(q, k, v, 4, 1, 0)[0][:, 0, 0], [4.0, 5.0])
    assert np.array_equal(win.attention(q, k, v, 4, 1, 1)[0][:, 0, 0], [2.0, 2.5])
    assert np.array_equal(win.attention(q, k, v, 4, 2, 0)[0][:, 0, 0], [3.5, 4.5])
    assert win.trim([1] * 4, [10], [[3, 2, 1, 0]], 4, 3, 0) == ([1, 1, 0, 0], [[-1, -1, 1, 0]])
    assert win.trim([1] * 4, [10], [[3, 2, 1, 0]], 4, 3, 1) == ([1, 1, 0, 1], [[3, -1, 1, 0]])
    assert win.trim([1] * 4, [10], [[3, 2, 1, 0]], 4, 4, 5) == ([1, 1, 1, 1], [[3, 2, 1, 0]])


def test_rotation_oracle():
    """The half layout over the whole head is the one of the cache's other oracle; pairs are a permutation of it; the rest stays."""
    r = np.random.Generator(np.random.Philox(2))
    bits = ref.f32_to_bf16_bits(r.standard_normal((3, 2, 128)).astype(np.float32))
    pos, freq = np.array([0, 7, 30000]), 1e6 ** (-2.0 * np.arange(64) / 128)
    x = ref.bf16_bits_to_f64(at.head_norm_rope(bits, ref.f32_to_bf16_bits(np.ones(128, np.float32)), 0.0, np.zeros(3), 1e6))
    want = at.head_norm_rope(bits, ref.f32_to_bf16_bits(np.ones(128, np.float32)), 0.0, pos, 1e6)
    assert np.array_equal(ref.f64_to_bf16_bits(win.rotate(x, pos, freq, "half")), want)
    perm = np.arange(128).reshape(2, 64).T.reshape(-1)                          # the half layout's pairs side by side
    assert np.allclose(win.rotate(x[..., perm], pos, freq, "interleaved"), win.rotate(x, pos, freq, "half")[..., perm], rtol=0, atol=0)
    part = win.rotate(x, pos, freq[:16], "interleaved", 2.0)
    assert np.array_equal(part[..., 32:], x[..., 32:]) and np.allclose(np.linalg.norm(part[..., :32], axis=-1), 2 * np.linalg.norm(x[..., :32], axis=-1))


# ------------------------------------------------------------------------------------------------- what is read

def test_blocks_that_rows_see(model):
    """Every unit that holds a position that some row sees is taken once, in order, and no other beyond those that hold first tokens or the window's end."""
    r = np.random.Generator(np.random.Philox(3))
    out = (ctypes.c_int * 600)()
    for trial in range(4000):
        shift = int(r.integers(5, 7))
        first, n = int(r.integers(0, [3, 70, 3000][trial % 3])), int(r.integers(1, 40))
        size, sinks = int(r.choice([1, 2, 31, 32, 33, 64, 100, 1000, 4000, MOST])), int(r.choice([0, 1, 4, 31, 32, 33, 64, 200, 5000, MOST]))
        units = min(((first + n - 1) >> shift) + 1, int(r.choice([1, 2, 5, 1000])))
        count = model.units_model(size, sinks, first, units, shift, out)
        got = list(out[:count])
        pos = np.arange(first + n)
        seen = np.zeros(first + n, bool)
        for row in range(first, first + n):
            seen |= (pos <= row) & ((row - pos < size) | (pos < sinks))
        want = sorted(u for u in {p >> shift for p in pos[seen]} if u < units) or [units - 1]       # (nothing: a block to write the zeros)
        assert got == want, (size, sinks, first, n, units, shift)


def test_steps_that_a_tile_sees(model):
    """The same for a tile of rows first .. last: all of them once; those ahead of `whole` are seen whole by every row, being in its window."""
    r = np.random.Generator(np.random.Philox(4))
    out, whole = (ctypes.c_int * 600)(), (ctypes.c_int * 1)()
    some = 0
    for trial in range(4000):
        first = int(r.integers(0, [3, 300, 6000][trial % 3]))
        last = first + int(r.integers(0, [1, 16, 130][int(r.integers(3))]))
        size, sinks = int(r.choice([1, 2, 63, 64, 65, 127, 128, 200, 1000, 4000, MOST])), int(r.choice([0, 1, 4, 63, 64, 65, 200, 5000, MOST]))
        units = min((last >> 6) + 1, int(r.choice([1, 3, 20, 1000])))
        count = model.tile_model(size, sinks, first, last, units, 6, out, whole)
        got = list(out[:count])
        pos = np.arange(last + 1)
        rows = np.arange(first, last + 1)[:, None]
        seen = (pos <= rows) & ((rows - pos < size) | (pos < sinks))
        want = {int(u) for u in pos[seen.any(axis=0)] >> 6 if u < units} or {units - 1}
        assert len(set(got)) == count and set(got) == want
        for u in got[:whole[0]]:
            assert seen[:, 64 * u:64 * u + 64].all() and 64 * u + 63 <= last
        assert got[whole[0]:] == sorted(got[whole[0]:]) and 0 <= whole[0] <= count
        some += whole[0]
    assert some > 1000


def test_positions_of_a_block(model):
    r = np.random.Generator(np.random.Philox(5))
    for trial in range(20000):
        size, sinks = int(r.choice([1, 2, 5, 31, 32, 33, 100, MOST])), int(r.choice([0, 1, 4, 31, 32, 33, 70, MOST]))
        pos0 = 32 * int(r.integers(0, 6))
        pos = int(r.integers(0, 260))
        bits = model.seen_model(size, sinks, pos, pos0)
        assert [bits >> i & 1 for i in range(32)] == [int(win.sees(pos, pos0 + i, size, sinks)) for i in range(32)]
    for size, sinks, pos, pos0 in ((1, 0, 1 << 24, 0), (MOST, MOST, (1 << 24) + 31, (1 << 24) - 32), (1, 0, 0, 1 << 24), (MOST, 0, 0, 1 << 24)):
        assert model.seen_model(size, sinks, pos, pos0) == (0xFFFFFFFF if size == MOST and pos > pos0 else 0)


def test_columns_given_back(model):
    r = np.random.Generator(np.random.Philox(6))
    out = (ctypes.c_int * 2)()
    for trial in range(1500):
        shift = int(r.integers(5, 8))
        length = int(r.integers(0, 1200))
        size, sinks = int(r.choice([1, 2, 32, 33, 100, 500, MOST])), int(r.choice([0, 1, 4, 31, 32, 33, 64, 200, MOST]))
        model.columns_model(size, sinks, length, shift, out)
        columns = 1300 >> shift
        refs, table = win.trim([1] * columns, [length], [list(range(columns))], 1 << shift, size, sinks)
        assert [c for c in range(columns) if table[0][c] < 0] == list(range(out[0], min(out[1], columns)))


# ---------------------------------------------------------------------------------------------------------- refusals

BAD_WINDOW = [(dict(window=0), SHAPE), (dict(window=-1), SHAPE), (dict(sinks=-1), SHAPE), (dict(window=-2 ** 63), SHAPE), (dict(sinks=-2 ** 63), SHAPE)]


@pytest.mark.parametrize("change,status", BAD_PAGED + BAD_WINDOW + [(dict(x=None), NULL), (dict(out=None), NULL), (dict(ldq=4088), SHAPE), (dict(new=33), SHAPE),
                                                                    (dict(ldo=4098), SHAPE), (dict(x=ODD_ADDRESS), ALIGN), (dict(ws=None), WORKSPACE), (dict(room=1000), WORKSPACE)])
def test_windowed_step_refuses(lib, change, status):
    c = dict(PAGED, x=A, T=5, ldq=4096, hq=32, hk=8, row_start=A, n_seqs=2, new=4, out=A, ldo=4096, ws=A, room=1 << 30, window=100, sinks=4) | change
    assert lib.quasar_paged_attention_window(c["x"], c["T"], c["ldq"], c["hq"], c["hk"], c["row_start"], c["n_seqs"], c["new"], *paged_args(c), c["window"], c["sinks"],
                                             c["out"], c["ldo"], c["ws"], c["room"], None) == status


@pytest.mark.parametrize("change,status", BAD_PAGED + BAD_WINDOW + [(dict(x=None), NULL), (dict(out=None), NULL), (dict(ldo=4098), SHAPE), (dict(out=ODD_ADDRESS), ALIGN),
                                                                    (dict(ws=ODD_ADDRESS), ALIGN)])
def test_windowed_prompt_refuses(lib, change, status):
    c = dict(PAGED, x=A, T=5, ldq=8192, hq=32, hk=8, row_start=A, n_seqs=2, out=A, ldo=8192, ws=None, window=100, sinks=4) | change
    assert lib.quasar_prompt_attention_window(c["x"], c["T"], c["ldq"], c["hq"], c["hk"], c["row_start"], c["n_seqs"], *paged_args(c), c["window"], c["sinks"],
                                              c["out"], c["ldo"], c["ws"], 1 << 30, None) == status


@pytest.mark.parametrize("change,status", BAD_BOOKS + BAD_WINDOW + [(dict(lengths=None), NULL), (dict(lengths=ODD_ADDRESS), ALIGN)])
def test_trim_refuses(lib, change, status):
    c = BOOKS | dict(window=10, sinks=0) | change
    assert lib.quasar_pages_trim(c["table"], c["table_ld"], c["n_seqs"], c["max_pages"], c["lengths"], c["window"], c["sinks"], c["refs"], c["n_pages"], c["page_len"], None) == status


@pytest.mark.parametrize("change,status", BAD_PAGED + [(dict(x=None), NULL), (dict(q=None), NULL), (dict(qg=None), NULL), (dict(kg=None), NULL), (dict(f=None), NULL),
                                                       (dict(ld=32 * 128), SHAPE), (dict(ldq=4090), SHAPE), (dict(eps=-1.0), SHAPE), (dict(layout=2), DTYPE), (dict(layout=-1), DTYPE),
                                                       (dict(dims=0), SHAPE), (dict(dims=8), SHAPE), (dict(dims=40), SHAPE), (dict(dims=144), SHAPE), (dict(mag=0.0), SHAPE),
                                                       (dict(mag=math.inf), SHAPE), (dict(mag=math.nan), SHAPE), (dict(x=ODD_ADDRESS), ALIGN), (dict(qg=ODD_ADDRESS), ALIGN),
                                                       (dict(f=ctypes.c_void_p(0x1004)), ALIGN)])
def test_rotary_prepare_refuses(lib, change, status):
    c = dict(PAGED, x=A, T=5, ld=48 * 128, hq=32, hk=8, row_start=A, n_seqs=2, qg=A, kg=A, eps=1e-6, layout=0, dims=64, f=A, mag=1.0, q=A, ldq=4096) | change
    assert lib.quasar_paged_prepare_rope(c["x"], c["T"], c["ld"], c["hq"], c["hk"], c["row_start"], c["n_seqs"], c["qg"], c["kg"], c["eps"], c["layout"], c["dims"], c["f"],
                                         c["mag"], c["q"], c["ldq"], *paged_args(c), None) == status


def test_rope_frequencies():
    """The frequencies that a Rope works out, by hand at the ends and against their formulas between; refusals."""
    from paper_2603_01399_amd import binding as qb
    f = qb.Rope(128, 1e6, device="cpu")
    assert f.magnitude == 1.0 and f.inv_freq[0] == 1.0 and np.allclose(f.inv_freq, [1e6 ** (-i / 64) for i in range(64)], rtol=1e-14)
    assert np.allclose(qb.Rope(64, 1e4, scaling="linear", factor=4.0, device="cpu").inv_freq, [1e4 ** (-i / 32) / 4 for i in range(32)], rtol=1e-14)
    ntk = qb.Rope(64, 1e4, scaling="ntk", factor=8.0, device="cpu").inv_freq
    assert ntk[0] == 1.0 and np.isclose(ntk[31], 1e4 ** (-31 / 32) / 8, rtol=1e-13)                     # the fastest as it was, the slowest divided
    parts = qb.Rope(128, 1e6, scaling="by_parts", factor=4.0, trained_len=32768, device="cpu")
    base = np.array([1e6 ** (-i / 64) for i in range(64)])
    turns = 32768 * base / (2 * math.pi)
    assert np.isclose(parts.magnitude, 1 + 0.1 * math.log(4.0))
    assert np.allclose(parts.inv_freq[turns >= 32], base[turns >= 32], rtol=1e-13) and np.allclose(parts.inv_freq[turns <= 1], base[turns <= 1] / 4, rtol=1e-13)
    i = int(np.flatnonzero((turns > 1) & (turns < 32))[0])
    g = (turns[i] - 1) / 31
    assert np.isclose(parts.inv_freq[i], base[i] * (g + (1 - g) / 4), rtol=1e-12)
    assert qb.Rope(64, scaling="by_parts", factor=8.0, trained_len=8192, fast=4.0, magnitude=1.0, device="cpu").magnitude == 1.0
    own = torch.linspace(1.0, 0.1, 16, dtype=torch.float64)
    assert torch.equal(qb.Rope(32, layout="interleaved", inv_freq=own, device="cpu").inv_freq, own)
    for bad in (dict(dims=24), dict(dims=0), dict(dims=144), dict(layout="pairs"), dict(scaling="other"), dict(theta=1.0), dict(factor=0.0), dict(scaling="by_parts"),
                dict(scaling="by_parts", trained_len=4096, slow=4.0, fast=4.0), dict(magnitude=0.0), dict(magnitude=math.inf), dict(inv_freq=own), dict(dims=32, inv_freq=own.float()),
                dict(dims=32, inv_freq=own, scaling="linear")):
        with pytest.raises(ValueError):
            qb.Rope(**(dict(device="cpu") | bad))
