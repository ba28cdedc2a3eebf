"""The line of buckets without a GPU (the library's own functions, csrc/token_math.hpp), also where logits are many times the temperature: neighbouring fp32 numbers
lie several buckets apart there, and a place on the line in fp32 was off by as many."""
import ctypes
import subprocess
from pathlib import Path

import numpy as np
import pytest

HERE = Path(__file__).resolve().parent
LARGEST = np.finfo(np.float32).max


@pytest.fixture(scope="module")
def model(tmp_path_factory):
    out = tmp_path_factory.mktemp("lines") / "libtoken_lines.so"
    subprocess.run(["g++", "-O2", "-std=c++17", "-ffp-contract=off", "-fPIC", "-shared", "-fsanitize=undefined", "-fno-sanitize-recover", "-o", str(out),
                    str(HERE / "token_lines_model.cpp")], check=True)
    lib = ctypes.CDLL(str(out))
    f, i = ctypes.c_float, ctypes.c_int
    lib.buckets_model.argtypes, lib.buckets_model.restype = [ctypes.c_void_p, ctypes.c_longlong, f, f, ctypes.c_void_p], None
    for name, result, args in (("least_model", f, [i, f, f]), ("last_model", i, [f]), ("least_left_model", f, [f, f, f])):
        getattr(lib, name).restype, getattr(lib, name).argtypes = result, args
    return lib


def buckets(model, z, most, t):
    z, out = np.ascontiguousarray(z, np.float32), np.empty(len(z), np.int32)
    model.buckets_model(z.ctypes.data, len(z), most, t, out.ctypes.data)
    return out


def below(most, n):
    """The n fp32 numbers from `most` on down."""
    bits = np.float32(most).view(np.int32).astype(np.int64)
    key = (bits if bits >= 0 else np.int64(-0x80000000) - bits) - np.arange(n)
    return np.where(key >= 0, key, np.int64(-0x80000000) - key).astype(np.int64).astype(np.uint64).astype(np.uint32).view(np.float32)


# (logits that lie apart by less than an fp32 place on their line, the same at temperatures of everyday use, signs, zero crossed, the largest numbers)
LINES = [(2097152.25, 1.0), (200.000015, 1e-4), (20.0000019, 1e-5), (413.573486, 3.93e-5), (30.7390366, 8.96e-7), (3.9999998, 1.4901161e-8), (4.0, 1.4901161e-8), (5.25, 1e-9), (1e9, 100.0),
         (-2097152.25, 1.0), (-20.0000019, 1e-5), (-3.9999998, 1.4901161e-8), (7.5, 1.0), (0.3, 0.7), (-0.2, 0.01), (0.0, 1.0), (1e-3, 1e-30), (0.0, 1e-45), (12.0, float("inf")), (40.0, 3e38),
         (float(LARGEST), 1.0), (float(-LARGEST), 1.0), (float(LARGEST), 1e30), (1e30, 1e22), (1e20, 1e-20)]


@pytest.mark.parametrize("most,t", LINES)
def test_an_interval_of_logits_is_what_its_bucket_holds(model, most, t):
    """From the smallest logit of buckets 0 .. j to the largest below the smallest of 0 .. j - 1: exactly those that bucket j holds."""
    most = np.float32(most)
    r = np.random.Generator(np.random.Philox(1))
    z = [below(most, 3000), (most - np.abs(r.standard_normal(3000)) * np.float32(min(t, 1e30)) * 10).astype(np.float32), (most - r.random(2000) * 33 * min(t, 1e30)).astype(np.float32)]
    z = np.concatenate(z)
    z = z[(z <= most) & (z >= -LARGEST)] + np.float32(0)
    at = buckets(model, z, most, t)
    assert at.min() == 0 and at.max() <= 512
    order = np.argsort(z, kind="stable")
    assert (np.diff(at[order]) <= 0).all()
    least = np.array([model.least_model(j, most, t) for j in range(512)], np.float32)
    for j in sorted({*range(40), *np.unique(at[at < 512]).tolist(), *(np.unique(at[at < 511]) + 1).tolist(), 511}):
        inside = (z >= least[j]) & (z < least[j - 1] if j else True)
        assert (inside == (at == j)).all(), j


@pytest.mark.parametrize("most,t", LINES)
def test_what_lies_beyond_the_buckets_weighs_less_than_2_to_the_minus_46(model, most, t):
    z = below(np.float32(most), 20000)
    z = z[z >= -LARGEST]
    away = (np.float64(np.float32(most)) - z) / np.float64(np.float32(t))
    beyond = buckets(model, z, most, t) == 512
    assert (away[beyond] > 46 * np.log(2)).all()
    assert beyond[away > 33].all() or 16 / float(np.float32(t)) > LARGEST                       # (where the line's scale ends)


def test_no_token_that_min_p_keeps_lies_behind_the_last_bucket_it_asks_for(model):
    r = np.random.Generator(np.random.Philox(2))
    cases = [(413.573486, 3.93e-5, 0.1654), (30.7390366, 8.96e-7, 1.95e-5)]
    cases += [(16 * 64 ** r.random(), 10 ** r.uniform(-8, -2), 10 ** r.uniform(-14, 0)) for _ in range(4000)]
    cases += [(r.normal() * 20, 10 ** r.uniform(-3, 2), 10 ** r.uniform(-14, 0)) for _ in range(4000)]
    for most, t, min_p in cases:
        most, t, min_p = np.float32(most), np.float32(t), np.float32(min_p)
        z = np.float32(model.least_left_model(most, t, min_p))
        assert min(buckets(model, [z], most, t)[0], 511) <= model.last_model(min_p), (most, t, min_p)      # (512: beyond the buckets, left out)
