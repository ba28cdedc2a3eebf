"""Drawing tokens without a GPU: the oracle, the arithmetic of the kernels (the library's own functions, csrc/token_math.hpp) and the calls that are
refused before anything is launched."""
import ctypes
import math
import subprocess
from pathlib import Path

import numpy as np
import pytest
import torch

from oracle import quasar_sampling_ref as one
from oracle import quasar_tokens_ref as tok

HERE = Path(__file__).resolve().parent
LARGEST = float(np.finfo(np.float32).max)
LOG2E = 1.4426950408889634


@pytest.fixture(scope="module")
def model(tmp_path_factory):
    out = tmp_path_factory.mktemp("token") / "libtoken_model.so"
    subprocess.run(["g++", "-O2", "-std=c++17", "-ffp-contract=off", "-fPIC", "-shared", "-fsanitize=undefined", "-fno-sanitize-recover", "-o", str(out),
                    str(HERE / "token_model.cpp")], check=True)
    lib = ctypes.CDLL(str(out))
    f, d, i, u = ctypes.c_float, ctypes.c_double, ctypes.c_int, ctypes.c_uint64
    for name, result, args in (("weight_model", d, [f, f, d]), ("units_model", u, [f, f, d, i]), ("value_model", f, [f]), ("key_model", u, [f, i, i]), ("key_value_model", f, [u, i]), ("last_key_model", u, [f, i]), ("first_key_model", u, [f, i]),
                               ("key_token_model", i, [u]), ("bucket_model", i, [f, f, f]), ("least_model", f, [f, d, f]),
                               ("filters_model", None, [f, i, f, f, i, ctypes.c_void_p])):
        getattr(lib, name).restype, getattr(lib, name).argtypes = result, args
    return lib


@pytest.fixture(scope="module")
def lib():
    from paper_2603_01399_amd import binding
    return binding.lib()


# ------------------------------------------------------------------------------------------------------------ oracle

def test_oracle_by_hand():
    z = np.log([1.0, 4.0, 2.0, 2.0, 1.0])
    t, p = tok.left(z)
    assert t.tolist() == [0, 1, 2, 3, 4] and np.allclose(p, [.1, .4, .2, .2, .1])
    assert tok.left(z, top_k=2)[0].tolist() == [1, 2] and tok.left(z, top_k=3)[0].tolist() == [1, 2, 3]     # of equal ones the first
    assert tok.left(z, top_p=0.39)[0].tolist() == [1] and tok.left(z, top_p=0.41)[0].tolist() == [1, 2] and tok.left(z, top_p=0.61)[0].tolist() == [1, 2, 3]
    assert tok.left(z, top_k=4, top_p=0.88)[0].tolist() == [1, 2, 3] and tok.left(z, top_k=4, top_p=0.89)[0].tolist() == [0, 1, 2, 3]     # of what top-k leaves: 8 / 9
    assert tok.left(z, min_p=0.49)[0].tolist() == [1, 2, 3] and tok.left(z, min_p=0.51)[0].tolist() == [1] and tok.left(z, min_p=7.0)[0].tolist() == [1]
    assert tok.left(z, temperature=0.0)[0].tolist() == [1] and tok.left(z, top_p=0.0)[0].tolist() == [1] and tok.left(np.zeros(4), temperature=0.0)[0].tolist() == [0]
    assert np.allclose(tok.left(z, temperature=0.5, top_k=2)[1], [.8, .2])
    assert len(tok.left(np.full(3, -np.inf))[0]) == 0 and tok.left([np.nan, 1.0, np.inf])[0].tolist() == [1, 2] and tok.left([np.nan, 1.0, np.inf])[1].tolist() == [0, 1]
    t, p = tok.left(z)
    assert [tok.draw(t, p, u) for u in (0.0, 0.09, 0.11, 0.49, 0.51, 0.99)] == [0, 0, 1, 1, 2, 4]


def test_oracle_without_filters_is_the_one_of_a_single_sequence():
    r = np.random.Generator(np.random.Philox(1))
    for trial in range(200):
        n, V = int(r.integers(1, 6)), int(r.integers(2, 30))
        z = r.standard_normal((n, V)) * 2
        drafts, ua, us, t = r.integers(0, V, n), r.random(n), r.random(n), float(r.uniform(0.5, 1.5))
        got = tok.verify(z, drafts, ua, us, temperature=t)
        want = one.speculative_verify(z, drafts[:n - 1], t, ua, us)
        assert (got[0], got[1]) == (want["n_acc"], want["token"]) and np.allclose(got[2][:n - 1], want["p_draft"])


def test_oracle_loses_nothing():
    """The token behind a candidate that is accepted or not is distributed as the filtered row is (integrated over the numbers)."""
    z = np.array([0.3, 1.0, -0.5, 0.9, 0.2])
    filters = dict(temperature=0.8, top_k=4, top_p=0.9)
    t, p = tok.left(z, **filters)
    for draft in (1, 2, 4):
        out, n = np.zeros(5), 60                             # (midpoints: off by at most half a step of either number)
        for ua in (np.arange(n) + 0.5) / n:
            for us in (np.arange(n) + 0.5) / n:
                a, token, _ = tok.verify(np.stack([z, z]), [draft, 0], [ua, 0], [us, us], **filters)
                out[draft if a else token] += 1 / (n * n)
        want = np.zeros(5)
        want[t] = p
        assert np.abs(out - want).max() <= 1 / n


# -------------------------------------------------------------------------------------------------------- arithmetic

def test_weights(model):
    """Within 2^-47 of the exponential relatively (31 units: the argument's two roundings are 2^-52 of 45 each), and its units to nearest."""
    r = np.random.Generator(np.random.Philox(2))
    for _ in range(5000):
        ref = np.float32(r.normal() * 10)
        z, t = np.float32(ref - np.float32(r.exponential() * 6)), float(np.float32(np.exp(r.normal())))
        rate = LOG2E / t
        x = (float(z) - float(ref)) / t
        w, want = model.weight_model(z, ref, rate), math.exp(x)
        assert abs(w - want) <= 2.0 ** -46 * want + 2.0 ** -59
        for bits in (42, 48):
            units = model.units_model(z, ref, rate, bits)
            assert abs(units - want * 2.0 ** bits) <= 0.5 + 2.0 ** -46 * want * 2.0 ** bits + 2.0 ** (bits - 59)
    assert model.weight_model(3.0, 3.0, LOG2E) == 1.0 and model.units_model(3.0, 3.0, LOG2E, 48) == 1 << 48 and model.units_model(-LARGEST, LARGEST, 1e45, 48) == 0
    assert model.units_model(-math.inf, 1.0, 0.0, 48) == 0 and model.units_model(-math.inf, 1.0, 1.0, 48) == 0 and model.units_model(-5.0, 1.0, 0.0, 42) == 1 << 42


def test_values_and_order(model):
    assert model.value_model(math.nan) == -math.inf and model.value_model(math.inf) == LARGEST and model.value_model(-math.inf) == -math.inf
    assert math.copysign(1, model.value_model(-0.0)) == 1.0
    r = np.random.Generator(np.random.Philox(3))
    z = np.concatenate([r.standard_normal(300) * np.exp(r.normal(size=300) * 20), [0.0, LARGEST, -LARGEST, 1e-45, -1e-45, 1.0, -1.0], np.repeat(2.5, 20)]).astype(np.float32)
    for bf16 in (0, 1):
        if bf16:
            z = np.unique(torch.from_numpy(z).bfloat16().float().numpy() + 0.0).clip(-3.3e38, 3.3e38)
            z = np.concatenate([z, np.repeat(z[50], 30)])
            z = torch.from_numpy(z).bfloat16().float().numpy()
        v = r.permutation(1 << 20)[:len(z)]
        keys = [model.key_model(a, int(b), bf16) for a, b in zip(z, v)]
        assert [int(i) for i in np.argsort(np.array(keys, np.uint64))] == [int(i) for i in np.lexsort((v, -z.astype(np.float64)))]
        for a, b, key in zip(z, v, keys):
            assert model.key_value_model(key, bf16) == a and model.key_token_model(key) == b and key < 1 << (36 if bf16 else 52)
        # a logit counts up to the last key of a bound exactly where it is not below it, and from the first on exactly where it is not above it
        for bound in np.concatenate([z[::7], (r.standard_normal(60) * np.exp(r.normal(size=60) * 20)).astype(np.float32), np.nextafter(z[::5], np.float32(math.inf)),
                                     np.nextafter(z[::5], np.float32(-math.inf))]).clip(-3.3e38, 3.3e38):
            last = model.last_key_model(bound, bf16)
            assert [key <= last for key in keys] == [bool(a >= bound) for a in z], bound
            first = model.first_key_model(bound, bf16)
            assert [key >= first for key in keys] == [bool(a <= bound) for a in z], bound


@pytest.mark.parametrize("scale", [16.0, 0.0, 1.0, 16000.0, 1e30, LARGEST, 3e-5])
def test_buckets(model, scale):
    """Fall never as logits grow, and are the same line from every part: a bucket in a part and the part's largest one's in the row add up to the bucket in the row."""
    r = np.random.Generator(np.random.Philox(4))
    for width in (1e-3, 1.0, 30.0, 1e5, 1e20, 1e38):
        z = np.sort((r.standard_normal(400) * width).clip(-LARGEST, LARGEST).astype(np.float32))
        most = z[-1]
        at = [model.bucket_model(x, scale, most) for x in z]
        assert at[-1] == 0 and all(a >= b for a, b in zip(at, at[1:])) and 0 <= min(at) and max(at) <= 512
        for part in z[r.integers(0, 400, 20)]:
            shift = model.bucket_model(part, scale, most)
            for x, row in zip(z, at):
                if x <= part:
                    inside = model.bucket_model(x, scale, part)
                    if inside < 512 and shift + inside < 512:
                        assert row == shift + inside
                    if row < 512:
                        assert row == shift + inside
        assert model.bucket_model(-math.inf, scale, most) == 512


def test_least_logit(model):
    r = np.random.Generator(np.random.Philox(5))
    for _ in range(3000):
        most, t, min_p = np.float32(r.normal() * 20), float(np.float32(np.exp(r.normal() * 2))), np.float32(r.choice([1.0, 0.5, 1e-3, 1e-14, float(r.random())]))
        rate = LOG2E / t
        z = np.float32(model.least_model(most, rate, min_p))
        assert z <= most and model.weight_model(z, most, rate) >= float(min_p)              # (numpy would round the weight to fp32)
        assert model.weight_model(np.nextafter(z, np.float32(-math.inf)), most, rate) < float(min_p)
    assert model.least_model(3.0, 0.0, 0.5) == -LARGEST and model.least_model(-LARGEST, LOG2E, 0.5) == -LARGEST


def test_filters(model):
    out = (ctypes.c_double * 5)()

    def f(*a):
        model.filters_model(*a, 100, out)
        return list(out)
    assert f(1.0, 0, 1.0, 0.0) == [LOG2E, 16.0, 0, 1, 0] and f(0.5, 7, 0.5, 0.25) == [2 * LOG2E, 32.0, 7, 0.5, 0.25]
    nan = math.nan
    for t in (0.0, -1.0, nan, -math.inf):
        assert f(t, 5, 1.0, 0.0) == [LOG2E, 16.0, 1, 1, 0]
    assert f(math.inf, 100, 1.0, 0.0)[:3] == [0, 0, 0] and f(1.0, -3, nan, nan)[2:] == [0, 1, 0] and f(1.0, 2 ** 31 - 1, 5.0, -1.0)[2:] == [0, 1, 0]
    assert f(1.0, 9, 0.0, 3.0)[2:] == [1, 1, 1] and f(1.0, 9, -1.0, 0.0)[2:] == [1, 1, 0] and f(1.0, 9, 1.0, 1e-30)[4] == 0 and f(1e-45, 9, 1.0, 0.0)[1] == LARGEST


# ---------------------------------------------------------------------------------------------------------- refusals

NULL, SHAPE, ALIGN, WORKSPACE, DTYPE = 1, 2, 3, 4, 5
A, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1002)
BAD = [(dict(z=None), NULL), (dict(u=None), NULL), (dict(token=None), NULL), (dict(dtype=2), DTYPE), (dict(dtype=-1), DTYPE), (dict(T=0), SHAPE), (dict(T=(1 << 20) + 1), SHAPE),
       (dict(V=0), SHAPE), (dict(V=(1 << 20) + 1, ld=1 << 21), SHAPE), (dict(ld=999), SHAPE), (dict(ld=-1), SHAPE), (dict(z=ODD), ALIGN), (dict(t=ODD), ALIGN), (dict(k=ODD), ALIGN),
       (dict(p=ODD), ALIGN), (dict(m=ODD), ALIGN), (dict(u=ODD), ALIGN), (dict(token=ODD), ALIGN), (dict(out_p=ODD), ALIGN), (dict(ws=None), WORKSPACE), (dict(room=1000), WORKSPACE),
       (dict(ws=ctypes.c_void_p(0x1008)), ALIGN), (dict(z=ctypes.c_void_p(0x1001), dtype=1), ALIGN)]
GOOD = dict(z=A, dtype=0, T=5, V=1000, ld=1000, t=A, k=A, p=A, m=A, u=A, token=A, out_p=A, ws=A, room=1 << 30)


@pytest.mark.parametrize("change,status", BAD)
def test_sample_refuses(lib, change, status):
    c = GOOD | change
    assert lib.quasar_sample_tokens(c["z"], c["dtype"], c["T"], c["V"], c["ld"], c["t"], c["k"], c["p"], c["m"], c["u"], c["token"], c["out_p"], c["ws"], c["room"], None) == status


@pytest.mark.parametrize("change,status", BAD + [(dict(starts=None), NULL), (dict(draft=None), NULL), (dict(ua=None), NULL), (dict(acc=None), NULL), (dict(n_seqs=0), SHAPE),
                                                 (dict(n_seqs=1025), SHAPE), (dict(starts=ODD), ALIGN), (dict(draft=ODD), ALIGN), (dict(ua=ODD), ALIGN), (dict(acc=ODD), ALIGN)])
def test_verify_refuses(lib, change, status):
    c = GOOD | dict(starts=A, n_seqs=2, draft=A, ua=A, acc=A) | change
    assert lib.quasar_verify_tokens(c["z"], c["dtype"], c["T"], c["V"], c["ld"], c["starts"], c["n_seqs"], c["draft"], c["t"], c["k"], c["p"], c["m"], c["ua"], c["u"], c["acc"],
                                    c["token"], c["out_p"], c["ws"], c["room"], None) == status


def test_workspaces(lib):
    for fn in (lib.quasar_sample_tokens_workspace_bytes, lib.quasar_verify_tokens_workspace_bytes):
        assert 0 < fn(1, 1) < fn(1, 151936) < fn(64, 151936) and fn(1 << 20, 1 << 20) < 1 << 33
        for bad in ((0, 100), (1, 0), (-1, 5), ((1 << 20) + 1, 5), (5, (1 << 20) + 1)):
            assert fn(*bad) == 0


def test_binding_refuses_host_tensors():
    from paper_2603_01399_amd import binding as qb
    z, u = torch.zeros(2, 50), torch.zeros(2)
    with pytest.raises(TypeError):
        qb.sample_tokens(z, u)
    with pytest.raises(TypeError):
        qb.verify_tokens(z, torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), u, u)


def test_native_calls_without_a_gpu_or_enough_arguments():
    from paper_2603_01399_amd import binding as qb
    z, u = torch.zeros(2, 8), torch.zeros(2)
    assert qb._fast.sample_tokens(z, u, None, None, None, None) == -1 and qb._fast.sample_tokens() == -1 and qb._fast.sample_tokens(None, u, None, None, None, None) == -1
    assert qb._fast.verify_tokens(z, u.int(), u.int(), u, u, None, None, None, None) == -1 and qb._fast.verify_tokens(z, u) == -1
    for call in (qb._fast.paged_prepare_rope, qb._fast.paged_attention_window, qb._fast.prompt_attention_window, qb._fast.pages_trim):
        assert call() == -1 and call(None) == -1
