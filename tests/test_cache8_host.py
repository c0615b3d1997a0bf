"""The 8-bit cache's rules on the host: the oracle's e4m3, the exponent of a block as the kernels form it, the angles in turns,
and what the entry points refuse."""
import ctypes as C
import math
import random
import subprocess
import types

import numpy as np
import pytest
import torch

from oracle import cache8 as O

SRC = """
#include "../../paper_2608_15943_b200/csrc/kvp_cache8.h"
#include "../../paper_2608_15943_b200/csrc/kvp_rope_freq.h"
extern "C" int exponent(unsigned bits) { return kvp::scale_exponent(bits); }
extern "C" int of_byte(unsigned b) { return kvp::exponent_of_byte(b); }
extern "C" unsigned power(int e) { return kvp::power_bits(e); }
extern "C" void turns(double theta, int dh, uint64_t* out) { kvp::rope_turns(theta, dh, out); }
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    d = tmp_path_factory.mktemp("cache8")
    (d / "r.cpp").write_text(SRC.replace("../../", root + "/"))
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-o", str(d / "r.so"), str(d / "r.cpp")], check=True)
    lib = C.CDLL(str(d / "r.so"))
    lib.power.restype = C.c_uint
    lib.turns.argtypes = [C.c_double, C.c_int, C.c_void_p]
    return lib


def bits(x):
    return int(np.float32(x).view(np.uint32))


def test_oracle_rounds_as_e4m3_does():
    every = torch.arange(256, dtype=torch.uint8)
    value = every.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(O.VALUE, value, equal_nan=True)
    fine = np.isfinite(value)
    assert (O.round_e4m3(value[fine]) == np.arange(256)[fine]).all()
    up = value[:127]
    ties = (up[1:] + up[:-1]) / 2
    x = np.concatenate([ties, -ties, np.nextafter(ties, 0), np.nextafter(ties, 1e3), np.random.default_rng(0).normal(size=20000) * 90])
    x = np.concatenate([x.astype(np.float32).astype(np.float64), ties])
    x = x[np.abs(x) <= 448]
    want = torch.tensor(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert (O.round_e4m3(x) == want).all()
    assert (O.round_e4m3([np.inf, -np.inf, np.nan]) == 0x7f).all()


def test_exponent_of_a_block(rules):
    rng = random.Random(3)
    xs = [0.0, 1e-45, 448.0, float(np.nextafter(np.float32(448), np.float32(1e9))), 3.4028234663852886e38, 2.0 ** -126]
    for k in range(-105, 120):
        edge = np.float32(448.0 * 2.0 ** k)
        xs += [float(edge), float(np.nextafter(edge, np.float32(0))), float(np.nextafter(edge, np.float32(np.inf))), math.ldexp(1 + rng.random(), k)]
    xs = [float(np.float32(x)) for x in xs]
    want = O.exponent(np.array(xs))
    for x, e in zip(xs, want):
        assert rules.exponent(bits(x)) == e, x
        assert e == O.LEAST or x > math.ldexp(448, int(e) - 1)
        assert x <= math.ldexp(448, int(e)) and O.LEAST <= e <= 120
    for b in range(256):
        assert rules.of_byte(b) == min(max(b - 127, -100), 120)
    for e in range(-126, 121):
        assert np.uint32(rules.power(e)).view(np.float32) == np.float32(2.0 ** e)
    assert rules.power(-247) == rules.power(-126)


@pytest.mark.parametrize("theta,dh", [(10000.0, 128), (10000.0, 64), (500000.0, 128), (1.0000001, 64), (3e38, 128)])
def test_angles_in_turns(rules, theta, dh):
    """A frequency is off by at most 2^-57 of itself and half of 2^-64 turns; the product modulo 2^64 adds nothing."""
    from decimal import Decimal, getcontext
    getcontext().prec = 60
    pi = Decimal("3.14159265358979323846264338327950288419716939937510582097494")
    out = (C.c_uint64 * (dh // 2))()
    rules.turns(theta, dh, out)
    for i in range(dh // 2):
        f = (Decimal(theta) ** (Decimal(-2 * i) / dh)) / (2 * pi)
        assert abs(Decimal(out[i]) / 2 ** 64 - f) <= f / 2 ** 57 + Decimal(2) ** -64


def test_rotation_of_the_oracle():
    x = np.random.default_rng(1).normal(size=(5, 3, 64))
    pos = np.array([0, 1, 7, 1000, 131071])
    y = O.rotate(x, pos, 10000.0)
    assert np.array_equal(y[0], x[0]) and np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
    i, p = 5, 3
    a = pos[p] * 10000.0 ** (-2 * i / 64)
    assert np.allclose(y[p, :, 2 * i], x[p, :, 2 * i] * math.cos(a) - x[p, :, 2 * i + 1] * math.sin(a))
    assert np.array_equal(O.rotate(x, pos, 0), x)


# ---------------------------------------------------------------------------------------------
# refusals
# ---------------------------------------------------------------------------------------------
def tokens_call(kvp, L=2, donor=(0, 0), B=2, Hq=4, Hkv=2, dh=64, page=16, max_pages=3, n_pages=7, T=2, dtype=0, bits8=True, **over):
    io = torch.float32 if dtype else torch.bfloat16
    cache = torch.uint8 if bits8 else torch.bfloat16
    lists = dict(k_new=[torch.zeros(T, Hkv, dh, dtype=io), None], v_new=[torch.zeros(T, Hkv, dh, dtype=io), None],
                 k_cache=[torch.zeros(n_pages, Hkv, page, dh, dtype=cache), None], v_cache=[torch.zeros(n_pages, Hkv, page, dh, dtype=cache), None],
                 block_table=torch.zeros(B, max_pages, dtype=torch.int32), lengths=torch.ones(B, dtype=torch.int32), first=None, theta=10000.0,
                 q=[torch.zeros(T, Hq, dh, dtype=io) for _ in range(L)], q_out=[torch.zeros(T, Hq, dh, dtype=io) for _ in range(L)],
                 k_scale=[torch.zeros(n_pages, Hkv, max(page // 16, 1), dtype=torch.uint8), None] if bits8 else None,
                 v_scale=[torch.zeros(n_pages, Hkv, max(page // 16, 1), dtype=torch.uint8), None] if bits8 else None)
    lists.update(over)
    desc = kvp.DecodeDesc(L, B, Hq, Hkv, dh, page, max_pages, n_pages, 0, dtype)
    return lambda: kvp.cache_append_tokens(desc, list(donor), **lists)


def decode_call(kvp, L=2, donor=(0, 0), B=2, Hq=4, Hkv=2, dh=64, page=16, max_pages=3, n_pages=7, dtype=0, splits=0, **over):
    io = torch.float32 if dtype else torch.bfloat16
    lists = dict(q=[torch.zeros(B, Hq, dh, dtype=io) for _ in range(L)], k_cache=[torch.zeros(n_pages, Hkv, page, dh, dtype=torch.uint8), None],
                 v_cache=[torch.zeros(n_pages, Hkv, page, dh, dtype=torch.uint8), None],
                 k_scale=[torch.zeros(n_pages, Hkv, max(page // 16, 1), dtype=torch.uint8), None],
                 v_scale=[torch.zeros(n_pages, Hkv, max(page // 16, 1), dtype=torch.uint8), None], block_table=torch.zeros(B, max_pages, dtype=torch.int32),
                 lengths=torch.ones(B, dtype=torch.int32), o=[torch.zeros(B, Hq, dh, dtype=io) for _ in range(L)],
                 lse=[torch.zeros(B, Hq) for _ in range(L)], ws=torch.zeros(1 << 22, dtype=torch.uint8))
    lists.update(over)
    desc = kvp.DecodeDesc(L, B, Hq, Hkv, dh, page, max_pages, n_pages, splits, dtype)
    return lambda: kvp.decode8(desc, list(donor), **lists)


@pytest.fixture(params=["native", "ctypes"])
def kvp(request, monkeypatch):
    from paper_2608_15943_b200 import kvp as mod
    if torch.cuda.is_available():
        pytest.skip("host tensors: refused before anything else where there is a device")
    if request.param == "ctypes":
        monkeypatch.setattr(mod, "_pack", types.SimpleNamespace(cache_append_tokens=lambda *a: NotImplemented, decode8=lambda *a: NotImplemented))
    return mod


def refused(kvp, call, status):
    with pytest.raises(kvp.KvpError) as e:
        call()
    assert e.value.status == status, e.value


def test_tokens_reach_the_device(kvp):
    """Valid calls pass every check and end at the launch, which has no device."""
    for call in (tokens_call(kvp), tokens_call(kvp, bits8=False), tokens_call(kvp, dtype=1), tokens_call(kvp, q=None, q_out=None, theta=0.0),
                 tokens_call(kvp, T=5, first=torch.tensor([0, 2, 5], dtype=torch.int32)), decode_call(kvp), decode_call(kvp, dtype=1),
                 decode_call(kvp, layer_begin=1, layer_end=2), decode_call(kvp, splits=3)):
        refused(kvp, call, kvp.ERR_CUDA)
    tokens_call(kvp, T=0, first=torch.zeros(3, dtype=torch.int32))()       # nothing to do


def test_tokens_refused_by_the_library(kvp):
    bad, one = kvp.ERR_INVALID_ARG, [None, None]
    for over in (dict(T=3), dict(theta=-1.0), dict(theta=1.0), dict(theta=math.inf), dict(theta=math.nan), dict(k_new=one), dict(v_new=one), dict(k_cache=one),
                 dict(v_cache=one), dict(k_scale=one), dict(v_scale=one), dict(v_scale=None), dict(q=None), dict(q_out=None), dict(q=[]), dict(q_out=[])):
        if over.get("k_new") is one:
            over["k_new"] = [None, torch.zeros(2, 2, 64, dtype=torch.bfloat16)]
        refused(kvp, tokens_call(kvp, **over), bad)
    for over in (dict(dh=32), dict(dh=256), dict(page=8), dict(Hq=3, Hkv=2)):
        if over.get("page"):
            over.update(k_scale=[torch.zeros(7, dtype=torch.uint8), None], v_scale=[torch.zeros(7, dtype=torch.uint8), None])
        refused(kvp, tokens_call(kvp, **over), kvp.ERR_UNSUPPORTED)
    odd = torch.zeros(2 * 2 * 64 + 4, dtype=torch.bfloat16)[4:].view(2, 2, 64)
    refused(kvp, tokens_call(kvp, k_new=[odd, None]), kvp.ERR_UNSUPPORTED)
    for donor in ((0,), (0, 2), (1, 1), (0, -1)):
        refused(kvp, tokens_call(kvp, donor=donor), kvp.ERR_BAD_DONOR)


def test_tensors_refused(kvp):
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    for over in (dict(v_new=[bf(3, 2, 64), None]), dict(k_new=[torch.zeros(2, 2, 64), None]), dict(k_new=[bf(2, 64, 2).transpose(1, 2), None]),
                 dict(k_cache=[bf(7, 2, 16, 64), None]), dict(v_cache=[u8(6, 2, 16, 64), None]), dict(k_scale=[u8(7, 2, 2), None]),
                 dict(v_scale=[torch.zeros(7, 2, 1), None]), dict(q=[bf(2, 4, 64), bf(2, 2, 64)]), dict(q_out=[bf(2, 4, 64), bf(4, 2, 64)[::2]]),
                 dict(lengths=i32(3)), dict(lengths=i32(2).long()), dict(block_table=i32(3, 2).t()), dict(first=i32(2))):
        with pytest.raises(ValueError):
            tokens_call(kvp, **over)()
    for over in (dict(q=[bf(2, 4, 64), torch.zeros(2, 4, 64)]), dict(k_cache=[bf(7, 2, 16, 64), None]), dict(v_scale=[u8(7, 3), None]), dict(lse=[bf(2, 4)] * 2),
                 dict(o=[bf(2, 4, 128)[..., ::2]] * 2), dict(lengths=i32(1)), dict(block_table=i32(2, 4))):
        with pytest.raises(ValueError):
            decode_call(kvp, **over)()


def test_decode8_refused_by_the_library(kvp):
    one = [None, None]
    for over in (dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(layer_begin=1, layer_end=1), dict(layer_begin=-1), dict(layer_end=3), dict(q=one),
                 dict(k_cache=one), dict(v_cache=one), dict(k_scale=one), dict(v_scale=one), dict(o=one), dict(lse=one), dict(q=[])):
        refused(kvp, decode_call(kvp, **over), kvp.ERR_INVALID_ARG)
    for over in (dict(dh=32), dict(page=24), dict(Hq=34, Hkv=2)):
        if over.get("page"):
            over.update(k_scale=[torch.zeros(21, dtype=torch.uint8), None], v_scale=[torch.zeros(21, dtype=torch.uint8), None])
        refused(kvp, decode_call(kvp, **over), kvp.ERR_UNSUPPORTED)
    refused(kvp, decode_call(kvp, ws=torch.zeros(16, dtype=torch.uint8)), kvp.ERR_WORKSPACE)
    refused(kvp, decode_call(kvp, ws=None), kvp.ERR_WORKSPACE)
    for donor in ((0,), (0, 2), (1, 1)):
        refused(kvp, decode_call(kvp, donor=donor), kvp.ERR_BAD_DONOR)
    d = kvp.DecodeDesc(2, 2, 4, 2, 64, 16, 3, 7)
    assert kvp.decode8_workspace_bytes(d, [0]) == 0 and kvp.decode8_workspace_bytes(d, [0, 2]) == 0 and kvp.decode8_workspace_bytes(d, [0, 0]) > 0
    assert kvp.decode8_workspace_bytes(kvp.DecodeDesc(2, 2, 4, 2, 64, 16, 1 << 27, 7), [0, 0]) == 0    # positions beyond 32 bits


def test_a_workspace_serves_every_layer_range(kvp):
    """Ranges leave members of groups out; none needs more than the whole stack's bytes."""
    rng = random.Random(5)
    for _ in range(60):
        L, G = rng.randint(1, 9), rng.choice((1, 2, 4, 8, 16))
        donor = []
        for l in range(L):
            donor.append(l if l == 0 or rng.random() < 0.4 else rng.choice([x for x in set(donor)]))
        desc = kvp.DecodeDesc(L, rng.randint(1, 40), 2 * G, 2, rng.choice((64, 128)), 16, rng.randint(1, 4000), 5, rng.choice((0, 0, 3)))
        need = kvp.decode8_workspace_bytes(desc, donor)
        for a in range(L):
            for b in range(a + 1, L + 1):
                got = kvp.lib.kvp_decode8(C.byref(desc), kvp._donors(donor), 0.0, *[(C.c_void_p * L)(*[4096] * L)] * 5, 4096, 4096,
                                          *[(C.c_void_p * L)(*[4096] * L)] * 2, a, b, 4096, need, None)
                assert got == kvp.ERR_CUDA, (donor, a, b)       # every check passed, the workspace's among them


# ---------------------------------------------------------------------------------------------
# what the native calls hand over
# ---------------------------------------------------------------------------------------------
FORMS = {"cache_append_tokens": "SDipfAAAAAAAAppp", "decode8": "SDfAAAAAppAAiiplp"}
TYPES = dict(i=C.c_int, l=C.c_size_t, f=C.c_float, p=C.c_void_p, S=C.c_void_p, D=C.c_void_p, A=C.c_void_p)


def test_both_paths_hand_over_the_same(monkeypatch):
    """Sizes, pointers and null arrays reach the library alike by the native and the ctypes path; unusual lists go by the latter."""
    from paper_2608_15943_b200 import kvp
    if torch.cuda.is_available():
        pytest.skip("host tensors")
    seen, keep = [], []
    for name, form in FORMS.items():
        def called(*args, name=name, form=form):
            layers = C.cast(args[0], C.POINTER(C.c_int32))[0]
            read = {"S": lambda v: C.string_at(v, C.sizeof(kvp.DecodeDesc)), "D": lambda v: C.string_at(v, 4 * layers),
                    "A": lambda v: v and C.string_at(v, 8 * layers)}
            seen.append([name] + [read.get(k, lambda v: v)(v) for k, v in zip(form, args)])
            return 0
        keep.append(C.CFUNCTYPE(C.c_int, *[TYPES[k] for k in form])(called))
        monkeypatch.setattr(kvp.lib, "kvp_" + name, keep[-1])
    real = kvp._pack
    original = [C.cast(getattr(C.CDLL(kvp.LIB_PATH), "kvp_" + n), C.c_void_p).value for n in FORMS]
    monkeypatch.setattr(kvp, "_call_place", lambda: (-2, 0x7f0000001238))
    none = types.SimpleNamespace(cache_append_tokens=lambda *a: NotImplemented, decode8=lambda *a: NotImplemented, pointers=real.pointers, donors=real.donors)
    real.bind_cache([C.cast(cb, C.c_void_p).value for cb in keep])
    try:
        first = torch.tensor([0, 1, 2], dtype=torch.int32)
        calls = [tokens_call(kvp, **o) for o in ({}, dict(bits8=False), dict(dtype=1), dict(q=None, q_out=None, theta=0.0), dict(first=first), dict(T=7, first=first),
                                                 dict(donor=(0, 1), k_new=[torch.zeros(2, 2, 64, dtype=torch.bfloat16)] * 2, L=2))]
        calls += [decode_call(kvp, **o) for o in ({}, dict(dtype=1), dict(scale=0.25, layer_begin=1), dict(layer_end=1), dict(splits=4))]
        for call in calls:
            del seen[:]
            monkeypatch.setattr(kvp, "_pack", real)
            call()
            monkeypatch.setattr(kvp, "_pack", none)
            call()
            a, b = seen
            for k, x, y in zip("." + FORMS[a[0]], a, b):
                if k != "A":
                    assert x == y, (a[0], k)
                    continue
                assert (x is None) == (y is None)
                for i in range(0, len(x or b""), 8):      # (the native path hands over what the call looks at alone)
                    assert x[i:i + 8] in (y[i:i + 8], bytes(8))
        monkeypatch.setattr(kvp, "_pack", real)

        class Sub(torch.Tensor):
            pass
        del seen[:]
        tokens_call(kvp, lengths=torch.ones(2, dtype=torch.int32).as_subclass(Sub))()
        decode_call(kvp, scale=0)()
        assert len(seen) == 2
    finally:
        real.bind_cache(original)


@pytest.mark.parametrize("bits8", [True, False])
def test_owners_without_rows_are_refused(kvp, bits8):
    """Runs of tokens whose rows are missing or are None: no number of tokens can be read off them, and nothing would be stored."""
    runs = dict(T=5, first=torch.tensor([0, 2, 5], dtype=torch.int32), q=None, q_out=None, bits8=bits8)
    none = torch.zeros(0, 2, 64, dtype=torch.bfloat16)
    for over in (dict(k_new=[None], v_new=[None]), dict(k_new=[], v_new=[]), dict(k_new=[None, None]), dict(v_new=[None, None], k_new=[none, None]),
                 dict(k_new=[None, none], v_new=[none, none]), dict(donor=(0, 1), k_new=[none, None], v_new=[none, none], k_cache=None, v_cache=None)):
        if "k_cache" in over:                                 # an owner above the first one
            pool = torch.zeros(7, 2, 16, 64, dtype=torch.uint8 if bits8 else torch.bfloat16)
            scale = torch.zeros(7, 2, 1, dtype=torch.uint8)
            over.update(k_cache=[pool] * 2, v_cache=[pool] * 2, k_scale=[scale] * 2 if bits8 else None, v_scale=[scale] * 2 if bits8 else None)
        refused(kvp, tokens_call(kvp, **(runs | over)), kvp.ERR_INVALID_ARG)
    tokens_call(kvp, **(runs | dict(k_new=[none, None], v_new=[none, None])))()      # rows there are, none of them: nothing to do
