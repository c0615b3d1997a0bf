"""What the calls on new tokens and on pages refuse, before anything reaches the device; the pages' oracle by itself."""
import ctypes as C
import random
import types

import pytest
import torch

from oracle.pages import Book


@pytest.fixture(scope="module")
def kvp():
    from paper_2608_15943_b200 import build
    build.build()
    from paper_2608_15943_b200 import kvp as mod
    return mod


@pytest.fixture
def as_on_a_device(kvp, monkeypatch):
    """Tensors on the host pass the look at their device, and the call stops at the library's own checks."""
    monkeypatch.setattr(kvp, "_call_place", lambda: (-2, 0))


NATIVE = ("attn_chunk", "pages_copy", "pages_fork", "pages_resize", "pages_trim", "pages_compact")


@pytest.fixture(params=["native", "ctypes"], autouse=True)
def path(request, kvp, monkeypatch):
    """Both ways into the library: the native module, and what it leaves to the binding."""
    if request.param == "ctypes":
        monkeypatch.setattr(kvp, "_pack", types.SimpleNamespace(**{n: lambda *a: NotImplemented for n in NATIVE}))


@pytest.fixture
def unseen(kvp, as_on_a_device, monkeypatch):
    """The binding does not look at the tensors: what the library itself refuses."""
    monkeypatch.setattr(kvp, "_fit", lambda *a: None)


BF, I32 = torch.bfloat16, torch.int32


def chunk_args(kvp, L=2, B=3, Hq=4, Hkv=2, dh=64, page=16, max_pages=4, n_pages=12, T=7, bits8=False, dtype=BF):
    a = types.SimpleNamespace()
    a.desc = kvp.DecodeDesc(L, B, Hq, Hkv, dh, page, max_pages, n_pages, 0, kvp.F32 if dtype == torch.float32 else kvp.BF16)
    a.donor = [0] * L
    rows = lambda *s, t=dtype: [torch.zeros(*s, dtype=t) for _ in range(L)]
    a.q, a.o, a.lse = rows(T, Hq, dh), rows(T, Hq, dh), rows(T, Hq, t=torch.float32)
    pool = lambda: [torch.zeros(n_pages, Hkv, page, dh, dtype=torch.uint8 if bits8 else BF)] + [None] * (L - 1)
    a.k, a.v = pool(), pool()
    scales = lambda: [torch.zeros(n_pages, Hkv, page // 16, dtype=torch.uint8)] + [None] * (L - 1)
    a.ks, a.vs = (scales(), scales()) if bits8 else (None, None)
    a.table, a.lengths, a.first = torch.zeros(B, max_pages, dtype=I32), torch.zeros(B, dtype=I32), torch.zeros(B + 1, dtype=I32)
    a.ws = torch.zeros(max(1, kvp.attn_chunk_workspace_bytes(a.desc, a.donor, T)), dtype=torch.uint8)
    a.kw = {}
    return a


def chunk(kvp, a):
    kvp.attn_chunk(a.desc, a.donor, a.q, a.k, a.v, a.table, a.lengths, a.o, a.lse, a.ws, first=a.first, k_scale=a.ks, v_scale=a.vs, **a.kw)


def set_(path, value):
    def change(a):
        *head, last = path.split(".")
        for name in head:
            a = getattr(a, name)
        if isinstance(value, dict):
            getattr(a, last).update(value)
        elif "[" in last:
            name, i = last[:-1].split("[")
            getattr(a, name)[int(i)] = value
        else:
            setattr(a, last, value)
    return change


INVALID, BAD_DONOR, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4


@pytest.mark.parametrize("change,status", [
    (set_("desc.dh", 96), UNSUPPORTED), (set_("desc.page_size", 24), UNSUPPORTED), (set_("desc.Hq", 5), UNSUPPORTED),
    (set_("desc.B", 0), INVALID), (set_("desc.max_pages", 1 << 27), UNSUPPORTED), (set_("desc.dtype", 7), UNSUPPORTED),
    (set_("donor", [0, 2]), BAD_DONOR), (set_("donor", [0]), BAD_DONOR), (set_("donor", [1, 1]), BAD_DONOR),
    (set_("kw", dict(window=-1)), INVALID), (set_("kw", dict(sinks=4)), INVALID), (set_("kw", dict(window=3, sinks=-1)), INVALID),
    (set_("kw", dict(scale=-1.0)), INVALID), (set_("kw", dict(scale=float("nan"))), INVALID), (set_("kw", dict(scale=float("inf"))), INVALID),
    (set_("kw", dict(layer_begin=1, layer_end=1)), INVALID), (set_("kw", dict(layer_end=3)), INVALID), (set_("kw", dict(layer_begin=-1)), INVALID),
    (set_("q[1]", None), INVALID), (set_("o[0]", None), INVALID), (set_("lse[1]", None), INVALID), (set_("k[0]", None), INVALID),
    (set_("v[0]", None), INVALID), (set_("ws", None), WORKSPACE), (set_("ws", torch.zeros(16, dtype=torch.uint8)), WORKSPACE),
    (set_("first", None), INVALID), (set_("ks", [torch.zeros(12, 2, 1, dtype=torch.uint8), None]), INVALID),
])
def test_refusals_of_attention(kvp, unseen, change, status):
    a = chunk_args(kvp)
    change(a)
    with pytest.raises(kvp.KvpError) as e:
        chunk(kvp, a)
    assert e.value.status == status


@pytest.mark.parametrize("change", [
    set_("q[0]", torch.zeros(7, 4, 64)), set_("q[1]", torch.zeros(6, 4, 64, dtype=BF)), set_("o[0]", torch.zeros(7, 64, 4, dtype=BF).transpose(1, 2)),
    set_("lse[0]", torch.zeros(7, 4, dtype=BF)), set_("lse[0]", torch.zeros(4, 4)), set_("k[0]", torch.zeros(11, 2, 16, 64, dtype=BF)),
    set_("k[0]", torch.zeros(12, 2, 16, 64, dtype=torch.uint8)), set_("table", torch.zeros(3, 5, dtype=I32)), set_("table", torch.zeros(3, 4)),
    set_("lengths", torch.zeros(3, dtype=torch.int64)), set_("lengths", torch.zeros(2, dtype=I32)), set_("first", torch.zeros(3, dtype=I32)),
])
def test_tensors_that_do_not_fit(kvp, as_on_a_device, change):
    a = chunk_args(kvp)
    change(a)
    with pytest.raises(ValueError):
        chunk(kvp, a)


def test_scales_come_in_pairs_and_alignment(kvp, as_on_a_device):
    a = chunk_args(kvp, bits8=True)
    a.vs = None
    with pytest.raises(kvp.KvpError) as e:
        chunk(kvp, a)
    assert e.value.status == INVALID
    a = chunk_args(kvp, bits8=True)
    a.vs = [None, None]
    with pytest.raises(kvp.KvpError) as e:
        chunk(kvp, a)
    assert e.value.status == INVALID
    a = chunk_args(kvp)
    a.q[0] = torch.zeros(7 * 4 * 64 + 1, dtype=BF)[1:].view(7, 4, 64)
    with pytest.raises(kvp.KvpError) as e:
        chunk(kvp, a)
    assert e.value.status == UNSUPPORTED


def test_more_rows_than_are_counted(kvp):
    some = (C.c_void_p * 1)(256)
    d = kvp.DecodeDesc(1, 1, 4, 2, 64, 16, 4, 12, 0, kvp.BF16)
    call = lambda T: kvp.lib.kvp_attn_chunk(C.byref(d), (C.c_int32 * 1)(0), T, 256, 0.0, 0, 0, some, some, some, None, None, 256, 256, some, some, 0, 1, None, 0, None)
    assert call(1 << 24) == UNSUPPORTED and call((1 << 31) - 1) == UNSUPPORTED and call((1 << 24) - 1) == WORKSPACE


def test_no_rows_are_no_work(kvp, as_on_a_device):
    a = chunk_args(kvp, T=0)
    chunk(kvp, a)
    assert kvp.attn_chunk_workspace_bytes(a.desc, [0, 2], 4) >= 0 and kvp.attn_chunk_workspace_bytes(a.desc, [0], 4) == 0
    assert kvp.attn_chunk_workspace_bytes(a.desc, a.donor, -1) == 0
    sizes = [kvp.attn_chunk_workspace_bytes(a.desc, a.donor, T) for T in (0, 1, 7, 100, 5000)]
    assert sizes == sorted(sizes)


# ---------------------------------------------------------------------------------------------
# pages
# ---------------------------------------------------------------------------------------------
def pages_args(kvp):
    a = chunk_args(kvp)
    a.refs, a.parent, a.to, a.one = torch.zeros(12, dtype=I32), torch.zeros(3, dtype=I32), torch.zeros(3, dtype=I32), torch.zeros(1, dtype=I32)
    a.src, a.dst = torch.zeros(2, dtype=I32), torch.zeros(2, dtype=I32)
    a.ws = torch.zeros(kvp.pages_workspace_bytes(a.desc), dtype=torch.uint8)
    return a


CALLS = {
    "copy": lambda k, a: k.pages_copy(a.desc, a.donor, a.src, a.dst, a.k, a.v, a.ks, a.vs),
    "fork": lambda k, a: k.pages_fork(a.desc, a.parent, a.refs, a.table, a.lengths, a.ws),
    "resize": lambda k, a: k.pages_resize(a.desc, a.donor, a.to, a.refs, a.table, a.lengths, a.one, a.ws, a.k, a.v, a.ks, a.vs),
    "trim": lambda k, a: k.pages_trim(a.desc, a.kw.get("window", 4), a.kw.get("sinks", 0), a.refs, a.table, a.lengths),
    "compact": lambda k, a: k.pages_compact(a.desc, a.donor, a.refs, a.table, a.lengths, a.one, a.ws, a.k, a.v, a.ks, a.vs),
}
POOLED, BOOKED = ("copy", "resize", "compact"), ("fork", "resize", "compact")


@pytest.mark.parametrize("calls,change,status", [
    (tuple(CALLS), set_("desc.dh", 32), UNSUPPORTED), (tuple(CALLS), set_("desc.page_size", 8), UNSUPPORTED), (tuple(CALLS), set_("desc.n_pages", 0), INVALID),
    (POOLED, set_("donor", [0, 2]), BAD_DONOR), (POOLED, set_("donor", [0]), BAD_DONOR), (POOLED, set_("k[0]", None), INVALID), (POOLED, set_("v[0]", None), INVALID),
    (POOLED, set_("vs", [torch.zeros(12, 2, 1, dtype=torch.uint8), None]), INVALID),
    (BOOKED, set_("ws", None), WORKSPACE), (BOOKED, set_("ws", torch.zeros(64, dtype=torch.uint8)), WORKSPACE),
    (("trim",), set_("kw", dict(window=0)), INVALID), (("trim",), set_("kw", dict(sinks=-1)), INVALID),
    (("fork", "resize", "trim", "compact"), set_("refs", None), INVALID), (("fork", "resize", "trim", "compact"), set_("table", None), INVALID),
    (("fork", "resize", "trim", "compact"), set_("lengths", None), INVALID), (("resize", "compact"), set_("one", None), INVALID),
    (("fork",), set_("parent", None), INVALID), (("resize",), set_("to", None), INVALID),
])
def test_refusals_of_pages(kvp, unseen, calls, change, status):
    for name in calls:
        a = pages_args(kvp)
        change(a)
        with pytest.raises(kvp.KvpError) as e:
            CALLS[name](kvp, a)
        assert e.value.status == status, name


@pytest.mark.parametrize("calls,change", [
    (("fork", "resize", "trim", "compact"), set_("refs", torch.zeros(11, dtype=I32))), (("fork", "resize", "trim", "compact"), set_("table", torch.zeros(3, 3, dtype=I32))),
    (("fork", "resize", "trim", "compact"), set_("lengths", torch.zeros(3))), (("fork",), set_("parent", torch.zeros(4, dtype=I32))),
    (("resize",), set_("to", torch.zeros(3, dtype=torch.int64))), (("resize", "compact"), set_("one", torch.zeros(2, dtype=I32))),
    (("copy",), set_("dst", torch.zeros(3, dtype=I32))), (("copy",), set_("src", torch.zeros(2))), (POOLED, set_("k[0]", torch.zeros(12, 2, 16, 32, dtype=BF))),
])
def test_book_tensors_that_do_not_fit(kvp, as_on_a_device, calls, change):
    for name in calls:
        a = pages_args(kvp)
        change(a)
        with pytest.raises(ValueError):
            CALLS[name](kvp, a)


def test_nothing_to_copy(kvp, as_on_a_device):
    a = pages_args(kvp)
    a.src = a.dst = torch.zeros(0, dtype=I32)
    CALLS["copy"](kvp, a)
    assert kvp.pages_workspace_bytes(kvp.DecodeDesc(1, (1 << 14) + 1, 4, 2, 64, 16, 4, 12)) == 0


def test_the_oracle_counts_every_place():
    r = random.Random(1)
    for _ in range(60):
        page, rows = r.choice((16, 32, 48)), r.randint(1, 7)
        book = Book(page, 6, r.randint(4, 40), rows)
        for _ in range(30):
            what = r.choice(("grow", "grow", "fork", "trim", "compact", "any"))
            if what in ("grow", "any"):
                before = (list(book.refs), [list(t) for t in book.table], list(book.lengths))
                short = book.resize([min(6 * page, n + r.randint(0, 2 * page)) if what == "grow" else r.randint(0, 6 * page) for n in book.lengths])
                assert short == 0 or before == (book.refs, book.table, book.lengths)
            elif what == "fork":
                book.fork([r.choice((b, b, -1, r.randrange(rows))) for b in range(rows)])
            elif what == "trim":
                book.trim(r.randint(1, 2 * page), r.choice((0, 4, 20)))
            else:
                used = book.compact()
                assert all(x > 0 for x in book.refs[:used]) and not any(book.refs[used:])
            assert book.consistent()


def test_the_oracle_by_hand():
    book = Book(16, 4, 8, 3)
    assert book.resize([20, 0, 0]) == 0 and book.table[0][:2] == [0, 1]
    book.fork([0, 0, 0])
    assert book.refs[:2] == [3, 3] and book.lengths == [20, 20, 20]
    assert book.resize([21, 21, 20]) == 0                     # the third row still holds page 1: both others take copies
    assert book.table[0][1] == 2 and book.table[1][1] == 3 and book.refs[:4] == [3, 1, 1, 1] and book.content[2:4] == [1, 1]
    book.fork([0, 0, -1])
    assert book.refs[:4] == [2, 0, 2, 0]
    assert book.resize([40, 22, 0]) == 0                      # both grow: the lower keeps the page
    assert book.table[0][:3] == [0, 2, 1] and book.table[1][:2] == [0, 3] and book.content[3] == 1
    assert book.resize([64, 64, 64]) == 1 + 2 + 4 - 4 and book.lengths == [40, 22, 0]
    assert book.resize([65, 0, 0]) == -1
    book.trim(3, 0)
    assert book.table[0][:3] == [-1, -1, 1] and book.table[1][:2] == [-1, 3]
    assert book.compact() == 2 and book.table[0][2] == 1 and book.table[1][1] == 0


# ---------------------------------------------------------------------------------------------
# what both paths hand over
# ---------------------------------------------------------------------------------------------
FORMS = {"attn_chunk": "SDipfiiAAAAAppAAiiplp", "pages_copy": "SDippAAAAp", "pages_fork": "Sppppplp", "pages_resize": "SDppppp" + "pl" + "AAAAp", "pages_trim": "Siipppp",
         "pages_compact": "SDpppp" + "pl" + "AAAAp"}
TYPES = dict(i=C.c_int, l=C.c_size_t, f=C.c_float, p=C.c_void_p, S=C.c_void_p, D=C.c_void_p, A=C.c_void_p)


def test_both_paths_hand_over_the_same(kvp, monkeypatch, request):
    if torch.cuda.is_available() or "ctypes" in request.node.name:
        pytest.skip("host tensors; both paths at once")
    seen, keep = [], []
    for name, form in FORMS.items():
        def called(*args, name=name, form=form):
            layers = C.cast(args[0], C.POINTER(C.c_int32))[0]
            read = {"S": lambda v: C.string_at(v, C.sizeof(kvp.DecodeDesc)), "D": lambda v: C.string_at(v, 4 * layers), "A": lambda v: v and C.string_at(v, 8 * layers)}
            seen.append([name] + [read.get(k, lambda v: v)(v) for k, v in zip(form, args)])
            return 0
        keep.append(C.CFUNCTYPE(C.c_int, *[TYPES[k] for k in form])(called))
        monkeypatch.setattr(kvp.lib, "kvp_" + name, keep[-1])
    real = kvp._pack
    original = [C.cast(getattr(C.CDLL(kvp.LIB_PATH), "kvp_" + n), C.c_void_p).value for n in FORMS]
    monkeypatch.setattr(kvp, "_call_place", lambda: (-2, 0x7f0000001238))
    none = types.SimpleNamespace(**{n: lambda *a: NotImplemented for n in NATIVE})
    real.bind_pages([C.cast(cb, C.c_void_p).value for cb in keep])
    try:
        calls = []
        for over, kw in (({}, {}), (dict(bits8=True), dict(window=9, sinks=3)), (dict(dtype=torch.float32), dict(scale=0.25, layer_begin=1)), ({}, dict(layer_end=1, window=2))):
            a = chunk_args(kvp, **over)
            a.kw = kw
            calls.append(lambda a=a: chunk(kvp, a))
        a = chunk_args(kvp, T=3)
        a.first = None
        calls.append(lambda a=a: chunk(kvp, a))
        for bits8 in (False, True):
            a = pages_args(kvp)
            if bits8:
                b = chunk_args(kvp, bits8=True)
                a.k, a.v, a.ks, a.vs = b.k, b.v, b.ks, b.vs
            a.kw = dict(window=7, sinks=2)
            calls += [lambda a=a, f=f: f(kvp, a) for f in CALLS.values()]
        for call in calls:
            del seen[:]
            monkeypatch.setattr(kvp, "_pack", real)
            call()
            monkeypatch.setattr(kvp, "_pack", none)
            call()
            x, y = seen
            assert len(x) == len(FORMS[x[0]]) + 1
            for k, u, w in zip("." + FORMS[x[0]], x, y):
                if k != "A":
                    assert u == w, (x[0], k)
                    continue
                assert (u is None) == (w is None)
                for i in range(0, len(u or b""), 8):          # (the native path hands over what the call looks at alone)
                    assert u[i:i + 8] in (w[i:i + 8], bytes(8))
    finally:
        real.bind_pages(original)
