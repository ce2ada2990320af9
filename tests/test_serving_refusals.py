"""Paged cache, tree attention, beam search: what is refused on the host, before anything is launched (no GPU needed; the
pointers are never followed), and the oracle's own definitions on cases small enough to do by hand."""
import ctypes as C

import numpy as np
import pytest

import paper_2604_15356_b200 as plc
from paper_2604_15356_b200 import serving

A, B, WS = 1 << 20, 1 << 24, 1 << 28                     # "device addresses"


@pytest.fixture(scope="module")
def lib():
    plc.build()
    return plc.lib()


def pool(L=2, H=4, d=64, pages=32, page=16, dtype=plc.OUT_F16, base=A, **strides):
    st = dict(layer=2 * pages * page * H * d, kv=pages * page * H * d, session=page * H * d, head=page * d, pos=d)
    st.update(strides)
    return serving.PagePoolC(plc.KVView(base, st["layer"], st["kv"], st["session"], st["head"], st["pos"]), L, H, d, pages, page, dtype)


def book(at=B, rows=3, cols=5):
    return serving.PageBookC(at, at + 4096, at + 8192, rows, cols)


def fork(lib, p, i, o, parent=A, ws=WS, ws_bytes=1 << 20, status=A):
    return lib.plc_pages_fork(C.byref(p), C.byref(i), C.c_void_p(parent), None, C.byref(o), C.c_void_p(ws), C.c_uint64(ws_bytes),
                              C.c_void_p(status), None)


@pytest.mark.parametrize("change, code", [
    (dict(base=0), plc.E_INVALID), (dict(base=A + 8), plc.E_ALIGN), (dict(d=48), plc.E_SHAPE), (dict(d=512), plc.E_SHAPE),
    (dict(pages=0), plc.E_INVALID), (dict(page=0), plc.E_INVALID), (dict(L=0), plc.E_INVALID), (dict(H=0), plc.E_INVALID),
    (dict(dtype=3), plc.E_INVALID), (dict(pos=68), plc.E_ALIGN), (dict(session=4), plc.E_ALIGN), (dict(pages=1 << 29), plc.E_SHAPE)])
def test_pools_that_are_refused(lib, change, code):
    p, o = pool(**change), book(B + (1 << 20))
    i = book()
    assert fork(lib, p, i, o) == code
    assert lib.plc_pages_keep(C.byref(p), C.byref(i), C.c_void_p(A), C.c_void_p(A), 4, C.byref(o), C.c_void_p(A), None) == code
    assert lib.plc_pages_compact(C.byref(p), C.byref(i), C.byref(o), C.c_void_p(A), C.c_void_p(WS), C.c_uint64(1 << 20), C.c_void_p(A), None) == code
    b = C.c_uint64()
    assert lib.plc_tree_attention_workspace(C.byref(p), 3, 4, 7, C.byref(b)) == code


def test_books_and_workspaces_that_are_refused(lib):
    p, i, o = pool(), book(), book(B + (1 << 20))
    assert fork(lib, p, i, i) == plc.E_INVALID                                     # the same arrays on both sides
    assert fork(lib, p, i, serving.PageBookC(B + 40, B + 9000000, B + 9100000, 3, 5)) == plc.E_INVALID   # overlapping tables
    assert fork(lib, p, i, book(B + (1 << 20), cols=6)) == plc.E_SHAPE
    assert fork(lib, p, book(rows=0), o) == plc.E_INVALID and fork(lib, p, i, book(B + (1 << 20), rows=1 << 21)) == plc.E_SHAPE
    assert fork(lib, p, i, o, parent=0) == plc.E_INVALID and fork(lib, p, i, o, status=0) == plc.E_INVALID
    assert fork(lib, p, i, o, ws=0) == plc.E_INVALID and fork(lib, p, i, o, ws=WS + 4) == plc.E_ALIGN
    b = C.c_uint64()
    assert lib.plc_pages_workspace(32, 3, 3, C.byref(b)) == plc.OK and b.value >= 4 * 32
    assert fork(lib, p, i, o, ws_bytes=b.value - 1) == plc.E_CAPACITY
    assert lib.plc_pages_workspace(0, 3, 3, C.byref(b)) == plc.E_INVALID
    k = lambda rows, stride: lib.plc_pages_keep(C.byref(p), C.byref(i), C.c_void_p(A), C.c_void_p(A), stride,  # noqa: E731
                                                C.byref(book(B + (1 << 20), rows=rows)), C.c_void_p(A), None)
    assert k(4, 4) == plc.E_SHAPE and k(3, 0) == plc.E_INVALID
    assert lib.plc_pages_compact(C.byref(p), C.byref(i), C.byref(o), None, C.c_void_p(WS), C.c_uint64(1 << 20), C.c_void_p(A), None) == plc.E_INVALID


def queries(**change):
    t = dict(q_dev=A, q_stride_row=512, q_stride_head=64, out_dev=B, out_stride_row=512, out_stride_head=64, lse_dev=None, begin_dev=A,
             mask_dev=A, n_rows=7, n_heads=8, mask_words=1)
    t.update(change)
    return serving.TreeQueries(**t)


@pytest.mark.parametrize("change, code", [
    (dict(q_dev=None), plc.E_INVALID), (dict(out_dev=None), plc.E_INVALID), (dict(begin_dev=None), plc.E_INVALID), (dict(n_rows=-1), plc.E_INVALID),
    (dict(n_heads=0), plc.E_INVALID), (dict(n_heads=6), plc.E_SHAPE), (dict(mask_words=0), plc.E_INVALID), (dict(q_dev=A + 2), plc.E_ALIGN),
    (dict(q_stride_row=516), plc.E_ALIGN), (dict(out_stride_head=68), plc.E_ALIGN)])
def test_queries_that_are_refused(lib, change, code):
    p, b, t, n = pool(), book(), queries(**change), C.c_uint64()
    assert lib.plc_tree_attention_workspace(C.byref(p), 3, 8, 7, C.byref(n)) == plc.OK
    call = lambda layer, scale, p, bytes_: lib.plc_tree_attention(C.byref(p), layer, C.byref(b), C.byref(t), C.c_float(scale), C.c_void_p(WS),  # noqa: E731
                                                                  C.c_uint64(bytes_), C.c_void_p(A), None)
    assert call(0, 0.125, p, n.value) == code
    t = queries()
    for layer, scale, q, bytes_, want in ((2, 0.1, p, n.value, plc.E_INVALID), (-1, 0.1, p, n.value, plc.E_INVALID), (0, 0.0, p, n.value, plc.E_INVALID),
                                          (0, float("nan"), p, n.value, plc.E_INVALID), (0, 0.1, pool(dtype=plc.OUT_F32), n.value, plc.E_INVALID),
                                          (0, 0.1, p, n.value - 1, plc.E_CAPACITY)):
        assert call(layer, scale, q, bytes_) == want


def test_beam_calls_that_are_refused(lib):
    def select(S=2, W=4, V=100, n_out=4, logits=A, dtype=plc.OUT_F16, score=A, done=0, eos=2, ws=WS, bytes_=1 << 20):
        return lib.plc_beam_select(C.c_void_p(logits), dtype, C.c_int64(V), S, W, V, C.c_void_p(score), C.c_void_p(done), eos, n_out, C.c_void_p(A),
                                   C.c_void_p(A), C.c_void_p(A), C.c_void_p(ws), C.c_uint64(bytes_), None)
    for kw in (dict(S=0), dict(W=0), dict(V=0), dict(n_out=0), dict(logits=0), dict(dtype=3), dict(score=0), dict(done=A, eos=-1), dict(done=A, eos=100),
               dict(ws=0)):
        assert select(**kw) == plc.E_INVALID, kw
    assert select(W=129) == plc.E_SHAPE and select(n_out=129) == plc.E_SHAPE
    assert select(logits=A + 1) == plc.E_ALIGN and select(logits=A + 2, dtype=plc.OUT_F32) == plc.E_ALIGN and select(ws=WS + 8) == plc.E_ALIGN
    b = C.c_uint64()
    assert lib.plc_beam_workspace(2, 4, 100, 4, C.byref(b)) == plc.OK and select(bytes_=b.value - 1) == plc.E_CAPACITY
    for S, W, V, n in ((1, 1, 1, 1), (1, 128, 128256, 128), (256, 16, 32000, 32), (1, 1, 10 ** 6, 1)):
        assert lib.plc_beam_workspace(S, W, V, n, C.byref(b)) == plc.OK and 0 < b.value < S * W * (V // 4096 + 1) * (8 * n + 12) + 1

    def reorder(src=A, dst=B, ss=100, ds=100, n=100, sets=1, rows=(4, 4), parent=A):
        arr = (serving.RowSet * 17)(*[serving.RowSet(src, dst, ss, ds, n)] * 17)
        return lib.plc_beam_reorder(arr, sets, C.c_void_p(parent), rows[0], rows[1], None, None)
    for kw in (dict(src=0), dict(dst=0), dict(n=0), dict(ss=-1), dict(ds=99), dict(dst=A + 399), dict(sets=0), dict(rows=(0, 1)), dict(rows=(1, 0)),
               dict(parent=0)):
        assert reorder(**kw) == plc.E_INVALID, kw
    assert reorder(sets=17) == plc.E_SHAPE


def test_the_oracle_by_hand():
    from oracle import serving as o
    table = np.array([[3, 1, -1], [3, 0, -1]], np.int32)                   # two rows share page 3, page 4 and 2 are free
    length, ref = np.array([5, 4], np.int32), np.array([1, 1, 0, 2, 0], np.int32)
    t, n, r, copies, bits = o.fork(table, length, ref, [0, 0, -1], [0, 4, 9], 4)
    assert t.tolist() == [[3, 1, -1], [3, 2, 4], [-1, -1, -1]] and n.tolist() == [5, 5, 0] and bits == 0
    assert copies == [(1, 2, 1)] and r.tolist() == [0, 1, 1, 2, 1]         # row 1's spare page 0 is released
    assert o.fork(table, length, ref, [0, 0, 0], [0, 4, 4], 4)[4] == o.CAPACITY
    t, n, r, moves, bits = o.keep(np.array([[3, 1, 0]], np.int32), np.array([3], np.int32), np.array([1, 1, 0, 1], np.int32), np.array([[1, 4]]), [2], 4)
    assert moves == [(0, 4, 3), (0, 7, 4)] and n.tolist() == [5] and t.tolist() == [[3, 1, -1]] and r.tolist() == [0, 1, 0, 1] and bits == 0
    t, r, moved = o.compact(table, ref)
    assert moved.tolist() == [0, 1, -1, 2, -1] and t.tolist() == [[2, 1, -1], [2, 0, -1]] and r.tolist() == [1, 1, 2, 0, 0]
    x = np.log(np.array([[[.5, .25, .25], [.2, .2, .6]]]))
    s, p, k = o.beam_select(x, np.log(np.array([[.4, .6]])), 4)
    assert np.allclose(np.exp(s), [[.36, .2, .12, .12]]) and p.tolist() == [[1, 0, 1, 1]] and k.tolist() == [[2, 0, 0, 1]]


def test_the_binding_checks_its_tensors():
    import torch
    kv = torch.zeros(1, 2, 4, 1, 8, 32, dtype=torch.float16)
    with pytest.raises(plc.PlcError) as e:
        plc.PagePool(kv)                                                   # not on a GPU
    assert e.value.code == plc.E_INVALID
    with pytest.raises(plc.PlcError):
        plc.PagePool(kv[0])
    i = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(plc.PlcError):
        plc.PageBook(i, i, i)
    with pytest.raises(plc.PlcError):
        plc.PageBook(i.view(1, 3), i[:1], i.long())
    with pytest.raises(plc.PlcError):
        plc.beam_select(torch.zeros(1, 2, 8), torch.zeros(1, 2), 2)
    with pytest.raises(plc.PlcError):
        plc.beam_reorder(i, [i])


@pytest.mark.parametrize("low", [float(np.finfo(np.float32).min), -3.3895313892515355e38, -65504.0, -1e9])
def test_the_oracle_at_the_lowest_values(low):
    """A beam whose tokens all are masked with one value has each at its own score less log V, and does not pass a live one."""
    from oracle import serving as o
    V = 32000
    x = np.full((1, 2, V), low)
    x[0, 1] = 0.0
    x[0, 1, 7] = 20.0
    s, p, k = o.beam_select(x, np.array([[-20.0, -30.0]]), 3)
    live = -30.0 - np.log(np.exp(-20.0) * (V - 1) + 1)
    assert p.tolist() == [[1, 0, 0]] and k.tolist() == [[7, 0, 1]]
    assert np.allclose(s, [[live, -20.0 - np.log(V), -20.0 - np.log(V)]], rtol=1e-13)


class _Reached:
    """Stands in for the library: notes which calls come through, and does nothing."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            return plc.OK
        return call


def _session_pages(kind, L=2, H=4, d=64, pages=12, page=16):
    import torch
    p = plc.PagePool.__new__(plc.PagePool)
    p.kv = torch.zeros(L, 2, pages, page, H, d, dtype={plc.OUT_F16: torch.float16, plc.OUT_BF16: torch.bfloat16, plc.OUT_F32: torch.float32}[kind]).transpose(3, 4)
    p._c = serving.PagePoolC(plc.kv_view(p.kv), L, H, d, pages, page, kind)
    return p


def _codec_calls(monkeypatch, out_dtype, L=2, H=4, d=64, V=8):
    """Context without a library behind it -> the calls that take a view, by name: (what it needs, the call)."""
    import torch
    ctx = plc.Context.__new__(plc.Context)
    ctx.cfg, ctx.T, ctx._h = plc.Config(L, H, d, V, 4, 0.02, 0.0, 32, 0, out_dtype), None, C.c_void_p()
    lib = _Reached()
    monkeypatch.setattr(plc, "lib", lambda: lib)
    monkeypatch.setattr(plc, "_stream", lambda: None)

    class St:
        c = staticmethod(plc.Streams)
    x = lambda S, n: torch.zeros(S, n, V, dtype=torch.float16)  # noqa: E731
    rec, par, tok = torch.zeros(16, dtype=torch.uint8), plc.RotqParams(), torch.zeros(4, dtype=torch.int32)
    return lib, {"plc_encode": (plc.OUT_F16, lambda v, S, n: ctx.encode(v, x(S, n), St)), "plc_decode": (out_dtype, lambda v, S, n: ctx.decode(St, x(S, n), v)),
                 "plc_encode_adaptive": (plc.OUT_F16, lambda v, S, n: ctx.encode(v, x(S, n), St, tokens=tok)),
                 "plc_decode_adaptive": (out_dtype, lambda v, S, n: ctx.decode(St, x(S, n), v, tokens=tok)),
                 "plc_encode_rotq": (plc.OUT_F16, lambda v, S, n: ctx.encode_rotq(v, x(S, n), par, rec)),
                 "plc_decode_rotq": (out_dtype, lambda v, S, n: ctx.decode_rotq(rec, x(S, n), par, v))}


@pytest.mark.parametrize("out_dtype", [plc.OUT_F16, plc.OUT_F32])
@pytest.mark.parametrize("kind", [plc.OUT_F16, plc.OUT_BF16, plc.OUT_F32])
def test_pages_of_another_type_are_not_coded(monkeypatch, kind, out_dtype):
    """A run of pages is taken by the codec's calls in the pool's own type alone, and as far as it reaches."""
    view = _session_pages(kind).sessions_view(1, 3, 40)
    lib, calls = _codec_calls(monkeypatch, out_dtype)
    for name, (needs, call) in calls.items():
        del lib.calls[:]
        if needs != kind:
            with pytest.raises(plc.PlcError) as e:
                call(view, 3, 40)
            assert e.value.code == plc.E_INVALID and lib.calls == [], name
            continue
        call(view, 3, 40)
        call(view, 1, 48)                                                  # a session has three pages
        assert lib.calls == [name, name]
        for S, n in ((4, 40), (3, 49)):
            with pytest.raises(plc.PlcError) as e:
                call(view, S, n)
            assert e.value.code == plc.E_SHAPE and lib.calls == [name, name], name


@pytest.mark.parametrize("change", [dict(L=3), dict(H=5), dict(d=128), dict(d=32)])
def test_pages_of_another_shape_are_not_coded(monkeypatch, change):
    view = _session_pages(plc.OUT_F16).sessions_view(0, 2, 20)
    lib, calls = _codec_calls(monkeypatch, plc.OUT_F16, **change)
    for name, (_, call) in calls.items():
        with pytest.raises(plc.PlcError) as e:
            call(view, 2, 20)
        assert e.value.code == plc.E_SHAPE and lib.calls == [], name


def test_status_words_that_are_refused(lib):
    take = lambda a, b: lib.plc_take_status(C.c_void_p(a), C.c_void_p(b), None)  # noqa: E731
    assert take(0, B) == plc.E_INVALID and take(A, 0) == plc.E_INVALID and take(A, A) == plc.E_INVALID
    assert take(A + 2, B) == plc.E_ALIGN and take(A, B + 1) == plc.E_ALIGN


@pytest.mark.parametrize("V", [2 ** 31 - 1, 2 ** 31 - 64, 2 ** 31 - 4096, 2 ** 31 - 2 ** 16 + 1])
def test_vocabularies_near_two_to_the_31_are_refused(lib, V):
    """A column with a block's logits added has to be an int."""
    b = C.c_uint64()
    assert lib.plc_beam_workspace(1, 1, V, 4, C.byref(b)) == plc.E_SHAPE
    assert lib.plc_beam_select(C.c_void_p(A), plc.OUT_F16, C.c_int64(V), 1, 1, V, C.c_void_p(A), None, -1, 4, C.c_void_p(A), C.c_void_p(A), C.c_void_p(A),
                               C.c_void_p(WS), C.c_uint64(1 << 20), None) == plc.E_SHAPE
    assert lib.plc_beam_workspace(1, 1, 2 ** 31 - 2 ** 16, 4, C.byref(b)) == plc.OK and 0 < b.value <= 64 * (8 * 4 + 12)


@pytest.mark.parametrize("out_dtype", [plc.OUT_F16, plc.OUT_F32])
def test_tensors_of_another_width_are_not_coded(monkeypatch, out_dtype):
    """Elements of half the size would be written past the tensor's end."""
    import torch
    lib, calls = _codec_calls(monkeypatch, out_dtype)
    for name, (needs, call) in calls.items():
        for dtype in (torch.float16, torch.bfloat16, torch.float32, torch.uint8):
            kv = torch.zeros(2, 2, 3, 4, 40, 64, dtype=dtype)
            del lib.calls[:]
            if dtype.itemsize == (4 if needs == plc.OUT_F32 else 2):
                call(kv, 3, 40)
                assert lib.calls == [name]
                continue
            with pytest.raises(plc.PlcError) as e:
                call(kv, 3, 40)
            assert e.value.code == plc.E_INVALID and lib.calls == [], (name, dtype)
