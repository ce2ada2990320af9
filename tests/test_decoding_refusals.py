"""Rotary positions, append, attention weights, eviction, log probabilities: what is refused on the host, before anything is launched (no GPU needed; the pointers
are never followed), the frequencies, and the oracle's own definitions on cases small enough to do by hand."""
import ctypes as C
import math
from fractions import Fraction

import numpy as np
import pytest

import paper_2604_15356_b200 as plc
from paper_2604_15356_b200 import serving

A, B, WS = 1 << 20, 1 << 24, 1 << 28                     # "device addresses"


@pytest.fixture(scope="module")
def lib():
    plc.build()
    return plc.lib()


def pool(L=2, H=4, d=64, pages=32, page=16, dtype=plc.OUT_F16, base=A):
    return serving.PagePoolC(plc.KVView(base, 2 * pages * page * H * d, pages * page * H * d, page * H * d, page * d, d), L, H, d, pages, page, dtype)


def book(at=B, rows=3, cols=5):
    return serving.PageBookC(at, at + 4096, at + 8192, rows, cols)


def rotary(turns=A, dim=64, inter=0, scale=1.0):
    return serving.RotaryC(turns, dim, inter, scale)


# 1 / (2 pi) to 160 bits, from the arctangents of 1/5 and 1/239 in integers
def _inverse_turn():
    one, bits = 1 << 400, 160

    def arctan(n):
        term, total, k = one // n, one // n, 1
        while term:
            term //= -n * n
            k += 2
            total += term // k
        return total
    return Fraction((one << bits) // (2 * (16 * arctan(5) - 4 * arctan(239))), 1 << bits)


def test_turns_are_exact(lib):
    inv = _inverse_turn()
    f = [0.0, 1.0, 2 * math.pi, 0.5, 1e-3, 1e-30, 2.0 ** -60, 5e-324, 65536.0, 12345.678, math.pi] + [500000.0 ** (-2 * i / 128) for i in range(64)]
    out = (C.c_uint64 * len(f))()
    assert lib.plc_rotary_turns((C.c_double * len(f))(*f), len(f), out) == plc.OK
    for x, t in zip(f, out):
        want = math.floor(Fraction(x) * inv * (1 << 64) + Fraction(1, 2)) % (1 << 64)
        assert t == want, x
    for bad in (-1.0, float("nan"), float("inf"), 65537.0):
        assert lib.plc_rotary_turns((C.c_double * 1)(bad), 1, out) == plc.E_INVALID
    assert lib.plc_rotary_turns(None, 1, out) == plc.E_INVALID and lib.plc_rotary_turns((C.c_double * 1)(1.0), 0, out) == plc.E_INVALID


def test_frequencies():
    f = plc.rotary_frequencies(8, 10000.0)
    assert np.allclose(f, [1, 0.1, 0.01, 0.001])
    assert np.allclose(plc.rotary_frequencies(8, 10000.0, "all", 4.0), np.array(f) / 4)
    assert np.allclose(plc.rotary_frequencies(8, 10000.0, "base", 4.0)[-1], f[-1] / 4)      # the slowest pair as if all were divided
    g = plc.rotary_frequencies(8, 10000.0, "turns", 8.0, context=628, slow=1.0, fast=15.0)   # 99.9, 9.99, 0.999, 0.0999 turns
    r = 628 * np.array(f) / (2 * math.pi)
    w = np.clip((r - 1) / 14, 0, 1)
    assert np.allclose(g, w * f + (1 - w) * np.array(f) / 8) and g[0] == f[0] and g[2] == f[2] / 8
    g = plc.rotary_frequencies(8, 10000.0, "index", 8.0, context=628, slow=1.0, fast=15.0)   # from pair 0 to pair 2
    assert np.allclose(g, np.array(f) * [1, (1 + 1 / 8) / 2, 1 / 8, 1 / 8])
    for kw in (dict(ramp="other"), dict(ramp="turns"), dict(ramp="index", context=0), dict(base=0.0), dict(factor=0.0, ramp="all"), dict(ramp="turns", context=9, slow=2, fast=1)):
        with pytest.raises(plc.PlcError) as e:
            plc.rotary_frequencies(8, **kw)
        assert e.value.code == plc.E_INVALID
    with pytest.raises(plc.PlcError):
        plc.rotary_frequencies(2, ramp="base", factor=2.0)


def test_rotary_objects_that_are_refused(lib):
    for kw in (dict(dim=7), dict(dim=0), dict(dim=8, frequencies=[1.0] * 3), dict(dim=8, scale=float("nan")), dict(dim=4, frequencies=[1.0, -1.0])):
        with pytest.raises(plc.PlcError):
            plc.Rotary(device="cpu", **kw)
    r = plc.Rotary(8, base=10.0, device="cpu")
    assert r.turns.shape == (4,) and r.turns[0] == round((1 << 64) / (2 * math.pi)) or abs(int(r.turns[0]) / (1 << 64) * 2 * math.pi - 1) < 1e-15


def apply(lib, r=None, sets=None, n_sets=1, pos=A, rows=3, d=64, dtype=plc.OUT_F16, **change):
    t = dict(x_dev=A, out_dev=B, x_stride_row=256, x_stride_head=64, out_stride_row=256, out_stride_head=64, heads=4)
    t.update(change)
    s = (serving.RotarySet * 5)(*[serving.RotarySet(**t)] * 5)
    return lib.plc_rotary_apply(C.byref(r or rotary()), s, n_sets, C.c_void_p(pos), rows, d, dtype, 0, None)


def test_turns_that_are_refused(lib):
    for kw in (dict(x_dev=None), dict(out_dev=None), dict(heads=0), dict(n_sets=0), dict(pos=0), dict(rows=-1), dict(d=1), dict(dtype=3), dict(r=rotary(turns=0)),
               dict(r=rotary(scale=float("inf"))), dict(out_dev=A, out_stride_row=512), dict(out_dev=A, out_stride_head=128),
               dict(out_stride_row=0), dict(out_stride_head=0)):
        assert apply(lib, **kw) == plc.E_INVALID, kw
    for kw in (dict(n_sets=5), dict(d=2048), dict(r=rotary(dim=66)), dict(r=rotary(dim=7)), dict(r=rotary(dim=0)), dict(heads=4097), dict(heads=2049, n_sets=2)):
        assert apply(lib, **kw) == plc.E_SHAPE, kw
    for kw in (dict(x_dev=A + 1), dict(out_dev=B + 1), dict(x_dev=A + 2, dtype=plc.OUT_F32), dict(r=rotary(turns=A + 4))):
        assert apply(lib, **kw) == plc.E_ALIGN, kw
    assert apply(lib, rows=0) == plc.OK and apply(lib, rows=0, out_dev=A) == plc.OK


def tokens(**change):
    t = dict(q_dev=A, q_stride_row=512, q_stride_head=64, out_dev=B, out_stride_row=512, out_stride_head=64, k_dev=A, k_stride_row=256, k_stride_head=64, v_dev=A,
             v_stride_row=256, v_stride_head=64, begin_dev=A, pos_dev=None, n_rows=7, n_heads=8)
    t.update(change)
    return serving.NewTokens(**t)


def test_appends_that_are_refused(lib):
    def call(layer=0, p=None, b=None, r=rotary(), status=A, **change):
        return lib.plc_pages_append(C.byref(p or pool()), layer, C.byref(b or book()), C.byref(r) if r else None, C.byref(tokens(**change)), C.c_void_p(status), None)
    for kw in (dict(layer=-1), dict(layer=2), dict(status=0), dict(q_dev=None), dict(out_dev=None), dict(k_dev=None), dict(v_dev=None), dict(begin_dev=None), dict(n_rows=-1),
               dict(n_heads=-1), dict(r=rotary(turns=0)), dict(b=book(rows=0)), dict(p=pool(base=0)), dict(out_dev=A, out_stride_row=1024), dict(out_stride_row=0), dict(out_stride_head=0)):
        assert call(**kw) == plc.E_INVALID, kw
    for kw in (dict(r=rotary(dim=128)), dict(r=rotary(dim=5)), dict(p=pool(d=48)), dict(n_heads=1 << 14), dict(b=book(rows=1 << 21))):
        assert call(**kw) == plc.E_SHAPE, kw
    for kw in (dict(k_dev=A + 1), dict(v_dev=A + 1), dict(q_dev=A + 1), dict(out_dev=B + 1), dict(p=pool(base=A + 8))):
        assert call(**kw) == plc.E_ALIGN, kw
    assert call(n_rows=0) == plc.OK and call(n_rows=0, n_heads=0, q_dev=None, out_dev=None, r=None) == plc.OK


def test_weights_that_are_refused(lib):
    def call(layer=0, p=None, b=None, scale=0.125, decay=1.0, base=B, n_pos=100, status=A, ws=WS, ws_bytes=1 << 20, strides=(800, 400, 100), **change):
        t = dict(q_dev=A, q_stride_row=512, q_stride_head=64, lse_dev=A, rows_dev=None, begin_dev=A, n_rows=7, n_list=7, n_heads=8)
        t.update(change)
        q, w = serving.WeighQueries(**t), serving.Weights(base, *strides, n_pos)
        return lib.plc_pages_weigh(C.byref(p or pool()), layer, C.byref(b or book()), C.byref(q), C.c_float(scale), C.c_float(decay), C.byref(w), C.c_void_p(ws),
                                   C.c_uint64(ws_bytes), C.c_void_p(status), None)
    for kw in (dict(layer=2), dict(layer=-1), dict(ws=0, n_rows=700, n_list=700), dict(scale=0.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(decay=-1.0), dict(decay=float("inf")), dict(base=0),
               dict(n_pos=0), dict(status=0), dict(q_dev=None), dict(lse_dev=None), dict(begin_dev=None), dict(n_rows=-1), dict(n_list=-1), dict(n_heads=0),
               dict(p=pool(dtype=plc.OUT_F32)), dict(b=book(rows=0)), dict(strides=(0, 400, 100)), dict(strides=(800, 0, 100)), dict(strides=(800, 400, 0))):
        assert call(**kw) == plc.E_INVALID, kw
    for kw in (dict(n_heads=6), dict(n_list=8), dict(n_rows=1 << 29, n_list=1 << 29, n_heads=16), dict(p=pool(d=48))):
        assert call(**kw) == plc.E_SHAPE, kw
    for kw in (dict(q_dev=A + 2), dict(q_stride_row=516), dict(q_stride_head=68), dict(base=B + 2), dict(ws=WS + 8)):
        assert call(**kw) == plc.E_ALIGN, kw
    n = C.c_uint64()
    assert lib.plc_pages_weigh_workspace(C.byref(pool()), 3, 8, 7, C.byref(n)) == plc.OK and n.value == 0
    assert lib.plc_pages_weigh_workspace(C.byref(pool()), 3, 8, 700, C.byref(n)) == plc.OK and n.value > 0
    assert call(n_rows=700, n_list=700, ws_bytes=n.value - 1) == plc.E_CAPACITY
    assert lib.plc_pages_weigh_workspace(C.byref(pool()), 0, 8, 7, C.byref(n)) == plc.E_INVALID and lib.plc_pages_weigh_workspace(C.byref(pool()), 3, 8, 7, None) == plc.E_INVALID
    assert lib.plc_pages_weigh_workspace(C.byref(pool()), 3, 6, 7, C.byref(n)) == plc.E_SHAPE
    assert call(n_list=0) == plc.OK


def test_evictions_that_are_refused(lib):
    def call(p=None, i=None, o=None, budgets=0, budget=5, recent=1, base=A, out=B, n_pos=100, ws=WS, ws_bytes=1 << 24, status=A):
        w = serving.Weights(base, 800, 400, 100, n_pos)
        return lib.plc_pages_evict(C.byref(p or pool()), C.byref(i or book()), C.byref(w), C.c_void_p(budgets), budget, recent, C.byref(o or book(B + (1 << 20))), C.c_void_p(out),
                                   C.c_void_p(ws), C.c_uint64(ws_bytes), C.c_void_p(status), None)
    for kw in (dict(budget=-1), dict(recent=-1), dict(base=0), dict(out=0), dict(out=A), dict(n_pos=0), dict(ws=0), dict(status=0), dict(o=book()), dict(i=book(rows=0)),
               dict(o=serving.PageBookC(B + 40, B + 9000000, B + 9100000, 3, 5))):
        assert call(**kw) == plc.E_INVALID, kw
    for kw in (dict(o=book(B + (1 << 20), rows=4)), dict(o=book(B + (1 << 20), cols=6)), dict(p=pool(d=48)), dict(n_pos=0x7fff0001),
               dict(p=pool(L=1 << 14, H=1 << 14), i=book(rows=4), o=book(B + (1 << 20), rows=4))):
        assert call(**kw) == plc.E_SHAPE, kw
    for kw in (dict(base=A + 2), dict(out=B + 2), dict(ws=WS + 8)):
        assert call(**kw) == plc.E_ALIGN, kw
    n = C.c_uint64()
    assert lib.plc_pages_evict_workspace(C.byref(pool()), 3, 100, C.byref(n)) == plc.OK and call(ws_bytes=n.value - 1) == plc.E_CAPACITY
    assert lib.plc_pages_evict_workspace(C.byref(pool()), 0, 100, C.byref(n)) == plc.E_INVALID
    assert lib.plc_pages_evict_workspace(C.byref(pool()), 3, 0, C.byref(n)) == plc.E_INVALID
    assert lib.plc_pages_evict_workspace(C.byref(pool()), 3, 100, None) == plc.E_INVALID
    assert lib.plc_pages_evict_workspace(C.byref(pool()), 1 << 21, 100, C.byref(n)) == plc.E_SHAPE


def test_log_probabilities_that_are_refused(lib):
    def call(rows=2, V=100, m=1, top=4, logits=A, dtype=plc.OUT_F16, toks=A, logp=A, entropy=A, top_logp=A, top_token=A, ws=WS, ws_bytes=1 << 20):
        return lib.plc_token_logprobs(C.c_void_p(logits), dtype, C.c_int64(V), rows, V, C.c_void_p(toks), m, top, C.c_void_p(logp), C.c_void_p(entropy), C.c_void_p(top_logp),
                                      C.c_void_p(top_token), C.c_void_p(ws), C.c_uint64(ws_bytes), None, None)
    for kw in (dict(rows=0), dict(V=0), dict(m=-1), dict(top=-1), dict(logits=0), dict(dtype=3), dict(toks=0), dict(logp=0), dict(top_logp=0), dict(top_token=0), dict(ws=0)):
        assert call(**kw) == plc.E_INVALID, kw
    for kw in (dict(rows=(1 << 24) + 1), dict(V=2 ** 31 - 2 ** 16 + 1), dict(top=129), dict(m=(1 << 20) + 1)):
        assert call(**kw) == plc.E_SHAPE, kw
    for kw in (dict(logits=A + 1), dict(logits=A + 2, dtype=plc.OUT_F32), dict(ws=WS + 8)):
        assert call(**kw) == plc.E_ALIGN, kw
    n = C.c_uint64()
    assert lib.plc_token_logprobs_workspace(2, 100, 4, C.byref(n)) == plc.OK and call(ws_bytes=n.value - 1) == plc.E_CAPACITY
    assert lib.plc_token_logprobs_workspace(0, 100, 4, C.byref(n)) == plc.E_INVALID and lib.plc_token_logprobs_workspace(2, 100, 4, None) == plc.E_INVALID


def test_the_binding_checks_its_tensors():
    import torch
    i = torch.zeros(3, dtype=torch.int32)
    r = plc.Rotary(8, device="cpu")
    x = torch.zeros(3, 2, 16)
    for bad in (lambda: r.apply(x, i.long()), lambda: r.apply(x[0], i), lambda: r.apply(x.double(), i), lambda: r.apply((x, x[:2]), i), lambda: r.apply((x,) * 5, i),
                lambda: r.apply((), i), lambda: r.apply(x, i, out=x[..., :8]), lambda: r.apply((x, x), i, out=(x,)), lambda: r.apply(x.transpose(1, 2), i),
                lambda: plc.token_logprobs(torch.zeros(3, 8), i)):
        with pytest.raises(plc.PlcError):
            bad()
    assert r.apply(x[:0], i[:0]).shape == (0, 2, 16)


def test_the_oracle_by_hand():
    from oracle import serving as o
    y = o.rotary(np.array([[[1.0, 2, 3, 4, 9]]]), [1], [math.pi / 2, math.pi])
    assert np.allclose(y, [[[-3, -2, 1, -4, 9]]])
    y = o.rotary(np.array([[[1.0, 2, 3, 4, 9]]]), [1], [math.pi / 2, math.pi], interleaved=True, scale=2.0, back=True)
    assert np.allclose(y, [[[4, -2, -6, -8, 9]]])
    table, ref = np.array([[3, 1, -1], [0, 2, -1]]), np.array([1, 1, 2, 1, 0])
    places, within, bits = o.append_places(table, [3, 4], ref, [0, 2, 4], 4, 5)
    assert places == [(3, 3), (1, 0), None, None, None] and within == [3, 4, 4, 5, None] and bits == o.RANGE
    q, lse = np.array([[[1.0, 0]], [[0.0, 1]]]), np.log(np.array([[2.0], [4.0]]))
    keys = np.log(np.array([[2.0, 3], [4, 5], [6, 7]]))
    w, _ = o.weigh(q, lse, lambda s, h, t: keys[t], [3], [0, 2], None, 1.0, 0.5, np.array([[[8.0, 100, 100, 7]]]))
    assert np.allclose(w, [[[4 + 2 / 2 + 3 / 4, 4 / 2 + 5 / 4, 7 / 4, 7]]])
    weight = np.array([[[[5.0, 1, 5, 9, 2, 0]]]])
    t, n, r, ww, moves, bits = o.evict(np.array([[3, 1, 0]]), np.array([5]), np.array([1, 2, 0, 1]), weight, [3], 1, 2)
    assert moves == [(0, 0, 0, (3, 0), (3, 0)), (0, 0, 0, (1, 1), (3, 1)), (0, 0, 0, (0, 0), (2, 0))] and n.tolist() == [3] and bits == 0
    assert t.tolist() == [[3, 2, -1]] and r.tolist() == [0, 1, 1, 1] and ww.tolist() == [[[[5, 9, 2, 0, 0, 0]]]]
    lp, h, tl, tt, _ = o.token_logprobs(np.log(np.array([[.5, .25, .25]])), np.array([[1, -1]]), 4)
    assert np.allclose(np.exp(lp), [[.25, 1]]) and np.allclose(h, 1.5 * math.log(2)) and tt.tolist() == [[0, 1, 2, -1]] and np.isinf(tl[0, 3])


def test_evictions_onto_the_weights_are_refused(lib):
    """Kept weights that lie among the old ones, shifted or between rows that are far apart: 3 rows, 2 layers, 4 heads, 100 positions, 9600 bytes where they are contiguous."""
    def call(base, out, strides=(800, 400, 100)):
        w = serving.Weights(base, *strides, 100)
        n = C.c_uint64()
        assert lib.plc_pages_evict_workspace(C.byref(pool()), 3, 100, C.byref(n)) == plc.OK
        return lib.plc_pages_evict(C.byref(pool()), C.byref(book()), C.byref(w), None, 5, 1, C.byref(book(B + (1 << 20))), C.c_void_p(out), C.c_void_p(WS), C.c_uint64(n.value - 1),
                                   C.c_void_p(A), None)
    at = 1 << 26
    for out in (at, at + 4, at + 9596, at - 4, at - 9596):
        assert call(at, out) == plc.E_INVALID, out
    for out in (at + 9600, at - 9600):
        assert call(at, out) == plc.E_CAPACITY, out             # past the check, to the workspace that is a byte short
    wide = (10000, 400, 100)                                     # rows 40000 bytes apart, the last one ends at 83200
    for out in (at + 83196, at + 4000, at - 9596):
        assert call(at, out, wide) == plc.E_INVALID, out
    assert call(at, at + 83200, wide) == plc.E_CAPACITY
    down = (-800, 400, 100)                                      # rows that go down
    assert call(at, at - 6400, down) == plc.E_INVALID and call(at, at - 6400 - 9600, down) == plc.E_CAPACITY and call(at, at + 3200, down) == plc.E_CAPACITY
    assert call(at, at + 3196, down) == plc.E_INVALID
    huge = (1 << 62, 1 << 62, 1 << 62)                           # no sum of these wraps
    assert call(at, at + 4096, huge) == plc.E_INVALID and call(at, at - 9600, huge) == plc.E_CAPACITY


def test_weights_on_top_of_each_other_are_refused(lib):
    """Against every pair of runs: strides of either sign, nested and not, from 0 on; one row or one head needs no stride."""
    rng = np.random.default_rng(1)
    seen = set()
    for i in range(4000):
        rows, H, n = int(rng.integers(1, 6)), int(rng.integers(1, 6)), int(rng.integers(1, 9))
        row, head = (int(x) for x in rng.integers(-6 * n, 6 * n + 1, 2))
        starts = sorted(r * row + h * head for r in range(rows) for h in range(H))
        apart = all(b - a >= n for a, b in zip(starts, starts[1:]))
        q = serving.WeighQueries(A, 64 * H, 64, A, None, A, 7, 0, H)
        rc = lib.plc_pages_weigh(C.byref(pool(L=1, H=H)), 0, C.byref(book(rows=rows)), C.byref(q), C.c_float(1.0), C.c_float(1.0),
                                 C.byref(serving.Weights(B, row, 0, head, n)), C.c_void_p(WS), C.c_uint64(1 << 20), C.c_void_p(A), None)
        assert rc == (plc.OK if apart else plc.E_INVALID), (rows, H, n, row, head)
        seen.add((apart, row < 0, head < 0, abs(row) > abs(head), rows > 1 and H > 1))
    assert len(seen) >= 28
    q = serving.WeighQueries(A, 256, 64, A, None, A, 7, 0, 4)
    for row, head, rc in ((1 << 62, 1 << 62, plc.E_INVALID), (-(1 << 63), 1 << 61, plc.OK), (1 << 62, 100, plc.OK), (400, 100, plc.OK), (399, 100, plc.E_INVALID), (100, 300, plc.OK),
                          (100, 299, plc.E_INVALID)):
        assert lib.plc_pages_weigh(C.byref(pool(L=1)), 0, C.byref(book()), C.byref(q), C.c_float(1.0), C.c_float(1.0), C.byref(serving.Weights(B, row, 0, head, 100)), C.c_void_p(WS),
                                   C.c_uint64(1 << 20), C.c_void_p(A), None) == rc, (row, head)


def test_results_on_top_of_each_other_are_refused(lib):
    """Turned rows and heads, against every pair of runs; so many rows that only the heads can be gone through."""
    rng = np.random.default_rng(2)
    answers = set()
    for i in range(3000):
        rows, heads, d = int(rng.integers(1, 6)), int(rng.integers(1, 6)), 2 * int(rng.integers(1, 5))
        row, head = (int(x) for x in rng.integers(-6 * d, 6 * d + 1, 2))
        starts = sorted(r * row + h * head for r in range(rows) for h in range(heads))
        apart = all(b - a >= d for a, b in zip(starts, starts[1:]))
        # the second set is looked at behind the first and is off its boundary, so that nothing is launched
        t = dict(x_dev=A, x_stride_row=4096, x_stride_head=256, heads=heads)
        s = (serving.RotarySet * 2)(serving.RotarySet(out_dev=B, out_stride_row=row, out_stride_head=head, **t),
                                    serving.RotarySet(out_dev=WS + 1, out_stride_row=1 << 20, out_stride_head=64, **t))
        rc = lib.plc_rotary_apply(C.byref(rotary(dim=2)), s, 2, C.c_void_p(A), rows, d, plc.OUT_F16, 0, None)
        assert rc == (plc.E_ALIGN if apart else plc.E_INVALID), (rows, heads, d, row, head)
        answers.add((apart, abs(row) > abs(head), row < 0, head < 0))
    assert len(answers) == 16
    s = (serving.RotarySet * 2)(serving.RotarySet(A, B, 64, 64, 128, (1 << 36) + 64, 2), serving.RotarySet(A, WS + 1, 64, 64, 1 << 20, 64, 1))
    assert lib.plc_rotary_apply(C.byref(rotary()), s, 2, C.c_void_p(A), 0x7fffffff, 64, plc.OUT_F16, 0, None) == plc.E_ALIGN     # between the rows
    s[0].out_stride_head += 64
    assert lib.plc_rotary_apply(C.byref(rotary()), s, 2, C.c_void_p(A), 0x7fffffff, 64, plc.OUT_F16, 0, None) == plc.E_INVALID
    for kw in (dict(out_stride_head=63), dict(out_stride_row=511), dict(out_stride_row=64)):
        assert lib.plc_pages_append(C.byref(pool()), 0, C.byref(book()), None, C.byref(tokens(**kw)), C.c_void_p(A), None) == plc.E_INVALID, kw


def test_shared_memory_that_is_read_in_wide_words_is_aligned():
    """Arrays of ints that kernels read as int4 or uint4 say so: where the compiler puts the next variable is no promise."""
    import os
    import re
    src = os.path.join(os.path.dirname(plc.__file__), "csrc")
    for name, array in (("plc_evict.cu", "bins"), ("plc_logits.cuh", "order")):
        text = open(os.path.join(src, name)).read()
        assert re.search(r"(alignas\(16\)|__align__\(16\)) (int|uint32_t) %s\[" % array, text), (name, array)


def test_turns_of_tensors_on_the_host_are_refused():
    import torch
    r = plc.Rotary(8, device="cpu")
    with pytest.raises(plc.PlcError) as e:
        r.apply(torch.zeros(3, 2, 16), torch.zeros(3, dtype=torch.int32))
    assert e.value.code == plc.E_INVALID
