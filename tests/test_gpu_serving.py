"""Paged cache, tree attention and beam search on the GPU against the oracle's literal definitions (binary64).

Tolerances.  Books, counts, moved pages, parents and tokens: equal.  Copied page data: equal bit for bit, everything else in
the pool untouched.  Attention, per output component, with u = half a step of the type (2^-11 f16, 2^-8 bf16, relative):
  * scores are sums of d binary32 products: off by at most d 2^-23 of the sum of |q k| scale (the tensor cores' alignment
    of addends loses at most one more bit than 2^-24 each), and the exponential of a binary32 argument x below
    the maximum by 2^-23 |x| + 2^-22: a weight is off by a relative e = 2 (d 2^-23 B + 2^-22 + 2^-23 X), B the row's largest sum of
    |q k| scale and X <= 2 B the span of its scores; twice, because the normaliser is off by as much;
  * each weight is rounded to the type (u), the sum over positions is binary32 (n 2^-23), the result is rounded (u):
    |out - exact| <= (u + e + n 2^-23) sum |p v| + u |exact| + half the smallest step of the type;
  * |lse - exact| <= e + n 2^-23 + 2^-22 |exact|.
Scores of beams: binary32 exponentials off by 2^-21 relative (argument up to 2^3 half steps where the terms count, 2 ulp of the
function), the result rounded: |score - exact| <= 2^-20 + 2^-23 |exact|.  Orders: the inputs' scores are farther apart than 2^-18 or equal
by construction, which is asserted on the oracle's.
"""
import math

import numpy as np
import pytest
import torch

import paper_2604_15356_b200 as plc
from paper_2604_15356_b200 import synth

pytestmark = pytest.mark.gpu

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    plc.build()
    return torch.device("cuda:0")


@pytest.fixture(scope="module")
def ora():
    from oracle import serving
    return serving


def i32(v, dev):
    return torch.as_tensor(np.asarray(v), dtype=torch.int32).to(dev)


def make_pool(rng, L, pages, H, page, d, dtype, dev, slots_first, fill=None):
    """kv [L][2][P][H][page][d] with a margin of one layer behind it that no call may touch."""
    shape = (L + 1, 2, pages, page, H, d) if slots_first else (L + 1, 2, pages, H, page, d)
    base = torch.full(shape, float("nan"), dtype=TYPES[dtype]) if fill == "nan" else torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(TYPES[dtype])
    base = base.to(dev)
    kv = base.transpose(3, 4) if slots_first else base
    return kv[:L], base


def make_book(rng, held, cols, pages, dev):
    order = rng.permutation(pages)
    table = np.full((len(held), cols), -1, np.int32)
    at = 0
    for s, n in enumerate(held):
        table[s, :n] = order[at:at + n]
        at += n
    ref = np.bincount(table[table >= 0], minlength=pages).astype(np.int32)
    return table, ref


def book_of(table, length, ref, dev):
    return plc.PageBook(i32(table, dev), i32(length, dev), i32(ref, dev))


def same_book(b, table, length, ref):
    assert np.array_equal(b.table.cpu().numpy(), table)
    assert np.array_equal(b.len.cpu().numpy(), length)
    assert np.array_equal(b.ref.cpu().numpy(), ref)


# ---------------------------------------------------------------------------------------------- attention

def tree_mask(rng, begin, words, empty=()):
    """Ancestors of random trees; the rows in `empty` see nothing drafted."""
    N = begin[-1]
    bits = np.zeros((N, words * 32), bool)
    for s in range(len(begin) - 1):
        for i in range(begin[s + 1] - begin[s]):
            up = rng.integers(-1, i) if i else -1
            if up >= 0:
                bits[begin[s] + i] = bits[begin[s] + up]
            if i < words * 32:
                bits[begin[s] + i, i] = True
    for r in empty:
        bits[r] = False
    w = np.packbits(bits, axis=1, bitorder="little").view(np.int32) if N else np.zeros((0, words), np.int32)
    return bits, w


def attention_case(dev, ora, seed, dtype, d, H, G, page, lens, n, tree=True, slots_first=False, words=None, layer=0, L=1, empty=(), scale=None,
                   spread=1.0, behind=0, strided=False, bad_pages=(), nan_masked=False):
    rng = np.random.default_rng(seed)
    S = len(lens)
    held = [-(-(a + b) // page) for a, b in zip(lens, n)]
    pages = sum(held) + 2
    kv, base = make_pool(rng, L, pages, H, page, d, dtype, dev, slots_first, fill="nan")
    cols = max(max(held), 1) + 1
    table, ref = make_book(rng, held, cols, pages, dev)
    begin = np.cumsum([0] + list(n)).astype(np.int32)
    N = int(begin[-1])
    vals = torch.from_numpy(rng.standard_normal((2, S, max(a + b for a, b in zip(lens, n)) + 1, H, d)).astype(np.float32) * spread).to(TYPES[dtype])
    for s in range(S):                                     # real values where positions are; NaN everywhere else
        t = torch.arange(lens[s] + n[s])
        if len(t):
            at = torch.as_tensor(table[s].astype(np.int64))[t // page]
            kv[layer][:, at.to(dev), :, (t % page).to(dev)] = vals[:, s, :len(t)].to(dev).transpose(0, 1)
    q = torch.from_numpy(rng.standard_normal((N + behind, H * G, d)).astype(np.float32) * spread).to(TYPES[dtype])
    words = words or max(1, -(-max(n) // 32))
    bits, w = tree_mask(rng, begin, words, empty) if tree else (None, None)
    if nan_masked:                                         # drafted positions of session 0 that only some rows see
        for j in range(n[0]):
            if not bits[begin[0]:begin[1], j][:2].any():
                p = lens[0] + j
                kv[layer, :, int(table[0, p // page]), :, p % page] = float("nan") if j % 2 else float("inf")
                vals[:, 0, p] = float("nan")
    for s, c in bad_pages:
        table[s, c] = pages + 7
    pool = plc.PagePool(kv)
    book = book_of(table, lens, ref, dev)
    qd = q.to(dev)
    if strided:
        wide = torch.full((N + behind, H * G + 3, d + 16), 9.0, dtype=TYPES[dtype], device=dev)
        wide[:, 1:H * G + 1, 8:d + 8] = qd
        qd = wide[:, 1:H * G + 1, 8:d + 8]
    out = torch.full((N + behind, H * G, d), 77.0, dtype=TYPES[dtype], device=dev)
    lse = torch.full((N + behind, H * G), 77.0, dtype=torch.float32, device=dev)
    m = None
    if tree:
        m = torch.zeros(N + behind, words, dtype=torch.int32)
        m[:N] = torch.from_numpy(w.copy()).view(N, words)
        m = m.to(dev)
    got, got_lse = pool.tree_attention(layer, book, qd, i32(begin, dev), mask=m, scale=scale, out=out, lse=lse)
    torch.cuda.synchronize()
    assert got.data_ptr() == out.data_ptr() and bool((out[N:] == 77).all()) and bool((lse[N:] == 77).all())

    class Of:
        heads = H

        def __init__(self, j):
            self.x = vals[j].float().numpy()

        def __call__(self, s, g, t):
            return None if (s, t // page) in bad_pages else self.x[s, t, g]

    if nan_masked:                                         # only the rows that see no such position are compared
        keep = [r for r in range(N) if r >= begin[1] or not any(bits[r, j] and bool(vals[0, 0, lens[0] + j].isnan().any()) for j in range(n[0]))]
        assert len(keep) >= 2
    else:
        keep = list(range(N))
    sc = 1 / math.sqrt(d) if scale is None else scale
    ex, exl, mag, big = ora.attention(q[:N].double().numpy(), Of(0), Of(1), [int(x) for x in lens], [int(x) for x in begin], bits, sc)
    got, got_lse = got[:N].double().cpu().numpy(), got_lse[:N].double().cpu().numpy()
    u = torch.finfo(TYPES[dtype]).eps / 2
    terms = max(a + b for a, b in zip(lens, n))
    e = 2 * (d * 2.0 ** -23 * big + 2.0 ** -22 + 2.0 ** -23 * 2 * big)
    tol = (u + e[..., None] + terms * 2.0 ** -23) * mag + u * np.abs(ex) + torch.finfo(TYPES[dtype]).smallest_normal * u
    none = np.isinf(exl)
    assert np.array_equal(got_lse[keep][none[keep]], exl[keep][none[keep]]) and not got[keep][none[keep]].any()
    bad = np.abs(got - ex)[keep] > tol[keep]
    assert not bad.any() and not np.isnan(got[keep]).any(), (np.argwhere(bad)[:5], np.abs(got - ex)[keep].max())
    fine = ~none[keep]
    off = np.abs(got_lse - np.where(none, 0, exl))[keep][fine]
    assert (off <= (e + terms * 2.0 ** -23 + 2.0 ** -22 * np.abs(np.where(none, 0, exl)))[keep][fine]).all(), off.max()
    return pool


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d, H, G, page, slots_first", [(32, 3, 1, 16, False), (64, 1, 5, 1, True), (128, 2, 8, 24, False), (128, 8, 1, 64, True),
                                                        (256, 1, 3, 100, False), (256, 2, 16, 32, True)])
def test_attention_of_ragged_trees(dev, ora, dtype, d, H, G, page, slots_first):
    """Lengths of zero and one, around tile and page ends; sessions without queries; trees of one to 40 nodes."""
    pool = attention_case(dev, ora, d + H, dtype, d, H, G, page, lens=[0, 1, 127, 128, 129, 300, 0, 63], n=[3, 1, 40, 0, 17, 2, 0, 1], slots_first=slots_first,
                          behind=2)
    pool.check()


@pytest.mark.parametrize("dtype, d, H, G, n", [("f16", 64, 1, 1, 1), ("bf16", 128, 2, 4, 1), ("f16", 128, 1, 8, 100), ("bf16", 64, 2, 7, 33), ("f16", 256, 1, 2, 150),
                                               ("bf16", 32, 1, 1, 260)])
def test_attention_of_chains(dev, ora, dtype, d, H, G, n):
    """No mask: single-token decoding, a drafted chain, a chunk of a prompt (several row tiles a session)."""
    attention_case(dev, ora, n, dtype, d, H, G, 16, lens=[200, 0, 37, 511], n=[n, n, 1, n], tree=False, behind=1).check()


def test_attention_over_longer_contexts(dev, ora):
    """One session whose positions are split over the whole GPU, and a ragged batch whose parts begin inside sessions."""
    attention_case(dev, ora, 1, "bf16", 128, 1, 2, 64, lens=[9001], n=[5]).check()
    attention_case(dev, ora, 2, "f16", 64, 2, 1, 48, lens=[4000, 10, 0, 2500, 700, 1], n=[1, 9, 4, 1, 0, 2]).check()
    attention_case(dev, ora, 3, "f16", 128, 1, 8, 256, lens=[3000, 5], n=[40, 37]).check()


def test_attention_masks(dev, ora):
    """Rows that see nothing drafted, rows that see nothing at all, masks of fewer and of more words than drafts."""
    attention_case(dev, ora, 4, "f16", 64, 1, 2, 16, lens=[0, 20, 0], n=[5, 6, 33], empty=(0, 3, 6, 12, 40)).check()
    attention_case(dev, ora, 5, "bf16", 128, 1, 1, 16, lens=[50, 0], n=[70, 40], words=1).check()
    attention_case(dev, ora, 6, "f16", 128, 2, 2, 16, lens=[50, 129], n=[7, 3], words=4).check()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_attention_does_not_look_at_what_is_masked(dev, ora, dtype):
    """Infinities and NaN at drafted positions that a row does not see leave it as it is, keys and values alike."""
    attention_case(dev, ora, 7, dtype, 128, 2, 2, 16, lens=[60, 10], n=[30, 4], nan_masked=True)
    attention_case(dev, ora, 8, dtype, 64, 1, 1, 8, lens=[0, 10], n=[12, 4], nan_masked=True)
    attention_case(dev, ora, 8, dtype, 256, 1, 1, 8, lens=[125, 10], n=[12, 4], nan_masked=True)


def test_attention_scales_and_strides(dev, ora):
    """Large scores (the running maximum rises late and by much), a small scale, strided queries, another layer."""
    attention_case(dev, ora, 9, "bf16", 128, 2, 2, 16, lens=[700, 33], n=[3, 1], spread=3.0, scale=1.0)
    attention_case(dev, ora, 10, "f16", 64, 2, 2, 16, lens=[300, 33], n=[3, 1], scale=0.001)
    attention_case(dev, ora, 11, "f16", 128, 2, 3, 32, lens=[300, 33], n=[9, 1], strided=True, L=3, layer=2, slots_first=True)


def test_attention_reports_pages_out_of_range(dev, ora):
    pool = attention_case(dev, ora, 12, "f16", 64, 1, 2, 16, lens=[100, 40], n=[4, 2], bad_pages=((0, 2), (1, 0)))
    with pytest.raises(plc.PlcError) as e:
        pool.check()
    assert e.value.code == plc.E_INVALID
    pool.check()                                           # the word has been cleared


def test_attention_cuts_ranges_and_lengths_to_what_there_is(dev):
    kv = torch.zeros(1, 2, 4, 1, 16, 64, dtype=torch.float16, device=dev)
    pool = plc.PagePool(kv)
    for length, begin in (([40], [0, 9]), ([-3], [0, 2]), ([30], [0, 4]), ([10], [2, 1]), ([10], [-2, 3]), ([1 << 30], [0, 4])):
        book = book_of(np.array([[0, 1]]), length, np.array([1, 1, 0, 0]), dev)
        out, lse = pool.tree_attention(0, book, torch.ones(4, 2, 64, dtype=torch.float16, device=dev), i32(begin, dev), out=torch.zeros(4, 2, 64, dtype=torch.float16, device=dev))
        assert not out.any()
        with pytest.raises(plc.PlcError) as e:
            pool.check()
        assert e.value.code == plc.E_INVALID


def test_attention_offsets_pass_32_bits(dev, ora):
    """Pages that lie farther apart than 2^31 elements and 2^32 bytes."""
    far = (1 << 31) + 64
    store = torch.empty(2 * far + 4 * 8 * 64, dtype=torch.float16, device=dev)
    kv = store.as_strided((1, 2, 3, 1, 8, 64), (0, 8 * 64, far, 8 * 64, 64, 1))
    rng = np.random.default_rng(3)
    x = torch.from_numpy(rng.standard_normal((2, 3, 1, 8, 64)).astype(np.float32)).half()
    kv[0] = x.to(dev)
    q = torch.from_numpy(rng.standard_normal((1, 1, 64)).astype(np.float32)).half()
    out, _ = plc.PagePool(kv).tree_attention(0, book_of(np.array([[2, 0]]), [14], np.array([1, 0, 1]), dev), q.to(dev), i32([0, 1], dev))
    K = torch.cat([x[0, 2, 0], x[0, 0, 0]])[:15].double()
    V = torch.cat([x[1, 2, 0], x[1, 0, 0]])[:15].double()
    want = torch.softmax(K @ q[0, 0].double() / 8, 0) @ V
    assert float((out.cpu().double()[0, 0] - want).abs().max()) < 2.0 ** -9


def test_attention_on_another_stream_and_in_graphs(dev):
    """Two captured graphs and an eager call, each with its own results: a replay reads the lengths that stand there then."""
    rng = np.random.default_rng(5)
    kv, _ = make_pool(rng, 1, 40, 2, 16, 128, "bf16", dev, False)
    pool, q = plc.PagePool(kv), torch.randn(6, 8, 128, device=dev).bfloat16()
    begin = i32([0, 1, 6], dev)
    table = rng.permutation(40)[:36].reshape(2, 18)
    book = book_of(table, [200, 100], np.ones(40), dev)
    want = [t.clone() for t in pool.tree_attention(0, book, q, begin)]
    side = torch.cuda.Stream(dev)
    side.wait_stream(torch.cuda.current_stream(dev))
    with torch.cuda.stream(side):
        here = pool.tree_attention(0, book, q, begin)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(here, want))
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = pool.tree_attention(0, book, q, begin)
        graphs.append((g, res))
    for g, res in graphs:
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(res, want))
    book.len.copy_(i32([17, 283], dev))
    want2 = [t.clone() for t in pool.tree_attention(0, book, q, begin)]
    for g, res in reversed(graphs):
        g.replay()
    torch.cuda.synchronize()
    for g, res in graphs:
        assert all(torch.equal(a, b) for a, b in zip(res, want2))
    assert not torch.equal(want[0], want2[0])


# ---------------------------------------------------------------------------------------------- pages

def forked(rng, S, W, page, pages, cols):
    """A book as beams leave it: rows of a session share their first pages."""
    table, length, at = np.full((S * W, cols), -1, np.int32), np.zeros(S * W, np.int32), 0
    order = rng.permutation(pages)
    for s in range(S):
        n = int(rng.integers(0, (cols - 1) * page)) if s else (cols - 2) * page   # the first session ends on a page's end
        full, part, shared = n // page, n % page > 0, n // page // 2
        first = order[at:at + shared]
        at += shared
        for w in range(W):
            mine = full - shared + part + (s % 3 == 1)     # some rows hold a page of room
            table[s * W + w, :shared + mine] = np.concatenate([first, order[at:at + mine]])
            at += mine
            length[s * W + w] = n
    ref = np.bincount(table[table >= 0], minlength=pages).astype(np.int32)
    return table, length, ref


@pytest.mark.parametrize("dtype, L, H, d, page, slots_first, S, W", [
    ("f16", 2, 2, 64, 16, False, 5, 3), ("bf16", 1, 3, 128, 5, True, 9, 4), ("f32", 3, 1, 32, 8, False, 4, 2), ("f32", 1, 2, 256, 100, True, 2, 5),
    ("f16", 1, 1, 128, 1, False, 6, 2), ("f16", 1, 1, 32, 4, True, 700, 2)])
def test_fork_copies_and_counts(dev, ora, dtype, L, H, d, page, slots_first, S, W):
    rng = np.random.default_rng(S * W + page)
    cols = 7
    pages = S * W * (cols + 3)
    table, length, ref = forked(rng, S, W, page, pages, cols)
    table[0, 6], ref[pages - 1] = -1, ref[pages - 1] + 2    # the caller holds on to a page itself
    kv, base = make_pool(rng, L, pages, H, page, d, dtype, dev, slots_first)
    before = base.clone()
    out_rows = S * W + 3                                     # more rows than before: a session gets more beams
    parent = rng.integers(-1, S * W, out_rows)
    parent[:S * W // 2] = np.arange(S * W // 2)              # these go on as they are
    room = np.minimum(rng.integers(0, 2 * page, out_rows), cols * page - np.where(parent < 0, 0, length[parent]))
    pool = plc.PagePool(kv)
    for r in (room, None):
        base.copy_(before)
        new = pool.fork(book_of(table, length, ref, dev), i32(parent, dev), None if r is None else i32(r, dev))
        t, n, f, copies, bits = ora.fork(table, length, ref, parent, r, page)
        assert bits == 0 and (page == 1 or len(copies) >= 1)
        same_book(new, t, n, f)
        want = before.transpose(3, 4).clone() if slots_first else before.clone()
        for src, dst, used in copies:
            want[:L, :, dst, :, :used] = want[:L, :, src, :, :used]
        assert torch.equal(base, want.transpose(3, 4) if slots_first else want)
    pool.check()


def test_fork_without_enough_pages_changes_nothing(dev, ora):
    rng = np.random.default_rng(8)
    table, ref = make_book(rng, [3, 2], 4, 7, dev)           # two pages are free
    length = np.array([33, 20], np.int32)
    kv, base = make_pool(rng, 1, 7, 1, 16, 64, "f16", dev, False)
    before, pool = base.clone(), plc.PagePool(kv)
    for parent, room, enough in (([0, 0, 0], None, True), ([0, 0, 0, 0], None, False), ([0, 1], [16, 16], True), ([0, 1, 1], [16, 16, 0], False),
                                 ([0], [32], False)):        # the last one needs a fifth column
        base.copy_(before)
        new = pool.fork(book_of(table, length, ref, dev), i32(parent, dev), None if room is None else i32(room, dev))
        t, n, f, copies, bits = ora.fork(table, length, ref, parent, room, 16)
        assert bits == (0 if enough else ora.CAPACITY)
        same_book(new, t, n, f)
        if enough:
            pool.check()
        else:
            assert torch.equal(base, before)
            with pytest.raises(plc.PlcError) as e:
                pool.check()
            assert e.value.code == plc.E_CAPACITY


def test_fork_refuses_what_is_out_of_range(dev, ora):
    rng = np.random.default_rng(9)
    table, ref = make_book(rng, [3, 2, 1], 4, 20, dev)
    kv, _ = make_pool(rng, 1, 20, 1, 16, 64, "f16", dev, False)
    pool = plc.PagePool(kv)
    wrong = table.copy()
    wrong[0, 1], wrong[2, 0] = 20, -5
    for t0, length, parent, room in ((table, [33, 20, 3], [0, 3, -2, 1], [0, 0, 0, 0]), (table, [33, -1, 65], [0, 1, 2, 0], [0, 0, 0, 0]),
                                     (table, [33, 20, 3], [0, 1, 2, 0], [0, -1, 1 << 30, 0]), (wrong, [33, 20, 3], [0, 0, 1, 2], [0, 0, 0, 0])):
        new = pool.fork(book_of(t0, length, ref, dev), i32(parent, dev), i32(room, dev))
        t, n, f, _, bits = ora.fork(t0, np.array(length, np.int32), ref, parent, room, 16)
        same_book(new, t, n, f)
        word = int(pool.status)
        pool.status.zero_()
        assert word == bits != 0


@pytest.mark.parametrize("dtype, L, H, d, page, slots_first, S, m", [
    ("f16", 2, 2, 64, 16, False, 5, 9), ("bf16", 1, 3, 128, 5, True, 9, 40), ("f32", 3, 1, 32, 8, False, 4, 2), ("f32", 1, 2, 256, 100, True, 1, 150),
    ("f16", 1, 40, 128, 1, False, 3, 70)])
def test_keep_moves_the_accepted_path(dev, ora, dtype, L, H, d, page, slots_first, S, m):
    rng = np.random.default_rng(S + m)
    length = rng.integers(0, 4 * page, S).astype(np.int32)
    held = [-(-(int(n) + m) // page) + (s % 2) for s, n in enumerate(length)]
    pages, cols = sum(held) + 2, max(held) + 1
    table, ref = make_book(rng, held, cols, pages, dev)
    kv, base = make_pool(rng, L, pages, H, page, d, dtype, dev, slots_first)
    before = base.clone()
    n_path = rng.integers(0, m + 1, S)
    n_path[0] = m                                            # everything is kept
    path = np.full((S, m), -9, np.int32)
    for s in range(S):
        path[s, :n_path[s]] = np.sort(rng.choice(m, n_path[s], replace=False))
    pool = plc.PagePool(kv)
    new = pool.keep(book_of(table, length, ref, dev), i32(path, dev), i32(n_path, dev))
    t, n, f, moves, bits = ora.keep(table, length, ref, path, n_path, page)
    assert bits == 0
    same_book(new, t, n, f)
    old = before.transpose(3, 4) if slots_first else before
    want = old.clone()
    for s, a, b in moves:
        want[:L, :, int(table[s, b // page]), :, b % page] = old[:L, :, int(table[s, a // page]), :, a % page]
    assert torch.equal(base, want.transpose(3, 4) if slots_first else want)
    pool.check()


def test_keep_leaves_rows_with_bad_paths_as_they_are(dev, ora):
    rng = np.random.default_rng(11)
    table, ref = make_book(rng, [3] * 9, 4, 40, dev)
    table[8, 1] = table[7, 1]                                # two rows hold the page that one of them would write to
    ref = np.bincount(table[table >= 0], minlength=40).astype(np.int32)
    length = np.array([20, 20, 20, 20, 20, -1, 65, 14, 14], np.int32)
    path = np.array([[0, 2, 5], [0, 0, 1], [3, 2, 5], [-1, 2, 5], [0, 2, 28], [0, 1, 2], [0, 1, 2], [1, 2, 5], [0, 1, 2]], np.int32)
    n_path = np.array([3, 3, 3, 3, 3, 1, 1, 3, 4], np.int32)
    kv, base = make_pool(rng, 1, 40, 2, 16, 64, "f16", dev, False)
    before, pool = base.clone(), plc.PagePool(kv)
    new = pool.keep(book_of(table, length, ref, dev), i32(path, dev), i32(n_path, dev))
    t, n, f, moves, bits = ora.keep(table, length, ref, path, n_path, 16)
    assert bits == ora.RANGE and {m[0] for m in moves} == {0}
    same_book(new, t, n, f)
    want = before.clone()
    for s, a, b in moves:
        want[:1, :, int(table[s, b // 16]), :, b % 16] = before[:1, :, int(table[s, a // 16]), :, a % 16]
    assert torch.equal(base, want)
    assert int(pool.status) == ora.RANGE


@pytest.mark.parametrize("dtype, L, H, d, page, slots_first, S, pages", [
    ("f16", 2, 2, 64, 16, False, 5, 60), ("bf16", 1, 3, 128, 5, True, 9, 100), ("f32", 1, 2, 256, 100, True, 2, 12), ("f16", 1, 1, 32, 2, False, 900, 5000),
    ("f16", 1, 1, 64, 16, False, 1, 1), ("f16", 1, 1, 64, 16, False, 3, 40)])
def test_compact_moves_pages_down(dev, ora, dtype, L, H, d, page, slots_first, S, pages):
    rng = np.random.default_rng(pages)
    held = [min(5, pages // S) if pages != 40 else 0 for s in range(S)]   # the last case: a pool without pages in use
    table, ref = make_book(rng, held, 6, pages, dev)
    if S > 1 and pages != 40:
        table[1, 0] = table[0, 0]                            # a shared page; row 1's own is still held by the caller
        ref[table[0, 0]] += 1
    length = rng.integers(0, 2 * page, S).astype(np.int32)
    kv, base = make_pool(rng, L, pages, H, page, d, dtype, dev, slots_first)
    before, pool = base.clone(), plc.PagePool(kv)
    new, moved = pool.compact(book_of(table, length, ref, dev))
    t, f, where = ora.compact(table, ref)
    same_book(new, t, length, f)
    assert np.array_equal(moved.cpu().numpy(), where)
    old = before.transpose(3, 4) if slots_first else before
    want = old.clone()
    for p in range(pages):
        if where[p] >= 0:
            want[:L, :, where[p]] = old[:L, :, p]
    assert torch.equal(base, want.transpose(3, 4) if slots_first else want)
    pool.check()


# ---------------------------------------------------------------------------------------------- beams

def check_beams(ora, x, cum, n_out, done=None, eos=-1, gap=2.0 ** -18):
    S, W, V = x.shape
    es, ep, et = ora.beam_select(x.double().cpu().numpy(), cum.cpu().numpy(), n_out, None if done is None else done.cpu().numpy(), eos)
    # neighbours in the order are equal logits of one row, equal rows, or farther apart than the kernel's error
    more = ora.beam_select(x.double().cpu().numpy(), cum.cpu().numpy(), min(n_out + 1, W * V), None if done is None else done.cpu().numpy(), eos)[0]
    with np.errstate(invalid="ignore"):
        step = more[:, :-1] - more[:, 1:]
    assert (np.isnan(step) | (step == 0) | (step > gap)).all(), "the case's scores are too near each other to say anything"
    s, p, t = plc.beam_select(x, cum, n_out, done=done, eos=eos)
    s, p, t = s.double().cpu().numpy(), p.cpu().numpy(), t.cpu().numpy()
    assert np.array_equal(p, ep) and np.array_equal(t, et)
    fine = ~np.isinf(es)
    assert np.array_equal(fine, ~np.isinf(s)) and (np.abs(s - es)[fine] <= 2.0 ** -20 + 2.0 ** -23 * np.abs(es[fine])).all()


def spaced(rng, S, W, V, dtype, dev, peak=None):
    """Logits whose large values are far apart across the rows of a session (multiples of 1/8 in a row; rows differ by the score)."""
    x = np.round(rng.standard_normal((S, W, V)) * 16) / 8
    return torch.from_numpy(x.astype(np.float32)).to(TYPES[dtype]).to(dev)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("S, W, V, n_out", [(1, 1, 1, 1), (2, 3, 7, 5), (1, 4, 257, 8), (5, 2, 1000, 3), (3, 8, 4099, 16), (1, 5, 20001, 64), (2, 16, 513, 32),
                                            (1, 3, 9000, 128), (1, 128, 300, 128)])
def test_beam_selection(dev, ora, dtype, S, W, V, n_out):
    """Odd vocabularies (rows off 16-byte boundaries), many equal logits (ties by column), several parts a row, n_out above the vocabulary."""
    rng = np.random.default_rng(V + n_out)
    x = spaced(rng, S, W, V, dtype, dev)
    for attempt in range(40):                                # scores of the beams that keep the rows' values apart
        cum = torch.from_numpy(rng.uniform(-9, -1, (S, W)).astype(np.float32)).to(dev)
        es = ora.beam_select(x.double().cpu().numpy(), cum.cpu().numpy(), min(n_out + 1, W * V))[0]
        with np.errstate(invalid="ignore"):
            step = es[:, :-1] - es[:, 1:]
        if (np.isnan(step) | (step == 0) | (step > 2.0 ** -17)).all():
            break
    check_beams(ora, x, cum, min(n_out, W * V))


def test_beam_selection_of_first_steps_and_ended_beams(dev, ora):
    rng = np.random.default_rng(2)
    x = spaced(rng, 4, 4, 500, "f16", dev)
    cum = torch.tensor([[-1.0, -math.inf, -math.inf, -math.inf], [-3.0, -2.03, -4.31, -1.77], [-math.inf] * 4, [-5.0, -5.13, -0.4, math.inf]], device=dev)
    done = torch.tensor([[False] * 4, [False, True, False, True], [False, True, False, False], [True, True, True, True]], device=dev)
    check_beams(ora, x, cum, 6, done=done, eos=3)
    s, p, t = plc.beam_select(x, cum, 6, done=done, eos=3)
    assert p[2].tolist() == [-1] * 6 and t[2].tolist() == [-1] * 6
    assert p[3].tolist() == [14, 12, 13, -1, -1, -1] and t[3].tolist() == [3, 3, 3, -1, -1, -1]


def test_equal_beams_tie_to_the_lower_one(dev):
    """Equal rows have equal sums wherever they start: their continuations alternate, the lower row first."""
    for V, dtype in ((1001, "f16"), (5003, "bf16"), (333, "f32"), (40001, "f16")):
        rng = np.random.default_rng(V)
        row = torch.from_numpy(rng.permutation(V).astype(np.float32) / 64).to(TYPES[dtype])
        x = row.expand(3, 4, V).contiguous().to(dev)
        order = torch.argsort(row.float(), descending=True, stable=True)
        s, p, t = plc.beam_select(x, torch.full((3, 4), -2.5, device=dev), 8)
        top = row.float()[order[:40]].tolist()
        want = sorted([(-v, w, int(c)) for w in range(4) for v, c in zip(top, order[:40].tolist())])[:8]
        for b in range(3):
            assert p[b].tolist() == [4 * b + w for _, w, _ in want] and t[b].tolist() == [c for _, _, c in want]


def test_beam_selection_with_infinities_and_nan(dev, ora):
    rng = np.random.default_rng(4)
    x = spaced(rng, 3, 4, 900, "f32", dev)
    x[0, :, 10:] = -math.inf                                 # all but ten tokens are banned
    x[1, 0, 5], x[1, 1, 7], x[1, 2] = math.nan, math.inf, -math.inf
    x[2, 1, :899] = -math.inf                                # one token left
    x[2, 0, 3], x[2, 0, 4] = -0.0, 0.0
    cum = torch.tensor([[-1.0, -2.1, -3.3, -4.7], [-1.0, -1.0, -1.0, -1.1], [-30.0, -1.2, math.nan, -50.0]], device=dev)
    check_beams(ora, x, cum, 50)
    s, p, t = plc.beam_select(x, cum, 50)
    assert (p[0] >= 0).sum() == 40 and (p[1][p[1] >= 0] == 7).all()


def test_beam_selection_where_everything_ties(dev, ora):
    """All logits equal: the lowest columns of the lowest rows."""
    for dtype in ("f16", "f32"):
        x = torch.full((2, 3, 6001), 1.5, dtype=TYPES[dtype], device=dev)
        s, p, t = plc.beam_select(x, torch.full((2, 3), -1.0, device=dev), 128)
        for b in range(2):
            assert p[b].tolist() == [3 * b] * 128 and t[b].tolist() == list(range(128))
        x = torch.arange(70000, device=dev).float().div(70000).to(TYPES[dtype]).expand(1, 1, -1).contiguous()   # rising: every step beats the last
        order = torch.argsort(x[0, 0].float(), descending=True, stable=True)[:100]
        s, p, t = plc.beam_select(x, torch.zeros(1, 1, device=dev), 100)
        assert torch.equal(t[0].long(), order)


def test_reordering_of_states(dev):
    rng = np.random.default_rng(6)
    R = 37
    states = [torch.randint(0, 9, (R, 5), dtype=torch.int32, device=dev), torch.randn(R, 3, 7, device=dev).half(), torch.randint(0, 255, (R, 33), dtype=torch.uint8, device=dev),
              torch.randn(R, 40000, device=dev), torch.randn(R, 64, device=dev)[:, :48], torch.randn(R, device=dev), torch.randn(R, 0, device=dev)] * 3
    for rows in (1, 37, 64):
        parent = i32(rng.integers(-1, R, rows), dev)
        got = plc.beam_reorder(parent, states)
        at = parent.long()
        for g, t in zip(got, states):
            want = t[at.clamp(min=0)].clone()
            want[at < 0] = 0
            assert g.shape == want.shape and torch.equal(g, want)
    word = torch.zeros(1, dtype=torch.int32, device=dev)
    got = plc.beam_reorder(i32([R, 0, -2], dev), states[:1], status=word)
    assert int(word) == 32 and not got[0][0].any() and not got[0][2].any() and torch.equal(got[0][1], states[0][0])


# ---------------------------------------------------------------------------------------------- together

def test_beams_over_a_restored_cache(dev, ora):
    """A coded cache is decoded into pages, beams fork it, attend, are selected, and drafted paths are kept: every row's keys and
    values stay those of its own history, which is kept beside it in plain tensors."""
    S, W, n, L, H, d, V, K, page = 2, 3, 40, 2, 2, 64, 400, 32, 16
    table = synth.markov_table(V, 8.0, 5, max_states=64)
    tokens = synth.sample_tokens(table, S, n, 6)
    logits = synth.position_logits(table, tokens).to(dev)
    T = synth.make_tables(L, H, V, d, 7)
    src = synth.make_kv(T, tokens, 0.05, 8).to(dev)
    ctx = plc.Context(T.to(dev), K, 0.02, chunk_pos=32, out_dtype=plc.OUT_F16)
    st = plc.StreamSet(S * ctx.W, ctx.max_chunks(n), 3 * S * n * ctx.W * d + 8192, dev)
    ctx.encode(src, logits, st)
    pages, each = 60, -(-n // page)
    kv = torch.zeros(L, 2, pages, page, H, d, dtype=torch.float16, device=dev).transpose(3, 4)
    pool = plc.PagePool(kv)
    ctx.decode(st, logits, pool.sessions_view(4, S, n))
    plain = torch.zeros(L, 2, S, H, n, d, dtype=torch.float16, device=dev)
    ctx.decode(st, logits, plain)
    assert ctx.sync_status() == plc.OK
    first = np.full((S, 8), -1, np.int32)
    for s in range(S):
        first[s, :each] = 4 + s * each + np.arange(each)
    book = book_of(first, [n] * S, np.bincount(first[first >= 0], minlength=pages), dev)
    history = [plain[:, :, s].float().cpu() for s in range(S)]                    # [L][2][H][positions][d]
    book = pool.fork(book, i32(np.repeat(np.arange(S), W), dev), torch.full((S * W,), 4, dtype=torch.int32, device=dev))
    history = [history[s].clone() for s in range(S) for _ in range(W)]
    score = torch.full((S, W), -math.inf, device=dev)
    score[:, 0] = 0
    toks = torch.zeros(S * W, 8, dtype=torch.int32, device=dev)
    gen = torch.Generator(device="cpu").manual_seed(3)
    proj = torch.randn(H * 2 * d, V, generator=gen).to(dev) * 0.3
    for step in range(3):
        R, m = S * W, 4                                                           # a tree of four drafts: 0 -> 1, 0 -> 2, 3
        new = torch.randn(L, 2, R, H, m, d, generator=gen).half()
        pos = book.len.long()[:, None] + torch.arange(m, device=dev)
        at = book.table.long().gather(1, pos // page)
        kv.permute(2, 4, 0, 1, 3, 5)[at, pos % page] = new.to(dev).permute(2, 4, 0, 1, 3, 5)
        q = torch.randn(R * m, 2 * H, d, generator=gen).half()
        mask = torch.tensor([0b0001, 0b0011, 0b0101, 0b1000], dtype=torch.int32).repeat(R)[:, None].to(dev)
        out, lse = pool.tree_attention(1, book, q.to(dev), torch.arange(0, R * m + 1, m, dtype=torch.int32, device=dev), mask=mask)
        bits = np.array([[1, 0, 0, 0], [1, 1, 0, 0], [1, 0, 1, 0], [0, 0, 0, 1]], bool)
        for r in range(R):
            k, v = (torch.cat([history[r][1, j], new[1, j, r].float()], 1).double() for j in (0, 1))   # [H][n + m][d]
            for i in range(m):
                sees = torch.cat([torch.ones(history[r].shape[3], dtype=torch.bool), torch.from_numpy(bits[i])])
                for h in range(2 * H):
                    w = torch.softmax(k[h // 2][sees] @ q[r * m + i, h].double() / math.sqrt(d), 0)
                    want = w @ v[h // 2][sees]
                    assert float((out[r * m + i, h].cpu().double() - want).abs().max()) < 2.0 ** -8
        # the path 0 -> 2 is accepted everywhere, then the beams go on from what was seen last
        book = pool.keep(book, i32([[0, 2]] * R, dev), i32([2] * R, dev))
        history = [torch.cat([history[r], new[:, :, r].float()[:, :, :, [0, 2]]], 3) for r in range(R)]
        x = (out.view(R, m, -1)[:, 2].float() @ proj).view(S, W, V)
        score, parent, token = plc.beam_select(x, score, W)
        assert bool((parent >= 0).all())
        toks, = plc.beam_reorder(parent, [toks])
        toks[:, step] = token.flatten()
        par = parent.flatten().tolist()
        book = pool.fork(book, parent.flatten(), torch.full((R,), 4, dtype=torch.int32, device=dev))
        history = [history[p].clone() for p in par]
        if step == 1:
            book, moved = pool.compact(book)
            live = int((book.ref > 0).sum())
            assert not book.ref[live:].any() and int(book.table.max()) == live - 1
        for r in range(R):                                                        # every row's pages hold its own history
            t = torch.arange(history[r].shape[3], device=dev)
            mine = kv[:, :, book.table[r].long()[t // page], :, t % page]
            assert torch.equal(mine.permute(1, 2, 3, 0, 4).float().cpu(), history[r])
        assert int(book.len[0]) == history[0].shape[3]
    pool.check()


def attention_in_64_bits(kv, layer, table, lens, q, begin, bits, scale):
    """The formula over one layer's pages, session by session; sums of magnitudes for the tolerance beside it."""
    H, page, d = kv.shape[3], kv.shape[4], kv.shape[5]
    G = q.shape[1] // H
    out, mag = (torch.zeros(q.shape, dtype=torch.float64, device=q.device) for _ in range(2))
    big = torch.zeros(q.shape[:2], dtype=torch.float64, device=q.device)
    for s, at in enumerate(lens):
        lo, hi = int(begin[s]), int(begin[s + 1])
        n, T = hi - lo, at + hi - lo
        if n == 0:
            continue
        pages = torch.as_tensor(table[s, :-(-T // page)].astype(np.int64), device=q.device)
        k, v = (kv[layer, j, pages].double().transpose(1, 2).reshape(-1, H, d)[:T].transpose(0, 1) for j in range(2))
        x = q[lo:hi].double().reshape(n, H, G, d).permute(1, 2, 0, 3)
        score = torch.einsum("hgnd,htd->hgnt", x, k) * scale
        most = torch.einsum("hgnd,htd->hgnt", x.abs(), k.abs()).amax(-1) * scale
        sees = torch.ones(n, T, dtype=torch.bool, device=q.device)
        sees[:, at:] = torch.ones(n, n, dtype=torch.bool, device=q.device).tril() if bits is None else torch.as_tensor(bits[lo:hi, :n], device=q.device).bool()
        w = score.masked_fill(~sees, -math.inf).softmax(-1)
        out[lo:hi] = torch.einsum("hgnt,htd->hgnd", w, v).permute(2, 0, 1, 3).reshape(n, H * G, d)
        mag[lo:hi] = torch.einsum("hgnt,htd->hgnd", w, v.abs()).permute(2, 0, 1, 3).reshape(n, H * G, d)
        big[lo:hi] = most.permute(2, 0, 1).reshape(n, H * G)
    return out, mag, big


@pytest.mark.parametrize("dtype, d, G, page, n", [("bf16", 128, 4, 32, 1), ("f16", 128, 3, 24, 9), ("f16", 64, 4, 16, 5), ("bf16", 64, 8, 64, 7), ("bf16", 256, 2, 32, 8),
                                                  ("f16", 32, 4, 32, 4), ("f16", 128, 4, 20, 3), ("bf16", 128, 8, 32, 14), ("f16", 128, 8, 64, 30), ("bf16", 64, 8, 32, 33),
                                                  ("f16", 256, 8, 32, 14), ("f16", 128, 8, 36, 31)])
def test_attention_of_batches_with_many_pieces_an_sm(dev, dtype, d, G, page, n):
    """Ragged batches that give every SM many pieces one after the other, most of which end inside a tile; the same call again and again."""
    rng = np.random.default_rng(d + n)
    H, S = 8, 160
    lens = [int(x) for x in rng.integers(0, 420, S)]
    drafts = [n if i % 5 else int(rng.integers(0, n + 1)) for i in range(S)]
    held = [-(-(a + b) // page) for a, b in zip(lens, drafts)]
    pages = sum(held) + 2
    table, ref = make_book(rng, held, max(held) + 1, pages, dev)
    gen = torch.Generator(device=dev).manual_seed(n)
    kv = torch.randn(1, 2, pages, H, page, d, device=dev, generator=gen).to(TYPES[dtype])
    begin = np.cumsum([0] + drafts).astype(np.int32)
    N = int(begin[-1])
    q = torch.randn(N, H * G, d, device=dev, generator=gen).to(TYPES[dtype])
    bits, w = tree_mask(rng, begin, -(-n // 32), ())
    mask = torch.from_numpy(w.copy()).view(N, -1).to(dev) if n > 1 else None
    ex, mag, big = attention_in_64_bits(kv, 0, table, lens, q, begin, bits if n > 1 else None, 1 / math.sqrt(d))
    for s in range(S):                                     # what stands behind a session's last position is not to be seen
        t = torch.arange(lens[s] + drafts[s], held[s] * page)
        kv[0, :, torch.as_tensor(table[s].astype(np.int64))[t // page].to(dev), :, (t % page).to(dev)] = float("nan")
    pool, book = plc.PagePool(kv), book_of(table, lens, ref, dev)
    u = torch.finfo(TYPES[dtype]).eps / 2
    terms = max(a + b for a, b in zip(lens, drafts))
    e = 2 * (d * 2.0 ** -23 * big + 2.0 ** -22 + 2.0 ** -23 * 2 * big)
    tol = (u + e[..., None] + terms * 2.0 ** -23) * mag + u * ex.abs() + torch.finfo(TYPES[dtype]).smallest_normal * u
    for _ in range(25):
        got = pool.tree_attention(0, book, q, i32(begin, dev), mask=mask)
        got = got[0] if isinstance(got, tuple) else got
        bad = ~((got.double() - ex).abs() <= tol)
        assert not bad.any(), (int(bad.any(-1).sum()), float((got.double() - ex).abs().max()))
    pool.check()


@pytest.mark.parametrize("dtype, d, G, page, n", [("f16", 128, 8, 16, 20), ("bf16", 128, 8, 24, 40), ("bf16", 128, 8, 20, 40), ("f16", 64, 8, 136, 20), ("bf16", 64, 8, 8, 40),
                                                  ("f16", 256, 8, 16, 20), ("bf16", 256, 4, 12, 40), ("f16", 32, 8, 32, 40)])
def test_attention_of_many_rows_does_not_look_at_what_is_masked(dev, ora, dtype, d, G, page, n):
    """Infinities and NaN at masked drafted positions, for row tiles of 128 and 256, with pages that boxes copy and others."""
    attention_case(dev, ora, n + d, dtype, d, 1, G, page, lens=[125, 300], n=[n, n // 4], nan_masked=True).check()
    attention_case(dev, ora, n + d, dtype, d, 2, G, page, lens=[0, 10, 7], n=[n, 2, n], empty=(1, n + 1, n + 3)).check()


@pytest.mark.parametrize("d, G, page, n", [(128, 8, 16, 20), (128, 8, 16, 40), (64, 8, 8, 40), (256, 8, 16, 20), (128, 8, 12, 40)])
def test_attention_of_many_rows_reports_pages_out_of_range(dev, ora, d, G, page, n):
    pool = attention_case(dev, ora, d, "bf16", d, 1, G, page, lens=[100, 40], n=[n, n], bad_pages=((0, 2), (1, 0)))
    with pytest.raises(plc.PlcError) as e:
        pool.check()
    assert e.value.code == plc.E_INVALID


def test_attention_of_wide_sessions_among_narrow_ones(dev):
    """Row tiles that are in use now and then only, infinities in what they have drafted: a row sees its own, and no row another's."""
    rng = np.random.default_rng(0)
    H, G, d, page, S = 4, 8, 128, 32, 80
    drafts = [60 if s % 8 == 0 else 3 for s in range(S)]
    lens = [int(x) for x in rng.integers(0, 300, S)]
    held = [-(-(a + b) // page) for a, b in zip(lens, drafts)]
    table, ref = make_book(rng, held, max(held), sum(held), dev)
    kv = torch.randn(1, 2, sum(held), H, page, d, device=dev, generator=torch.Generator(device=dev).manual_seed(0)).bfloat16()
    begin = np.cumsum([0] + drafts).astype(np.int32)
    q = torch.randn(int(begin[-1]), H * G, d, device=dev, generator=torch.Generator(device=dev).manual_seed(1)).bfloat16()
    pool, book = plc.PagePool(kv), book_of(table, lens, ref, dev)
    plain = pool.tree_attention(0, book, q, i32(begin, dev))[0].clone()
    hit = torch.zeros(q.shape[0], dtype=torch.bool, device=dev)
    for s in range(0, S, 8):                               # the last drafted position's value: only the last row sees it
        t = lens[s] + drafts[s] - 1
        kv[0, 1, int(table[s, t // page]), :, t % page, 5] = math.inf
        hit[int(begin[s + 1]) - 1] = True
    for _ in range(10):
        got = pool.tree_attention(0, book, q, i32(begin, dev))[0]
        assert bool(torch.isinf(got[hit][..., 5]).all()) and bool((got[~hit] == plain[~hit]).all())
        got[hit, :, 5] = 0
        assert bool(torch.isfinite(got).all())
    pool.check()


def test_page_calls_in_graphs_and_on_streams(dev):
    """Fork, draft, attend, keep, compact as one captured graph, replayed over new contents; a second graph on another stream beside it."""
    rng = np.random.default_rng(3)
    S, H, d, page, P = 6, 2, 64, 16, 90

    def state(seed):
        gen = torch.Generator(device=dev).manual_seed(seed)
        kv = torch.randn(2, 2, P, H, page, d, device=dev, generator=gen).half()
        table, ref = make_book(np.random.default_rng(seed), [3] * S, 6, P, dev)
        return kv, table, ref, [20 + 4 * i for i in range(S)]

    parent, room = i32([0, 0, 2, 3, 3, 5], dev), i32([5] * S, dev)
    begin, q = i32([0] + [5 * (i + 1) for i in range(S)], dev), torch.randn(5 * S, 2 * H, d, device=dev).half()
    path, n_path = i32(rng.permutation(5)[:2].repeat(S).reshape(2, S).T.copy(), dev).sort(1).values.contiguous(), i32([2, 1, 0, 2, 2, 1], dev)

    def steps(pool, book):
        new = pool.fork(book, parent, room)
        out = pool.tree_attention(1, new, q, begin)
        kept = pool.keep(new, path, n_path)
        small, moved = pool.compact(kept)
        return out + (kept.table, kept.len, kept.ref, small.table, small.len, small.ref, moved)

    def eager(seed):
        kv, table, ref, lens = state(seed)
        pool = plc.PagePool(kv)
        res = [t.clone() for t in steps(pool, book_of(table, lens, ref, dev))]
        pool.check()
        return res + [kv]

    want = {seed: eager(seed) for seed in range(3)}
    held = []
    for seed in range(2):
        kv, table, ref, lens = state(seed)
        pool, book, g = plc.PagePool(kv), book_of(table, lens, ref, dev), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = steps(pool, book)
        held.append((g, pool, book, res, kv))
    sides = [torch.cuda.Stream(dev), torch.cuda.Stream(dev)]
    torch.cuda.synchronize()
    for (g, *_), side in zip(held, sides):                 # both at once
        with torch.cuda.stream(side):
            g.replay()
    torch.cuda.synchronize()
    for seed, (g, pool, book, res, kv) in enumerate(held):
        assert all(torch.equal(a, b) for a, b in zip(list(res) + [kv], want[seed]))
    for g, pool, book, res, kv in held:                    # other contents in the same places
        kv2, table, ref, lens = state(2)
        kv.copy_(kv2)
        book.table.copy_(i32(table, dev)), book.ref.copy_(i32(ref, dev)), book.len.copy_(i32(lens, dev))
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(list(res) + [kv], want[2]))
        pool.check()


def test_beam_calls_in_graphs_and_on_streams(dev):
    gen = torch.Generator(device=dev).manual_seed(4)
    sets = [(torch.randn(3, 8, 5003, device=dev, generator=gen).half(), torch.randn(3, 8, device=dev, generator=gen), torch.randn(24, 7, device=dev, generator=gen)) for _ in range(3)]

    def steps(logits, score, tokens):
        s, parent, token = plc.beam_select(logits, score, 8)
        return [s, parent, token] + plc.beam_reorder(parent.view(-1), [tokens])

    want = [[t.clone() for t in steps(*x)] for x in sets]
    held = []
    for i in range(2):
        x = [t.clone() for t in sets[i]]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = steps(*x)
        held.append((g, x, res))
    torch.cuda.synchronize()
    for g, _, _ in held:
        with torch.cuda.stream(torch.cuda.Stream(dev)):
            g.replay()
    torch.cuda.synchronize()
    for i, (g, x, res) in enumerate(held):
        assert all(torch.equal(a, b) for a, b in zip(res, want[i]))
        for a, b in zip(x, sets[2]):
            a.copy_(b)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(res, want[2]))


def test_reordering_of_many_states_and_odd_rows(dev):
    """More tensors than one launch takes, rows of one to 4099 bytes, rows without anything, expanded rows, one parent for all."""
    gen = torch.Generator(device=dev).manual_seed(6)
    states = [torch.randint(0, 255, (5, n), device=dev, generator=gen, dtype=torch.uint8) for n in (1, 2, 3, 5, 7, 15, 16, 17, 31, 33, 64, 127, 255, 1025, 4096, 4099, 12, 9, 0)]
    states += [torch.randn(5, 3, 2, device=dev, generator=gen)[:, 1], torch.randn(1, 9, device=dev, generator=gen).expand(5, 9), torch.arange(5, device=dev)]
    for parent in ([4, 4, 4], [0, -1, 2, 3, 4, 1, 0], [-1]):
        rows = torch.tensor(parent, device=dev)
        for a, b in zip(plc.beam_reorder(i32(parent, dev), states), states):
            want = b[rows.clamp(min=0)].clone()
            want[rows < 0] = 0
            assert torch.equal(a, want)


def test_lengths_near_two_to_the_31(dev):
    """One page named by 2^17 entries of a row: lengths that an int holds, but not with a tile's positions added, are refused."""
    page, cols = 1 << 14, (1 << 17) + 2
    pool = plc.PagePool(torch.zeros(1, 2, 2, 1, page, 32, dtype=torch.float16, device=dev))
    table = torch.zeros(1, cols, dtype=torch.int32, device=dev)
    q, begin = torch.zeros(1, 1, 32, dtype=torch.float16, device=dev), i32([0, 0], dev)
    for length in (0x7fffffff, 0x7fff0001):
        book = plc.PageBook(table, i32([length], dev), i32([cols, 0], dev))
        for call in (lambda: pool.fork(book, i32([0], dev)), lambda: pool.keep(book, i32([[1]], dev), i32([1], dev)), lambda: pool.tree_attention(0, book, q, begin)):
            call()
            with pytest.raises(plc.PlcError) as e:
                pool.check()
            assert e.value.code == plc.E_INVALID


@pytest.mark.parametrize("pages, page, L", [(40, 4, 1), (40, 64, 2), (17000, 4, 1)])
def test_small_and_large_page_calls_alike(dev, ora, pages, page, L):
    """Calls that one cluster does, and the same ones that more blocks do because of a page's bytes or the pages' number."""
    rng = np.random.default_rng(pages + page)
    kv, _ = make_pool(rng, L, pages, 2, page, 32, "f16", dev, False)
    lens = [page * 2 + 1]
    table, ref = np.full((1, 8), -1, np.int32), np.zeros(pages, np.int32)
    held = pages - 1 - np.arange(4)
    table[0, :4] = held
    ref[held] = 1
    pool = plc.PagePool(kv)
    book = book_of(table, lens, ref, dev)
    was = kv[:, :, torch.as_tensor(held.astype(np.int64)).to(dev)].clone()
    two = pool.fork(book, i32([0, 0], dev), i32([page, 1], dev))
    t, n, r = (x.cpu().numpy() for x in (two.table, two.len, two.ref))
    assert n.tolist() == [page * 2 + 1] * 2 and (t[:, :2] == held[:2]).all() and r[held[:2]].tolist() == [2, 2] and r.sum() == (t >= 0).sum()
    assert t[0, 2] == held[2] and t[1, 2] != held[2] and len(set(t[t >= 0])) == len(t[t >= 0]) - 2
    assert torch.equal(kv[:, :, int(t[1, 2]), :, :1], was[:, :, 2, :, :1])
    got = pool.keep(book, i32([[1, 2]], dev), i32([2], dev))
    x = was.permute(0, 1, 3, 2, 4, 5).reshape(L, 2, 2, 4 * page, 32)[:, :, :, page * 2 + 2:page * 2 + 4]
    at = [page * 2 + 1, page * 2 + 2]
    for i, p in enumerate(at):
        assert torch.equal(kv[:, :, int(held[p // page]), :, p % page], x[:, :, :, i])
    assert got.len.tolist() == [page * 2 + 3] and got.table.cpu().numpy()[0].tolist() == [*held[:3], -1, -1, -1, -1, -1] and int(got.ref.sum()) == 3
    low, moved = pool.compact(got)
    assert sorted(low.table.cpu().numpy()[0, :3].tolist()) == [0, 1, 2] and low.ref[:3].tolist() == [1, 1, 1] and int(low.ref.sum()) == 3
    m = moved.cpu().numpy()
    assert (m[held[:3]] == low.table.cpu().numpy()[0, :3]).all()
    for i in range(2):
        assert torch.equal(kv[:, :, int(m[held[i]])], was[:, :, i])
    pool.check()


@pytest.mark.parametrize("dtype, d, H, G, page, cols, n", [("f16", 64, 1, 1, 16, 24, [1]), ("bf16", 128, 8, 4, 32, 12, [1, 0, 3]), ("f16", 128, 4, 8, 12, 32, [9, 1]),
                                                           ("bf16", 128, 4, 8, 128, 3, [30, 2]), ("f16", 256, 2, 8, 64, 6, [40, 0, 0, 1]), ("bf16", 32, 8, 2, 8, 48, [1] * 18)])
def test_attention_of_few_short_items(dev, dtype, d, H, G, page, cols, n):
    """Calls whose rows of pages are so short that no item is split, beside the same contents in a longer book, where they are."""
    rng = np.random.default_rng(cols)
    S = len(n)
    lens = [int(rng.integers(0, page * cols - max(n) + 1)) for _ in range(S)]
    lens[0] = page * cols - n[0]
    held = [-(-(a + b) // page) for a, b in zip(lens, n)]
    table, ref = make_book(rng, held, cols, sum(held) + 1, dev)
    gen = torch.Generator(device=dev).manual_seed(0)
    kv = torch.randn(1, 2, sum(held) + 1, H, page, d, device=dev, generator=gen).to(TYPES[dtype])
    begin = np.cumsum([0] + n).astype(np.int32)
    q = torch.randn(int(begin[-1]), H * G, d, device=dev, generator=gen).to(TYPES[dtype])
    ex, mag, big = attention_in_64_bits(kv, 0, table, lens, q, begin, None, 1 / math.sqrt(d))
    u = torch.finfo(TYPES[dtype]).eps / 2
    e = 2 * (d * 2.0 ** -23 * big + 2.0 ** -22 + 2.0 ** -23 * 2 * big)
    tol = (u + e[..., None] + page * cols * 2.0 ** -23) * mag + u * ex.abs() + torch.finfo(TYPES[dtype]).smallest_normal * u
    pool = plc.PagePool(kv)
    for t in (table, np.concatenate([table, np.full((S, 1000), -1, np.int32)], 1)):
        got = pool.tree_attention(0, book_of(t, lens, ref, dev), q, i32(begin, dev))[0]
        assert bool(((got.double() - ex).abs() <= tol).all())
    pool.check()


@pytest.mark.parametrize("n, lens", [([2, 1], [300, 40]), ([40, 3], [1000, 7]), ([5, 60], [0, 2000])])
def test_attention_into_strided_results_and_from_expanded_queries(dev, n, lens):
    """Results as a view of a wider tensor whose other elements stay as they are; one query row for all."""
    rng = np.random.default_rng(1)
    H, G, d, page = 2, 8, 128, 32
    held = [-(-(a + b) // page) for a, b in zip(lens, n)]
    table, ref = make_book(rng, held, max(held), sum(held), dev)
    gen = torch.Generator(device=dev).manual_seed(2)
    kv = torch.randn(1, 2, sum(held), H, page, d, device=dev, generator=gen).half()
    begin = np.cumsum([0] + n).astype(np.int32)
    N = int(begin[-1])
    pool, book = plc.PagePool(kv), book_of(table, lens, ref, dev)
    q = torch.randn(1, H * G, d, device=dev, generator=gen).half().expand(N, H * G, d)
    want, lse = pool.tree_attention(0, book, q.contiguous(), i32(begin, dev))
    wide = torch.full((N, H * G + 2, d + 24), 5.0, dtype=torch.float16, device=dev)
    got, lse2 = pool.tree_attention(0, book, q, i32(begin, dev), out=wide[:, 1:-1, 16:-8])
    assert torch.equal(got, want) and torch.equal(lse, lse2)
    wide[:, 1:-1, 16:-8] = 5.0
    assert bool((wide == 5).all())
    pool.check()


# ---------------------------------------------------------------------------------------------- calls at the borders

@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("V", [259, 32000, 70001])
def test_beam_selection_at_the_lowest_values(dev, dtype, V):
    """Tokens masked with the type's lowest finite value: all of a beam's, all but one, some, of several sessions.  A beam that is masked as a
    whole has each token at its score less log V.  Exact values by the formula in binary64, the row's maximum taken off first; tolerance as above."""
    low = torch.finfo(TYPES[dtype]).min
    rng = np.random.default_rng(V)
    x = spaced(rng, 4, 4, V, dtype, dev)
    x[0, 0] = low
    x[0, 2] = low
    x[0, 2, V - 2] = 1.5
    x[0, 3, ::2] = low
    x[1] = low                                               # nothing else in the session
    x[2, 1:] = low
    x[2, 0] = low
    x[2, 0, 17] = -4.0
    x[3, :, 1:] = low
    cum = torch.tensor([[-5.0, -20.0, -9.3, -30.17], [-20.0, -math.inf, -20.0, -19.51], [-7.0, -math.inf, -math.inf, -math.inf], [-4.0, -3.0, -2.0, -1.0]], device=dev)
    n_out = 40
    f = x.double()
    f = f - f.amax(-1, keepdim=True)
    f = ((f - f.exp().sum(-1, keepdim=True).log()) + cum.double()[..., None]).flatten(1)
    best, at = f.sort(dim=1, descending=True, stable=True)
    step = (best[:, :n_out] - best[:, 1:n_out + 1]).cpu()
    assert bool((torch.isnan(step) | (step == 0) | (step > 2.0 ** -18)).all())
    best, at = best[:, :n_out], at[:, :n_out]
    none = best == -math.inf
    s, p, t = plc.beam_select(x, cum, n_out)
    assert torch.equal(p.long(), torch.where(none, -1, at // V + 4 * torch.arange(4, device=dev)[:, None])) and torch.equal(t.long(), torch.where(none, -1, at % V))
    assert bool((s[none] == -math.inf).all()) and bool(((s.double() - best).abs() <= 2.0 ** -20 + 2.0 ** -23 * best.abs())[~none].all())
    assert p[1, 0] == 7 and abs(float(s[1, 0]) - (-19.51 - math.log(V))) < 1e-4


def test_no_status_is_lost_while_it_is_read(dev, monkeypatch):
    """A call that finds something wrong between the reading of the word and the end of check() is told of by the next check()."""
    pool = plc.PagePool(torch.zeros(1, 2, 8, 1, 4, 32, dtype=torch.float16, device=dev))
    book, side, real, late = pool.new_book(2, 3), torch.cuda.Stream(dev), torch.Tensor.item, [True]
    torch.cuda.synchronize()

    def wrong():                                           # a parent that there is not
        with torch.cuda.stream(side):
            pool.fork(book, i32([5, 0], dev))
        side.synchronize()

    def item(self):
        value = real(self)
        if late:
            late.clear()
            wrong()
        return value

    with monkeypatch.context() as m:
        m.setattr(torch.Tensor, "item", item)
        pool.check()                                       # nothing was wrong when the word was read
    for _ in range(2):
        with pytest.raises(plc.PlcError) as e:
            pool.check()
        assert e.value.code == plc.E_INVALID
        pool.check()
        wrong()
    with pytest.raises(plc.PlcError):
        pool.check()


def test_numbers_that_are_no_int32_are_refused(dev):
    """Layers, end tokens and counts that hold the number of a valid one in their low 32 bits."""
    kv = torch.zeros(2, 2, 4, 1, 16, 64, dtype=torch.float16, device=dev)
    pool, q, begin = plc.PagePool(kv), torch.zeros(1, 1, 64, dtype=torch.float16, device=dev), i32([0, 1], dev)
    book = pool.fork(pool.new_book(1, 2), i32([0], dev), i32([4], dev))
    x, score, done = torch.zeros(1, 2, 8, device=dev), torch.zeros(1, 2, device=dev), torch.tensor([[True, False]], device=dev)
    for wide in (1 << 32, -(1 << 32), 1 << 63):
        for code, call in ((plc.E_INVALID, lambda: pool.tree_attention(wide + 1, book, q, begin)), (plc.E_INVALID, lambda: plc.beam_select(x, score, 2, done=done, eos=wide + 3)),
                           (plc.E_SHAPE, lambda: plc.beam_select(x, score, wide + 2))):
            with pytest.raises(plc.PlcError) as e:
                call()
            assert e.value.code == code
    pool.check()


@pytest.mark.parametrize("cols", [2, 40])
@pytest.mark.parametrize("dtype, d, H, G, page", [("f16", 64, 1, 2, 16), ("bf16", 128, 2, 8, 16), ("bf16", 128, 2, 24, 16), ("f16", 128, 1, 40, 16), ("bf16", 256, 1, 16, 16),
                                                  ("f16", 32, 1, 2, 12), ("bf16", 64, 1, 40, 12)])
def test_attention_answers_for_what_is_left_of_ranges_and_lengths(dev, dtype, d, H, G, page, cols):
    """Row ranges, lengths and pages out of range: the rows that are left get the formula's value over the positions that are left (tolerance as above), the
    others stay as they were, and each call is told of.  Items taken whole and split, few rows and many, boxes and single positions."""
    rng = np.random.default_rng(d + G + cols)
    most, P, N = cols * page, 4, 5
    kv = torch.from_numpy(rng.standard_normal((1, 2, P, H, page, d)).astype(np.float32)).to(TYPES[dtype]).to(dev)
    q = torch.from_numpy(rng.standard_normal((N, H * G, d)).astype(np.float32)).to(TYPES[dtype]).to(dev)
    pool, scale = plc.PagePool(kv), 1 / math.sqrt(d)
    for lens, begin, missing in (([most + 8], [0, 9], ()), ([-3], [0, 2], ()), ([most - 2], [1, 5], ()), ([10], [2, 1], ()), ([10], [-2, 3], ()), ([1 << 30], [0, 4], ()),
                                 ([3, most], [0, 3, 2], ()), ([most - 1, 7], [1, 3, 77], ()), ([page + 3], [0, 2], ((0, 1),)), ([-7, -7], [-5, -4, 2], ())):
        S = len(lens)
        table = rng.integers(0, P, (S, cols)).astype(np.int32)
        for s, c in missing:
            table[s, c] = P + 3
        out, lse = torch.full((N, H * G, d), 5.0, dtype=TYPES[dtype], device=dev), torch.full((N, H * G), 7.0, device=dev)
        pool.tree_attention(0, book_of(table, lens, np.ones(P), dev), q, i32(begin, dev), out=out, lse=lse)
        with pytest.raises(plc.PlcError) as e:
            pool.check()
        assert e.value.code == plc.E_INVALID
        rest = torch.ones(N, dtype=torch.bool, device=dev)
        for s in range(S):
            lo = min(max(begin[s], 0), N)
            hi = min(max(begin[s + 1], lo), N)
            at = min(max(lens[s], 0), most)
            t = np.arange(min(at + hi - lo, most))
            t = t[table[s, t // page] < P]
            pages, slots = torch.as_tensor(table[s, t // page].astype(np.int64), device=dev), torch.as_tensor(t % page, device=dev)
            k, v = (kv[0, j, pages, :, slots].double().transpose(0, 1) for j in range(2))       # [H][positions][d]
            for row in range(lo, hi):
                rest[row] = False
                sees = torch.as_tensor(t <= at + row - lo, device=dev)
                x = q[row].double().view(H, G, d)
                z = (torch.einsum("hgd,htd->hgt", x, k) * scale).masked_fill(~sees, -math.inf)
                big = (torch.einsum("hgd,htd->hgt", x.abs(), k.abs()) * scale).amax(-1).flatten()
                want, mag = (torch.einsum("hgt,htd->hgd", z.softmax(-1), y).reshape(H * G, d) for y in (v, v.abs()))
                u, err = torch.finfo(TYPES[dtype]).eps / 2, 2 * (d * 2.0 ** -23 * big + 2.0 ** -22 + 2.0 ** -23 * 2 * big) + len(t) * 2.0 ** -23
                tol = (u + err[:, None]) * mag + u * want.abs() + torch.finfo(TYPES[dtype]).smallest_normal * u
                assert bool(((out[row].double() - want).abs() <= tol).all()), (lens, begin, row)
                exl = z.logsumexp(-1).flatten()
                assert bool(((lse[row].double() - exl).abs() <= err + 2.0 ** -22 * exl.abs()).all()), (lens, begin, row)
        assert bool((out[rest] == 5).all()) and bool((lse[rest] == 7).all()), (lens, begin)


def test_attention_over_two_to_the_31_positions(dev):
    """The longest row that is taken, its entries naming four pages over and over: the softmax over the four, each as often as it stands there.  The
    sums: a CTA (148 or more) has at most 2^24 / 148 tiles, whose sums a thread adds in binary32 and whose eight products each are added to the
    result at a step of 2^-23 at most."""
    page, d, cols = 1 << 14, 64, 131068                    # 131068 * 2^14 = 2^31 - 2^16
    gen = torch.Generator(device=dev).manual_seed(8)
    kv = torch.randn(1, 2, 4, 1, page, d, device=dev, generator=gen).half()
    kv[0, 1] += torch.arange(4, device=dev)[:, None, None, None]
    table = torch.randint(0, 4, (1, cols), dtype=torch.int32, device=dev, generator=gen)
    q = torch.randn(1, 2, d, device=dev, generator=gen).half()
    pool = plc.PagePool(kv)
    times = torch.bincount(table[0], minlength=4)
    out, lse = pool.tree_attention(0, plc.PageBook(table, i32([cols * page - 1], dev), times.int()), q, i32([0, 1], dev))
    pool.check()
    k, v = (kv[0, j, :, 0].double() for j in range(2))
    z = torch.einsum("hd,ptd->hpt", q[0].double(), k) / 8
    big = (torch.einsum("hd,ptd->hpt", q[0].double().abs(), k.abs()) / 8).amax((1, 2))
    z = (z + times.double().log()[:, None]).flatten(1)
    p, tiles = z.softmax(-1), -(-(1 << 24) // 148)
    want, mag = p @ v.reshape(-1, d), p @ v.reshape(-1, d).abs()
    e = 2 * (d * 2.0 ** -23 * big + 2.0 ** -22 + 2.0 ** -23 * 2 * big)
    assert bool(((lse[0].double() - z.logsumexp(-1)).abs() <= e + tiles * 2.0 ** -24 + 2.0 ** -22 * 32).all())
    tol = (2.0 ** -11 + e[:, None] + tiles * 2.0 ** -24 + 8 * tiles * 2.0 ** -23) * mag + 2.0 ** -11 * want.abs()
    assert bool(((out[0].double() - want).abs() <= tol).all())
