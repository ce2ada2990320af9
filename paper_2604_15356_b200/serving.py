"""Paged KV cache, attention of drafted tokens over it, and beam search: binding of the plc_pages_*, plc_tree_attention
and plc_beam_* calls.

As in the rest of the binding nothing is computed here: tensors become pointers, and the work runs on the current stream
of the tensors' device.  Results and workspaces are allocated by torch on that stream, so that calls on several streams
and captured graphs do not share any.
"""
import ctypes as C

from . import E_ALIGN, E_CAPACITY, E_CUDA, E_INVALID, E_SHAPE, OUT_BF16, OUT_F16, OUT_F32, KVView, PlcError, PoolView, _check, lib


class PagePoolC(C.Structure):
    _fields_ = [("view", KVView), ("n_layers", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("n_pages", C.c_int32),
                ("page_pos", C.c_int32), ("dtype", C.c_int32)]


class PageBookC(C.Structure):
    _fields_ = [("table_dev", C.c_void_p), ("len_dev", C.c_void_p), ("ref_dev", C.c_void_p), ("rows", C.c_int32), ("max_pages", C.c_int32)]


class TreeQueries(C.Structure):
    _fields_ = [("q_dev", C.c_void_p), ("q_stride_row", C.c_int64), ("q_stride_head", C.c_int64), ("out_dev", C.c_void_p),
                ("out_stride_row", C.c_int64), ("out_stride_head", C.c_int64), ("lse_dev", C.c_void_p), ("begin_dev", C.c_void_p),
                ("mask_dev", C.c_void_p), ("n_rows", C.c_int32), ("n_heads", C.c_int32), ("mask_words", C.c_int32)]


class RowSet(C.Structure):
    _fields_ = [("src_dev", C.c_void_p), ("dst_dev", C.c_void_p), ("src_stride", C.c_int64), ("dst_stride", C.c_int64), ("row_bytes", C.c_int64)]


def _need(ok, code, where):
    if not ok:
        raise PlcError(code, where)


def _int32(code, where, *values):
    """What the library takes as int32: ctypes would cut larger numbers to their low bits."""
    for v in values:
        if not -0x80000000 <= v <= 0x7fffffff:
            raise PlcError(code, where)


_api = None


def _lib():
    """The library with the argument types of this module's calls set, so that plain integers can be passed."""
    global _api
    if _api is None:
        api, P, I, L, F = lib(), C.c_void_p, C.c_int32, C.c_int64, C.c_float
        U = C.c_uint64
        for name, types in (("plc_pages_fork", [P, P, P, P, P, P, U, P, P]), ("plc_pages_keep", [P, P, P, P, I, P, P, P]),
                            ("plc_pages_compact", [P, P, P, P, P, U, P, P]), ("plc_pages_workspace", [I, I, I, P]), ("plc_take_status", [P, P, P]),
                            ("plc_tree_attention", [P, I, P, P, F, P, U, P, P]), ("plc_tree_attention_workspace", [P, I, I, I, P]),
                            ("plc_beam_select", [P, I, L, I, I, I, P, P, I, I, P, P, P, P, U, P]), ("plc_beam_workspace", [I, I, I, I, P]),
                            ("plc_beam_reorder", [P, I, P, I, I, P, P])):
            getattr(api, name).argtypes = types
        _api = api
    return _api


_KINDS = {}


def _kind(dtype, where, wide=True):
    import torch
    if not _KINDS:
        _KINDS.update({torch.float16: OUT_F16, torch.bfloat16: OUT_BF16, torch.float32: OUT_F32})
    kind = _KINDS.get(dtype)
    _need(kind is not None and (wide or kind != OUT_F32), E_INVALID, where)
    return kind


def _i32(t, device, where):
    """t as what the library reads: int32, contiguous, on the device."""
    import torch
    if t.dtype != torch.int32 or t.device != device or not t.is_contiguous():
        raise PlcError(E_INVALID, where)
    return t


def _run(device, call, *args):
    """The call on the current stream of the tensors' device, with that device current."""
    import torch
    if torch.cuda.current_device() == device.index:
        return call(*args, torch._C._cuda_getCurrentRawStream(device.index))
    with torch.cuda.device(device):
        return call(*args, torch._C._cuda_getCurrentRawStream(device.index))


_sizes = {}


def _bytes(device, call, *args):
    """A workspace size, asked for once a device (it may go by the device's size)."""
    import torch
    key = (device.index, call.__name__) + args
    n = _sizes.get(key)
    if n is None:
        b = C.c_uint64()
        with torch.cuda.device(device):
            _check(call(*args, C.byref(b)), call.__name__)
        if len(_sizes) >= 4096:
            _sizes.clear()
        n = _sizes[key] = b.value
    return n


class PageBook:
    """Who holds which page: table [rows][max_pages], len [rows], ref [pages] (int32 on the device).  Calls return new
    books; an old one stays valid until a page that only it names is taken by a later call.  A book that a call has made is
    one allocation, with that call's workspace (about 16 bytes a page) behind it for as long as the book lives."""

    def __init__(self, table, len, ref):
        dev = table.device
        for t, n, dim in ((table, "table", 2), (len, "len", 1), (ref, "ref", 1)):
            _i32(t, dev, "PageBook." + n)
            _need(t.dim() == dim, E_SHAPE, "PageBook." + n)
        _need(len.shape[0] == table.shape[0], E_SHAPE, "PageBook.len")
        _int32(E_SHAPE, "PageBook", *table.shape, *ref.shape)
        self._parts = (table, len, ref)
        self.rows, self.max_pages = table.shape
        self.n_pages, self.device = ref.shape[0], dev
        self._c = PageBookC(table.data_ptr(), len.data_ptr(), ref.data_ptr(), self.rows, self.max_pages)
        self._by = C.byref(self._c)

    @classmethod
    def _new(cls, rows, max_pages, n_pages, device, extra=0):
        """A book that a call fills, in one allocation; (book, address of `extra` bytes behind it)."""
        import torch
        self = cls.__new__(cls)
        n = rows * max_pages
        words = (n + rows + n_pages + 3) & ~3
        self._store = torch.empty(words + (extra + 3) // 4, dtype=torch.int32, device=device)
        at = self._store.data_ptr()
        self._parts = None
        self.rows, self.max_pages, self.n_pages, self.device = rows, max_pages, n_pages, device
        self._c = PageBookC(at, at + 4 * n, at + 4 * (n + rows), rows, max_pages)
        self._by = C.byref(self._c)
        return self, at + 4 * words

    def _views(self):
        if self._parts is None:
            n, s = self.rows * self.max_pages, self._store
            self._parts = (s.as_strided((self.rows, self.max_pages), (self.max_pages, 1), 0), s.as_strided((self.rows,), (1,), n),
                           s.as_strided((self.n_pages,), (1,), n + self.rows))
        return self._parts

    @property
    def table(self):
        return self._views()[0]

    @property
    def len(self):
        return self._views()[1]

    @property
    def ref(self):
        return self._views()[2]


class PagePool:
    """Pages of a KV cache: kv indexed [layer][2][page][head][slot][component], any strides with the components
    contiguous and every vector on a 16-byte boundary (float16, bfloat16; float32 for everything but attention)."""

    def __init__(self, kv):
        import torch
        _need(kv.dim() == 6 and kv.shape[1] == 2 and kv.stride(5) == 1, E_SHAPE, "PagePool")
        _need(kv.is_cuda, E_INVALID, "PagePool")
        self.kv, self.device, self.n_pages = kv, kv.device, kv.shape[2]
        s = kv.stride()
        L, _, P, H, page, d = kv.shape
        _int32(E_SHAPE, "PagePool", L, P, H, page, d)
        self._c = PagePoolC(KVView(kv.data_ptr(), s[0], s[1], s[2], s[3], s[4]), L, H, d, P, page, _kind(kv.dtype, "PagePool"))
        self._by = C.byref(self._c)
        self.status = torch.zeros(1, dtype=torch.int32, device=kv.device)
        self._word = self.status.data_ptr()
        self._need_bytes = {}

    def new_book(self, rows, max_pages):
        """A book of empty rows over a pool whose pages are all free."""
        import torch
        dev = self.device
        return PageBook(torch.full((rows, max_pages), -1, dtype=torch.int32, device=dev), torch.zeros(rows, dtype=torch.int32, device=dev),
                        torch.zeros(self.n_pages, dtype=torch.int32, device=dev))

    def sessions_view(self, first_page, sessions, n):
        """KVView of consecutive pages as plain sessions of n positions, for Context.encode / Context.decode: session i
        has the pages first_page + i * ceil(n / page) ....  Needs slots before heads, so that a page follows the other.
        The pool's type has to be what the call works in: float16 for encoding, the context's out_dtype for decoding (a
        pool that attention reads: out_dtype=OUT_F16; bfloat16 pools have no such calls)."""
        c, page = self._c, self.kv.shape[4]
        each = -(-n // page)
        _need(c.view.stride_session == page * c.view.stride_pos, E_SHAPE, "sessions_view")
        _need(first_page >= 0 and sessions >= 1 and n >= 1 and first_page + sessions * each <= c.n_pages, E_INVALID, "sessions_view")
        v = c.view
        view = PoolView(self.kv.data_ptr() + first_page * v.stride_session * self.kv.element_size(), v.stride_layer, v.stride_kv,
                        each * v.stride_session, v.stride_head, v.stride_pos)
        view.dtype, view.extents = c.dtype, (c.n_layers, c.n_kv_heads, c.head_dim, sessions, each * page)
        return view

    def _book(self, book, where):
        _need(book.device == self.device, E_INVALID, where)
        _need(book.n_pages == self.n_pages, E_SHAPE, where)
        return book._by

    def fork(self, book, parent, room=None):
        """New book whose row s continues row parent[s] (-1: empty), with pages for room[s] positions more."""
        where, dev, api = "plc_pages_fork", self.device, _lib()
        a = self._book(book, where)
        rows = _i32(parent, dev, where).numel()
        _need(rows >= 1, E_INVALID, where)
        _int32(E_SHAPE, where, rows)
        if room is not None:
            _need(_i32(room, dev, where).numel() == rows, E_SHAPE, where)
        need = _bytes(dev, api.plc_pages_workspace, self.n_pages, book.rows, rows)
        new, ws = PageBook._new(rows, book.max_pages, self.n_pages, dev, need)
        _check(_run(dev, api.plc_pages_fork, self._by, a, parent.data_ptr(), None if room is None else room.data_ptr(), new._by, ws, need, self._word), where)
        return new

    def keep(self, book, path, n_path):
        """New book after the drafted positions path[s][:n_path[s]] of every row have been accepted (path: one column or more)."""
        where, dev, api = "plc_pages_keep", self.device, _lib()
        a = self._book(book, where)
        _i32(path, dev, where)
        _i32(n_path, dev, where)
        _need(path.dim() == 2 and path.shape[0] == book.rows == n_path.numel(), E_SHAPE, where)
        _int32(E_SHAPE, where, path.shape[1])
        new, _ = PageBook._new(book.rows, book.max_pages, self.n_pages, dev)
        _check(_run(dev, api.plc_pages_keep, self._by, a, path.data_ptr(), n_path.data_ptr(), path.shape[1], new._by, self._word), where)
        return new

    def compact(self, book):
        """(new book, moved): the pages in use have the lowest numbers; moved[p] is page p's new number (-1: free)."""
        import torch
        where, dev, api = "plc_pages_compact", self.device, _lib()
        a = self._book(book, where)
        need = _bytes(dev, api.plc_pages_workspace, self.n_pages, book.rows, book.rows)
        new, ws = PageBook._new(book.rows, book.max_pages, self.n_pages, dev, need)
        moved = torch.empty(self.n_pages, dtype=torch.int32, device=dev)
        _check(_run(dev, api.plc_pages_compact, self._by, a, new._by, moved.data_ptr(), ws, need, self._word), where)
        return new, moved

    def tree_attention(self, layer, book, q, begin, mask=None, scale=None, out=None, lse=None):
        """(out, lse) of the query rows q [N][heads][d]; session s has the rows begin[s] .. begin[s+1]-1, whose keys and
        values stand behind its length.  mask [N][words] int32: bit j of row i = drafted position j is seen (None: j <= i).
        scale: positive, 1 / sqrt(d) if not given.  out, lse: written where given.  Chunks of prompts go into a call of
        their own: one call's work is cut by the mean number of rows."""
        import torch
        where, dev, api = "plc_tree_attention", self.device, _lib()
        a = self._book(book, where)
        _need(q.dim() == 3, E_SHAPE, where)
        (N, heads, d), (row, head, one) = q.shape, q.stride()
        _need(d == self._c.head_dim, E_SHAPE, where)
        _int32(E_INVALID, where, layer)
        _int32(E_SHAPE, where, N, heads)
        _need(q.device == dev and q.dtype == self.kv.dtype and one == 1, E_INVALID, where)
        _kind(q.dtype, where, wide=False)
        _need(_i32(begin, dev, where).numel() == book.rows + 1, E_SHAPE, where)
        words, bits = 0, None
        if mask is not None:
            _i32(mask, dev, where)
            _need(mask.dim() == 2 and mask.shape[0] == N, E_SHAPE, where)
            words, bits = mask.shape[1], mask.data_ptr()
            _int32(E_SHAPE, where, words)
        if out is None:
            out = torch.empty((N, heads, d), dtype=q.dtype, device=dev)
            out_row, out_head = heads * d, d
        else:
            _need(out.shape == q.shape and out.dtype == q.dtype and out.device == dev and out.stride(2) == 1, E_INVALID, where)
            out_row, out_head, _ = out.stride()
        if lse is None:
            lse = torch.empty((N, heads), dtype=torch.float32, device=dev)
        else:
            _need(lse.shape == (N, heads) and lse.dtype == torch.float32 and lse.device == dev and lse.is_contiguous(), E_INVALID, where)
        if N == 0:
            return out, lse
        need = self._need_bytes.get((book.rows, heads, N))
        if need is None:
            b = C.c_uint64()
            with torch.cuda.device(dev):
                _check(api.plc_tree_attention_workspace(self._by, book.rows, heads, N, C.byref(b)), "plc_tree_attention_workspace")
            if len(self._need_bytes) >= 4096:
                self._need_bytes.clear()
            need = self._need_bytes[(book.rows, heads, N)] = b.value
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
        t = TreeQueries(q.data_ptr(), row, head, out.data_ptr(), out_row, out_head, lse.data_ptr(), begin.data_ptr(), bits, N, heads, words)
        _check(_run(dev, api.plc_tree_attention, self._by, layer, a, C.byref(t), d ** -0.5 if scale is None else scale, ws.data_ptr(), need, self._word), where)
        return out, lse

    def check(self):
        """Waits for the current stream's work and raises where a call has found something wrong on the device; clears the word.
        What a call that still runs on another stream finds stays there for the next check."""
        import torch
        taken = torch.empty(1, dtype=torch.int32, device=self.device)
        _check(_run(self.device, _lib().plc_take_status, self._word, taken.data_ptr()), "plc_take_status")
        bits = int(taken.item())
        for bit, code in ((8, E_CUDA), (1, E_CAPACITY), (32, E_INVALID)):
            _need(not bits & bit, code, f"status word {bits}")


def beam_select(logits, score, n_out, done=None, eos=-1):
    """(score, parent, token), each [sessions][n_out], of the n_out best continuations of every session: logits
    [sessions][beams][vocab], score [sessions][beams] float32, done [sessions][beams] bool.  parent counts the rows of all
    sessions (-1, with token -1 and score -inf: no continuation)."""
    import torch
    where, dev, api = "plc_beam_select", logits.device, _lib()
    _need(logits.is_cuda and logits.dim() == 3, E_INVALID, where)
    (S, W, V), (session, row, one) = logits.shape, logits.stride()
    _need(one == 1, E_INVALID, where)
    _int32(E_SHAPE, where, S, W, V, n_out)
    _int32(E_INVALID, where, eos)
    _need(S < 2 or W < 2 or session == W * row, E_SHAPE, where)
    if W < 2:
        row = session
    _need(score.dtype == torch.float32 and score.device == dev and score.is_contiguous() and score.shape == (S, W), E_INVALID, where)
    if done is not None:
        _need(done.dtype == torch.bool and done.device == dev and done.is_contiguous() and done.shape == (S, W), E_INVALID, where)
    kind = _kind(logits.dtype, where)
    need = _bytes(dev, api.plc_beam_workspace, S, W, V, n_out)
    n = S * n_out
    ws = torch.empty(need, dtype=torch.uint8, device=dev)
    out = torch.empty((S, n_out), dtype=torch.float32, device=dev)
    store = torch.empty(2 * n, dtype=torch.int32, device=dev)
    at = store.data_ptr()
    _check(_run(dev, api.plc_beam_select, logits.data_ptr(), kind, row, S, W, V, score.data_ptr(), None if done is None else done.data_ptr(), eos, n_out,
                out.data_ptr(), at, at + 4 * n, ws.data_ptr(), need), where)
    return out, store.as_strided((S, n_out), (n_out, 1), 0), store.as_strided((S, n_out), (n_out, 1), n)


def beam_reorder(parent, states, status=None):
    """New tensors whose row r is row parent[r] of each of `states` (zeros for -1): state tensors that follow their beams,
    indexed by the row first, the rest of a row contiguous.  status: int32 word that receives 32 for a parent out of range."""
    import torch
    where, dev, api = "plc_beam_reorder", parent.device, _lib()
    _need(parent.is_cuda and len(states) > 0, E_INVALID, where)
    rows, rows_in = _i32(parent, dev, where).numel(), states[0].shape[0] if states[0].dim() else 0
    _need(rows > 0 and rows_in > 0, E_INVALID, where)
    _int32(E_SHAPE, where, rows, rows_in)
    word = None if status is None else _i32(status, dev, where).data_ptr()
    out, sets = [], []
    for t in states:
        _need(t.device == dev and t.dim() >= 1 and t.shape[0] == rows_in and (t.is_contiguous() or t[0].is_contiguous()), E_INVALID, where)
        o = torch.empty((rows,) + t.shape[1:], dtype=t.dtype, device=dev)
        out.append(o)
        size = t.element_size()
        row = t.numel() // rows_in * size
        if row:
            sets += (t.data_ptr(), o.data_ptr(), t.stride(0) * size, row, row)
    for i in range(0, len(sets), 80):                        # sixteen plc_row_set of five 64-bit words
        some = sets[i:i + 80]
        _check(_run(dev, api.plc_beam_reorder, (C.c_int64 * len(some))(*some), len(some) // 5, parent.data_ptr(), rows_in, rows, word), where)
    return out
