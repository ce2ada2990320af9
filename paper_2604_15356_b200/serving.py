"""Paged KV cache, attention of drafted tokens over it, beam search, rotary positions, eviction and log probabilities: binding of
the plc_pages_*, plc_tree_attention, plc_beam_*, plc_rotary_* and plc_token_logprobs calls.

As in the rest of the binding nothing is computed here: tensors become pointers, and the work runs on the current stream
of the tensors' device.  Results and workspaces are allocated by torch on that stream, so that calls on several streams
and captured graphs do not share any.  No call is recorded for autograd.
"""
import ctypes as C
import math
import struct

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


class RotaryC(C.Structure):
    _fields_ = [("turns_dev", C.c_void_p), ("dim", C.c_int32), ("interleaved", C.c_int32), ("scale", C.c_float)]


class RotarySet(C.Structure):
    _fields_ = [("x_dev", C.c_void_p), ("out_dev", C.c_void_p), ("x_stride_row", C.c_int64), ("x_stride_head", C.c_int64), ("out_stride_row", C.c_int64),
                ("out_stride_head", C.c_int64), ("heads", C.c_int32)]


class NewTokens(C.Structure):
    _fields_ = [("q_dev", C.c_void_p), ("q_stride_row", C.c_int64), ("q_stride_head", C.c_int64), ("out_dev", C.c_void_p), ("out_stride_row", C.c_int64),
                ("out_stride_head", C.c_int64), ("k_dev", C.c_void_p), ("k_stride_row", C.c_int64), ("k_stride_head", C.c_int64), ("v_dev", C.c_void_p),
                ("v_stride_row", C.c_int64), ("v_stride_head", C.c_int64), ("begin_dev", C.c_void_p), ("pos_dev", C.c_void_p), ("n_rows", C.c_int32),
                ("n_heads", C.c_int32)]


class Weights(C.Structure):
    _fields_ = [("base_dev", C.c_void_p), ("stride_row", C.c_int64), ("stride_layer", C.c_int64), ("stride_head", C.c_int64), ("n_pos", C.c_int32)]


class WeighQueries(C.Structure):
    _fields_ = [("q_dev", C.c_void_p), ("q_stride_row", C.c_int64), ("q_stride_head", C.c_int64), ("lse_dev", C.c_void_p), ("rows_dev", C.c_void_p),
                ("begin_dev", C.c_void_p), ("n_rows", C.c_int32), ("n_list", C.c_int32), ("n_heads", C.c_int32)]


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
                            ("plc_beam_reorder", [P, I, P, I, I, P, P]), ("plc_rotary_apply", [P, P, I, P, I, I, I, I, P]), ("plc_pages_append", [P, I, P, P, P, P, P]),
                            ("plc_pages_weigh", [P, I, P, P, F, F, P, P, U, P, P]), ("plc_pages_weigh_workspace", [P, I, I, I, P]), ("plc_pages_evict", [P, P, P, P, I, I, P, P, P, U, P, P]),
                            ("plc_pages_evict_workspace", [P, I, I, P]), ("plc_token_logprobs", [P, I, L, I, I, P, I, I, P, P, P, P, P, U, P, P]),
                            ("plc_token_logprobs_workspace", [I, I, I, P])):
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

    def append(self, layer, book, q, k, v, begin, rotary=None, pos=None, out=None):
        """Writes the new tokens' keys k, turned by `rotary` (None: as they are), and values v [N][kv heads][d] into the layer's pages behind their
        sessions' lengths, and returns the turned queries q [N][heads][d] (q None: None).  Session s has the rows begin[s] .. begin[s+1]-1.  pos [N] int32: the
        positions that they turn by (drafted trees: their depths; after evictions), len + i if not given.  out: where the queries go, q itself is allowed.
        The book stays as it is; keep counts the tokens in."""
        import torch
        where, dev, api = "plc_pages_append", self.device, _lib()
        a = self._book(book, where)
        H, d = self._c.n_kv_heads, self._c.head_dim
        N = k.shape[0]
        for t in (k, v):
            _need(t.dim() == 3 and t.shape == (N, H, d), E_SHAPE, where)
            _need(t.device == dev and t.dtype == self.kv.dtype and t.stride(2) == 1, E_INVALID, where)
        _int32(E_INVALID, where, layer)
        _int32(E_SHAPE, where, N)
        _need(_i32(begin, dev, where).numel() == book.rows + 1, E_SHAPE, where)
        if pos is not None:
            _need(_i32(pos, dev, where).numel() == N, E_SHAPE, where)
        heads, queries = 0, (None, 0, 0, None, 0, 0)
        if q is not None:
            _need(q.dim() == 3 and q.shape[0] == N and q.shape[2] == d and q.shape[1] > 0, E_SHAPE, where)
            _need(q.device == dev and q.dtype == self.kv.dtype and q.stride(2) == 1, E_INVALID, where)
            heads = q.shape[1]
            _int32(E_SHAPE, where, heads)
            if out is None:
                out = torch.empty_strided((N, heads, d), (heads * d, d, 1), dtype=q.dtype, device=dev)
            else:
                _need(out.shape == q.shape and out.dtype == q.dtype and out.device == dev and out.stride(2) == 1, E_INVALID, where)
            queries = (q.data_ptr(), q.stride(0), q.stride(1), out.data_ptr(), out.stride(0), out.stride(1))
        else:
            _need(out is None, E_INVALID, where)
        by = None
        if rotary is not None:
            _need(rotary.device == dev, E_INVALID, where)
            by = rotary._by
        if N == 0:
            return out
        t = NewTokens(*queries, k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(), v.stride(0), v.stride(1), begin.data_ptr(),
                      None if pos is None else pos.data_ptr(), N, heads)
        _check(_run(dev, api.plc_pages_append, self._by, layer, a, by, C.byref(t), self._word), where)
        return out

    def new_weights(self, rows, n_pos):
        """Weights of empty rows: [rows][layers][kv heads][n_pos] float32, rows first, so that they follow beams through beam_reorder."""
        import torch
        return torch.zeros((rows, self._c.n_layers, self._c.n_kv_heads, n_pos), dtype=torch.float32, device=self.device)

    def _weights(self, weight, book, where):
        import torch
        _need(weight.dim() == 4 and weight.shape[:3] == (book.rows, self._c.n_layers, self._c.n_kv_heads), E_SHAPE, where)
        _need(weight.dtype == torch.float32 and weight.device == self.device and (weight.stride(3) == 1 or weight.shape[3] == 1), E_INVALID, where)
        _int32(E_SHAPE, where, weight.shape[3])
        row, layer, head, _ = weight.stride()
        return Weights(weight.data_ptr(), row, layer, head, weight.shape[3])

    def attention_weights(self, layer, book, q, lse, begin, weight, rows=None, scale=None, decay=1.0):
        """Adds to weight [rows][layers][kv heads][positions] (in place, and returned) what the layer's positions receive from the sessions' newest tokens:
        weight = decay * weight + sum of exp(scale q.k - lse).  q [N][heads][d] and lse [N][heads] as tree_attention had and left them.  Session s has the
        entries begin[s] .. begin[s+1]-1, which stand at its last positions (the book after keep); entry e is row e of q and lse, or row rows[e] (int32; -1: none):
        the accepted ones of a draft.  decay 0: nothing of the old weights is read."""
        import torch
        where, dev, api = "plc_pages_weigh", self.device, _lib()
        a = self._book(book, where)
        _need(q.dim() == 3, E_SHAPE, where)
        (N, heads, d), (row, head, one) = q.shape, q.stride()
        _need(d == self._c.head_dim and lse.shape == (N, heads), E_SHAPE, where)
        _int32(E_INVALID, where, layer)
        _int32(E_SHAPE, where, N, heads)
        _need(q.device == dev and q.dtype == self.kv.dtype and one == 1, E_INVALID, where)
        _kind(q.dtype, where, wide=False)
        _need(lse.dtype.itemsize == 4 and lse.is_floating_point() and lse.device == dev and lse.is_contiguous(), E_INVALID, where)
        _need(_i32(begin, dev, where).numel() == book.rows + 1, E_SHAPE, where)
        n_list = N if rows is None else _i32(rows, dev, where).numel()
        _int32(E_SHAPE, where, n_list)
        w = self._weights(weight, book, where)
        if n_list == 0:
            return weight
        need = self._need_bytes.get((book.rows, heads, n_list, "weigh"))
        if need is None:
            b = C.c_uint64()
            with torch.cuda.device(dev):
                _check(api.plc_pages_weigh_workspace(self._by, book.rows, heads, n_list, C.byref(b)), "plc_pages_weigh_workspace")
            if len(self._need_bytes) >= 4096:
                self._need_bytes.clear()
            need = self._need_bytes[(book.rows, heads, n_list, "weigh")] = b.value
        ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
        t = WeighQueries(q.data_ptr(), row, head, lse.data_ptr(), None if rows is None else rows.data_ptr(), begin.data_ptr(), N, n_list, heads)
        _check(_run(dev, api.plc_pages_weigh, self._by, layer, a, C.byref(t), d ** -0.5 if scale is None else scale, decay, C.byref(w),
                    None if ws is None else ws.data_ptr(), need,
                    self._word), where)
        return weight

    def evict(self, book, weight, budget, recent=0):
        """(new book, new weights): rows longer than `budget` (an int, or int32 [rows] on the device, negative: the row stays) keep, in every layer and head by
        itself, their last `recent` positions and those of the largest weights; what is kept moves together.  Tokens appended later turn by
        positions of their own (append's pos): len no longer counts what was evicted."""
        import torch
        where, dev, api = "plc_pages_evict", self.device, _lib()
        a = self._book(book, where)
        w = self._weights(weight, book, where)
        _int32(E_INVALID, where, recent)
        budgets, scalar = None, budget
        if torch.is_tensor(budget):                          # (held on to by its own name: what is allocated below must not take its place)
            _need(_i32(budget, dev, where).numel() == book.rows, E_SHAPE, where)
            budgets, scalar = budget.data_ptr(), 0
        _int32(E_INVALID, where, scalar)
        n_pos = weight.shape[3]
        need = self._need_bytes.get((book.rows, n_pos))
        if need is None:
            b = C.c_uint64()
            _check(api.plc_pages_evict_workspace(self._by, book.rows, n_pos, C.byref(b)), "plc_pages_evict_workspace")
            if len(self._need_bytes) >= 4096:
                self._need_bytes.clear()
            need = self._need_bytes[(book.rows, n_pos)] = b.value
        new, _ = PageBook._new(book.rows, book.max_pages, self.n_pages, dev)
        (rows, layers, heads, _), n = weight.shape, weight.numel() + 3 & ~3
        store = torch.empty_strided((n + (need + 3) // 4,), (1,), dtype=torch.float32, device=dev)     # the workspace behind them: 18, 13 or 8 times smaller (pieces of 128, 64, 32 positions), and 4 bytes for each page of the pool and of the rows
        out = store.as_strided((rows, layers, heads, n_pos), (layers * heads * n_pos, heads * n_pos, n_pos, 1), 0)
        at = store.data_ptr()
        _check(_run(dev, api.plc_pages_evict, self._by, a, C.byref(w), budgets, scalar, recent, new._by, at, at + 4 * n, need, self._word), where)
        return new, out

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


class Rotary:
    """Rotary positions: pair i of `dim` components turns by a frequency f_i a position, pairs being (i, i + dim/2), or neighbours where `interleaved`.
    f_i = base ** (-2 i / dim), stretched for contexts longer than the trained one by `ramp`:

      "none"   as they are
      "all"    f / factor
      "base"   base * factor ** (dim / (dim - 2)) in place of base
      "turns"  pairs that turn at least `fast` times over `context` positions stay, those that turn at most `slow` times are divided by factor, between them
               blended linearly in the number of turns
      "index"  the same, blended linearly in the pair's number, between those (rounded outwards) that turn `fast` and `slow` times

    scale multiplies what turns.  frequencies: dim/2 numbers in radians a position, in place of all of these."""

    def __init__(self, dim, base=10000.0, interleaved=False, ramp="none", factor=1.0, context=None, slow=1.0, fast=32.0, scale=1.0, frequencies=None, device="cuda"):
        import torch
        where = "Rotary"
        _need(dim >= 2 and dim % 2 == 0, E_SHAPE, where)
        f = rotary_frequencies(dim, base, ramp, factor, context, slow, fast) if frequencies is None else [float(x) for x in frequencies]
        _need(len(f) == dim // 2, E_SHAPE, where)
        _need(math.isfinite(scale), E_INVALID, where)
        turns = (C.c_uint64 * len(f))()
        _check(_lib().plc_rotary_turns((C.c_double * len(f))(*f), len(f), turns), "plc_rotary_turns")
        signed = [x - (1 << 64) if x >> 63 else x for x in turns]
        self.dim, self.interleaved, self.scale, self.frequencies = dim, bool(interleaved), float(scale), f
        self.turns = torch.tensor(signed, dtype=torch.int64).to(device)
        self.device = self.turns.device
        self._on_gpu = self.turns.is_cuda
        self._c = RotaryC(self.turns.data_ptr(), dim, int(self.interleaved), self.scale)
        self._by = C.byref(self._c)

    def apply(self, x, pos, back=False, out=None):
        """x [N][heads][d], or up to four of them (queries and keys, any strides with the components contiguous), turned at positions pos [N] (int32);
        back: by the opposite angles, which turns a gradient of the results into x's.  Nothing is recorded for autograd, also where x requires a gradient:
        a function of the caller's joins the two.  out: where the results go, x itself is allowed."""
        import torch
        where, dev = "plc_rotary_apply", self.device
        single = isinstance(x, torch.Tensor)
        xs = (x,) if single else x
        outs = (None,) * len(xs) if out is None else (out,) if isinstance(out, torch.Tensor) else out
        _need(len(xs) >= 1, E_INVALID, where)
        _need(len(xs) <= 4 and len(outs) == len(xs), E_SHAPE, where)
        if xs[0].dim() != 3:
            raise PlcError(E_SHAPE, where)
        N, dtype, d = _i32(pos, dev, where).numel(), xs[0].dtype, xs[0].shape[2]
        kind, sets, got = _kind(dtype, where), [], []
        for t, o in zip(xs, outs):
            shape = t.shape
            if len(shape) != 3 or shape[0] != N or shape[2] != d or N > 0x7fffffff or shape[1] > 0x7fffffff:
                raise PlcError(E_SHAPE, where)
            heads, (row, head, one) = shape[1], t.stride()
            if one != 1 or t.dtype != dtype or t.device != dev:
                raise PlcError(E_INVALID, where)
            if o is None:
                out_row, out_head = heads * d, d
                o = torch.empty_strided(shape, (out_row, d, 1), dtype=dtype, device=dev)
            else:
                _need(o.shape == shape and o.dtype == dtype and o.device == dev and o.stride(2) == 1, E_INVALID, where)
                out_row, out_head, _ = o.stride()
            got.append(o)
            sets += (t.data_ptr(), o.data_ptr(), row, head, out_row, out_head, heads)     # a plc_rotary_set, seven 64-bit words
        if N:
            if not self._on_gpu:
                raise PlcError(E_INVALID, where)
            rc = _run(dev, _lib().plc_rotary_apply, self._by, _SETS[len(xs)].pack(*sets), len(xs), pos.data_ptr(), N, d, kind, 1 if back else 0)
            if rc:
                raise PlcError(rc, where)
        return got[0] if single else tuple(got)


_SETS = [struct.Struct("%dq" % (7 * n)) for n in range(5)]


def rotary_frequencies(dim, base=10000.0, ramp="none", factor=1.0, context=None, slow=1.0, fast=32.0):
    """The dim/2 frequencies of Rotary, in radians a position."""
    where = "rotary_frequencies"
    _need(ramp in ("none", "all", "base", "turns", "index") and base > 0 and factor > 0, E_INVALID, where)
    if ramp == "base":
        _need(dim > 2, E_SHAPE, where)
        base *= factor ** (dim / (dim - 2))
    f = [base ** (-2.0 * i / dim) for i in range(dim // 2)]
    if ramp == "all":
        return [x / factor for x in f]
    if ramp in ("none", "base"):
        return f
    _need(context is not None and context > 0 and 0 < slow < fast, E_INVALID, where)
    if ramp == "turns":
        keep = [(context * x / (2 * math.pi) - slow) / (fast - slow) for x in f]
    else:
        _need(base > 1, E_INVALID, where)
        lo, hi = (dim * math.log(context / (2 * math.pi * x)) / (2 * math.log(base)) for x in (fast, slow))
        lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), dim - 1)
        keep = [1 - (i - lo) / max(hi - lo, 0.001) for i in range(dim // 2)]
    keep = [min(max(g, 0.0), 1.0) for g in keep]
    return [g * x + (1 - g) * x / factor for g, x in zip(keep, f)]


def token_logprobs(logits, tokens, n_top=0, status=None):
    """(logp, entropy, top_logp, top_token) of rows of logits [N][vocab]: the log probabilities [N][m] of tokens [N][m] (or [N]; int32, -1: none, 0),
    the rows' entropies [N] in nats, and the n_top likeliest tokens [N][n_top] with their log probabilities.  status: int32 word that receives 32 for a token
    out of range.  The four are views of one allocation, with the call's workspace behind them for as long as one of them lives."""
    import torch
    where, dev, api = "plc_token_logprobs", logits.device, _lib()
    _need(logits.is_cuda and logits.dim() == 2, E_INVALID, where)
    (N, V), (row, one) = logits.shape, logits.stride()
    _need(one == 1 or V == 1, E_INVALID, where)
    _need(_i32(tokens, dev, where).dim() in (1, 2) and tokens.shape[0] == N, E_SHAPE, where)
    m = 1 if tokens.dim() == 1 else tokens.shape[1]
    _int32(E_SHAPE, where, N, V, m, n_top)
    _need(n_top >= 0, E_INVALID, where)
    word = None if status is None else _i32(status, dev, where).data_ptr()
    kind = _kind(logits.dtype, where)
    # one allocation: log probabilities, entropies, the alternatives' and their tokens, and the workspace behind them
    need = _bytes(dev, api.plc_token_logprobs_workspace, N, V, n_top) if N else 0
    tops = N * n_top
    a, b, c = N * m, N * m + N, N * m + N + tops
    d = c + tops + 3 & ~3
    store = torch.empty_strided((d + (need + 3) // 4,), (1,), dtype=torch.float32, device=dev)
    logp, entropy = store.as_strided(tokens.shape, tokens.stride(), 0), store.as_strided((N,), (1,), a)
    top_logp = store.as_strided((N, n_top), (n_top, 1), b)
    top_token = store.view(torch.int32).as_strided((N, n_top), (n_top, 1), c)
    if N:
        at = store.data_ptr()
        _check(_run(dev, api.plc_token_logprobs, logits.data_ptr(), kind, row, N, V, tokens.data_ptr(), m, n_top, at, at + 4 * a, at + 4 * b, at + 4 * c,
                    at + 4 * d, need, word), where)
    return logp, entropy, top_logp, top_token
