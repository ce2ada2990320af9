"""Paged KV cache, attention of drafted tokens over it, and beam search: binding of the plc_pages_*, plc_tree_attention
and plc_beam_* calls.

As in the rest of the binding nothing is computed here: tensors become pointers, and the work runs on the current stream
of the tensors' device.  Results and workspaces are allocated by torch on that stream, so that calls on several streams
and captured graphs do not share any.
"""
import ctypes as C
import math

from . import E_ALIGN, E_CAPACITY, E_CUDA, E_INVALID, E_SHAPE, OUT_BF16, OUT_F16, OUT_F32, KVView, PlcError, _check, _ptr, lib


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


def _dtype(t, where, wide=True):
    import torch
    kinds = {torch.float16: OUT_F16, torch.bfloat16: OUT_BF16}
    if wide:
        kinds[torch.float32] = OUT_F32
    _need(t.dtype in kinds, E_INVALID, where)
    return kinds[t.dtype]


def _i32(t, shape, device, where):
    """t as what the library reads: int32, contiguous, on the device, of the shape (None: any extent)."""
    import torch
    _need(t.dtype == torch.int32 and t.device == device and t.is_contiguous(), E_INVALID, where)
    _need(t.dim() == len(shape) and all(w is None or n == w for n, w in zip(t.shape, shape)), E_SHAPE, where)
    return t


class _On:
    """The device of a call: made current for it, with its current stream."""

    def __init__(self, device):
        import torch
        self.guard = torch.cuda.device(device)
        self.device = device

    def __enter__(self):
        import torch
        self.guard.__enter__()
        return C.c_void_p(torch.cuda.current_stream(self.device).cuda_stream)

    def __exit__(self, *e):
        return self.guard.__exit__(*e)


class PageBook:
    """Who holds which page: table [rows][max_pages], len [rows], ref [pages] (int32 on the device).  Calls return new
    books; an old one stays valid until a page that only it names is taken by a later call."""

    def __init__(self, table, len, ref):
        dev = table.device
        _i32(table, (None, None), dev, "PageBook.table")
        _i32(len, (table.shape[0],), dev, "PageBook.len")
        _i32(ref, (None,), dev, "PageBook.ref")
        self.table, self.len, self.ref = table, len, ref

    def c(self):
        return PageBookC(self.table.data_ptr(), self.len.data_ptr(), self.ref.data_ptr(), self.table.shape[0], self.table.shape[1])


class PagePool:
    """Pages of a KV cache: kv indexed [layer][2][page][head][slot][component], any strides with the components
    contiguous and every vector on a 16-byte boundary (float16, bfloat16; float32 for everything but attention)."""

    def __init__(self, kv):
        import torch
        _need(kv.dim() == 6 and kv.shape[1] == 2 and kv.stride(5) == 1, E_SHAPE, "PagePool")
        _need(kv.is_cuda, E_INVALID, "PagePool")
        self.kv = kv
        s = kv.stride()
        L, _, P, H, page, d = kv.shape
        self._c = PagePoolC(KVView(kv.data_ptr(), s[0], s[1], s[2], s[3], s[4]), L, H, d, P, page, _dtype(kv, "PagePool"))
        self.status = torch.zeros(1, dtype=torch.int32, device=kv.device)

    def new_book(self, rows, max_pages):
        """A book of empty rows over a pool whose pages are all free."""
        import torch
        dev = self.kv.device
        return PageBook(torch.full((rows, max_pages), -1, dtype=torch.int32, device=dev), torch.zeros(rows, dtype=torch.int32, device=dev),
                        torch.zeros(self.kv.shape[2], dtype=torch.int32, device=dev))

    def sessions_view(self, first_page, sessions, n):
        """KVView of consecutive pages as plain sessions of n positions, for Context.encode / Context.decode: session i
        has the pages first_page + i * ceil(n / page) ....  Needs slots before heads, so that a page follows the other."""
        c, page = self._c, self.kv.shape[4]
        each = -(-n // page)
        _need(c.view.stride_session == page * c.view.stride_pos, E_SHAPE, "sessions_view")
        _need(first_page >= 0 and sessions >= 1 and n >= 1 and first_page + sessions * each <= c.n_pages, E_INVALID, "sessions_view")
        v = c.view
        return KVView(self.kv.data_ptr() + first_page * v.stride_session * self.kv.element_size(), v.stride_layer, v.stride_kv,
                      each * v.stride_session, v.stride_head, v.stride_pos)

    def _book(self, book, where):
        _need(book.table.device == self.kv.device, E_INVALID, where)
        _need(book.ref.shape[0] == self.kv.shape[2], E_SHAPE, where)
        return book.c()

    def _new(self, book, rows):
        import torch
        return PageBook(torch.empty(rows, book.table.shape[1], dtype=torch.int32, device=self.kv.device),
                        torch.empty(rows, dtype=torch.int32, device=self.kv.device), torch.empty_like(book.ref))

    def _workspace(self, book, rows):
        import torch
        b = C.c_uint64()
        _check(lib().plc_pages_workspace(self.kv.shape[2], book.table.shape[0], rows, C.byref(b)), "plc_pages_workspace")
        return torch.empty(b.value, dtype=torch.uint8, device=self.kv.device)

    def fork(self, book, parent, room=None):
        """New book whose row s continues row parent[s] (-1: empty), with pages for room[s] positions more."""
        import torch
        where, dev = "plc_pages_fork", self.kv.device
        a = self._book(book, where)
        rows = _i32(parent.reshape(-1), (None,), dev, where).shape[0]
        _need(rows >= 1, E_INVALID, where)
        if room is not None:
            _i32(room, (rows,), dev, where)
        with _On(dev) as st:
            new = self._new(book, rows)
            ws, b = self._workspace(book, rows), new.c()
            _check(lib().plc_pages_fork(C.byref(self._c), C.byref(a), _ptr(parent), _ptr(room), C.byref(b), _ptr(ws),
                                        C.c_uint64(ws.numel()), _ptr(self.status), st), where)
        return new

    def keep(self, book, path, n_path):
        """New book after the drafted positions path[s][:n_path[s]] of every row have been accepted."""
        where, dev = "plc_pages_keep", self.kv.device
        a = self._book(book, where)
        rows = book.table.shape[0]
        _i32(path, (rows, None), dev, where)
        _i32(n_path, (rows,), dev, where)
        with _On(dev) as st:
            new = self._new(book, rows)
            b = new.c()
            _check(lib().plc_pages_keep(C.byref(self._c), C.byref(a), _ptr(path), _ptr(n_path), path.shape[1], C.byref(b),
                                        _ptr(self.status), st), where)
        return new

    def compact(self, book):
        """(new book, moved): the pages in use have the lowest numbers; moved[p] is page p's new number (-1: free)."""
        import torch
        where = "plc_pages_compact"
        a = self._book(book, where)
        with _On(self.kv.device) as st:
            new = self._new(book, book.table.shape[0])
            moved = torch.empty_like(book.ref)
            ws, b = self._workspace(book, book.table.shape[0]), new.c()
            _check(lib().plc_pages_compact(C.byref(self._c), C.byref(a), C.byref(b), _ptr(moved), _ptr(ws), C.c_uint64(ws.numel()),
                                           _ptr(self.status), st), where)
        return new, moved

    def tree_attention(self, layer, book, q, begin, mask=None, scale=None, out=None, lse=None):
        """(out, lse) of the query rows q [N][heads][d]; session s has the rows begin[s] .. begin[s+1]-1, whose keys and
        values stand behind its length.  mask [N][words] int32: bit j of row i = drafted position j is seen (None: j <= i).
        scale: 1 / sqrt(d) if not given.  out, lse: written where given."""
        import torch
        where, dev = "plc_tree_attention", self.kv.device
        a = self._book(book, where)
        _need(q.dim() == 3 and q.shape[2] == self.kv.shape[5], E_SHAPE, where)
        _need(q.device == dev and q.dtype == self.kv.dtype and q.stride(2) == 1, E_INVALID, where)
        _dtype(q, where, wide=False)
        N, heads, d = q.shape
        _i32(begin, (book.table.shape[0] + 1,), dev, where)
        words = 0
        if mask is not None:
            words = _i32(mask, (N, None), dev, where).shape[1]
        with _On(dev) as st:
            if out is None:
                out = torch.empty(N, heads, d, dtype=q.dtype, device=dev)
            _need(out.shape == q.shape and out.dtype == q.dtype and out.device == dev and out.stride(2) == 1, E_INVALID, where)
            if lse is None:
                lse = torch.empty(N, heads, dtype=torch.float32, device=dev)
            _need(lse.shape == (N, heads) and lse.dtype == torch.float32 and lse.device == dev and lse.is_contiguous(), E_INVALID, where)
            if N == 0:
                return out, lse
            b = C.c_uint64()
            _check(lib().plc_tree_attention_workspace(C.byref(self._c), book.table.shape[0], heads, N, C.byref(b)), "plc_tree_attention_workspace")
            ws = torch.empty(b.value, dtype=torch.uint8, device=dev)
            t = TreeQueries(q.data_ptr(), q.stride(0), q.stride(1), out.data_ptr(), out.stride(0), out.stride(1), lse.data_ptr(),
                            begin.data_ptr(), None if mask is None else mask.data_ptr(), N, heads, words)
            _check(lib().plc_tree_attention(C.byref(self._c), int(layer), C.byref(a), C.byref(t), C.c_float(1 / math.sqrt(d) if scale is None else scale),
                                            _ptr(ws), C.c_uint64(ws.numel()), _ptr(self.status), st), where)
        return out, lse

    def check(self):
        """Waits for the work and raises where a call has found something wrong on the device; clears the word."""
        bits = int(self.status.item())
        self.status.zero_()
        for bit, code in ((8, E_CUDA), (1, E_CAPACITY), (32, E_INVALID)):
            _need(not bits & bit, code, f"status word {bits}")


def beam_select(logits, score, n_out, done=None, eos=-1):
    """(score, parent, token), each [sessions][n_out], of the n_out best continuations of every session: logits
    [sessions][beams][vocab], score [sessions][beams] float32, done [sessions][beams] bool.  parent counts the rows of all
    sessions (-1, with token -1 and score -inf: no continuation)."""
    import torch
    where, dev = "plc_beam_select", logits.device
    _need(logits.is_cuda and logits.dim() == 3 and logits.stride(2) == 1, E_INVALID, where)
    S, W, V = logits.shape
    _need(S < 2 or logits.stride(0) == W * logits.stride(1), E_SHAPE, where)
    _need(score.dtype == torch.float32 and score.device == dev and score.is_contiguous() and score.shape == (S, W), E_INVALID, where)
    if done is not None:
        _need(done.dtype == torch.bool and done.device == dev and done.is_contiguous() and done.shape == (S, W), E_INVALID, where)
    kind = _dtype(logits, where)
    b = C.c_uint64()
    _check(lib().plc_beam_workspace(S, W, V, int(n_out), C.byref(b)), "plc_beam_workspace")
    with _On(dev) as st:
        ws = torch.empty(b.value, dtype=torch.uint8, device=dev)
        out = torch.empty(S, n_out, dtype=torch.float32, device=dev)
        parent, token = (torch.empty(S, n_out, dtype=torch.int32, device=dev) for _ in range(2))
        _check(lib().plc_beam_select(_ptr(logits), kind, C.c_int64(logits.stride(1) if S * W > 1 else V), S, W, V, _ptr(score), _ptr(done), int(eos), int(n_out),
                                     _ptr(out), _ptr(parent), _ptr(token), _ptr(ws), C.c_uint64(ws.numel()), st), where)
    return out, parent, token


def beam_reorder(parent, states, status=None):
    """New tensors whose row r is row parent[r] of each of `states` (zeros for -1): state tensors that follow their beams,
    indexed by the row first, the rest of a row contiguous.  status: int32 word that receives 32 for a parent out of range."""
    import torch
    where, dev = "plc_beam_reorder", parent.device
    _need(parent.is_cuda and parent.dtype == torch.int32 and parent.is_contiguous() and parent.numel() > 0, E_INVALID, where)
    rows = parent.numel()
    _need(len(states) > 0, E_INVALID, where)
    for t in states:
        _need(t.device == dev and t.dim() >= 1 and t.shape[0] == states[0].shape[0] and (t.shape[0] == 0 or t[0].is_contiguous()), E_INVALID, where)
    with _On(dev) as st:
        out = [torch.empty((rows,) + tuple(t.shape[1:]), dtype=t.dtype, device=dev) for t in states]
        todo = [(t, o) for t, o in zip(states, out) if o.numel()]
        if status is not None:
            _i32(status, (1,), dev, where)
        for i in range(0, len(todo), 16):
            some = todo[i:i + 16]
            sets = (RowSet * len(some))(*[RowSet(t.data_ptr(), o.data_ptr(), t.stride(0) * t.element_size(), o.stride(0) * o.element_size(),
                                                 o[0].numel() * o.element_size()) for t, o in some])
            _check(lib().plc_beam_reorder(sets, len(some), _ptr(parent), states[0].shape[0], rows, _ptr(status), st), where)
    return out
