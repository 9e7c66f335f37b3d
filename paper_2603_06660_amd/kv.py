"""The 8-bit key/value cache of include/pag.h: argument marshalling only.

A decoding step, in order (every call goes onto the current stream and returns without waiting):

    tables = KvTables(requests, max_pages, num_pages, page_tokens)      # who holds which pages
    cache = KvCache(num_pages, kv_heads, head_dim, page_tokens)         # one for each layer, with the same tables
    step = tables.extend(add, total)                                    # add: new tokens of each request
    cache.append(k, v, step.slots)
    out, lse = cache.attend(q, step)                                    # reads everything
    out, lse = cache.attend_selected(q, ids, step, window=64)           # reads what a search found, and the last 64 tokens
    tables.commit(step)

None of it has a backward: tensors that require a gradient are refused unless gradients are switched off (torch.no_grad).
"""
from __future__ import annotations

import ctypes as C

import torch

from .binding import PagError, _check, load_library

_FORMATS = {"int8": 0, "fp8": 1}
_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_ROW_DTYPES = (torch.float16, torch.bfloat16)


class _Cache(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("format", C.c_uint32), ("kv_heads", C.c_uint32), ("head_dim", C.c_uint32),
                ("page_tokens", C.c_uint32), ("reserved", C.c_uint32), ("num_pages", C.c_uint64), ("data", C.c_void_p),
                ("exponents", C.c_void_p)]


class _Tables(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("requests", C.c_uint32), ("max_pages", C.c_uint32), ("page_tokens", C.c_uint32),
                ("table_stride", C.c_uint64), ("num_pages", C.c_uint64), ("table", C.c_void_p), ("lengths", C.c_void_p),
                ("free_pages", C.c_void_p), ("free_count", C.c_void_p)]


class _Step(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("requests", C.c_uint32), ("max_pages", C.c_uint32), ("max_new", C.c_uint32),
                ("table_stride", C.c_uint64), ("tokens", C.c_uint64), ("table", C.c_void_p), ("offsets", C.c_void_p),
                ("context", C.c_void_p), ("request", C.c_void_p), ("positions", C.c_void_p), ("slots", C.c_void_p),
                ("granted", C.c_void_p), ("lengths", C.c_void_p), ("free_count", C.c_void_p), ("scratch", C.c_void_p)]


class _Attention(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_uint32), ("heads", C.c_uint32), ("window", C.c_uint32),
                ("scale", C.c_float), ("softcap", C.c_float), ("slopes", C.c_void_p),
                ("q", C.c_void_p), ("q_token_stride", C.c_int64), ("q_head_stride", C.c_int64),
                ("out", C.c_void_p), ("out_token_stride", C.c_int64), ("out_head_stride", C.c_int64),
                ("lse", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64)]


def _gpu(device):
    device = torch.device("cuda" if device is None else device)
    if device.type != "cuda":
        raise PagError("the cache lives on a GPU, not on %s" % device)
    return device if device.index is not None else torch.device("cuda", torch.cuda.current_device())


def _no_graph(t, what):
    """The cache is 8 bits, written once, and its calls have no backward: a graph that ends here would be a silent zero."""
    if t.requires_grad and torch.is_grad_enabled():
        raise PagError("%s requires a gradient, and the cache has no backward: detach it, or call under torch.no_grad()" % what)


def _array(t, dtype, shape, device, what):
    """The address of a dense tensor of this type, shape and device."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.shape != shape or t.device != device or not t.is_contiguous():
        raise PagError("%s must be a contiguous %s tensor of shape %s on %s" % (what, dtype, tuple(shape), device))
    _no_graph(t, what)
    return t.data_ptr()


def _rows(t, shape, device, what, dtypes=_DTYPES):
    """Checks a [tokens, heads, dim] tensor whose last dimension is dense; the other strides are free."""
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes or t.shape != shape or t.device != device:
        raise PagError("%s must be a tensor of shape %s on %s, of type %s" %
                       (what, tuple(shape), device, ", ".join(str(x) for x in dtypes)))
    if t.stride(2) != 1 and t.shape[2] > 1:
        raise PagError("%s: the last dimension must be dense" % what)
    _no_graph(t, what)


# the number of a GPU's current stream, without an object around it where torch offers that
_stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)

_P, _I = C.c_void_p, C.c_int64
_ARGTYPES = {"pag_kv_extend": [_P, _P, _P, _P], "pag_kv_release": [_P, _P, _P],
             "pag_kv_append": [_P, C.c_uint32, _P, _I, _I, _P, _I, _I, _P, C.c_uint64, _P],
             "pag_kv_read": [_P, _P, C.c_uint64, C.c_uint32, _P, _I, _I, _P, _I, _I, _P],
             "pag_kv_workspace_bytes": [_P, _P, _P, C.c_int, C.c_uint32, C.c_uint32, _P],
             "pag_kv_attend": [_P, _P, _P, _P], "pag_kv_attend_selected": [_P, _P, _P, _P, _I, _I, C.c_uint32, C.c_uint32, _P]}
_calls = {}


def _call(name, device, *args):
    """One call of the library with `device` current, on its current stream (the last argument of every call)."""
    f = _calls.get(name)
    if f is None:
        f = C.CFUNCTYPE(C.c_int, *_ARGTYPES[name])((name, load_library()))
        _calls[name] = f
    index = device.index
    before = torch.cuda.current_device()
    if before == index:
        rc = f(*args, _stream_of(index))
    else:
        with torch.cuda.device(index):
            rc = f(*args, _stream_of(index))
    if rc:
        _check(rc, name)


class KvStep:
    """One step of a batch (pag_kv_step): its new tokens, request after request, padding at the end.

    table [requests, max_pages], offsets [requests + 1], context [requests], request and positions [tokens], all int32; slots int64
    [tokens].  KvTables.extend makes them; a program with tables of its own passes them in.  attend needs offsets and context,
    attend_selected request and positions.
    """

    def __init__(self, table, offsets=None, context=None, requests=None, positions=None, slots=None, max_new=0, granted=None,
                 lengths=None, free_count=None, scratch=None, tokens=None):
        self.table, self.offsets, self.context = None, offsets, context
        self.requests, self.positions, self.slots = requests, positions, slots
        self.granted, self.lengths, self.free_count, self.scratch = granted, lengths, free_count, scratch
        self.max_new = int(max_new)
        for t in (positions, requests, slots):
            if tokens is None and t is not None:
                tokens = t.shape[0]
        self._s = _Step(struct_size=C.sizeof(_Step), max_new=self.max_new)
        self.tokens = tokens
        self._holders = []          # tables that took over lengths and free_count
        if table is not None:
            self._bind(table)

    @classmethod
    def empty(cls, requests, total, device=None):
        """Room for a step of `requests` requests and `total` tokens, for KvTables.extend(out=...)."""
        device = _gpu(device)
        ints = torch.empty(5 * requests + 3 + 2 * total, dtype=torch.int32, device=device)
        offsets, context, granted, lengths, scratch, free_count, request, positions = ints.split(
            [requests + 1, requests, requests, requests, requests + 1, 1, total, total])
        return cls(None, offsets, context, request, positions, torch.empty(total, dtype=torch.int64, device=device), 0, granted,
                   lengths, free_count, scratch, total)

    def _bind(self, table):
        """Takes over a table and looks the arrays over."""
        if not isinstance(table, torch.Tensor) or table.dtype != torch.int32 or table.dim() != 2 or not table.is_cuda or \
                (table.stride(1) != 1 and table.shape[1] > 1) or table.shape[0] == 0 or table.shape[1] == 0:
            raise PagError("table must be an int32 CUDA tensor [requests, max_pages] with dense rows")
        device, n = table.device, table.shape[0]
        fields = dict(requests=n, max_pages=table.shape[1], table_stride=table.stride(0) if n > 1 else max(table.stride(0), table.shape[1]),
                      table=table.data_ptr())
        for name, shape, field in (("offsets", (n + 1,), "offsets"), ("context", (n,), "context"), ("granted", (n,), "granted"),
                                   ("lengths", (n,), "lengths"), ("free_count", (1,), "free_count"), ("scratch", (n + 1,), "scratch"),
                                   ("requests", (self.tokens,), "request"), ("positions", (self.tokens,), "positions")):
            t = getattr(self, name)
            if t is not None:
                fields[field] = _array(t, torch.int32, shape, device, name)
        if self.slots is not None:
            fields["slots"] = _array(self.slots, torch.int64, (self.tokens,), device, "slots")
        # everything fits: a step that is refused stays what it was
        for field, value in fields.items():
            setattr(self._s, field, value)
        self.table, self.device = table, device

    def _with(self, tokens):
        if self.table is None:
            raise PagError("the step has no table: it comes from KvStep.empty and KvTables.extend has not filled it")
        if self.tokens is not None and tokens != self.tokens:
            raise PagError("the step has %d tokens, q has %d" % (self.tokens, tokens))
        self._s.tokens = tokens
        return self._s


class KvTables:
    """The block tables of `requests` requests over a pool of pages, on the GPU (pag_kv_tables)."""

    def __init__(self, requests, max_pages, num_pages, page_tokens=64, device=None):
        device = _gpu(device)
        self._set(torch.zeros(requests, dtype=torch.int32, device=device),
                  torch.full((requests, max_pages), -1, dtype=torch.int32, device=device),
                  torch.arange(num_pages - 1, -1, -1, dtype=torch.int32, device=device),
                  torch.full((1,), num_pages, dtype=torch.int32, device=device), page_tokens)

    @classmethod
    def from_tensors(cls, lengths, table, free_pages, free_count, page_tokens):
        """Tables over the caller's own int32 tensors: [requests], [requests, max_pages], [num_pages], [1]."""
        self = cls.__new__(cls)
        self._set(lengths, table, free_pages, free_count, page_tokens)
        return self

    def _set(self, lengths, table, free_pages, free_count, page_tokens):
        if not isinstance(table, torch.Tensor) or table.dtype != torch.int32 or table.dim() != 2 or not table.is_cuda or \
                (table.stride(1) != 1 and table.shape[1] > 1):
            raise PagError("table must be an int32 CUDA tensor [requests, max_pages] with dense rows")
        self.device, self.page_tokens = table.device, int(page_tokens)
        n = table.shape[0]
        self.table, self.free_pages = table, free_pages
        self._t = _Tables(C.sizeof(_Tables), n, table.shape[1], self.page_tokens, table.stride(0) if n > 1 else max(table.stride(0), table.shape[1]),
                          free_pages.numel(), table.data_ptr())
        self._t.free_pages = _array(free_pages, torch.int32, (free_pages.numel(),), self.device, "free_pages")
        self._take(lengths, free_count)

    def _take(self, lengths, free_count):
        where = (_array(lengths, torch.int32, (self._t.requests,), self.device, "lengths"),
                 _array(free_count, torch.int32, (1,), self.device, "free_count"))
        self._t.lengths, self._t.free_count = where
        self.lengths, self.free_count = lengths, free_count

    def extend(self, add, total, max_new=0, out=None, commit=False):
        """-> KvStep for add[r] (int32 [requests]) new tokens of each request, `total` rows in all (more than the sum: padding; fewer: the
        requests whose tokens do not all have rows are refused, as those are for which there are no pages).
        max_new: no request gets more tokens (0: not known).  out: a step whose arrays are written again.  The tables keep their
        lengths and free pages until commit(step); commit=True writes them in place, as a captured loop needs it."""
        if out is None:
            out = KvStep.empty(self._t.requests, total, self.device)
        elif out.tokens != total:
            raise PagError("the step has %s tokens, not %d" % (out.tokens, total))
        if out.slots is None or out.granted is None or out.scratch is None:
            raise PagError("out has no room for slots: use KvStep.empty")
        add = _array(add, torch.int32, (self._t.requests,), self.device, "add")
        if out.table is not self.table:
            out._bind(self.table)
        s = out._s
        out.max_new = s.max_new = int(max_new)
        s.tokens = total
        if commit:
            out.lengths, out.free_count = self.lengths, self.free_count
            s.lengths, s.free_count = self._t.lengths, self._t.free_count
            out._holders = [self]
        elif any(t.lengths is out.lengths or t.free_count is out.free_count for t in (self, *out._holders)):
            out.lengths, out.free_count = torch.empty_like(self.lengths), torch.empty_like(self.free_count)
            s.lengths, s.free_count = out.lengths.data_ptr(), out.free_count.data_ptr()
            out._holders = []
        _call("pag_kv_extend", self.device, C.addressof(self._t), add, C.addressof(s))
        return out

    def commit(self, step):
        """Takes over the lengths and the free pages of a step that extend() made for these tables."""
        if step.table is not self.table or step.lengths is None or step.free_count is None:
            raise PagError("the step belongs to other tables")
        self._take(step.lengths, step.free_count)
        step._holders = [t for t in step._holders if t is not self] + [self]

    def release(self, done):
        """The requests with done[r] != 0 (int32 [requests]) give their pages back."""
        _call("pag_kv_release", self.device, C.addressof(self._t), _array(done, torch.int32, (self._t.requests,), self.device, "done"))


class KvCache:
    """Keys and values in 8 bits, in pages (pag_kv_cache).  format: "int8" or "fp8" (4 exponent and 3 mantissa bits)."""

    def __init__(self, num_pages, kv_heads, head_dim, page_tokens=64, format="int8", device=None):
        device = _gpu(device)
        width = -(-head_dim // 64) * 64
        self._set(torch.zeros((num_pages, kv_heads, page_tokens, 2, width), dtype=torch.uint8, device=device),
                  torch.zeros((num_pages, kv_heads, page_tokens // 16, 2), dtype=torch.int8, device=device), head_dim, format)

    @classmethod
    def from_tensors(cls, data, exponents, head_dim, format="int8"):
        """A cache over the caller's tensors: uint8 [num_pages, kv_heads, page_tokens, 2, width], int8 [num_pages, kv_heads, page_tokens / 16, 2];
        width is head_dim rounded up to a multiple of 64, with zeros behind head_dim."""
        self = cls.__new__(cls)
        self._set(data, exponents, head_dim, format)
        return self

    def _set(self, data, exponents, head_dim, format):
        if format not in _FORMATS:
            raise PagError("format must be one of %s" % ", ".join(sorted(_FORMATS)))
        if not isinstance(data, torch.Tensor) or data.dim() != 5 or not data.is_cuda:
            raise PagError("data must be a uint8 CUDA tensor [num_pages, kv_heads, page_tokens, 2, width]")
        pages, heads, tokens = data.shape[:3]
        self.device = data.device
        self.num_pages, self.kv_heads, self.page_tokens, self.head_dim, self.format = pages, heads, tokens, int(head_dim), format
        self._c = _Cache(C.sizeof(_Cache), _FORMATS[format], heads, self.head_dim, tokens, 0, pages,
                         _array(data, torch.uint8, (pages, heads, tokens, 2, -(-self.head_dim // 64) * 64), self.device, "data"),
                         _array(exponents, torch.int8, (pages, heads, tokens // 16, 2), self.device, "exponents"))
        self.data, self.exponents = data, exponents
        _check(load_library().pag_kv_read(C.byref(self._c), None, C.c_uint64(0), C.c_uint32(0), *[C.c_void_p(None), C.c_int64(0), C.c_int64(0)] * 2,
                                          None), "KvCache")      # of nothing: looks the cache over
        self._rooms = {}        # sizes of workspaces

    def append(self, k, v, slots):
        """Writes k and v [tokens, kv_heads, head_dim] (float32, float16 or bfloat16) into slots (int64 [tokens], -1: left out)."""
        tokens = slots.shape[0]
        shape = (tokens, self.kv_heads, self.head_dim)
        _rows(k, shape, self.device, "k")
        _rows(v, shape, self.device, "v", (k.dtype,))
        _call("pag_kv_append", self.device, C.addressof(self._c), _DTYPES[k.dtype], k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(),
              v.stride(0), v.stride(1), _array(slots, torch.int64, (tokens,), self.device, "slots"), tokens)

    def read(self, slots, dtype=torch.float32, out=None):
        """-> (k, v) [tokens, kv_heads, head_dim]: the rows in these slots as numbers; zeros for -1.  out: (k, v) to write into, of any
        token and head strides; one of them may be None."""
        tokens = slots.shape[0]
        shape = (tokens, self.kv_heads, self.head_dim)
        if out is None:
            out = (torch.empty(shape, dtype=dtype, device=self.device), torch.empty(shape, dtype=dtype, device=self.device))
        k, v = out
        some = k if k is not None else v
        if some is None:
            raise PagError("read: both outputs are None")
        dtype = some.dtype
        if dtype not in _DTYPES:
            raise PagError("read gives float32, float16 or bfloat16, not %s" % dtype)
        args = []
        for t, what in ((k, "k"), (v, "v")):
            if t is None:
                args += [None, 0, 0]
            else:
                _rows(t, shape, self.device, what, (dtype,))
                args += [t.data_ptr(), t.stride(0), t.stride(1)]
        _call("pag_kv_read", self.device, C.addressof(self._c), _array(slots, torch.int64, (tokens,), self.device, "slots"), tokens, _DTYPES[dtype], *args)
        return k, v

    def _attention(self, q, step, scale, window, softcap, slopes, out, id_heads=0, k=-1):
        """Checks a call's tensors -> out, its arguments, and its workspace, which has to live until the call is made."""
        if not isinstance(q, torch.Tensor) or q.dim() != 3:
            raise PagError("q must be a tensor [tokens, heads, head_dim]")
        tokens, heads, dim = shape = q.shape
        device = self.device
        if dim != self.head_dim:
            raise PagError("q has rows of %d numbers, the cache of %d" % (dim, self.head_dim))
        _rows(q, shape, device, "q", _ROW_DTYPES)
        if step.table is not None and step.device != device:
            raise PagError("the step is on %s, the cache on %s" % (step.device, device))
        if not 0 <= window < 1 << 31:
            raise PagError("window must be between 0 and 2^31 - 1")
        if out is None:
            o, lse = out = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty((tokens, heads), dtype=torch.float32, device=device)
        else:
            o, lse = out
            _rows(o, shape, device, "out", (q.dtype,))
            if lse is not None:
                _array(lse, torch.float32, (tokens, heads), device, "lse")
        s = step._with(tokens)
        a = _Attention(C.sizeof(_Attention), _DTYPES[q.dtype], heads, window, dim ** -0.5 if scale is None else scale, softcap,
                       None if slopes is None else _array(slopes, torch.float32, (heads,), device, "slopes"),
                       q.data_ptr(), q.stride(0), q.stride(1), o.data_ptr(), o.stride(0), o.stride(1), None if lse is None else lse.data_ptr())
        key = (tokens, heads, window, s.requests, s.max_new, s.max_pages, id_heads, k)
        size = self._rooms.get(key)
        if size is None:
            n = C.c_uint64()
            with torch.cuda.device(device):
                _check(load_library().pag_kv_workspace_bytes(C.byref(self._c), C.byref(s), C.byref(a), C.c_int(k >= 0), C.c_uint32(id_heads),
                                                             C.c_uint32(max(k, 0)), C.byref(n)), "pag_kv_workspace_bytes")
            if len(self._rooms) > 4096:
                self._rooms.clear()
            size = self._rooms[key] = n.value
        room = None
        if size:
            room = torch.empty(size, dtype=torch.uint8, device=device)
            a.workspace, a.workspace_bytes = room.data_ptr(), size
        return out, a, room

    def attend(self, q, step, scale=None, window=0, softcap=0.0, slopes=None, out=None):
        """-> (out like q, lse float32 [tokens, heads]): every token of q [tokens, heads, head_dim] (float16 or bfloat16) attends to its request's
        tokens up to itself.  window > 0: to the last `window` of them.  softcap > 0: scores become softcap * tanh(score / softcap).
        slopes (float32 [heads]): minus slope * distance.  scale: head_dim ** -0.5.  out: (out, lse) to write into; lse may be None."""
        if step.offsets is None or step.context is None:
            raise PagError("attend needs the step's offsets and context")
        out, a, room = self._attention(q, step, scale, window, softcap, slopes, out)
        _call("pag_kv_attend", self.device, C.addressof(self._c), C.addressof(step._s), C.addressof(a))
        return out

    def attend_selected(self, q, ids, step, scale=None, window=0, softcap=0.0, slopes=None, out=None):
        """attend(), but a token reads the positions that ids (int64 [tokens, id_heads, k], -1: none; what a search of the request's keys
        returned) lists for its head, and the last `window` tokens.  id_heads: kv_heads, heads, or a multiple of the one that
        divides the other."""
        if step.requests is None or step.positions is None:
            raise PagError("attend_selected needs the step's requests and positions")
        if not isinstance(ids, torch.Tensor) or ids.dtype != torch.int64 or ids.dim() != 3 or ids.device != self.device or ids.shape[0] != q.shape[0] or \
                (ids.shape[2] > 1 and ids.stride(2) != 1):
            raise PagError("ids must be an int64 tensor [tokens, id_heads, k] on %s whose last dimension is dense" % self.device)
        out, a, room = self._attention(q, step, scale, window, softcap, slopes, out, ids.shape[1], ids.shape[2])
        _call("pag_kv_attend_selected", self.device, C.addressof(self._c), C.addressof(step._s), C.addressof(a), ids.data_ptr(), ids.stride(0), ids.stride(1),
              ids.shape[1], ids.shape[2])
        return out
