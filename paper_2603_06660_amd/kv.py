"""The key/value cache of include/pag.h, 8 or 4 bits a number: argument marshalling only.

A decoding step, in order (every call goes onto the current stream and returns without waiting):

    tables = KvTables(requests, max_pages, num_pages, page_tokens)      # who holds which pages
    cache = KvCache(num_pages, kv_heads, head_dim, page_tokens)         # one for each layer, with the same tables
    step = tables.extend(add, total)                                    # add: new tokens of each request
    cache.append(k, v, step.slots)
    out, lse = cache.attend(q, step)                                    # reads everything
    out, lse = cache.attend_selected(q, ids, step, window=64)           # reads what a search found, and the last 64 tokens
    tables.commit(step)

None of it has a backward: tensors that require a gradient are refused unless gradients are switched off (torch.no_grad), and so are tensors that carry a
tangent (torch.autograd.forward_ad) unless forward derivatives are (torch.inference_mode; torch.no_grad leaves them on).
"""
from __future__ import annotations

import ctypes as C

import torch
from torch.autograd import forward_ad

from .binding import PagError, _check, load_library

_FORMATS = {"int8": 0, "fp8": 1, "fp4": 4}
_PAIRS = {"halves": 0, "neighbours": 1}
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


class _Rotation(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("pairs", C.c_uint32), ("turned", C.c_uint32), ("heads", C.c_uint32), ("frequencies", C.c_void_p),
                ("positions", C.c_void_p), ("q", C.c_void_p), ("q_token_stride", C.c_int64), ("q_head_stride", C.c_int64), ("out", C.c_void_p),
                ("out_token_stride", C.c_int64), ("out_head_stride", C.c_int64)]


class _Blocks(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("block_tokens", C.c_uint32), ("codes", C.c_void_p), ("exponents", C.c_void_p)]


def _gpu(device):
    device = torch.device("cuda" if device is None else device)
    if device.type != "cuda":
        raise PagError("the cache lives on a GPU, not on %s" % device)
    return device if device.index is not None else torch.device("cuda", torch.cuda.current_device())


def _no_graph(t, what):
    """The cache is 8 or 4 bits, written once, and its calls have no backward: a graph that ends here would be a silent zero."""
    if torch.is_grad_enabled():
        raise PagError("%s requires a gradient, and the cache has no backward: detach it, or call under torch.no_grad()" % what)


def _no_tangent(t, what):
    """Forward derivatives would end here as well: a dual tensor's address is that of its value alone, and says nothing of its tangent."""
    if torch._C._is_fwd_grad_enabled() and forward_ad.unpack_dual(t).tangent is not None:
        raise PagError("%s carries a tangent, and the cache has no forward derivative: pass torch.autograd.forward_ad.unpack_dual(t).primal" % what)


def _array(t, dtype, shape, device, what):
    """The address of a dense tensor of this type, shape and device."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.shape != shape or t.device != device or not t.is_contiguous():
        raise PagError("%s must be a contiguous %s tensor of shape %s on %s" % (what, dtype, tuple(shape), device))
    if t.requires_grad:
        _no_graph(t, what)
    if forward_ad._current_level >= 0:
        _no_tangent(t, what)
    return t.data_ptr()


def _rows(t, shape, device, what, dtypes=_DTYPES):
    """Checks a [tokens, heads, dim] tensor whose last dimension is dense; the other strides are free. -> its address, those two strides."""
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes or t.shape != shape or t.device != device:
        raise PagError("%s must be a tensor of shape %s on %s, of type %s" %
                       (what, tuple(shape), device, ", ".join(str(x) for x in dtypes)))
    token, head, one = t.stride()
    if one != 1 and shape[2] > 1:
        raise PagError("%s: the last dimension must be dense" % what)
    if t.requires_grad:
        _no_graph(t, what)
    if forward_ad._current_level >= 0:
        _no_tangent(t, what)
    return t.data_ptr(), token, head


def _empty_rows(like):
    """A dense tensor of the same shape and type."""
    return torch.empty_like(like) if like.is_contiguous() else torch.empty_like(like, memory_format=torch.contiguous_format)


# the number of a GPU's current stream, without an object around it where torch offers that
_stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)

_P, _I = C.c_void_p, C.c_int64
_ARGTYPES = {"pag_kv_extend": [_P, _P, _P, _P], "pag_kv_release": [_P, _P, _P],
             "pag_kv_append": [_P, C.c_uint32, _P, _I, _I, _P, _I, _I, _P, C.c_uint64, _P],
             "pag_kv_append_rotated": [_P, C.c_uint32, _P, _I, _I, _P, _I, _I, _P, C.c_uint64, _P, _P],
             "pag_kv_read": [_P, _P, C.c_uint64, C.c_uint32, _P, _I, _I, _P, _I, _I, _P],
             "pag_kv_blocks_update": [_P, _P, _P, C.c_uint64, _P],
             "pag_kv_blocks_select": [_P, _P, _P, _P, C.c_uint32, C.c_uint32, _P, _I, _I, _P],
             "pag_kv_attend_blocks": [_P, _P, _P, _P, _I, _I, C.c_uint32, C.c_uint32, C.c_uint32, _P],
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


class KvRotation:
    """How rows are turned by their positions (pag_kv_rotation): frequencies float32 [turned / 2] on the GPU, of the first `turned` numbers of a row;
    pairs: "halves" (numbers i and i + turned / 2) or "neighbours" (2 i and 2 i + 1)."""

    def __init__(self, frequencies, pairs="halves"):
        if pairs not in _PAIRS:
            raise PagError("pairs must be one of %s" % ", ".join(sorted(_PAIRS)))
        if not isinstance(frequencies, torch.Tensor) or frequencies.dim() != 1 or not frequencies.is_cuda or frequencies.numel() == 0:
            raise PagError("frequencies must be a float32 CUDA tensor [turned / 2]")
        self.device, self.pairs, self.turned = frequencies.device, pairs, 2 * frequencies.numel()
        self._where = _array(frequencies, torch.float32, (frequencies.numel(),), self.device, "frequencies")
        self.frequencies = frequencies


def _cache_shapes(num_pages, kv_heads, page_tokens, head_dim, format):
    """Of data and exponents."""
    width = -(-head_dim // 64) * 64
    if format == "fp4":
        return (num_pages, kv_heads, page_tokens, 2, width // 2), (num_pages, kv_heads, page_tokens // 16, 2, width // 32, 16)
    return (num_pages, kv_heads, page_tokens, 2, width), (num_pages, kv_heads, page_tokens // 16, 2)


class KvCache:
    """Keys and values in pages (pag_kv_cache).  format: "int8", "fp8" (4 exponent and 3 mantissa bits), each with an exponent for 16 tokens, or
    "fp4" (2 exponent bits and 1 mantissa bit) with one for 32 numbers of a row."""

    def __init__(self, num_pages, kv_heads, head_dim, page_tokens=64, format="int8", device=None):
        device = _gpu(device)
        data, exponents = _cache_shapes(num_pages, kv_heads, page_tokens, head_dim, format)
        self._set(torch.zeros(data, dtype=torch.uint8, device=device), torch.zeros(exponents, dtype=torch.int8, device=device), head_dim, format)

    @classmethod
    def from_tensors(cls, data, exponents, head_dim, format="int8"):
        """A cache over the caller's tensors: uint8 [num_pages, kv_heads, page_tokens, 2, width], int8 [num_pages, kv_heads, page_tokens / 16, 2];
        width is head_dim rounded up to a multiple of 64, with zeros behind head_dim.  "fp4": uint8 [num_pages, kv_heads, page_tokens, 2, width / 2], int8
        [num_pages, kv_heads, page_tokens / 16, 2, width / 32, 16]."""
        self = cls.__new__(cls)
        self._set(data, exponents, head_dim, format)
        return self

    def _set(self, data, exponents, head_dim, format):
        if format not in _FORMATS:
            raise PagError("format must be one of %s" % ", ".join(sorted(_FORMATS)))
        if not isinstance(data, torch.Tensor) or data.dim() != 5 or not data.is_cuda:
            raise PagError("data must be a uint8 CUDA tensor [num_pages, kv_heads, page_tokens, 2, bytes of a row]")
        pages, heads, tokens = data.shape[:3]
        self.device = data.device
        data_shape, exponents_shape = _cache_shapes(pages, heads, tokens, int(head_dim), format)
        self.num_pages, self.kv_heads, self.page_tokens, self.head_dim, self.format = pages, heads, tokens, int(head_dim), format
        self._c = _Cache(C.sizeof(_Cache), _FORMATS[format], heads, self.head_dim, tokens, 0, pages,
                         _array(data, torch.uint8, data_shape, self.device, "data"), _array(exponents, torch.int8, exponents_shape, self.device, "exponents"))
        self.data, self.exponents = data, exponents
        _check(load_library().pag_kv_read(C.byref(self._c), None, C.c_uint64(0), C.c_uint32(0), *[C.c_void_p(None), C.c_int64(0), C.c_int64(0)] * 2,
                                          None), "KvCache")      # of nothing: looks the cache over
        self._rooms = {}        # sizes of workspaces

    def append(self, k, v, slots):
        """Writes k and v [tokens, kv_heads, head_dim] (float32, float16 or bfloat16) into slots (int64 [tokens], -1: left out)."""
        tokens = slots.shape[0]
        shape = (tokens, self.kv_heads, self.head_dim)
        keys = _rows(k, shape, self.device, "k")
        values = _rows(v, shape, self.device, "v", (k.dtype,))
        _call("pag_kv_append", self.device, C.addressof(self._c), _DTYPES[k.dtype], *keys, *values,
              _array(slots, torch.int64, (tokens,), self.device, "slots"), tokens)

    def append_rotated(self, k, v, slots, positions, rotation, q=None, out=None):
        """append() of k turned by `rotation` (a KvRotation) at positions (int32 [tokens]; a step's, or others) and of v as it is.
        -> q [tokens, heads, head_dim], of k's type, turned likewise: a new tensor, or `out` (q itself: in place; otherwise apart from q, k and v); None if there is no q."""
        tokens = slots.shape[0]
        shape = (tokens, self.kv_heads, self.head_dim)
        keys = _rows(k, shape, self.device, "k")
        values = _rows(v, shape, self.device, "v", (k.dtype,))
        if not isinstance(rotation, KvRotation) or rotation.device != self.device:
            raise PagError("rotation must be a KvRotation on %s" % self.device)
        r = _Rotation(C.sizeof(_Rotation), _PAIRS[rotation.pairs], rotation.turned, 0, rotation._where,
                      _array(positions, torch.int32, (tokens,), self.device, "positions"))
        if q is None:
            if out is not None:
                raise PagError("out is for a q")
        else:
            if not isinstance(q, torch.Tensor) or q.dim() != 3:
                raise PagError("q must be a tensor [tokens, heads, head_dim]")
            rows = (tokens, q.shape[1], self.head_dim)
            r.q, r.q_token_stride, r.q_head_stride = _rows(q, rows, self.device, "q", (k.dtype,))
            if out is None:
                out = _empty_rows(q)
            r.out, r.out_token_stride, r.out_head_stride = _rows(out, rows, self.device, "out", (k.dtype,))
            r.heads = rows[1]
        _call("pag_kv_append_rotated", self.device, C.addressof(self._c), _DTYPES[k.dtype], *keys, *values,
              _array(slots, torch.int64, (tokens,), self.device, "slots"), tokens, C.addressof(r))
        return out

    def read(self, slots, dtype=torch.float32, out=None):
        """-> (k, v) [tokens, kv_heads, head_dim]: the rows in these slots as numbers; zeros for -1.  out: (k, v) to write into, of any
        token and head strides; one of them may be None."""
        tokens = slots.shape[0]
        shape = (tokens, self.kv_heads, self.head_dim)
        if out is None:
            k = torch.empty(shape, dtype=dtype, device=self.device)
            out = (k, torch.empty_like(k))
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
                args += _rows(t, shape, self.device, what, (dtype,))
        _call("pag_kv_read", self.device, C.addressof(self._c), _array(slots, torch.int64, (tokens,), self.device, "slots"), tokens, _DTYPES[dtype], *args)
        return k, v

    def _queries(self, q, step, window):
        """Checks what every call over a step looks at. -> q's address and strides."""
        if not isinstance(q, torch.Tensor) or q.dim() != 3:
            raise PagError("q must be a tensor [tokens, heads, head_dim]")
        if q.shape[2] != self.head_dim:
            raise PagError("q has rows of %d numbers, the cache of %d" % (q.shape[2], self.head_dim))
        rows = _rows(q, q.shape, self.device, "q", _ROW_DTYPES)
        if step.table is not None and step.device != self.device:
            raise PagError("the step is on %s, the cache on %s" % (step.device, self.device))
        if not 0 <= window < 1 << 31:
            raise PagError("window must be between 0 and 2^31 - 1")
        return rows

    def _attention(self, q, step, scale, window, softcap, slopes, out, id_heads=0, k=-1, block=0):
        """Checks a call's tensors -> out, its arguments, and its workspace, which has to live until the call is made."""
        queries = self._queries(q, step, window)
        tokens, heads, dim = shape = q.shape
        device = self.device
        if out is None:
            o, lse = out = _empty_rows(q), torch.empty((tokens, heads), dtype=torch.float32, device=device)
        else:
            o, lse = out
            if lse is not None:
                _array(lse, torch.float32, (tokens, heads), device, "lse")
        s = step._with(tokens)
        a = _Attention(C.sizeof(_Attention), _DTYPES[q.dtype], heads, window, dim ** -0.5 if scale is None else scale, softcap,
                       None if slopes is None else _array(slopes, torch.float32, (heads,), device, "slopes"),
                       *queries, *_rows(o, shape, device, "out", (q.dtype,)), None if lse is None else lse.data_ptr())
        return out, a, self._room(a, s, (tokens, heads, window, s.requests, s.max_new, s.max_pages, id_heads, k, block), id_heads, k, block)

    def _room(self, a, s, key, id_heads, k, block=0, select=False):
        """The workspace of a call, None if it needs none."""
        size = self._rooms.get(key)
        if size is None:
            n = C.c_uint64()
            with torch.cuda.device(self.device):
                if block:
                    _check(load_library().pag_kv_blocks_workspace_bytes(C.byref(self._c), C.byref(s), C.byref(a), C.c_uint32(id_heads), C.c_uint32(k), C.c_uint32(block),
                                                                        C.byref(n) if select else None, None if select else C.byref(n)),
                           "pag_kv_blocks_workspace_bytes")
                else:
                    _check(load_library().pag_kv_workspace_bytes(C.byref(self._c), C.byref(s), C.byref(a), C.c_int(k >= 0), C.c_uint32(id_heads),
                                                                 C.c_uint32(max(k, 0)), C.byref(n)), "pag_kv_workspace_bytes")
            if len(self._rooms) > 4096:
                self._rooms.clear()
            size = self._rooms[key] = n.value
        if not size:
            return None
        room = torch.empty(size, dtype=torch.uint8, device=self.device)
        a.workspace, a.workspace_bytes = room.data_ptr(), size
        return room

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


class KvBlocks:
    """Summaries of a cache's blocks of `block_tokens` tokens, and attention over those that are chosen by them (pag_kv_blocks).  After each append:

        blocks.update(step.slots)
        ids = blocks.select(q, step, k, window)             # int32 [tokens, id_heads, k], ascending, -1 behind them
        out, lse = blocks.attend(q, ids, step, window=window)
    """

    def __init__(self, cache, block_tokens=64):
        if not isinstance(cache, KvCache) or block_tokens <= 0 or block_tokens % 16 or cache.page_tokens % block_tokens:
            raise PagError("block_tokens must be a multiple of 16 that divides the cache's page_tokens")
        per = cache.page_tokens // block_tokens
        self._set(cache, torch.zeros((cache.num_pages, cache.kv_heads, per, 2, -(-cache.head_dim // 64) * 64), dtype=torch.int8, device=cache.device),
                  torch.zeros((cache.num_pages, cache.kv_heads, per), dtype=torch.int8, device=cache.device))

    @classmethod
    def from_tensors(cls, cache, codes, exponents):
        """Over the caller's tensors: int8 [num_pages, kv_heads, page_tokens / block_tokens, 2, width] (largest and smallest), int8 [num_pages, kv_heads,
        page_tokens / block_tokens]."""
        self = cls.__new__(cls)
        self._set(cache, codes, exponents)
        return self

    def _set(self, cache, codes, exponents):
        if not isinstance(cache, KvCache) or not isinstance(codes, torch.Tensor) or codes.dim() != 5 or codes.shape[2] == 0 or cache.page_tokens % codes.shape[2] or \
                cache.page_tokens // codes.shape[2] % 16:
            raise PagError("codes must be an int8 tensor [num_pages, kv_heads, page_tokens / block_tokens, 2, width] for a KvCache")
        per = codes.shape[2]
        self.cache, self.block_tokens = cache, cache.page_tokens // per
        self._b = _Blocks(C.sizeof(_Blocks), self.block_tokens,
                          _array(codes, torch.int8, (cache.num_pages, cache.kv_heads, per, 2, -(-cache.head_dim // 64) * 64), cache.device, "codes"),
                          _array(exponents, torch.int8, (cache.num_pages, cache.kv_heads, per), cache.device, "exponents"))
        _check(load_library().pag_kv_blocks_update(C.byref(cache._c), C.byref(self._b), None, C.c_uint64(0), None), "KvBlocks")      # of nothing: looks them over
        self.codes, self.exponents = codes, exponents

    def update(self, slots):
        """Summarises the blocks that slots (int64 [tokens], of the append before) lie in.  A block's tokens stand side by side in ascending order; the last of them is
        the last that the block holds."""
        c = self.cache
        _call("pag_kv_blocks_update", c.device, C.addressof(c._c), C.addressof(self._b), _array(slots, torch.int64, (slots.shape[0],), c.device, "slots"), slots.shape[0])

    def select(self, q, step, k, window=0, id_heads=None, out=None):
        """-> int32 [tokens, id_heads, k]: for each token the k blocks of the best scores among those that begin before its last `window` tokens.
        id_heads: lists of a token, kv_heads if not given, else as attend_selected takes them; a list's heads share it by the largest of their scores."""
        c = self.cache
        queries = c._queries(q, step, window)
        if step.requests is None or step.positions is None:
            raise PagError("select needs the step's requests and positions")
        tokens, heads = q.shape[:2]
        if id_heads is None:
            id_heads = c.kv_heads
        if k < 0 or id_heads <= 0:
            raise PagError("k must not be negative, id_heads positive")
        if out is None:
            out = torch.empty((tokens, id_heads, k), dtype=torch.int32, device=c.device)
        elif not isinstance(out, torch.Tensor) or out.dtype != torch.int32 or out.shape != (tokens, id_heads, k) or out.device != c.device or \
                (k > 1 and out.stride(2) != 1):
            raise PagError("out must be an int32 tensor [tokens, id_heads, k] on %s whose last dimension is dense" % c.device)
        s = step._with(tokens)
        a = _Attention(C.sizeof(_Attention), _DTYPES[q.dtype], heads, window, 0.0, 0.0, None, *queries)
        room = c._room(a, s, ("select", tokens, heads, window, s.requests, s.max_pages, id_heads, k, self.block_tokens), id_heads, k, self.block_tokens, True)
        _call("pag_kv_blocks_select", c.device, C.addressof(c._c), C.addressof(self._b), C.addressof(s), C.addressof(a), id_heads, k, out.data_ptr(),
              out.stride(0), out.stride(1))
        del room
        return out

    def attend(self, q, ids, step, scale=None, window=0, softcap=0.0, slopes=None, out=None):
        """KvCache.attend_selected over the tokens of listed blocks: ids int32 [tokens, id_heads, k] (-1: none), as select() returns them."""
        c = self.cache
        if step.requests is None or step.positions is None:
            raise PagError("attend needs the step's requests and positions")
        if not isinstance(ids, torch.Tensor) or ids.dtype != torch.int32 or ids.dim() != 3 or ids.device != c.device or ids.shape[0] != q.shape[0] or \
                (ids.shape[2] > 1 and ids.stride(2) != 1):
            raise PagError("ids must be an int32 tensor [tokens, id_heads, k] on %s whose last dimension is dense" % c.device)
        out, a, room = c._attention(q, step, scale, window, softcap, slopes, out, ids.shape[1], ids.shape[2], self.block_tokens)
        _call("pag_kv_attend_blocks", c.device, C.addressof(c._c), C.addressof(step._s), C.addressof(a), ids.data_ptr(), ids.stride(0), ids.stride(1), ids.shape[1],
              ids.shape[2], self.block_tokens)
        del room
        return out
