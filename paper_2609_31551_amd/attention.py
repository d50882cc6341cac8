"""ctypes binding of the language side's attention in libeas.so (include/eas_attention.h): prompt attention
and the 8-bit key / value cache.  Argument marshalling and checks of what the C ABI cannot see (tensor types,
shapes, devices); PyTorch supplies device memory and the stream.

All tensors of a call are on the current device.  Work is enqueued on ``stream`` (a torch stream; None: the
current one); tensors made here are known to it, the caller's own are kept alive by the caller.
"""
import array
import ctypes
import struct

import torch

from .eas import EAS_MAX_SEQS, EAS_OK, LIB, EasError  # noqa: F401  (EAS_MAX_SEQS: the most packed prompts)

P, I32, I64, VP = ctypes.POINTER, ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
EAS_FP32, EAS_BF16, EAS_FP16 = range(3)
EAS_KV_INT8, EAS_KV_E4M3 = range(2)
SPLIT_KEYS, SPLIT_TOKENS = 2048, 1024   # calls below / up to these need no workspace
_INT_MAX = 2 ** 31 - 1
_DTYPE = {torch.float32: EAS_FP32, torch.bfloat16: EAS_BF16, torch.float16: EAS_FP16}
_FORMAT = {torch.int8: EAS_KV_INT8, torch.float8_e4m3fn: EAS_KV_E4M3}


class Strides(ctypes.Structure):
    _fields_ = [("row", I64), ("head", I64)]


class AttnShape(ctypes.Structure):
    _fields_ = [("dtype", I32), ("heads", I32), ("kv_heads", I32), ("head_dim", I32), ("causal", I32),
                ("scale", ctypes.c_float), ("q", Strides), ("k", Strides), ("v", Strides), ("out", Strides)]


class Kv8CacheStruct(ctypes.Structure):
    _fields_ = [("format", I32), ("kv_heads", I32), ("head_dim", I32), ("page_tokens", I32), ("n_pages", I32),
                ("k", VP), ("v", VP), ("k_scale", VP), ("v_scale", VP)]


# the structures' fields: made one by one, a structure takes 0.3 - 0.8 us more
_pack_shape, _pack_cache = struct.Struct("5if8q").pack, struct.Struct("5i4x4P").pack
_SIG = {
    "eas_prompt_attention": [P(AttnShape), VP, VP, VP, VP, VP, I32, VP, VP, VP, I64, VP],
    "eas_prompt_attention_workspace": [P(AttnShape), VP, VP, I32, P(I64)],
    "eas_kv8_append": [P(Kv8CacheStruct), I32, VP, Strides, VP, Strides, I32, VP, I32, VP, VP, I32, I32, VP],
    "eas_kv8_rows": [P(Kv8CacheStruct), I32, VP, I32, I32, VP, VP, I32, I32, VP, Strides, VP, Strides, VP],
    "eas_kv8_attention": [P(Kv8CacheStruct), P(AttnShape), VP, I32, VP, I32, VP, I32, VP, I32, I32, VP, VP, VP, I64,
                          VP],
    "eas_kv8_attention_workspace": [P(AttnShape), I32, I32, I32, P(I64)],
}
for _name, _args in _SIG.items():
    _fn = getattr(LIB, _name)
    _fn.argtypes = _args
    _fn.restype = I32
EXPORTS = tuple(sorted(_SIG))


def _check(status, what):
    if status != EAS_OK:
        raise EasError(status, what)


_current_stream = torch._C._cuda_getCurrentRawStream   # of a device; torch.cuda.current_stream takes 3 us


def _rows(t, name, heads, dim, dtype, index):
    """(row, head) strides of [rows, heads, dim] (heads None: any) with consecutive dims."""
    shape, strides = t.shape, t.stride()
    if len(strides) == 3 and t.dtype == dtype and t.get_device() == index:
        n, h, d = shape
        row, head, one = strides
        if d == dim and (heads is None or h == heads) and (one == 1 or not t.numel()):
            # a stride that no step is taken by says nothing
            return row if n > 1 else 0, head if h > 1 else 0
    raise ValueError("%s must be [rows, %s, %d], the values of a head consecutive, %s on cuda:%d: got %s, strides %s, %s "
                     "on %s" % (name, heads or "heads", dim, dtype, index, tuple(shape), strides, t.dtype, t.device))


def _device(t):
    """Index of the tensor's device, which has to be the current one."""
    index = t.get_device()
    if index < 0 or index != torch.cuda.current_device():
        raise ValueError("tensors must be on the current CUDA device, got %s" % t.device)
    return index


def _ints(t, name, index, shape):
    if t.dtype != torch.int32 or t.get_device() != index or t.shape != shape or not t.is_contiguous():
        raise ValueError("%s must be a contiguous int32 tensor of shape %s on cuda:%d, got %s %s on %s"
                         % (name, tuple(shape), index, t.dtype, tuple(t.shape), t.device))
    return t.data_ptr()


def _count(most, rows, name):
    """A bound of a batch (None: ``rows``) as a C int: what is more than that holds is as good as its largest."""
    if rows > _INT_MAX:
        raise ValueError("%d rows are more than the calls take" % rows)
    most = rows if most is None else min(int(most), _INT_MAX)
    if most < 0:
        raise ValueError("%s must not be negative" % name)
    return most


def _dtype(dtype):
    if dtype not in _DTYPE:
        raise ValueError("element type must be bfloat16 or float16, got %s" % dtype)
    return _DTYPE[dtype]


def _on(stream, make):
    """make() with its tensors known to ``stream`` (None: the current one)."""
    if stream is None:
        return make()
    with torch.cuda.stream(stream):
        return make()


def _outputs(q, out, lse, with_lse, index, stream):
    """The output tensors -- the caller's, or new ones -- the strides of out, and lse's address."""
    if stream is not None and (out is None or lse is None):
        with torch.cuda.stream(stream):
            return _outputs(q, out, lse, with_lse, index, None)
    rows, heads, dim = q.shape
    if out is None:
        out = torch.empty_like(q)
        row, head, _ = out.stride()   # empty_like keeps q's order
        strides = row if rows > 1 else 0, head if heads > 1 else 0
    elif out.shape[0] != rows:
        raise ValueError("out has %d rows, q %d" % (out.shape[0], rows))
    else:
        strides = _rows(out, "out", heads, dim, q.dtype, index)
    if lse is None:
        if not with_lse:
            return out, None, strides, None
        lse = torch.empty_strided((rows, heads), (heads, 1), dtype=torch.float32, device=q.device)   # 0.4 us below empty
    elif lse.dtype != torch.float32 or lse.get_device() != index or lse.shape != (rows, heads) \
            or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous float32 tensor [%d, %d] on cuda:%d" % (rows, heads, index))
    return out, lse, strides, lse.data_ptr()


def _workspace(workspace, need, index, device, stream):
    """The workspace of a call that needs ``need`` bytes -- the caller's or a new one --, its address and size."""
    if workspace is None:
        if not need:
            return None, None, 0
        workspace = _on(stream, lambda: torch.empty((need,), dtype=torch.uint8, device=device))
        return workspace, workspace.data_ptr(), need
    if workspace.dtype != torch.uint8 or workspace.get_device() != index or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on cuda:%d" % index)
    return workspace, workspace.data_ptr(), workspace.numel()


def _shape(code, heads, kv_heads, dim, causal, scale, q, k, v, out):
    try:
        return AttnShape.from_buffer_copy(_pack_shape(code, heads, kv_heads, dim, 1 if causal else 0,
                                                      dim ** -0.5 if scale is None else scale, *q, *k, *v, *out))
    except (struct.error, OverflowError):
        raise ValueError("scale must be a finite 32-bit float, got %r" % (scale,)) from None


def _cu(cu, rows, name):
    """Host prefix sums as an array of C ints."""
    cu = array.array("i", cu)
    if not cu or cu[-1] > rows:
        raise ValueError("%s must be [n_seqs + 1] prefix sums of at most %d rows" % (name, rows))
    return cu


def prompt_attention(q, k, v, cu_q, cu_k=None, *, causal=True, scale=None, out=None, lse=None, with_lse=False,
                     workspace=None, stream=None):
    """Attention over packed prompts (eas_prompt_attention).  q [rows, heads, head_dim] and k, v [rows, kv_heads,
    head_dim] in bfloat16 or float16, any row and head strides; cu_q, cu_k: host prefix sums of the sequences'
    queries and keys (cu_k None: the same).  scale None: head_dim ** -0.5.  Returns (out, lse): out like q, in
    ``out`` where given, rows behind the last sequence untouched; lse [rows, heads] float32 with with_lse or where
    given, else None.  workspace: a uint8 device tensor to use instead of a new one where one is needed, for few queries
    over 2,048 keys or more: up to 258 MiB for such a sequence with heads of 128."""
    index, dtype = _device(q), q.dtype
    code = _dtype(dtype)
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("q and k must be [rows, heads, head_dim]")
    rows, heads, dim = q.shape
    keys, kv_heads = k.shape[0], k.shape[1]
    cu_q = _cu(cu_q, rows, "cu_q")
    keys = min(keys, v.shape[0])
    cu_k = cu_q if cu_k is None else _cu(cu_k, keys, "cu_k")
    if len(cu_k) != len(cu_q) or cu_k[-1] > keys:
        raise ValueError("cu_q and cu_k: of the same sequences, keys within k and v")
    qs = _rows(q, "q", None, dim, dtype, index)
    ks = _rows(k, "k", None, dim, dtype, index)
    vs = _rows(v, "v", kv_heads, dim, dtype, index)
    out, lse, strides, lse_ptr = _outputs(q, out, lse, with_lse, index, stream)
    shape = _shape(code, heads, kv_heads, dim, causal, scale, qs, ks, vs, strides)
    n, cu_q_ptr, cu_k_ptr = len(cu_q) - 1, cu_q.buffer_info()[0], cu_k.buffer_info()[0]
    need = I64()
    if cu_k[-1] >= SPLIT_KEYS:
        _check(LIB.eas_prompt_attention_workspace(shape, cu_q_ptr, cu_k_ptr, n, need), "prompt_attention")
    workspace, ws_ptr, ws_bytes = _workspace(workspace, need.value, index, q.device, stream)
    _check(LIB.eas_prompt_attention(shape, q.data_ptr(), k.data_ptr(), v.data_ptr(), cu_q_ptr, cu_k_ptr, n,
                                    out.data_ptr(), lse_ptr, ws_ptr, ws_bytes,
                                    _current_stream(index) if stream is None else stream.cuda_stream),
           "prompt_attention")
    return out, lse


class Kv8Cache:
    """A key / value cache in 8 bits (include/eas_attention.h): int8 or float8_e4m3fn codes k [pages, kv_heads,
    page_tokens, head_dim] and v [pages, kv_heads, head_dim, page_tokens], float32 scales [pages, kv_heads].
    Made from the caller's tensors, or by ``Kv8Cache.empty``.  Page tables are int32 device tensors [n_seqs,
    max_pages]; an entry that is no page (-1) is not held."""

    def __init__(self, k, v, k_scale, v_scale):
        if k.dim() != 4 or k.dtype not in _FORMAT:
            raise ValueError("k must be int8 or float8_e4m3fn codes [pages, kv_heads, page_tokens, head_dim]")
        (n, h, p, d), codes, index = k.shape, k.dtype, k.get_device()
        if not (v.shape == (n, h, d, p) and v.dtype == codes and k_scale.shape == v_scale.shape == (n, h)
                and k_scale.dtype == v_scale.dtype == torch.float32
                and v.get_device() == k_scale.get_device() == v_scale.get_device() == index
                and k.is_contiguous() and v.is_contiguous() and k_scale.is_contiguous() and v_scale.is_contiguous()):
            raise ValueError("wanted contiguous v %s, %s, and k_scale, v_scale %s, float32, on %s: got %s" % (
                (n, h, d, p), codes, (n, h), k.device,
                ", ".join("%s %s on %s" % (tuple(t.shape), t.dtype, t.device) for t in (k, v, k_scale, v_scale))))
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.kv_heads, self.page_tokens, self.head_dim = n, h, p, d
        self.device, self._index = k.device, index
        self._c = Kv8CacheStruct.from_buffer_copy(_pack_cache(_FORMAT[codes], h, d, p, n, k.data_ptr(), v.data_ptr(),
                                                              k_scale.data_ptr(), v_scale.data_ptr()))

    @classmethod
    def empty(cls, n_pages, kv_heads, head_dim, page_tokens=64, dtype=torch.int8, device="cuda"):
        """A cache that holds nothing yet; its contents are whatever the memory held."""
        def new(shape, kind):
            return torch.empty(shape, dtype=kind, device=device)
        return cls(new((n_pages, kv_heads, page_tokens, head_dim), dtype),
                   new((n_pages, kv_heads, head_dim, page_tokens), dtype),
                   new((n_pages, kv_heads), torch.float32), new((n_pages, kv_heads), torch.float32))

    def _table(self, pages):
        shape = pages.shape
        if len(shape) != 2 or pages.dtype != torch.int32 or not pages.is_contiguous():
            raise ValueError("pages must be a contiguous int32 tensor [n_seqs, max_pages], got %s %s"
                             % (pages.dtype, tuple(shape)))
        if _device(pages) != self._index:
            raise ValueError("pages on %s, the cache on %s" % (pages.device, self.device))
        return pages.data_ptr(), shape[1], shape[0]

    def _split(self, cu, most, rows, n, name):
        """(pointer to the prefix sums or None, the most rows of a sequence)"""
        if cu is not None:
            return _ints(cu, name, self._index, (n + 1,)), _count(most, rows, "the most rows of a sequence")
        if most is None:
            most = rows // n if n else 0
        if most * n != rows:
            raise ValueError("without %s every sequence has the same number of rows: %d rows, %d sequences of %d"
                             % (name, rows, n, most))
        return None, _count(most, rows, "the most rows of a sequence")

    def append(self, k, v, held, pages, cu_new=None, max_new=None, stream=None):
        """New tokens' keys and values [rows, kv_heads, head_dim] behind the ``held`` (int32 device [n_seqs]) tokens
        of each sequence (eas_kv8_append).  cu_new: int32 device prefix sums of the new tokens; None: the same
        number for all.  max_new: the most of a sequence (None: all rows)."""
        table, max_pages, n = self._table(pages)
        index, dtype, rows = self._index, k.dtype, k.shape[0]
        code = _dtype(dtype)
        ks = _rows(k, "k", self.kv_heads, self.head_dim, dtype, index)
        vs = _rows(v, "v", self.kv_heads, self.head_dim, dtype, index)
        if v.shape[0] != rows:
            raise ValueError("k has %d rows, v %d" % (rows, v.shape[0]))
        cu, most = self._split(cu_new, max_new, rows, n, "cu_new")
        _check(LIB.eas_kv8_append(self._c, code, k.data_ptr(), Strides(*ks), v.data_ptr(), Strides(*vs), rows, cu, most,
                                  _ints(held, "held", index, (n,)), table, max_pages, n,
                                  _current_stream(index) if stream is None else stream.cuda_stream),
               "Kv8Cache.append")

    def rows(self, pages, cu_rows, n_rows, first=None, max_len=None, dtype=torch.bfloat16, k=None, v=None, stream=None):
        """Cached tokens back as rows (eas_kv8_rows): rows cu_rows[r] .. cu_rows[r+1] (int32 device [n_seqs + 1]) of
        the ``n_rows`` receive sequence r's tokens from first[r] (int32 device; None: 0) on.  max_len: the most of a
        sequence (None: n_rows); the launch grows with it * n_seqs.  Returns (k, v) [n_rows, kv_heads, head_dim]; rows
        of no sequence are not written."""
        table, max_pages, n = self._table(pages)
        index, code = self._index, _dtype(dtype)
        shape = (int(n_rows), self.kv_heads, self.head_dim)
        row = self.kv_heads * self.head_dim

        def new():
            return torch.empty_strided(shape, (row, self.head_dim, 1), dtype=dtype, device=self.device)
        ks = vs = row, self.head_dim
        if k is None:
            k = _on(stream, new)
        else:
            ks = _rows(k, "k", self.kv_heads, self.head_dim, dtype, index)
        if v is None:
            v = _on(stream, new)
        else:
            vs = _rows(v, "v", self.kv_heads, self.head_dim, dtype, index)
        if k.shape[0] != shape[0] or v.shape[0] != shape[0]:
            raise ValueError("k has %d rows, v %d, wanted %d" % (k.shape[0], v.shape[0], shape[0]))
        _check(LIB.eas_kv8_rows(self._c, code, table, max_pages, n, _ints(cu_rows, "cu_rows", index, (n + 1,)),
                                None if first is None else _ints(first, "first", index, (n,)),
                                _count(max_len, shape[0], "max_len"), shape[0], k.data_ptr(),
                                Strides(*ks), v.data_ptr(), Strides(*vs),
                                _current_stream(index) if stream is None else stream.cuda_stream),
               "Kv8Cache.rows")
        return k, v

    def attention(self, q, lens, pages, cu_q=None, max_q=None, max_len=None, *, causal=True, scale=None, out=None,
                  lse=None, with_lse=False, workspace=None, stream=None):
        """Attention of q [rows, heads, head_dim] over the first ``lens`` (int32 device [n_seqs]) tokens of each
        sequence, the queries' own among them (eas_kv8_attention).  cu_q, max_q: as cu_new and max_new of append;
        max_len: the most tokens of a sequence (None: what the page table holds).  The launch and the workspace grow
        with max_q * n_seqs and max_len, so give them where cu_q is given.  workspace: a uint8 device tensor to use
        instead of a new one.  Returns (out, lse) as prompt_attention, which over rows() is faster from 128 queries of
        a sequence on."""
        table, max_pages, n = self._table(pages)
        index, dtype, dim = self._index, q.dtype, self.head_dim
        code = _dtype(dtype)
        qs = _rows(q, "q", None, dim, dtype, index)
        rows, heads = q.shape[0], q.shape[1]
        cu, most_q = self._split(cu_q, max_q, rows, n, "cu_q")
        most = min(_count(max_len, max_pages * self.page_tokens, "max_len"), max_pages * self.page_tokens)
        out, lse, strides, lse_ptr = _outputs(q, out, lse, with_lse, index, stream)
        shape = _shape(code, heads, self.kv_heads, dim, causal, scale, qs, (0, 0), (0, 0), strides)
        need = I64()
        if most > SPLIT_TOKENS:
            _check(LIB.eas_kv8_attention_workspace(shape, most_q, most, n, need), "Kv8Cache.attention")
        workspace, ws_ptr, ws_bytes = _workspace(workspace, need.value, index, self.device, stream)
        _check(LIB.eas_kv8_attention(self._c, shape, q.data_ptr(), rows, cu, most_q, _ints(lens, "lens", index, (n,)),
                                     most, table, max_pages, n, out.data_ptr(), lse_ptr, ws_ptr, ws_bytes,
                                     _current_stream(index) if stream is None else stream.cuda_stream),
               "Kv8Cache.attention")
        return out, lse
