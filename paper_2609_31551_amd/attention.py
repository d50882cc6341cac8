"""ctypes binding of the language side's attention in libeas.so (include/eas_attention.h): prompt attention
and the 8-bit key / value cache.  Argument marshalling and checks of what the C ABI cannot see (tensor types,
shapes, devices); PyTorch supplies device memory and the stream.

All tensors of a call are on the current device.  Work is enqueued on ``stream`` (a torch stream; None: the
current one); tensors made here are known to it, the caller's own are kept alive by the caller.
"""
import ctypes

import numpy as np
import torch

from .eas import EAS_MAX_SEQS, EAS_OK, LIB, EasError  # noqa: F401  (EAS_MAX_SEQS: the most packed prompts)

P, I32, I64, VP = ctypes.POINTER, ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
EAS_FP32, EAS_BF16, EAS_FP16 = range(3)
EAS_KV_INT8, EAS_KV_E4M3 = range(2)
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


_SIG = {
    "eas_prompt_attention": [P(AttnShape), VP, VP, VP, P(I32), P(I32), I32, VP, VP, VP],
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


def _rows(t, name, heads=None, dim=None, dtype=None, device=None):
    """[rows, heads, dim] with consecutive dims; its strides."""
    if t.dim() != 3 or (heads is not None and t.shape[1] != heads) or (dim is not None and t.shape[2] != dim):
        raise ValueError("%s has shape %s, wanted [rows, %s, %s]" % (name, tuple(t.shape), heads or "heads",
                                                                     dim or "head_dim"))
    if (dtype is not None and t.dtype != dtype) or (device is not None and t.device != device):
        raise ValueError("%s is %s on %s, wanted %s on %s" % (name, t.dtype, t.device, dtype, device))
    row, head, one = t.stride()
    if one != 1 and t.numel():
        raise ValueError("%s: the values of a head must be consecutive" % name)
    # a stride that no step is taken by says nothing
    return Strides(row if t.shape[0] > 1 else 0, head if t.shape[1] > 1 else 0)


def _device(t):
    """The calls run on the current device."""
    if not t.is_cuda or t.device.index != torch.cuda.current_device():
        raise ValueError("tensors must be on the current CUDA device, got %s" % t.device)
    return t.device


def _ints(t, name, device, shape):
    if t.dtype != torch.int32 or t.device != device or tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError("%s must be a contiguous int32 tensor of shape %s on %s, got %s %s on %s"
                         % (name, shape, device, t.dtype, tuple(t.shape), t.device))
    return t.data_ptr()


def _dtype(dtype):
    if dtype not in _DTYPE:
        raise ValueError("element type must be bfloat16 or float16, got %s" % dtype)
    return _DTYPE[dtype]


def _scale(scale, dim):
    return dim ** -0.5 if scale is None else float(scale)


class _On:
    """The stream of a call, and tensors that it may use."""

    def __init__(self, stream):
        self.stream = stream
        self.ptr = (stream if stream is not None else torch.cuda.current_stream()).cuda_stream

    def empty(self, shape, dtype, device):
        if self.stream is None:
            return torch.empty(shape, dtype=dtype, device=device)
        with torch.cuda.stream(self.stream):
            return torch.empty(shape, dtype=dtype, device=device)


def _lse_ptr(lse, rows, heads, device):
    if lse.dtype != torch.float32 or lse.device != device or tuple(lse.shape) != (rows, heads) \
            or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous float32 tensor [%d, %d] on %s" % (rows, heads, device))
    return lse.data_ptr()


def _outputs(on, q, rows, heads, out, lse, with_lse):
    """The output tensors: the caller's, or new ones."""
    if out is None:
        out = on.empty((rows, heads, q.shape[2]), q.dtype, q.device)
    elif out.shape[0] != rows:
        raise ValueError("out has %d rows, q %d" % (out.shape[0], rows))
    if lse is None and with_lse:
        lse = on.empty((rows, heads), torch.float32, q.device)
    return out, lse, None if lse is None else _lse_ptr(lse, rows, heads, q.device)


def _cu(cu, rows, name):
    cu = np.ascontiguousarray(cu, dtype=np.int32)
    if cu.ndim != 1 or cu.shape[0] < 1 or cu[-1] > rows:
        raise ValueError("%s must be [n_seqs + 1] prefix sums of at most %d rows" % (name, rows))
    return cu


def prompt_attention(q, k, v, cu_q, cu_k=None, *, causal=True, scale=None, out=None, lse=None, with_lse=False,
                     stream=None):
    """Attention over packed prompts (eas_prompt_attention).  q [rows, heads, head_dim] and k, v [rows, kv_heads,
    head_dim] in bfloat16 or float16, any row and head strides; cu_q, cu_k: host prefix sums of the sequences'
    queries and keys (cu_k None: the same).  scale None: head_dim ** -0.5.  Returns (out, lse): out like q, in
    ``out`` where given, rows behind the last sequence untouched; lse [rows, heads] float32 with with_lse or where
    given, else None."""
    device, dt = _device(q), _dtype(q.dtype)
    s = AttnShape(dt, q.shape[1] if q.dim() == 3 else 0, k.shape[1] if k.dim() == 3 else 0, q.shape[-1],
                  1 if causal else 0, _scale(scale, q.shape[-1]))
    s.q = _rows(q, "q")
    s.k = _rows(k, "k", None, s.head_dim, q.dtype, device)
    s.v = _rows(v, "v", s.kv_heads, s.head_dim, q.dtype, device)
    cu_q = _cu(cu_q, q.shape[0], "cu_q")
    cu_k = cu_q if cu_k is None else _cu(cu_k, min(k.shape[0], v.shape[0]), "cu_k")
    if cu_k.shape != cu_q.shape or cu_k[-1] > min(k.shape[0], v.shape[0]):
        raise ValueError("cu_q and cu_k: of the same sequences, keys within k and v")
    on = _On(stream)
    out, lse, lse_ptr = _outputs(on, q, q.shape[0], s.heads, out, lse, with_lse)
    s.out = _rows(out, "out", s.heads, s.head_dim, q.dtype, device)
    _check(LIB.eas_prompt_attention(ctypes.byref(s), q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                    cu_q.ctypes.data_as(P(I32)), cu_k.ctypes.data_as(P(I32)), cu_q.shape[0] - 1,
                                    out.data_ptr(), lse_ptr, on.ptr), "prompt_attention")
    return out, lse


class Kv8Cache:
    """A key / value cache in 8 bits (include/eas_attention.h): int8 or float8_e4m3fn codes k [pages, kv_heads,
    page_tokens, head_dim] and v [pages, kv_heads, head_dim, page_tokens], float32 scales [pages, kv_heads].
    Made from the caller's tensors, or by ``Kv8Cache.empty``.  Page tables are int32 device tensors [n_seqs,
    max_pages]; an entry that is no page (-1) is not held."""

    def __init__(self, k, v, k_scale, v_scale):
        if k.dim() != 4 or k.dtype not in _FORMAT:
            raise ValueError("k must be int8 or float8_e4m3fn codes [pages, kv_heads, page_tokens, head_dim]")
        n, h, p, d = k.shape
        for t, name, shape, dtype in ((k, "k", (n, h, p, d), k.dtype), (v, "v", (n, h, d, p), k.dtype),
                                      (k_scale, "k_scale", (n, h), torch.float32),
                                      (v_scale, "v_scale", (n, h), torch.float32)):
            if tuple(t.shape) != shape or t.dtype != dtype or t.device != k.device or not t.is_contiguous():
                raise ValueError("%s must be a contiguous %s tensor of shape %s on %s" % (name, dtype, shape, k.device))
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.kv_heads, self.page_tokens, self.head_dim = n, h, p, d
        self.device = k.device
        self._c = Kv8CacheStruct(_FORMAT[k.dtype], h, d, p, n, k.data_ptr(), v.data_ptr(), k_scale.data_ptr(),
                                 v_scale.data_ptr())
        self._ref = ctypes.byref(self._c)

    @classmethod
    def empty(cls, n_pages, kv_heads, head_dim, page_tokens=64, dtype=torch.int8, device="cuda"):
        """A cache that holds nothing yet; its contents are whatever the memory held."""
        def new(shape, kind):
            return torch.empty(shape, dtype=kind, device=device)
        return cls(new((n_pages, kv_heads, page_tokens, head_dim), dtype),
                   new((n_pages, kv_heads, head_dim, page_tokens), dtype),
                   new((n_pages, kv_heads), torch.float32), new((n_pages, kv_heads), torch.float32))

    def _table(self, pages):
        if pages.dim() != 2:
            raise ValueError("pages must be [n_seqs, max_pages]")
        if _device(pages) != self.device:
            raise ValueError("pages on %s, the cache on %s" % (pages.device, self.device))
        return _ints(pages, "pages", self.device, tuple(pages.shape)), pages.shape[1], pages.shape[0]

    def _split(self, cu, most, rows, n, name):
        """(pointer to the prefix sums or None, the most rows of a sequence)"""
        if cu is not None:
            return _ints(cu, name, self.device, (n + 1,)), rows if most is None else int(most)
        if most is None:
            most = rows // n if n else 0
        if most * n != rows:
            raise ValueError("without %s every sequence has the same number of rows: %d rows, %d sequences of %d"
                             % (name, rows, n, most))
        return None, int(most)

    def append(self, k, v, held, pages, cu_new=None, max_new=None, stream=None):
        """New tokens' keys and values [rows, kv_heads, head_dim] behind the ``held`` (int32 device [n_seqs]) tokens
        of each sequence (eas_kv8_append).  cu_new: int32 device prefix sums of the new tokens; None: the same
        number for all.  max_new: the most of a sequence (None: all rows)."""
        table, max_pages, n = self._table(pages)
        dt = _dtype(k.dtype)
        ks = _rows(k, "k", self.kv_heads, self.head_dim, k.dtype, self.device)
        vs = _rows(v, "v", self.kv_heads, self.head_dim, k.dtype, self.device)
        if v.shape[0] != k.shape[0]:
            raise ValueError("k has %d rows, v %d" % (k.shape[0], v.shape[0]))
        cu, most = self._split(cu_new, max_new, k.shape[0], n, "cu_new")
        _check(LIB.eas_kv8_append(self._ref, dt, k.data_ptr(), ks, v.data_ptr(), vs, k.shape[0], cu, most,
                                  _ints(held, "held", self.device, (n,)), table, max_pages, n, _On(stream).ptr),
               "Kv8Cache.append")

    def rows(self, pages, cu_rows, n_rows, first=None, max_len=None, dtype=torch.bfloat16, k=None, v=None, stream=None):
        """Cached tokens back as rows (eas_kv8_rows): rows cu_rows[r] .. cu_rows[r+1] (int32 device [n_seqs + 1]) of
        the ``n_rows`` receive sequence r's tokens from first[r] (int32 device; None: 0) on.  max_len: the most of a
        sequence (None: n_rows).  Returns (k, v) [n_rows, kv_heads, head_dim]; rows of no sequence are not written."""
        table, max_pages, n = self._table(pages)
        on = _On(stream)
        shape = (int(n_rows), self.kv_heads, self.head_dim)
        k = on.empty(shape, dtype, self.device) if k is None else k
        v = on.empty(shape, dtype, self.device) if v is None else v
        ks = _rows(k, "k", self.kv_heads, self.head_dim, dtype, self.device)
        vs = _rows(v, "v", self.kv_heads, self.head_dim, dtype, self.device)
        if k.shape[0] != shape[0] or v.shape[0] != shape[0]:
            raise ValueError("k has %d rows, v %d, wanted %d" % (k.shape[0], v.shape[0], shape[0]))
        _check(LIB.eas_kv8_rows(self._ref, _dtype(dtype), table, max_pages, n,
                                _ints(cu_rows, "cu_rows", self.device, (n + 1,)),
                                None if first is None else _ints(first, "first", self.device, (n,)),
                                shape[0] if max_len is None else int(max_len), shape[0], k.data_ptr(), ks,
                                v.data_ptr(), vs, on.ptr), "Kv8Cache.rows")
        return k, v

    def attention(self, q, lens, pages, cu_q=None, max_q=None, max_len=None, *, causal=True, scale=None, out=None,
                  lse=None, with_lse=False, workspace=None, stream=None):
        """Attention of q [rows, heads, head_dim] over the first ``lens`` (int32 device [n_seqs]) tokens of each
        sequence, the queries' own among them (eas_kv8_attention).  cu_q, max_q: as cu_new and max_new of append;
        max_len: the most tokens of a sequence (None: what the page table holds).  workspace: a uint8 device tensor
        to use instead of a new one.  Returns (out, lse) as prompt_attention."""
        table, max_pages, n = self._table(pages)
        dt = _dtype(q.dtype)
        qs = _rows(q, "q", None, self.head_dim, q.dtype, self.device)
        rows, heads = q.shape[0], q.shape[1]
        cu, most_q = self._split(cu_q, max_q, rows, n, "cu_q")
        most = max_pages * self.page_tokens
        most = most if max_len is None else min(int(max_len), most)
        on = _On(stream)
        out, lse, lse_ptr = _outputs(on, q, rows, heads, out, lse, with_lse)
        s = AttnShape(dt, heads, self.kv_heads, self.head_dim, 1 if causal else 0, _scale(scale, self.head_dim))
        s.q, s.out = qs, _rows(out, "out", heads, self.head_dim, q.dtype, self.device)
        need = I64()
        _check(LIB.eas_kv8_attention_workspace(ctypes.byref(s), most_q, most, n, ctypes.byref(need)),
               "Kv8Cache.attention")
        if need.value and workspace is None:
            workspace = on.empty((need.value,), torch.uint8, self.device)
        elif workspace is not None and (workspace.dtype != torch.uint8 or workspace.device != self.device
                                        or not workspace.is_contiguous()):
            raise ValueError("workspace must be a contiguous uint8 tensor on %s" % self.device)
        _check(LIB.eas_kv8_attention(self._ref, ctypes.byref(s), q.data_ptr(), rows, cu, most_q,
                                     _ints(lens, "lens", self.device, (n,)), most, table, max_pages, n,
                                     out.data_ptr(), lse_ptr, None if workspace is None else workspace.data_ptr(),
                                     0 if workspace is None else workspace.numel(), on.ptr), "Kv8Cache.attention")
        return out, lse
