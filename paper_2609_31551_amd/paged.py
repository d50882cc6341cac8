"""ctypes binding of prompts in pieces in libeas.so (include/eas_paged.h): rotary positions with several axes, and the
paged 16-bit key / value cache.  Argument marshalling and checks of what the C ABI cannot see (tensor types, shapes,
devices), as in attention.py; all tensors of a call are on the current device.
"""
import ctypes
import struct

import torch

from .attention import (AttnShape, I32, I64, P, Strides, VP, _DTYPE, _check, _count, _current_stream, _device, _dtype,
                        _ints, _on, _outputs, _rows, _shape, _workspace)
from .eas import LIB

MAX_PAIRS, MAX_AXES = 128, 4
SPLIT_TOKENS = 1024   # calls of up to these need no workspace


class RotaryStruct(ctypes.Structure):
    _fields_ = [("pairs", I32), ("axes", I32), ("adjacent", I32), ("reserved", I32),
                ("step", ctypes.c_uint64 * MAX_PAIRS), ("axis", ctypes.c_uint8 * MAX_PAIRS)]


class Kv16CacheStruct(ctypes.Structure):
    _fields_ = [("dtype", I32), ("kv_heads", I32), ("head_dim", I32), ("page_tokens", I32), ("n_pages", I32),
                ("k", VP), ("v", VP)]


_pack_cache = struct.Struct("5i4x2P").pack
_SIG = {
    "eas_rotary_make": [VP, VP, I32, I32, I32, P(RotaryStruct)],
    "eas_rotary_rows": [P(RotaryStruct), I32, I32, I32, VP, I64, I32, VP, Strides, I32, VP, Strides, VP, Strides, I32, VP,
                        Strides, VP],
    "eas_kv16_append": [P(Kv16CacheStruct), P(RotaryStruct), VP, I64, VP, Strides, I32, VP, Strides, VP, Strides, VP,
                        Strides, I32, VP, I32, VP, VP, I32, I32, VP],
    "eas_kv16_attention": [P(Kv16CacheStruct), P(AttnShape), VP, I32, VP, I32, VP, I32, VP, I32, I32, VP, VP, VP, I64, VP],
    "eas_kv16_attention_workspace": [P(AttnShape), I32, I32, I32, I32, P(I64)],
}
for _name, _args in _SIG.items():
    _fn = getattr(LIB, _name)
    _fn.argtypes = _args
    _fn.restype = I32
EXPORTS = tuple(sorted(_SIG))
_NO_STRIDES = Strides(0, 0)


def _turned(x, name, out, heads, dim, dtype, index, stream):
    """The tensor that rotated rows go to -- the caller's or a new one --, its address and strides."""
    if out is None:
        out = torch.empty_like(x) if stream is None else _on(stream, lambda: torch.empty_like(x))
        row, head, _ = out.stride()   # empty_like keeps x's order
        return out, out.data_ptr(), Strides(row if x.shape[0] > 1 else 0, head if heads > 1 else 0)
    if out.shape[0] != x.shape[0]:
        raise ValueError("%s has %d rows, wanted %d" % (name, out.shape[0], x.shape[0]))
    return out, out.data_ptr(), Strides(*_rows(out, name, heads, dim, dtype, index))


class Rotary:
    """What a model's positions do to a head (include/eas_paged.h, eas_rotary): pair i of its dimensions turns by
    positions[axis[i]] * freqs[i] radians (|freqs[i]| < 2 ** 60).  Pair i is dimensions (i, i + pairs) or, adjacent,
    (2 i, 2 i + 1); dimensions behind the pairs pass.  Made once for a model; holds no device memory."""

    def __init__(self, freqs, axis=None, axes=None, adjacent=False):
        freqs = [float(f) for f in freqs]
        axis = [0] * len(freqs) if axis is None else [int(a) for a in axis]
        if len(axis) != len(freqs):
            raise ValueError("%d frequencies, %d axes of pairs" % (len(freqs), len(axis)))
        n = len(freqs)
        self.pairs, self.adjacent = n, bool(adjacent)
        self.axes = max(axis, default=0) + 1 if axes is None else int(axes)
        self._c = RotaryStruct()
        _check(LIB.eas_rotary_make((ctypes.c_double * n)(*freqs), (ctypes.c_int32 * n)(*axis), n, self.axes,
                                   1 if adjacent else 0, self._c), "Rotary")

    @classmethod
    def sections(cls, sections, theta=10000.0, *, per_axis=False, adjacent=False):
        """sections: the pairs that each axis turns, the first axis's first ((16, 24, 24): time, height, width).  Pair i
        of n turns by theta ** (-i / n) for one position; per_axis: pair j of an axis's m by theta ** (-j / m)."""
        sections = [int(n) for n in sections]
        if not sections or min(sections) < 0:
            raise ValueError("sections must be the numbers of pairs of the axes, got %r" % (sections,))
        axis = [a for a, n in enumerate(sections) for _ in range(n)]
        if per_axis:
            freqs = [float(theta) ** (-j / n) for n in sections for j in range(n)]
        else:
            freqs = [float(theta) ** (-i / len(axis)) for i in range(len(axis))]
        return cls(freqs, axis, len(sections), adjacent)

    def _positions(self, positions, rows, index):
        """Address and axis stride of int32 [axes, rows], or [rows] for all axes."""
        shape, strides = positions.shape, positions.stride()
        if positions.dtype == torch.int32 and positions.get_device() == index and strides and shape[-1] == rows \
                and (strides[-1] == 1 or rows <= 1):
            if len(shape) == 1:
                return positions.data_ptr(), 0
            if len(shape) == 2 and shape[0] == self.axes:
                return positions.data_ptr(), strides[0] if self.axes > 1 else 0
        raise ValueError("positions must be int32 [%d, %d], or [%d] for all axes, a row's neighbours consecutive, on cuda:%d:"
                         " got %s %s, strides %s, on %s"
                         % (self.axes, rows, rows, index, positions.dtype, tuple(shape), strides, positions.device))

    def rows(self, q, positions, k=None, *, inverse=False, q_out=None, k_out=None, stream=None):
        """q [rows, heads, head_dim] and, where given, k [rows, kv_heads, head_dim], in bfloat16 or float16, rotated by
        positions (int32 device [axes, rows], or [rows] for all axes) (eas_rotary_rows).  inverse: by the opposite
        angles, which takes a rotation back, and turns the gradients of rotated rows into the rows'.  q_out, k_out: where
        the results go (q and k themselves are fine); None: new tensors.  Returns (q_out, k_out), k_out None without k."""
        index, dtype = _device(q), q.dtype
        code = _dtype(dtype)
        if q.dim() != 3 or (k is not None and k.dim() != 3):
            raise ValueError("q and k must be [rows, heads, head_dim]")
        rows, heads, dim = q.shape
        qs = Strides(*_rows(q, "q", None, dim, dtype, index))
        at, axis_stride = self._positions(positions, rows, index)
        q_out, q_ptr, qos = _turned(q, "q_out", q_out, heads, dim, dtype, index, stream)
        if k is None:
            if k_out is not None:
                raise ValueError("k_out without k")
            kv_heads, k_in, k_ptr, ks, kos = 0, None, None, _NO_STRIDES, _NO_STRIDES
        else:
            if k.shape[0] != rows:
                raise ValueError("q has %d rows, k %d" % (rows, k.shape[0]))
            kv_heads, k_in = k.shape[1], k.data_ptr()
            ks = Strides(*_rows(k, "k", None, dim, dtype, index))
            k_out, k_ptr, kos = _turned(k, "k_out", k_out, kv_heads, dim, dtype, index, stream)
        _check(LIB.eas_rotary_rows(self._c, code, dim, 1 if inverse else 0, at, axis_stride, _count(None, rows, "rows"),
                                   q.data_ptr(), qs, heads, q_ptr, qos, k_in, ks, kv_heads, k_ptr, kos,
                                   _current_stream(index) if stream is None else stream.cuda_stream), "Rotary.rows")
        return q_out, k_out


class Kv16Cache:
    """A paged key / value cache in bfloat16 or float16 (include/eas_paged.h): k and v [pages, kv_heads, page_tokens,
    head_dim].  Made from the caller's tensors, or by ``Kv16Cache.empty``.  Page tables are int32 device tensors [n_seqs,
    max_pages]; an entry that is no page (-1) is not held."""

    def __init__(self, k, v):
        index, shape, dtype = k.get_device(), k.shape, k.dtype
        if not (len(shape) == 4 and (dtype == torch.bfloat16 or dtype == torch.float16) and v.shape == shape
                and v.dtype == dtype and v.get_device() == index and k.is_contiguous() and v.is_contiguous()):
            raise ValueError("wanted contiguous k and v [pages, kv_heads, page_tokens, head_dim], bfloat16 or "
                             "float16, on one device: got " +
                             ", ".join("%s %s on %s" % (tuple(t.shape), t.dtype, t.device) for t in (k, v)))
        n, h, p, d = shape
        code = _DTYPE[dtype]
        self.k, self.v, self.dtype = k, v, dtype
        self.n_pages, self.kv_heads, self.page_tokens, self.head_dim = n, h, p, d
        self._index, self._code = index, code
        self._c = Kv16CacheStruct.from_buffer_copy(_pack_cache(code, h, d, p, n, k.data_ptr(), v.data_ptr()))

    @property
    def device(self):
        return self.k.device

    @classmethod
    def empty(cls, n_pages, kv_heads, head_dim, page_tokens=64, dtype=torch.bfloat16, device="cuda"):
        """A cache that holds nothing yet; its contents are whatever the memory held."""
        shape = (n_pages, kv_heads, page_tokens, head_dim)
        return cls(torch.empty(shape, dtype=dtype, device=device), torch.empty(shape, dtype=dtype, device=device))

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

    def append(self, k, v, held, pages, cu_new=None, max_new=None, *, rotary=None, positions=None, q=None, q_out=None,
               stream=None):
        """New tokens' keys and values [rows, kv_heads, head_dim] behind the ``held`` (int32 device [n_seqs]) tokens of
        each sequence (eas_kv16_append).  cu_new: int32 device prefix sums of the new tokens; None: the same number for
        all.  max_new: the most of a sequence (None: all rows).  rotary: a Rotary by which the keys are rotated on the
        way, and the queries q [rows, heads, head_dim], where given, into q_out (q itself is fine; None: a new tensor,
        whose rows of no sequence are whatever the memory held); positions: int32 device [axes, rows], or [rows] for all
        axes; None: a token's place in its sequence.  Returns the rotated queries, or None without q."""
        table, max_pages, n = self._table(pages)
        index, dtype, rows, dim = self._index, self.dtype, k.shape[0], self.head_dim
        ks = _rows(k, "k", self.kv_heads, dim, dtype, index)
        vs = _rows(v, "v", self.kv_heads, dim, dtype, index)
        if v.shape[0] != rows:
            raise ValueError("k has %d rows, v %d" % (rows, v.shape[0]))
        cu, most = self._split(cu_new, max_new, rows, n, "cu_new")
        plan = at = q_ptr = out_ptr = None
        axis_stride = heads = 0
        qs = qos = _NO_STRIDES
        if rotary is not None:
            plan = rotary._c
            if positions is not None:
                at, axis_stride = rotary._positions(positions, rows, index)
        elif positions is not None or q is not None:
            raise ValueError("positions and q are for a rotation: rotary is None")
        if q is not None:
            if q.dim() != 3 or q.shape[0] != rows:
                raise ValueError("q must be [%d, heads, %d], got %s" % (rows, dim, tuple(q.shape)))
            heads = q.shape[1]
            q_ptr, qs = q.data_ptr(), Strides(*_rows(q, "q", None, dim, dtype, index))
            q_out, out_ptr, qos = _turned(q, "q_out", q_out, heads, dim, dtype, index, stream)
        elif q_out is not None:
            raise ValueError("q_out without q")
        _check(LIB.eas_kv16_append(self._c, plan, at, axis_stride, q_ptr, qs, heads, out_ptr, qos, k.data_ptr(),
                                   Strides(*ks), v.data_ptr(), Strides(*vs), rows, cu, most,
                                   _ints(held, "held", index, (n,)), table, max_pages, n,
                                   _current_stream(index) if stream is None else stream.cuda_stream), "Kv16Cache.append")
        return q_out

    def attention(self, q, lens, pages, cu_q=None, max_q=None, max_len=None, *, causal=True, scale=None, out=None,
                  lse=None, with_lse=False, workspace=None, stream=None):
        """Attention of q [rows, heads, head_dim] over the first ``lens`` (int32 device [n_seqs]) tokens of each
        sequence, the queries' own among them (eas_kv16_attention): single tokens, a few, or chunks, as they come.  cu_q,
        max_q: as cu_new and max_new of append; max_len: the most tokens of a sequence (None: what the page table holds).
        The launch and the workspace grow with max_q * n_seqs and max_len, so give them where cu_q is given.  workspace: a
        uint8 device tensor to use instead of a new one.  Returns (out, lse) as attention.prompt_attention."""
        table, max_pages, n = self._table(pages)
        index, dtype, dim = self._index, self.dtype, self.head_dim
        qs = _rows(q, "q", None, dim, dtype, index)
        rows, heads = q.shape[0], q.shape[1]
        cu, most_q = self._split(cu_q, max_q, rows, n, "cu_q")
        most = min(_count(max_len, max_pages * self.page_tokens, "max_len"), max_pages * self.page_tokens)
        out, lse, strides, lse_ptr = _outputs(q, out, lse, with_lse, index, stream)
        shape = _shape(self._code, heads, self.kv_heads, dim, causal, scale, qs, (0, 0), (0, 0), strides)
        need = I64()
        if most > SPLIT_TOKENS:
            _check(LIB.eas_kv16_attention_workspace(shape, rows, most_q, most, n, need), "Kv16Cache.attention")
        workspace, ws_ptr, ws_bytes = _workspace(workspace, need.value, index, self.device, stream)
        _check(LIB.eas_kv16_attention(self._c, shape, q.data_ptr(), rows, cu, most_q, _ints(lens, "lens", index, (n,)),
                                      most, table, max_pages, n, out.data_ptr(), lse_ptr, ws_ptr, ws_bytes,
                                      _current_stream(index) if stream is None else stream.cuda_stream),
               "Kv16Cache.attention")
        return out, lse
