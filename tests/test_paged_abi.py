"""Host-side checks of prompts in pieces (include/eas_paged.h): exports, refused arguments, calls with nothing to do,
workspace sizes, the plan's turns; and pins of the float64 reference.  No GPU: every call here returns before any HIP
call, so made-up device addresses do."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from oracle import paged as OP
from paper_2609_31551_amd import attention as A
from paper_2609_31551_amd import eas
from paper_2609_31551_amd import paged as B
from test_attention_abi import BAD, CAPACITY, PTR, SHAPE_REFUSALS, TABLE_REFUSALS, UNSUPPORTED, shape

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PI = 314159265358979323846264338327950288419716939937510582097494   # of 10^-59


def test_every_declared_symbol_is_exported():
    text = open(os.path.join(ROOT, "include", "eas_paged.h")).read()
    names = sorted(set(re.findall(r"^\s*eas_status\s+(eas_\w+)\s*\(", text, re.M)))
    assert len(names) == 5
    for n in names:
        assert hasattr(eas.LIB, n), n
    assert list(B.EXPORTS) == names


def plan(**over):
    r = B.Rotary.sections((16, 24, 24))._c
    copy = B.RotaryStruct.from_buffer_copy(r)
    for k, v in over.items():
        setattr(copy, k, v)
    return copy


def make(freqs=(1.0,) * 8, axis=None, pairs=None, axes=1, adjacent=0):
    r = B.RotaryStruct()
    n = len(freqs)
    status = eas.LIB.eas_rotary_make((ctypes.c_double * n)(*freqs), None if axis is None else (ctypes.c_int32 * n)(*axis),
                                     n if pairs is None else pairs, axes, adjacent, ctypes.byref(r))
    return status, r


@pytest.mark.parametrize("over,status", [
    (dict(freqs=(1.0,) * 7), UNSUPPORTED), (dict(freqs=(1.0,) * 136), UNSUPPORTED), (dict(pairs=0), BAD),
    (dict(pairs=-8), BAD), (dict(axes=0), BAD), (dict(axes=5), UNSUPPORTED), (dict(adjacent=2), BAD),
    (dict(freqs=(float("nan"),) * 8), BAD), (dict(freqs=(1.0,) * 7 + (float("inf"),)), BAD),
    (dict(axis=(0,) * 7 + (1,)), BAD), (dict(axis=(-1,) * 8), BAD), (dict(axis=(2,) * 8, axes=2), BAD),
], ids=lambda x: str(x))
def test_rotary_make_refuses(over, status):
    assert make(**over)[0] == status


def test_rotary_make_refuses_nothing_at_all():
    r = B.RotaryStruct()
    assert eas.LIB.eas_rotary_make(None, None, 8, 1, 0, ctypes.byref(r)) == BAD
    assert eas.LIB.eas_rotary_make((ctypes.c_double * 8)(), None, 8, 1, 0, None) == BAD


def test_a_plan_holds_turns_to_64_bits():
    """Against the quotient by 2 pi in whole numbers, pi to 59 decimals."""
    freqs = [1.0, 0.5, 1e-4, 1e-7, 3.0, 123456.789, -0.25, 0.0]
    status, r = make(freqs)
    assert status == eas.EAS_OK and r.pairs == 8 and r.axes == 1 and list(r.axis[:8]) == [0] * 8
    for f, got in zip(freqs, r.step):
        num, den = f.as_integer_ratio()
        turns = (num * 10 ** 59 << 64) // (den * 2 * PI)                # 2^-64 turns
        off = (got - turns) % (1 << 64)
        off = min(off, (1 << 64) - off)
        assert off <= 2 + abs(f) * 4, (f, got, turns)


def test_sections_put_the_frequencies_where_they_say():
    r = B.Rotary.sections((8, 16, 8), 10000.0)
    want = B.Rotary([10000.0 ** (-i / 32) for i in range(32)], [0] * 8 + [1] * 16 + [2] * 8)
    assert bytes(r._c) == bytes(want._c) and r.axes == 3 and r.pairs == 32
    r = B.Rotary.sections((8, 16, 8), 10000.0, per_axis=True)
    want = B.Rotary([10000.0 ** (-j / n) for n in (8, 16, 8) for j in range(n)], [0] * 8 + [1] * 16 + [2] * 8)
    assert bytes(r._c) == bytes(want._c)
    r = B.Rotary.sections((0, 16), adjacent=True)
    assert r.axes == 2 and r._c.adjacent == 1 and list(r._c.axis[:16]) == [1] * 16
    for bad in ((), (-8, 16), (12,), (136,)):
        with pytest.raises((ValueError, eas.EasError)):
            B.Rotary.sections(bad)
    with pytest.raises(ValueError):
        B.Rotary([1.0] * 8, [0] * 7)


def rows(rot=None, dtype=A.EAS_FP16, dim=128, inverse=0, positions=PTR, axis_stride=8, n=8, q=PTR, qs=(3584, 128), heads=28,
         q_out=PTR, qos=(3584, 128), k=PTR, ks=(512, 128), kv_heads=4, k_out=PTR, kos=(512, 128)):
    return eas.LIB.eas_rotary_rows(ctypes.byref(plan() if rot is None else rot), dtype, dim, inverse, positions, axis_stride,
                                   n, q, A.Strides(*qs), heads, q_out, A.Strides(*qos), k, A.Strides(*ks), kv_heads, k_out,
                                   A.Strides(*kos), None)


def bad_axis():
    r = plan()
    r.axis[5] = 3
    return r


PLAN_REFUSALS = [dict(pairs=0), dict(pairs=12), dict(pairs=136), dict(axes=0), dict(axes=5), dict(adjacent=2),
                 dict(reserved=1), dict(pairs=72)]


@pytest.mark.parametrize("over", PLAN_REFUSALS, ids=str)
def test_calls_refuse_plans(over):
    assert rows(plan(**over)) == BAD
    assert append(rot=plan(**over)) == BAD


def test_calls_refuse_plans_whose_axes_are_not_there():
    assert rows(bad_axis()) == append(rot=bad_axis()) == BAD
    assert eas.LIB.eas_rotary_rows(None, A.EAS_FP16, 128, 0, PTR, 8, 8, PTR, A.Strides(128, 128), 1, PTR,
                                   A.Strides(128, 128), None, A.Strides(0, 0), 0, None, A.Strides(0, 0), None) == BAD


@pytest.mark.parametrize("over,status", [
    (dict(dtype=A.EAS_FP32), UNSUPPORTED), (dict(dtype=7), BAD), (dict(dim=0), BAD), (dict(dim=136), UNSUPPORTED),
    (dict(dim=272), UNSUPPORTED), (dict(dim=112), BAD), (dict(inverse=2), BAD), (dict(positions=None), BAD),
    (dict(positions=PTR + 2), BAD), (dict(axis_stride=-1), BAD), (dict(n=-1), BAD), (dict(heads=0), BAD),
    (dict(heads=1025), BAD), (dict(kv_heads=0), BAD), (dict(q=None), BAD), (dict(q_out=None), BAD),
    (dict(q=PTR + 8), BAD), (dict(q_out=PTR + 8), BAD), (dict(k_out=None), BAD), (dict(k=PTR + 4, k_out=PTR + 4), BAD),
    (dict(qs=(3580, 128)), BAD), (dict(qos=(3584, 64), q_out=PTR + 4096), BAD), (dict(qos=(0, 128), q_out=PTR + 4096), BAD),
    (dict(qs=(1 << 24, 128)), UNSUPPORTED), (dict(kos=(512, 64)), BAD),
    (dict(qs=(7168, 128)), BAD), (dict(ks=(1024, 128)), BAD),       # in place, but not with the same strides
], ids=lambda x: str(x))
def test_rotary_rows_refuses(over, status):
    assert rows(**over) == status


def test_rotary_rows_refuses_more_threads_than_a_launch_holds():
    assert rows(n=(1 << 31) - 1, k=None) == UNSUPPORTED


def cache(**over):
    c = B.Kv16CacheStruct(A.EAS_BF16, 4, 128, 64, 10, PTR, PTR)
    for k, v in over.items():
        setattr(c, k, v)
    return c


CACHE_REFUSALS = [
    (dict(dtype=A.EAS_FP32), UNSUPPORTED), (dict(dtype=9), BAD), (dict(kv_heads=0), BAD), (dict(kv_heads=1025), BAD),
    (dict(n_pages=0), BAD), (dict(page_tokens=0), BAD), (dict(page_tokens=48), UNSUPPORTED),
    (dict(page_tokens=8), UNSUPPORTED), (dict(page_tokens=256), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED),
    (dict(head_dim=-1), BAD), (dict(k=None), BAD), (dict(v=PTR + 8), BAD),
]


def append(c=None, rot=None, positions=None, axis_stride=8, q=None, qs=(3584, 128), heads=28, q_out=None, qos=(3584, 128),
           k=PTR, v=PTR, strides=(512, 128), rows=8, cu=None, most=4, held=PTR, pages=PTR, max_pages=5, n=2):
    return eas.LIB.eas_kv16_append(ctypes.byref(c or cache()), None if rot is None else ctypes.byref(rot), positions,
                                   axis_stride, q, A.Strides(*qs), heads, q_out, A.Strides(*qos), k, A.Strides(*strides), v,
                                   A.Strides(*strides), rows, cu, most, held, pages, max_pages, n, None)


def attend(c=None, s=None, q=PTR, rows=2, cu=None, most_q=1, lens=PTR, most=4000, pages=PTR, max_pages=70, n=2, out=PTR,
           lse=None, ws=PTR, ws_bytes=1 << 62):
    return eas.LIB.eas_kv16_attention(ctypes.byref(c or cache()), ctypes.byref(s or shape()), q, rows, cu, most_q, lens,
                                      most, pages, max_pages, n, out, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("over,status", CACHE_REFUSALS, ids=lambda x: str(x))
def test_cache_calls_refuse_caches(over, status):
    assert append(cache(**over)) == status
    assert attend(cache(**over)) == status


@pytest.mark.parametrize("call", [append, attend])
@pytest.mark.parametrize("over,status", TABLE_REFUSALS, ids=lambda x: str(x))
def test_cache_calls_refuse_page_tables(call, over, status):
    assert call(**over) == status


@pytest.mark.parametrize("over,status", [
    (dict(k=None), BAD), (dict(v=PTR + 4), BAD), (dict(strides=(510, 128)), BAD), (dict(strides=(-8, 128)), BAD),
    (dict(rows=-1), BAD), (dict(most=-1), BAD), (dict(held=None), BAD), (dict(held=PTR + 2), BAD), (dict(cu=PTR + 2), BAD),
    (dict(q=PTR, q_out=PTR), BAD),                                       # queries without a rotation
    (dict(rot=1, q=PTR, q_out=None), BAD), (dict(rot=1, q=PTR + 8, q_out=PTR + 8), BAD),
    (dict(rot=1, q=PTR, q_out=PTR, heads=0), BAD), (dict(rot=1, q=PTR, q_out=PTR, heads=1025), BAD),
    (dict(rot=1, q=PTR, q_out=PTR, qs=(7168, 128)), BAD), (dict(rot=1, q=PTR, q_out=PTR + 16, qos=(3584, 64)), BAD),
    (dict(rot=1, positions=PTR + 2), BAD), (dict(rot=1, positions=PTR, axis_stride=-8), BAD),
    (dict(rows=(1 << 31) - 1, most=(1 << 31) - 1, n=1), UNSUPPORTED),
], ids=lambda x: str(x))
def test_append_refuses_arguments(over, status):
    if "rot" in over:
        over = dict(over, rot=plan())
    assert append(**over) == status


@pytest.mark.parametrize("over,status", [
    (dict(s=shape(kv_heads=2)), BAD), (dict(s=shape(head_dim=64)), BAD), (dict(s=shape(dtype=A.EAS_FP16)), BAD),
    (dict(q=None), BAD), (dict(out=None), BAD), (dict(q=PTR + 8), BAD), (dict(lens=None), BAD), (dict(lens=PTR + 1), BAD),
    (dict(cu=PTR + 1), BAD), (dict(most=-1), BAD), (dict(most_q=-1), BAD), (dict(rows=-1), BAD), (dict(ws=None), BAD),
    (dict(ws=PTR + 8), BAD), (dict(ws_bytes=0), CAPACITY), (dict(lse=PTR + 2), BAD),
    (dict(rows=(1 << 31) - 1, most_q=(1 << 31) - 1, n=(1 << 31) - 1), UNSUPPORTED), (dict(s=shape(out=(1024, 128))), BAD),
], ids=lambda x: str(x))
def test_attention_refuses_arguments(over, status):
    assert attend(**over) == status


@pytest.mark.parametrize("over,status", SHAPE_REFUSALS, ids=lambda x: str(x))
def test_attention_refuses_shapes(over, status):
    assert attend(s=shape(**over)) == status


def test_calls_with_nothing_to_do():
    for over in (dict(rows=0), dict(n=0)):
        assert append(k=None, v=None, **over) == eas.EAS_OK
        assert attend(q=None, out=None, ws=None, **over) == eas.EAS_OK
    assert append(most=0) == attend(most_q=0) == rows(n=0, q=None, q_out=None, positions=None) == eas.EAS_OK
    assert append(n=0, held=None, pages=None) == attend(n=0, lens=None, pages=None) == eas.EAS_OK


def workspace(max_q, max_len, n, s=None, rows=None):
    """rows: of the batch; None: max_q of each sequence."""
    b = ctypes.c_int64(-1)
    rows = min(max_q * n, (1 << 31) - 1) if rows is None else rows
    assert eas.LIB.eas_kv16_attention_workspace(ctypes.byref(s or shape()), rows, max_q, max_len, n, ctypes.byref(b)) == 0
    return b.value


def test_workspace_sizes_grow_with_rows_and_tokens_up_to_a_bound():
    assert workspace(1, 64, 3) == 0                        # short: nothing is split
    one = workspace(1, 4000, 1)
    assert one > 0 and workspace(1, 4000, 5) == 5 * one
    assert workspace(1, 1 << 20, 1) >= workspace(1, 9000, 1) >= one
    assert workspace(1 << 20, 1 << 30, 1) == workspace(1 << 21, 1 << 30, 1) <= 1200 << 20
    # single tokens beside one chunk: by the rows there are
    assert workspace(500, 8000, 64, rows=563) < workspace(500, 8000, 64) / 4
    assert workspace(0, 8000, 4) == workspace(5, 8000, 0) == 0
    assert attend(ws_bytes=workspace(1, 4000, 2) - 1) == CAPACITY
    b = ctypes.c_int64()
    call = eas.LIB.eas_kv16_attention_workspace
    assert call(None, 1, 1, 1, 1, ctypes.byref(b)) == BAD
    assert call(ctypes.byref(shape()), 1, -1, 1, 1, ctypes.byref(b)) == BAD
    assert call(ctypes.byref(shape()), -1, 1, 1, 1, ctypes.byref(b)) == BAD
    assert call(ctypes.byref(shape()), 1, 1, 1, 1, None) == BAD
    assert call(ctypes.byref(shape(head_dim=80)), 1, 1, 1, 1, ctypes.byref(b)) == UNSUPPORTED


def test_the_binding_knows_where_no_workspace_is_needed():
    for heads, kv_heads in ((1, 1), (28, 4), (1024, 8)):
        for max_q in (1, 7, 300, 5000):
            assert workspace(max_q, B.SPLIT_TOKENS, 64, shape(heads=heads, kv_heads=kv_heads)) == 0


def test_binding_refuses_tensors_of_other_devices_and_kinds():
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    rot = B.Rotary.sections((32,))
    with pytest.raises((ValueError, RuntimeError)):        # not on a GPU
        rot.rows(x, torch.zeros(4, dtype=torch.int32))
    k = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16)
    B.Kv16Cache(k, k.clone())
    for bad in ((k.float(), k.float()), (k, k.half()), (k[0], k[0]), (k, k[:2]), (k.transpose(1, 2), k.transpose(1, 2))):
        with pytest.raises(ValueError):
            B.Kv16Cache(*bad)


# ---- the reference ---------------------------------------------------------------

def test_reference_rotation():
    rng = np.random.default_rng(0)
    x = rng.normal(size=(5, 2, 40))
    freqs, axis = [10000.0 ** (-i / 16) for i in range(16)], [0] * 4 + [1] * 6 + [2] * 6
    pos = rng.integers(-50, 100, (3, 5))
    for adjacent in (False, True):
        y = OP.rotate(x, pos, freqs, axis, adjacent)
        np.testing.assert_allclose(OP.rotate(y, pos, freqs, axis, adjacent, inverse=True), x, atol=1e-13)
        np.testing.assert_array_equal(y[..., 32:], x[..., 32:])
        i, j = (6, 7) if adjacent else (3, 19)                       # pair 3: the first axis
        a = pos[0] * freqs[3]
        np.testing.assert_allclose(y[:, 0, i], x[:, 0, i] * np.cos(a) - x[:, 0, j] * np.sin(a), atol=1e-12)
        np.testing.assert_allclose(y[:, 0, j], x[:, 0, i] * np.sin(a) + x[:, 0, j] * np.cos(a), atol=1e-12)
    # q . k depends on the positions' differences alone
    q, k = x[:1], x[1:2]
    one = (OP.rotate(q, [[7], [1], [2]], freqs, axis) * OP.rotate(k, [[3], [5], [2]], freqs, axis)).sum()
    two = (OP.rotate(q, [[1007], [11], [0]], freqs, axis) * OP.rotate(k, [[1003], [15], [0]], freqs, axis)).sum()
    assert abs(one - two) < 1e-10
    # the angle of a far position: 2^31 - 1 at one radian, its sine to 25 digits from integer reduction
    p = (1 << 31) - 1
    rest = (p * 10 ** 59) % (2 * PI) / 10 ** 59
    assert abs(np.sin(OP.angles([[p]], [1.0], [0])[0, 0]) - np.sin(rest)) < 1e-8


def test_reference_cache_equals_plain_attention():
    from oracle import attention as O
    rng = np.random.default_rng(1)
    k, v, q = rng.normal(size=(37, 2, 8)), rng.normal(size=(37, 2, 8)), rng.normal(size=(5, 4, 8))
    c = OP.Cache(5, 2, 16, 8, np.nan)
    c.append(k[:20], v[:20], 0, [3, 0, 4])
    c.append(k[20:], v[20:], 20, [3, 0, 4])
    out, lse, size = c.attention(q, 37, [3, 0, 4], 0.3, True)
    want, want_lse = O.prompt_attention(q, k, v, [0, 5], [0, 37], 0.3, True)
    np.testing.assert_allclose(out, want, atol=1e-14)
    np.testing.assert_allclose(lse, want_lse, atol=1e-14)
    out, lse, _ = c.attention(q, 37, [3, -1, 4], 0.3, True)          # a page that is not held
    gone = np.r_[0:16, 32:37]
    want, want_lse = O.prompt_attention(q, k[gone], v[gone], [0, 5], [0, 21], 0.3, True)
    np.testing.assert_allclose(out, want, atol=1e-14)
