"""Host-side checks of the language side's attention (include/eas_attention.h): exports, refused arguments, calls
with nothing to do, workspace sizes; and pins of its float64 reference.  No GPU: every call here returns before any
HIP call, so made-up device addresses do."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from oracle import attention as O
from paper_2609_31551_amd import attention as A
from paper_2609_31551_amd import eas

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BAD, SHAPE, CAPACITY, UNSUPPORTED = (eas.EAS_ERR_INVALID_ARG, eas.EAS_ERR_SHAPE, eas.EAS_ERR_CAPACITY,
                                     eas.EAS_ERR_UNSUPPORTED)
PTR = 0x10000   # an aligned address that nothing reads


def test_every_declared_symbol_is_exported():
    text = open(os.path.join(ROOT, "include", "eas_attention.h")).read()
    names = sorted(set(re.findall(r"^\s*eas_status\s+(eas_\w+)\s*\(", text, re.M)))
    assert len(names) == 6
    for n in names:
        assert hasattr(eas.LIB, n), n
    assert list(A.EXPORTS) == names


def shape(**over):
    s = A.AttnShape(A.EAS_BF16, 28, 4, 128, 1, 0.1)
    for n in ("q", "k", "v", "out"):
        h = 28 if n in ("q", "out") else 4
        setattr(s, n, A.Strides(h * 128, 128))
    for k, v in over.items():
        setattr(s, k, A.Strides(*v) if isinstance(v, tuple) else v)
    return s


def ints(*v):
    return (ctypes.c_int32 * len(v))(*v)


def prompt(s=None, q=PTR, k=PTR, v=PTR, cu_q=(0, 5, 9), cu_k=None, n=None, out=PTR, lse=None, ws=PTR,
           ws_bytes=1 << 30):
    cu = None if cu_q is None else ints(*cu_q)
    return eas.LIB.eas_prompt_attention(ctypes.byref(s or shape()), q, k, v, cu, None if cu_k is None else ints(*cu_k),
                                        (len(cu_q) - 1 if cu_q else 1) if n is None else n, out, lse, ws, ws_bytes,
                                        None)


SHAPE_REFUSALS = [
    (dict(dtype=A.EAS_FP32), UNSUPPORTED), (dict(dtype=3), BAD), (dict(dtype=-1), BAD),
    (dict(heads=27), BAD), (dict(heads=0), BAD), (dict(kv_heads=0), BAD), (dict(kv_heads=-4), BAD),
    (dict(heads=1028), BAD), (dict(head_dim=0), BAD), (dict(head_dim=80), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED),
    (dict(causal=2), BAD), (dict(scale=float("nan")), BAD), (dict(scale=float("inf")), BAD),
    (dict(q=(3580, 128)), BAD), (dict(q=(-3584, 128)), BAD), (dict(q=(3584, 100)), BAD),
    (dict(q=((1 << 23) + 8, 128)), UNSUPPORTED), (dict(out=(3584, 64)), BAD), (dict(out=(1024, 128)), BAD),
    (dict(out=(0, 128)), BAD),
]


@pytest.mark.parametrize("over,status", SHAPE_REFUSALS, ids=lambda x: str(x))
def test_prompt_attention_refuses_shapes(over, status):
    assert prompt(shape(**over)) == status


@pytest.mark.parametrize("over,status", [
    (dict(cu_q=None), BAD), (dict(cu_q=(1, 5)), SHAPE), (dict(cu_q=(0, 5, 4)), SHAPE),
    (dict(cu_k=(0, 5, 4)), SHAPE), (dict(cu_k=(2, 5, 8)), SHAPE), (dict(n=-1), CAPACITY),
    (dict(cu_q=tuple(range(66))), CAPACITY), (dict(q=None), BAD), (dict(k=None), BAD), (dict(v=None), BAD),
    (dict(out=None), BAD), (dict(q=PTR + 8), BAD), (dict(k=PTR + 2), BAD), (dict(out=PTR + 8), BAD),
    (dict(lse=PTR + 2), BAD), (dict(cu_q=(0, 9), cu_k=(0, 90000), ws=None), BAD),
    (dict(cu_q=(0, 9), cu_k=(0, 90000), ws=PTR + 8), BAD), (dict(cu_q=(0, 9), cu_k=(0, 90000), ws_bytes=64), CAPACITY),
    (dict(cu_q=(0, 9), cu_k=(0, (1 << 30) + 1)), UNSUPPORTED),
], ids=lambda x: str(x))
def test_prompt_attention_refuses_arguments(over, status):
    assert prompt(**over) == status
    assert eas.LIB.eas_prompt_attention(None, PTR, PTR, PTR, ints(0, 5), None, 1, PTR, None, None, 0,
                                        None) == BAD


def test_prompt_attention_refuses_more_work_items_than_a_launch_holds():
    s = shape(heads=1024, kv_heads=1024, q=(1 << 17, 128), k=(1 << 17, 128), v=(1 << 17, 128), out=(1 << 17, 128))
    assert prompt(s, cu_q=(0, 2147483647)) == UNSUPPORTED


def test_prompt_attention_workspace():
    def size(cu_q, cu_k, s=None):
        b = ctypes.c_int64(-1)
        assert eas.LIB.eas_prompt_attention_workspace(ctypes.byref(s or shape()), ints(*cu_q), ints(*cu_k),
                                                      len(cu_q) - 1, ctypes.byref(b)) == 0
        return b.value
    assert size((0, 100, 300), (0, 100, 300)) == 0 and size((0,), (0,)) == 0
    assert size((0, 8000), (0, 8000)) == 0                  # many queries fill the chip
    one = size((0, 100), (0, 100000))
    assert one > 0 and size((0, 100, 200), (0, 100000, 200000)) == 2 * one
    assert size((0, 0, 100), (0, 50000, 150000)) == one
    assert prompt(cu_q=(0, 100), cu_k=(0, 100000), ws_bytes=one - 1) == CAPACITY
    call, b = eas.LIB.eas_prompt_attention_workspace, ctypes.c_int64()
    assert call(None, ints(0, 5), None, 1, ctypes.byref(b)) == BAD
    assert call(ctypes.byref(shape()), None, None, 1, ctypes.byref(b)) == BAD
    assert call(ctypes.byref(shape()), ints(0, 5), None, 1, None) == BAD
    assert call(ctypes.byref(shape()), ints(1, 5), None, 1, ctypes.byref(b)) == SHAPE
    assert call(ctypes.byref(shape()), ints(0, 5), None, 65, ctypes.byref(b)) == CAPACITY


def test_prompt_attention_with_nothing_to_do():
    assert prompt(cu_q=(0,), n=0, q=None, k=None, v=None, out=None) == eas.EAS_OK
    assert prompt(cu_q=(0, 0, 0), cu_k=(0, 3, 9), q=None, out=None) == eas.EAS_OK


def cache(**over):
    c = A.Kv8CacheStruct(A.EAS_KV_INT8, 4, 128, 64, 10, PTR, PTR, PTR, PTR)
    for k, v in over.items():
        setattr(c, k, v)
    return c


CACHE_REFUSALS = [
    (dict(format=2), BAD), (dict(kv_heads=0), BAD), (dict(n_pages=0), BAD), (dict(page_tokens=0), BAD),
    (dict(page_tokens=48), UNSUPPORTED), (dict(page_tokens=8), UNSUPPORTED), (dict(page_tokens=256), UNSUPPORTED),
    (dict(head_dim=96), UNSUPPORTED), (dict(k=None), BAD), (dict(v=PTR + 8), BAD), (dict(k_scale=None), BAD),
    (dict(v_scale=PTR + 2), BAD),
]


def append(c=None, dtype=A.EAS_FP16, k=PTR, v=PTR, strides=(512, 128), rows=8, cu=None, most=4, held=PTR, pages=PTR,
           max_pages=5, n=2):
    return eas.LIB.eas_kv8_append(ctypes.byref(c or cache()), dtype, k, A.Strides(*strides), v, A.Strides(*strides),
                                  rows, cu, most, held, pages, max_pages, n, None)


def rows(c=None, dtype=A.EAS_FP16, pages=PTR, max_pages=5, n=2, cu=PTR, first=None, most=4, rows=8, k=PTR, v=PTR,
         strides=(512, 128)):
    return eas.LIB.eas_kv8_rows(ctypes.byref(c or cache()), dtype, pages, max_pages, n, cu, first, most, rows, k,
                                A.Strides(*strides), v, A.Strides(*strides), None)


def attend(c=None, s=None, q=PTR, rows=2, cu=None, most_q=1, lens=PTR, most=4000, pages=PTR, max_pages=70, n=2, out=PTR,
           lse=None, ws=PTR, ws_bytes=1 << 30):
    return eas.LIB.eas_kv8_attention(ctypes.byref(c or cache()), ctypes.byref(s or shape()), q, rows, cu, most_q, lens,
                                     most, pages, max_pages, n, out, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("over,status", CACHE_REFUSALS, ids=lambda x: str(x))
def test_cache_calls_refuse_caches(over, status):
    assert append(cache(**over)) == status
    assert rows(cache(**over)) == status
    assert attend(cache(**over)) == status


TABLE_REFUSALS = [(dict(pages=None), BAD), (dict(max_pages=0), BAD), (dict(n=-1), BAD), (dict(pages=PTR + 1), BAD),
                  (dict(max_pages=(1 << 24) + 1), UNSUPPORTED)]


@pytest.mark.parametrize("call", [append, rows, attend])
@pytest.mark.parametrize("over,status", TABLE_REFUSALS, ids=lambda x: str(x))
def test_cache_calls_refuse_page_tables(call, over, status):
    assert call(**over) == status


@pytest.mark.parametrize("over,status", [
    (dict(dtype=A.EAS_FP32), UNSUPPORTED), (dict(dtype=9), BAD), (dict(k=None), BAD), (dict(v=PTR + 4), BAD),
    (dict(strides=(510, 128)), BAD), (dict(strides=(-8, 128)), BAD), (dict(rows=-1), BAD), (dict(most=-1), BAD),
    (dict(held=None), BAD), (dict(held=PTR + 2), BAD), (dict(cu=PTR + 2), BAD),
], ids=lambda x: str(x))
def test_append_refuses_arguments(over, status):
    assert append(**over) == status


@pytest.mark.parametrize("over,status", [
    (dict(dtype=A.EAS_FP32), UNSUPPORTED), (dict(k=None, v=None), BAD), (dict(v=PTR + 4), BAD),
    (dict(strides=(512, 64)), BAD), (dict(strides=(0, 128)), BAD), (dict(rows=-1), BAD), (dict(most=-1), BAD),
    (dict(cu=None), BAD), (dict(first=PTR + 2), BAD),
], ids=lambda x: str(x))
def test_rows_refuses_arguments(over, status):
    assert rows(**over) == status


@pytest.mark.parametrize("over,status", [
    (dict(s=shape(kv_heads=2)), BAD), (dict(s=shape(head_dim=64)), BAD), (dict(q=None), BAD), (dict(out=None), BAD),
    (dict(q=PTR + 8), BAD), (dict(lens=None), BAD), (dict(lens=PTR + 1), BAD), (dict(cu=PTR + 1), BAD),
    (dict(most=-1), BAD), (dict(most_q=-1), BAD), (dict(rows=-1), BAD), (dict(ws=None), BAD), (dict(ws=PTR + 8), BAD),
    (dict(ws_bytes=0), CAPACITY), (dict(lse=PTR + 2), BAD), (dict(most_q=1 << 30), UNSUPPORTED),
    (dict(s=shape(out=(1024, 128))), BAD),
], ids=lambda x: str(x))
def test_attention_refuses_arguments(over, status):
    assert attend(**over) == status


@pytest.mark.parametrize("over,status", SHAPE_REFUSALS, ids=lambda x: str(x))
def test_attention_refuses_shapes(over, status):
    assert attend(s=shape(**over)) == status


def test_cache_calls_with_nothing_to_do():
    for over in (dict(rows=0), dict(n=0)):
        assert append(k=None, v=None, **over) == eas.EAS_OK
        assert rows(k=None, v=None, **over) == eas.EAS_OK
        assert attend(q=None, out=None, ws=None, **over) == eas.EAS_OK
    assert append(most=0) == rows(most=0) == attend(most_q=0) == eas.EAS_OK
    # no sequences: their arrays may be empty
    assert append(n=0, held=None, pages=None) == attend(n=0, lens=None, pages=None) == rows(n=0, pages=None) == eas.EAS_OK


def workspace(max_q, max_len, n, s=None):
    b = ctypes.c_int64(-1)
    assert eas.LIB.eas_kv8_attention_workspace(ctypes.byref(s or shape()), max_q, max_len, n, ctypes.byref(b)) == 0
    return b.value


def test_workspace_sizes_grow_with_queries_and_tokens_up_to_a_bound():
    assert workspace(1, 64, 3) == 0                        # short: nothing is split
    one = workspace(1, 4000, 1)
    assert one > 0 and workspace(1, 4000, 5) == 5 * one
    assert workspace(1, 1 << 20, 1) >= workspace(1, 9000, 1) >= one
    assert workspace(1 << 20, 1 << 30, 1) == workspace(1 << 21, 1 << 30, 1)
    assert attend(ws_bytes=workspace(1, 4000, 2) - 1) == CAPACITY
    b = ctypes.c_int64()
    call = eas.LIB.eas_kv8_attention_workspace
    assert call(None, 1, 1, 1, ctypes.byref(b)) == BAD
    assert call(ctypes.byref(shape()), -1, 1, 1, ctypes.byref(b)) == BAD
    assert call(ctypes.byref(shape()), 1, 1, 1, None) == BAD
    assert call(ctypes.byref(shape(head_dim=80)), 1, 1, 1, ctypes.byref(b)) == UNSUPPORTED


def test_the_binding_knows_where_no_workspace_is_needed():
    b = ctypes.c_int64(-1)
    for heads, kv_heads in ((1, 1), (28, 4), (1024, 8)):
        s = shape(heads=heads, kv_heads=kv_heads)
        for lq in (1, 100, 128, 1000):
            assert eas.LIB.eas_prompt_attention_workspace(ctypes.byref(s), ints(0, lq), ints(0, A.SPLIT_KEYS - 1), 1,
                                                          ctypes.byref(b)) == 0 and b.value == 0
        for max_q in (1, 7, 300):
            assert workspace(max_q, A.SPLIT_TOKENS, 64, s) == 0


def test_binding_refuses_tensors_of_other_devices_and_kinds():
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises((ValueError, RuntimeError)):        # not on a GPU
        A.prompt_attention(x, x, x, [0, 4])
    k = torch.zeros(3, 2, 16, 64, dtype=torch.int8)
    v, s = torch.zeros(3, 2, 64, 16, dtype=torch.int8), torch.zeros(3, 2)
    A.Kv8Cache(k, v, s, s)
    for bad in ((k.float(), v, s, s), (k, k, s, s), (k, v.to(torch.float8_e4m3fn), s, s), (k, v, s[:2], s),
                (k, v, s, s.double()), (k[0], v, s, s), (k.transpose(1, 2), v, s, s)):
        with pytest.raises(ValueError):
            A.Kv8Cache(*bad)


# ---- the reference ---------------------------------------------------------------

def test_reference_codes_equal_torch_rounding():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.normal(0, 1, 4000) * 2.0 ** rng.integers(-12, 9, 4000), np.arange(-300, 300) / 512.0,
                        O.E4M3, (O.E4M3[1:] + O.E4M3[:-1]) / 2, [448.0, 464.0, -1e9, np.inf, -np.inf, np.nan]])
    x32 = np.clip(x, -448, 448).astype(np.float32)
    want = torch.from_numpy(np.nan_to_num(x32)).to(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(O.encode(np.where(np.isnan(x), x, x32.astype(np.float64)), 1.0, "e4m3"), want)
    want = torch.round(torch.from_numpy(np.nan_to_num(np.clip(x, -127, 127)))).numpy()
    np.testing.assert_array_equal(O.encode(x, 1.0, "int8"), want)
    every = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(O.E4M3, every)


def test_reference_scale_is_the_smallest_that_fits():
    for most in (127.0, 448.0):
        for top in (1e-30, 0.3, 1.0, most, np.nextafter(most, 1e9), most * 2.0 ** 40):
            s = O.scale_of(top, most)
            assert top <= most * s and (top > most * s / 2 or s == 2.0 ** -126)
    assert O.scale_of(0.0, 127.0) == 0.0 and O.scale_of(1e-300, 127.0) == 2.0 ** -126


def test_reference_attention_equals_torch_in_float64():
    rng = np.random.default_rng(1)
    q, k, v = rng.normal(size=(7, 16)), rng.normal(size=(11, 16)), rng.normal(size=(11, 16))
    out, lse = O.attention(q, k, v, 0.3, O.visible(7, 11, True))
    mask = torch.ones(7, 11, dtype=torch.bool).tril(4)
    want = torch.nn.functional.scaled_dot_product_attention(*(torch.from_numpy(x)[None] for x in (q, k, v)),
                                                            attn_mask=mask, scale=0.3)[0].numpy()
    np.testing.assert_allclose(out, want, atol=1e-14)
    s = torch.from_numpy(0.3 * q @ k.T).masked_fill(~mask, -np.inf)
    np.testing.assert_allclose(lse, torch.logsumexp(s, 1).numpy(), atol=1e-13)
    out, lse = O.attention(q, k[:3], v[:3], 0.3, O.visible(7, 3, True))   # the first four see nothing
    assert (out[:4] == 0).all() and (lse[:4] == -np.inf).all() and np.isfinite(lse[4:]).all()


def test_reference_cache_in_pieces_holds_what_it_holds_at_once_where_the_scale_is_set_first():
    rng = np.random.default_rng(2)
    k, v = rng.normal(size=(40, 2, 8)), rng.normal(size=(40, 2, 8))
    k[0::16] = v[0::16] = 3.0       # every page's first token has its largest value
    for form in ("int8", "e4m3"):
        one, many = O.Cache(3, 2, 16, 8, form), O.Cache(3, 2, 16, 8, form)
        one.append(k, v, 0, [2, 0, 1])
        for a, b in ((0, 1), (1, 17), (17, 30), (30, 40)):
            many.append(k[a:b], v[a:b], a, [2, 0, 1])
        for n, x in (("k", k), ("v", v)):
            np.testing.assert_array_equal(one.rows(n, [2, 0, 1], 0, 40), many.rows(n, [2, 0, 1], 0, 40))
            err = np.abs(one.rows(n, [2, 0, 1], 0, 40) - x)
            s = np.repeat(one.scale[n][[2, 0, 1]], 16, axis=0)[:40, :, None]
            assert (err <= (0.5 * s if form == "int8" else np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * s))).all()
