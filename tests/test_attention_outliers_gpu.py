"""Queries with one value far above the others, over the 8-bit cache: values are taken to fp16 relative to the row's
largest, so each is good to 2^-39 of it, and a score to scale * 2^-39 * largest * sum |k|."""
import numpy as np
import pytest

from oracle import attention as O
from test_attention_gpu import FORMATS, HALF, Both, f64, i32, lib, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("dtype,top", [("bfloat16", 2.0 ** 20), ("bfloat16", 1.5 * 2.0 ** 26), ("bfloat16", 2.0 ** 33),
                                       ("float16", 40000.0)])
def test_a_channel_far_above_the_others(form, dtype, top):
    torch, A = lib()
    n, dim, dt = 600, 128, getattr(torch, dtype)
    both = Both(form, 10, 1, 64, dim)
    k, v = make(torch, (n, 1, dim), torch.bfloat16, 1), make(torch, (n, 1, dim), torch.bfloat16, 2)
    k[:, :, 5] = 0.0                                   # the channel itself does not count
    table = np.arange(10)[None]
    both.append(k, v, [0, n], [0], table)
    q = make(torch, (4, 2, dim), dt, 3)
    q[:, :, 5] = top
    scale = dim ** -0.5
    out, lse = both.gpu.attention(q, i32(torch, [n]), i32(torch, table), scale=scale, causal=False, with_lse=True)
    K, V, Q = both.ref.rows("k", table[0], 0, n)[:, 0], both.ref.rows("v", table[0], 0, n)[:, 0], f64(q)
    for h in range(2):
        ref, ref_lse = O.attention(Q[:, h], K, V, scale, np.ones((4, n), bool))
        size, _ = O.attention(Q[:, h], K, np.abs(V), scale, np.ones((4, n), bool))
        rest = np.linalg.norm(np.delete(Q[:, h], 5, 1), axis=1)
        # the values' rounding, and fp32 sums of the other channels' products
        error = scale * (2.0 ** -39 * top * np.abs(K).sum(1).max() + (dim + 2) * 2.0 ** -24 * rest * np.linalg.norm(K, axis=1).max())
        most = both.ref.scale["v"].max() * O.MOST[form] * n
        growth = np.expm1(2 * error)[:, None]          # of a weight's share, both ways
        tol = HALF[dtype] * np.abs(ref) + (2.0 ** -11 + 2.0 ** -21 + growth) * size + 2.0 ** -40 * most + 2.0 ** -25
        print("[kv8] one channel at %g: scores good to %.2g, worst %.3g of the tolerance" % (
            top, error.max(), (np.abs(f64(out)[:, h] - ref) / tol).max()), flush=True)
        assert (np.abs(f64(out)[:, h] - ref) <= tol).all()
        assert (np.abs(f64(lse)[:, h] - ref_lse) <= error + 2.0 ** -21 * (1 + np.abs(ref_lse)) + n * 2.0 ** -24).all()
