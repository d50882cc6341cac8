"""Rows that NaN or infinities in hidden tokens send on the careful way: right to the same bounds as others (see
test_attention_gpu.py), and not a walk key by key."""
import numpy as np
import pytest

from oracle import attention as O
from test_attention_gpu import HALF, check, f64, lib, make, prompt_bounds

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("what", ["nan", "inf", "-inf"])
@pytest.mark.parametrize("lq,lk,at", [(33, 33, 32), (200, 200, 130), (90, 90, 64), (129, 700, 600), (64, 2500, 2440),
                                      (300, 130, 90), (40, 4200, 4170)])
@pytest.mark.parametrize("dtype,dim", [("bfloat16", 64), ("bfloat16", 128), ("float16", 64), ("float16", 128)])
def test_hidden_tokens_against_float64(dtype, dim, lq, lk, at, what):
    """The tokens from `at` on hold NaN or infinities: earlier queries against the reference."""
    torch, A = lib()
    dt = getattr(torch, dtype)
    q, k, v = make(torch, (lq, 4, dim), dt, 1), make(torch, (lk, 2, dim), dt, 2, 2.0), make(torch, (lk, 2, dim), dt, 3)
    first = at - (lk - lq)                       # the first query that sees one
    assert 0 < first < lq
    ref, ref_lse = O.prompt_attention(f64(q), f64(k), f64(v), [0, lq], [0, lk], dim ** -0.5, True)
    u = HALF[dtype]
    size, delta, total, count = prompt_bounds(f64(q), f64(k), f64(v), [0, lq], [0, lk], dim ** -0.5, True, u)
    k[at:, :, 3], v[at:, :, 5] = float(what), float(what)
    out, lse = A.prompt_attention(q, k, v, [0, lq], [0, lk], with_lse=True)
    s = slice(0, first)
    check(f64(out)[s], f64(lse)[s], ref[s], ref_lse[s], size[s], delta[s], total[s], count[s], u,
          2.0 ** -32 if dt == torch.float16 else 0.0)
    assert not torch.isfinite(out[first:, :, 5]).any()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_small_weights_count_on_the_careful_way(dtype, dim):
    """4,095 keys of 2^-25.3 of the first key's weight each, whose value is 0, and a hidden NaN behind them."""
    torch, A = lib()
    n, dt = 4096, getattr(torch, dtype)
    k, v = torch.zeros(n, 1, dim, dtype=dt, device="cuda"), torch.ones(n, 1, dim, dtype=dt, device="cuda")
    k[0], v[0] = 16.0, 0.0
    q = torch.zeros(40, 1, dim, dtype=dt, device="cuda")
    q[:, :, 0] = 1.0
    scale = float(np.float32(25.3 * np.log(2.0) / 16))
    ref, ref_lse = O.prompt_attention(f64(q), f64(k), f64(v), [0, 40], [0, n], scale, True)
    size, delta, total, count = prompt_bounds(f64(q), f64(k), f64(v), [0, 40], [0, n], scale, True, HALF[dtype])
    v[n - 1] = float("nan")
    out, lse = A.prompt_attention(q, k, v, [0, 40], [0, n], scale=scale, with_lse=True)
    s = slice(0, 39)
    check(f64(out)[s], f64(lse)[s], ref[s], ref_lse[s], size[s], delta[s], total[s], count[s], HALF[dtype],
          2.0 ** -32 if dt == torch.float16 else 0.0)


def test_a_nan_does_not_make_a_call_hundreds_of_times_longer():
    """2,048 tokens, 8 heads: 6 times the time of a call without (key by key it was over 200 times)."""
    torch, A = lib()
    q, k, v = (make(torch, (2048, h, 128), torch.bfloat16, 10 + h) for h in (8, 4, 4))

    def ms(k, v):
        best = []
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            A.prompt_attention(q, k, v, [0, 2048])
            b.record()
            b.synchronize()
            best.append(a.elapsed_time(b))
        return min(best)
    plain = ms(k, v)
    for x in ("k", "v"):
        k2, v2 = k.clone(), v.clone()
        (k2 if x == "k" else v2)[0, :, 3] = float("nan")
        assert ms(k2, v2) < 60 * plain
