"""Keys whose score is -inf -- a dimension that holds -inf, or products that overflow -- weigh nothing, wherever they
stand: the result is that of the other keys alone.  Tolerances as in test_attention_gpu.py."""
import numpy as np
import pytest

from oracle import attention as O
from test_attention_gpu import HALF, check, cu, f64, i32, lib, make, prompt_bounds, run_prompt

pytestmark = pytest.mark.gpu


def inputs(torch, dtype, dim, lq, lk, masked, low, what):
    """Queries with 1 in their first dimension; keys with -low there, or with what makes the score -inf."""
    dt = getattr(torch, dtype)
    q = make(torch, (lq, 2, dim), dt, 1)
    k, v = make(torch, (lk, 1, dim), dt, 2, 0.1), make(torch, (lk, 1, dim), dt, 3)
    one = 4.0 if what == "overflow" else 1.0
    q[:, :, 0] = one
    k[:, :, 0] = -low / one
    k[masked, :, 0] = -3e38 if what == "overflow" else -np.inf
    return q, k, v


def compare(torch, q, k, v, masked, causal):
    """Against the reference over the keys that are not masked; the queries are the last tokens either way."""
    lq, lk = q.shape[0], k.shape[0]
    out, lse = run_prompt(q, k, v, [0, lq], [0, lk], causal, 1.0, check_bounds=False)
    keep = np.delete(np.arange(lk), masked)
    Q, K, V = f64(q), f64(k)[keep], f64(v)[keep]
    cu_q, cu_k = [0, lq], [0, len(keep)]
    if causal:   # queries before the masked keys' end see fewer of the others than the shift of the end says
        assert masked.stop <= lk - lq + 1 or masked.start == 0
    ref, ref_lse = O.prompt_attention(Q, K, V, cu_q, cu_k, 1.0, causal)
    u = HALF[str(q.dtype)[6:]]
    size, delta, total, count = prompt_bounds(Q, K, V, cu_q, cu_k, 1.0, causal, u)
    check(f64(out), f64(lse), ref, ref_lse, size, delta, total, count, u, 2.0 ** -32 if q.dtype == torch.float16 else 0.0)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n", [64, 128, 4096])
@pytest.mark.parametrize("low", [16.0, 20.0, 100.0])
@pytest.mark.parametrize("dtype,dim,what", [("bfloat16", 128, "inf"), ("float16", 128, "inf"), ("float16", 64, "inf"),
                                            ("bfloat16", 64, "overflow")])
def test_masked_prefix(dtype, dim, what, low, n, causal):
    torch, _ = lib()
    print("[prompt] %d keys of score -inf, %s" % (n, dtype), flush=True)
    compare(torch, *inputs(torch, dtype, dim, 40, n + 200, slice(0, n), low, what), slice(0, n), causal)


@pytest.mark.parametrize("low", [16.0, 100.0])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_masked_keys_at_the_start_of_a_later_run(dtype, low):
    """9,000 keys in 8 runs of 18 tiles: the second begins at key 1,152."""
    torch, _ = lib()
    compare(torch, *inputs(torch, dtype, 128, 20, 9000, slice(1100, 1400), low, "inf"), slice(1100, 1400), True)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_queries_that_see_only_masked_keys(dtype):
    torch, _ = lib()
    q, k, v = inputs(torch, dtype, 64, 150, 150, slice(0, 70), 20.0, "inf")
    compare(torch, q, k, v, slice(0, 70), True)
    out, lse = run_prompt(q, k, v, [0, 150], None, True, 1.0, check_bounds=False)
    assert (out[:70] == 0).all() and torch.isneginf(lse[:70]).all()


@pytest.mark.parametrize("what", ["inf", "-inf"])
def test_infinite_queries(what):
    """A query with an infinite dimension: keys of one sign there weigh nothing where the score is -inf; any +inf makes
    the result NaN, and no other query's."""
    torch, A = lib()
    q = make(torch, (70, 2, 64), torch.bfloat16, 11)
    k, v = make(torch, (70, 1, 64), torch.bfloat16, 12), make(torch, (70, 1, 64), torch.bfloat16, 13)
    k[:, :, 3] = k[:, :, 3].abs() + 0.1
    want, want_lse = A.prompt_attention(q, k, v, [0, 70], causal=False, with_lse=True)
    q2 = q.clone()
    q2[20, :, 3] = float(what)
    got, lse = A.prompt_attention(q2, k, v, [0, 70], causal=False, with_lse=True)
    others = [i for i in range(70) if i != 20]
    assert torch.equal(got[others], want[others]) and torch.equal(lse[others], want_lse[others])
    if what == "inf":
        assert torch.isnan(got[20]).all() and torch.isnan(lse[20]).all()
    else:
        assert (got[20] == 0).all() and torch.isneginf(lse[20]).all()


@pytest.mark.parametrize("form", ["int8", "e4m3"])
def test_infinite_queries_over_the_cache(form):
    torch, A = lib()
    cache = A.Kv8Cache.empty(8, 1, 64, 16, torch.int8 if form == "int8" else torch.float8_e4m3fn)
    k, v = make(torch, (100, 1, 64), torch.float16, 14), make(torch, (100, 1, 64), torch.float16, 15)
    k[:, :, 3] = k[:, :, 3].abs() + 1.0      # no code 0
    pages = i32(torch, [list(range(8))])
    cache.append(k, v, i32(torch, [0]), pages)
    q = make(torch, (3, 2, 64), torch.float16, 16)
    want, want_lse = cache.attention(q, i32(torch, [100]), pages, causal=False, with_lse=True)
    q[0, :, 3], q[2, :, 3] = float("inf"), float("-inf")
    got, lse = cache.attention(q, i32(torch, [100]), pages, causal=False, with_lse=True)
    assert torch.equal(got[1], want[1]) and torch.equal(lse[1], want_lse[1])
    assert torch.isnan(got[0]).all() and torch.isnan(lse[0]).all()
    assert (got[2] == 0).all() and torch.isneginf(lse[2]).all()
