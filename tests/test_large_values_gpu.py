"""Values near the largest that bf16 holds: a result is a mean of values, so it is finite wherever they are, whichever kernel
takes the sequence and in however many runs.  What is held on the way are sums of weighted values, over all tokens of a run
and over all runs.

Tolerances.  Equal values c of a dimension: the weights are rounded to the element type, their sum is not, so the result is
off by half a step of a weight and half a step of its own, 2 * 2^-8, and by what fp32 adds over n tokens, n * 2^-24 at most
and 2^-12 here.  Others: as in test_paged_large_gpu.py, whose bounds grow with the values."""
import numpy as np
import pytest

from test_attention_gpu import make
from test_paged_gpu import i32, lib
from test_paged_large_gpu import check_on_gpu, random_cache

pytestmark = pytest.mark.gpu

TOL = 2.0 ** -7 + 2.0 ** -12


def columns(torch, dim, size=2.0 ** 127):
    want = torch.full((dim,), size, device="cuda")
    want[::2] *= -1.0
    return want


# (new tokens, tokens): whole and in runs, of the kernel for few rows of a key head and of that for many
FEW = [(1, 1023), (1, 32768), (3, 70000), (5, 3000)]
MANY = [(40, 70), (70, 70), (300, 700), (1024, 5000), (64, 4096), (300, 33000)]


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,length", FEW + MANY)
def test_paged_attention_of_equal_values(new, length, dim):
    torch, _ = lib()
    cache, table = random_cache("bfloat16", [length], 128, 1, dim, 400)
    want = columns(torch, dim)
    cache.v.copy_(want.to(torch.bfloat16))
    for size in (0.0, 1.0):   # equal scores, and others
        q = make(torch, (new, 4, dim), torch.bfloat16, 401, size)
        for causal in (True, False):
            out, _ = cache.attention(q, i32(torch, [length]), i32(torch, table), causal=causal)
            assert ((out.double() / want.double() - 1).abs() <= TOL).all(), (size, causal)


@pytest.mark.parametrize("new,length", FEW + MANY)
def test_paged_attention_of_large_values(new, length):
    """Random ones, of up to 2^128 (5.6 deviations), and what is hidden among them."""
    torch, _ = lib()
    cache, table = random_cache("bfloat16", [length], 64, 1, 64, 410)
    cache.v.copy_((cache.v.float().clamp(-5, 5) * 2.0 ** 125).to(torch.bfloat16))
    q = make(torch, (new, 4, 64), torch.bfloat16, 411)
    out, lse = cache.attention(q, i32(torch, [length]), i32(torch, table), with_lse=True)
    assert torch.isfinite(out).all()
    check_on_gpu(cache, q, [length], table, [new], out, lse, [0])


@pytest.mark.parametrize("new", [1, 40, 300])
def test_the_size_of_values_does_not_change_what_is_made_of_them(new):
    """Powers of two apart, results are powers of two apart, bit for bit, as long as no sum leaves fp32's range."""
    torch, _ = lib()
    cache, table = random_cache("bfloat16", [9000], 64, 2, 64, 420)
    q = make(torch, (new, 8, 64), torch.bfloat16, 421)
    t, n = i32(torch, table), i32(torch, [9000])
    want, want_lse = cache.attention(q, n, t, with_lse=True)
    for power in (-60, 40, 100):
        cache.v.mul_(2.0 ** power)
        out, lse = cache.attention(q, n, t, with_lse=True)
        cache.v.mul_(2.0 ** -power)
        assert torch.equal(out.double(), want.double() * 2.0 ** power) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("queries,keys", [(1, 500), (300, 300), (700, 700), (64, 5000), (1, 70000), (300, 33000), (2000, 2000)])
@pytest.mark.parametrize("dim", [64, 128])
def test_causal_prompt_attention_of_equal_values(queries, keys, dim):
    torch, _ = lib()
    from paper_2609_31551_amd import attention as A
    want = columns(torch, dim)
    k = make(torch, (keys, 1, dim), torch.bfloat16, 430)
    v = want.to(torch.bfloat16).expand(keys, 1, dim).contiguous()
    for size in (0.0, 1.0):
        q = make(torch, (queries, 4, dim), torch.bfloat16, 431, size)
        out, _ = A.prompt_attention(q, k, v, [0, queries], [0, keys])
        assert ((out.double() / want.double() - 1).abs() <= TOL).all(), size
