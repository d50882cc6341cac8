"""Pages that are not held: a sequence's result is its own tokens', to the bit, whatever any page of the cache holds that is
none of its own."""
import numpy as np
import pytest

from test_attention_gpu import make
from test_paged_gpu import i32, lib
from test_paged_large_gpu import random_cache

pytestmark = pytest.mark.gpu

FILL = [0.0, float("nan"), float("inf"), -float("inf"), 3e38, 1.0]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("new", [[1], [6], [30], [150], [1, 5, 140], [1500, 1, 900]], ids=str)
@pytest.mark.parametrize("dtype,dim", [("bfloat16", 64), ("float16", 128), ("bfloat16", 128)])
def test_what_other_pages_hold_does_not_matter(dtype, dim, new, page, causal):
    torch, B = lib()
    lens = [n + x for n, x in zip(new, (700, 1300, 260))]
    cache, table = random_cache(dtype, lens, page, 2, dim, 500)
    k, v = cache.k.clone(), cache.v.clone()
    heads = 64 if sum(new) > 1000 else 8                # 256 rows a workgroup, and 128
    q = make(torch, (sum(new), heads, dim), getattr(torch, dtype), 501)
    rng = np.random.default_rng(502)
    gone = np.where(rng.random(table.shape) < 0.4, rng.choice([-1, 1 << 30, cache.n_pages], table.shape), table)
    gone[0, 0], gone[:, 1] = -1, table[:, 1]
    mine = np.unique(gone[(gone >= 0) & (gone < cache.n_pages)])
    others = torch.tensor(np.setdiff1d(np.arange(cache.n_pages), mine), device="cuda")
    # page 0 among the others: the tokens of the sequence's page 0 are moved elsewhere
    if 0 in mine:
        at = int(others[0])
        k[at], v[at] = k[0], v[0]
        gone[gone == 0] = at
        others = torch.cat([others[1:], others.new_zeros(1)])
    c = i32(torch, np.cumsum([0] + new))
    want = None
    for fill in FILL:
        cache.k.copy_(k), cache.v.copy_(v)
        cache.k[others], cache.v[others] = fill, fill
        out, lse = cache.attention(q, i32(torch, lens), i32(torch, gone), c, max(new), max(lens), causal=causal, with_lse=True)
        assert torch.isfinite(out).all()
        if want is None:
            want = out, lse
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]), fill


@pytest.mark.parametrize("new", [1, 40, 600])
def test_no_page_is_held(new):
    """Zeros and -inf, whatever page 0 holds."""
    torch, _ = lib()
    cache, table = random_cache("bfloat16", [2000], 32, 1, 64, 510)
    cache.k.fill_(float("nan"))
    cache.v.fill_(float("nan"))
    q = make(torch, (new, 4, 64), torch.bfloat16, 511)
    out, lse = cache.attention(q, i32(torch, [2000]), torch.full_like(i32(torch, table), -1), with_lse=True)
    assert (out == 0).all() and torch.isneginf(lse).all()
