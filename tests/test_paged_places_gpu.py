"""Mixed batches whose bounds allow far more than there is: how many workgroups are launched for chunks goes by the rows that
there are, as only sequences with many of them have one.  Too many would be slow, and more than a launch holds refused."""
import numpy as np
import pytest

from test_attention_gpu import cu, make
from test_paged_gpu import i32, lib
from test_paged_large_gpu import check_on_gpu, random_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv_heads,dim", [(16, 16, 64), (28, 4, 128), (40, 1, 64)])
@pytest.mark.parametrize("chunks", [(512,), (33, 34, 40, 8), (300, 2, 1, 1200)], ids=str)
def test_far_bounds_of_mixed_batches(heads, kv_heads, dim, chunks):
    """Chunks at the ends and between, down to the fewest rows that are many: as with bounds that fit, bit for bit."""
    torch, _ = lib()
    new = [1] * 90
    for i, n in enumerate(chunks):
        new[(i * 89 // max(1, len(chunks) - 1))] = n
    rng = np.random.default_rng(600)
    lens = [n + int(x) for n, x in zip(new, rng.choice([0, 40, 700, 1500, 2500], 90))]
    cache, table = random_cache("bfloat16", lens, 64, kv_heads, dim, 601)
    far = np.full((90, 2048), -1)                                   # 131,072 tokens
    far[:, :table.shape[1]] = table
    q = make(torch, (sum(new), heads, dim), torch.bfloat16, 602)
    n, c = i32(torch, lens), i32(torch, cu(new))
    want = cache.attention(q, n, i32(torch, table), c, max(new), max(lens), with_lse=True)
    got = cache.attention(q, n, i32(torch, far), c, max(new), with_lse=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    check_on_gpu(cache, q, lens, table, new, *got, [r for r in range(90) if new[r] > 1 or r % 20 == 0])


@pytest.mark.parametrize("first,rows", [(-20, 130), (-60, 75), (5, 110)])
def test_sequences_cut_at_both_ends_of_the_rows(first, rows):
    """Prefix sums that begin before the rows and end behind them: what lies in the rows is computed, and nothing else."""
    torch, _ = lib()
    new = [40, 1, 70, 1, 60]
    lens = [n + 50 for n in new]
    cache, table = random_cache("float16", lens, 16, 2, 64, 610)
    c = np.array(cu(new)) + first
    whole = make(torch, (c[-1] - min(first, 0) + 10, 2, 64), torch.float16, 611)
    want = cache.attention(whole, i32(torch, lens), i32(torch, table), i32(torch, c - min(first, 0)), 70)[0]
    before = max(-first, 0)
    out = torch.full((rows, 2, 64), 7.0, dtype=torch.float16, device="cuda")
    cache.attention(whole[before:before + rows], i32(torch, lens), i32(torch, table), i32(torch, c), 70, out=out)
    a, b = max(first, 0), min(rows, int(c[-1]))
    assert (out[:a] == 7.0).all() and (out[b:] == 7.0).all()
    # a sequence that is cut has fewer rows, whose tokens are the same
    assert ((out[a:b].double() - want[a + before:b + before].double()).abs() <= 2.0 ** -9 * 8).all()


def test_a_batch_of_8200_sequences_of_1024_heads():
    """One of 40 tokens among them: as in parts, bit for bit."""
    torch, B = lib()
    n, heads = 8200, 1024
    new = np.ones(n, np.int64)
    new[n // 2] = 40
    rng = np.random.default_rng(620)
    cache = B.Kv16Cache.empty(4, heads, 64, 16)
    for x, seed in ((cache.k, 621), (cache.v, 622)):
        x.copy_(make(torch, x.shape, torch.bfloat16, seed))
    table = np.argsort(rng.random((n, 4)), 1)[:, :3]                 # shared for reading
    lens = i32(torch, rng.integers(1, 48, n).clip(new))
    table = i32(torch, table)
    q = make(torch, (int(new.sum()), heads, 64), torch.bfloat16, 623)
    out, _ = cache.attention(q, lens, table, i32(torch, cu(new)), 40)
    c = cu(new)
    for a, b in ((0, 3000), (3000, 6000), (6000, n)):
        part, _ = cache.attention(q[c[a]:c[b]], lens[a:b], table[a:b], i32(torch, cu(new[a:b])), 40)
        assert torch.equal(part, out[c[a]:c[b]])


def test_prefix_sums_that_decrease_end():
    """What the rows get is open then; nothing else is written, and no sum of the pieces of work wraps, of which these 27,000
    sequences of 20,000 queries and of less than none count 2 * 10^9."""
    torch, B = lib()
    n, rows, heads = 27000, 20000, 1024
    assert (n // 2) * (rows * heads // 128) > 1 << 31
    cache = B.Kv16Cache.empty(4, 1, 64, 16)
    cache.k.fill_(1.0)
    cache.v.fill_(2.0)
    out = torch.full((rows + 8, heads, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((rows + 8, heads), 7.0, device="cuda")
    q = make(torch, (1, 1, 64), torch.bfloat16, 630).expand(rows, heads, 64)
    lens, table = i32(torch, np.full(n, 40)), i32(torch, np.tile([0, 1, 2, 3], (n, 1)))
    print("[decreasing] %d sequences" % n, flush=True)
    cache.attention(q, lens, table, i32(torch, np.arange(n + 1) % 2 * rows), rows, causal=False, out=out[4:-4], lse=lse[4:-4])
    torch.cuda.synchronize()
    for x in (out, lse):
        assert (x[:4] == 7.0).all() and (x[-4:] == 7.0).all()
    assert ((out[4:-4] == 2.0) | (out[4:-4] == 7.0)).all()           # all values are 2: what is computed is
    # a batch as it should be, behind it
    c = i32(torch, [0, 5, 5, 45])
    one, _ = cache.attention(q[:45, :8], lens[:3], table[:3], c, 40, causal=False)
    assert (one == 2.0).all()
