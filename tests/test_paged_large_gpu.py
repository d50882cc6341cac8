"""Prompts in pieces at sizes that small tests do not reach: 256 rows a workgroup, batches whose runs are joined by rows,
sequences in many runs, strides and offsets past 32 bits, large values, a page table that changes between replays.
References in float64 on the GPU; bounds as in test_paged_gpu.py."""
import numpy as np
import pytest

from test_attention_gpu import HALF, cu, make
from test_paged_gpu import i32, lib, pages_of

pytestmark = pytest.mark.gpu


def random_cache(dtype, lens, page, heads, dim, seed):
    """A cache full of noise and the page table of sequences of `lens` tokens."""
    torch, B = lib()
    table, n_pages = pages_of(lens, page, seed, extra=1)
    dt = getattr(torch, dtype)
    k, v = make(torch, (n_pages, heads, page, dim), dt, seed, 2.0), make(torch, (n_pages, heads, page, dim), dt, seed + 1)
    return B.Kv16Cache(k, v), table


def check_on_gpu(cache, q, lens, table, new, out, lse, only):
    """Sequences `only` against float64 (causal)."""
    torch, _ = lib()
    c, u = cu(new), HALF[str(q.dtype)[6:]]
    dim, group = q.shape[2], q.shape[1] // cache.kv_heads
    for r in only:
        a, n = slice(c[r], c[r + 1]), lens[r]
        where = torch.tensor(table[r][:-(-n // cache.page_tokens)], device="cuda")
        i, j = torch.arange(new[r], device="cuda")[:, None], torch.arange(n, device="cuda")[None]
        hidden = j > i + (n - new[r])
        for h in range(q.shape[1]):
            k = cache.k[where, h // group].reshape(-1, dim)[:n].double()
            v = cache.v[where, h // group].reshape(-1, dim)[:n].double()
            x = q[a, h].double()
            s = (x @ k.t().contiguous() * dim ** -0.5).masked_fill(hidden, -np.inf)
            want_lse = torch.logsumexp(s, 1)
            p = torch.exp(s - want_lse[:, None])
            want, size = p @ v, p @ v.abs()
            delta = (dim * 2.0 ** -24 * dim ** -0.5 * x.norm(dim=1) * k.norm(dim=1).max())[:, None]
            tol = u * (want.abs() + size) + (2 * delta + 2.0 ** -21) * size + 2.0 ** -25
            if q.dtype == torch.float16:
                tol = tol + 2.0 ** -32 * v.abs().sum(0)
            assert ((out[a, h].double() - want).abs() <= tol).all(), (r, h)
            ltol = delta[:, 0] + 2.0 ** -21 * (1 + want_lse.abs()) + n * 2.0 ** -24
            assert ((lse[a, h].double() - want_lse).abs() <= ltol).all(), (r, h)


@pytest.mark.parametrize("dtype,heads,kv_heads,dim", [("bfloat16", 32, 4, 128), ("float16", 32, 8, 64)])
def test_wide_workgroups_beside_single_tokens(dtype, heads, kv_heads, dim):
    """Enough rows for 256 a workgroup, alone and beside single tokens: against float64, and bit for bit what the sequences
    give alone."""
    torch, B = lib()
    new, lens = [1500, 1, 1333, 1, 800], [1500, 700, 2000, 2500, 801]
    cache, table = random_cache(dtype, lens, 32, kv_heads, dim, 300)
    q = make(torch, (sum(new), heads, dim), getattr(torch, dtype), 301)
    assert sum(new) * heads >= 256 * 256 and sum(new) * heads // kv_heads >= 1024 * len(new)
    print("[wide] %s" % dtype, flush=True)
    out, lse = cache.attention(q, i32(torch, lens), i32(torch, table), i32(torch, cu(new)), max(new), max(lens), with_lse=True)
    check_on_gpu(cache, q, lens, table, new, out, lse, range(5))
    c = cu(new)
    for r in range(5):
        a = slice(c[r], c[r + 1])
        one, one_lse = cache.attention(q[a], i32(torch, lens[r:r + 1]), i32(torch, table[r:r + 1]), with_lse=True)
        assert torch.equal(one, out[a]) and torch.equal(one_lse, lse[a]), r


def test_runs_of_large_batches_are_joined_by_rows():
    """Sequences in runs beside others that are not split, few rows and many, more than 64 of them."""
    torch, B = lib()
    rng = np.random.default_rng(310)
    new = [int(x) for x in rng.choice([1, 1, 2, 60, 200], 70)]
    lens = [n + int(x) for n, x in zip(new, rng.choice([10, 900, 1100, 2300, 5000], 70))]
    cache, table = random_cache("bfloat16", lens, 64, 2, 64, 311)
    q = make(torch, (sum(new), 16, 64), torch.bfloat16, 312)
    out, lse = cache.attention(q, i32(torch, lens), i32(torch, table), i32(torch, cu(new)), max(new), max(lens), with_lse=True)
    check_on_gpu(cache, q, lens, table, new, out, lse, range(0, 70, 3))
    c = cu(new)
    for r in range(0, 70, 7):
        a = slice(c[r], c[r + 1])
        one, one_lse = cache.attention(q[a], i32(torch, lens[r:r + 1]), i32(torch, table[r:r + 1]), with_lse=True)
        assert torch.equal(one, out[a]) and torch.equal(one_lse, lse[a]), r


@pytest.mark.parametrize("new,length", [(1, 150001), (3, 70000), (20, 40000), (300, 33000)])
@pytest.mark.parametrize("dtype,dim", [("bfloat16", 128), ("float16", 64)])
def test_long_sequences(dtype, dim, new, length):
    """The most runs, and runs of many tiles."""
    torch, B = lib()
    cache, table = random_cache(dtype, [length], 128, 1, dim, 320)
    q = make(torch, (new, 4, dim), getattr(torch, dtype), 321)
    out, lse = cache.attention(q, i32(torch, [length]), i32(torch, table), with_lse=True)
    check_on_gpu(cache, q, [length], table, [new], out, lse, [0])


def test_large_values_do_not_overflow():
    """Values up to 2^122: weighted sums of 70 to 500 of them are finite where the weights' sum is not taken first."""
    torch, B = lib()
    for new, length in ((1, 500), (1, 3000), (40, 70), (70, 70)):
        cache, table = random_cache("bfloat16", [length], 16, 2, 64, 330)
        cache.v.fill_(2.0 ** 120)
        cache.v[..., ::2] *= -4.0
        q = make(torch, (new, 4, 64), torch.bfloat16, 331)
        out, lse = cache.attention(q, i32(torch, [length]), i32(torch, table), with_lse=True)
        want = torch.full((64,), 2.0 ** 120, device="cuda")
        want[::2] *= -4.0
        # weights that sum to 1 up to a half step each, and the result's own rounding
        assert ((out.float() - want).abs() <= 2.0 ** -6.9 * want.abs()).all(), (new, length)


def test_strides_past_32_bits():
    """Rows 2^23 values apart: 300 of them over 5 GB."""
    torch, B = lib()
    rows, step = 300, 1 << 23
    big = torch.empty(rows * step, dtype=torch.bfloat16, device="cuda")
    far = big.as_strided((rows, 5, 64), (step, 64, 1))
    x = make(torch, (rows, 5, 64), torch.bfloat16, 340)
    far.copy_(x)
    rot = B.Rotary.sections((8, 12, 12))
    pos = i32(torch, np.random.default_rng(0).integers(0, 9000, (3, rows)))
    q, k, v = (slice(0, 2), slice(2, 3), slice(3, 4))
    want = rot.rows(x[:, q], pos, x[:, k])
    got = rot.rows(far[:, q], pos, far[:, k])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    rot.rows(far[:, q], pos, q_out=far[:, q])
    assert torch.equal(far[:, q], want[0])
    far.copy_(x)
    caches = []
    for t in (x, far):
        c = B.Kv16Cache.empty(20, 1, 64, 16)
        table = i32(torch, [list(range(19, -1, -1))])
        out = c.append(t[:, k], t[:, v], i32(torch, [5]), table, rotary=rot, positions=pos, q=t[:, q])
        c.k[table[0, 0].long(), :, :5], c.v[table[0, 0].long(), :, :5] = 1.0, 1.0
        result = c.attention(t[:, q], i32(torch, [305]), table, out=far[:, q] if t is far else None, with_lse=True)
        caches.append((out, *result, c.k[1:], c.v[1:]))
    assert all(torch.equal(a, b) for a, b in zip(*caches))


def test_a_page_table_that_changes_between_replays():
    """Lengths, page tables and prefix sums are read when the kernels run: single tokens and chunks, split and not."""
    torch, B = lib()
    lens = [[1500, 40, 900], [300, 1300, 2000], [2048, 1, 1025]]
    news = [[1, 40, 100], [90, 1, 60], [150, 1, 1]]
    cache, whole = random_cache("bfloat16", [2048] * 3, 32, 2, 128, 350)
    rng = np.random.default_rng(351)
    n, c, t = i32(torch, lens[0]), i32(torch, cu(news[0])), i32(torch, whole)
    q = make(torch, (160, 8, 128), torch.bfloat16, 352)

    def call():
        return cache.attention(q, n, t, c, 150, 2048, with_lse=True)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = call()
    for i in (1, 2, 0, 1):
        n.copy_(i32(torch, lens[i]))
        c.copy_(i32(torch, cu(news[i])))
        t.copy_(i32(torch, whole[rng.permutation(3)][:, rng.permutation(whole.shape[1])]))
        graph.replay()
        want, want_lse = call()
        torch.cuda.synchronize()
        rows = sum(news[i])
        assert torch.equal(out[:rows], want[:rows]) and torch.equal(lse[:rows], want_lse[:rows])
        check_on_gpu(cache, q, lens[i], t.cpu().numpy(), news[i], out, lse, range(3))


@pytest.mark.parametrize("mixed", [False, True])
def test_bounds_far_above_the_lengths(mixed):
    """A page table and max_len for 65,536 tokens: as with bounds that fit, bit for bit; fewer workgroups than places."""
    torch, B = lib()
    rng = np.random.default_rng(360)
    new = [int(x) for x in rng.choice([1, 1, 3, 80] if mixed else [1, 2], 150)]
    lens = [n + int(x) for n, x in zip(new, rng.choice([0, 60, 900, 1500, 2600], 150))]
    cache, table = random_cache("bfloat16", lens, 16, 2, 64, 361)
    far = np.full((150, 4096), -1)
    far[:, :table.shape[1]] = table
    q = make(torch, (sum(new), 8, 64), torch.bfloat16, 362)
    n, c = i32(torch, lens), i32(torch, cu(new))
    want = cache.attention(q, n, i32(torch, table), c, max(new), max(lens), with_lse=True)
    got = cache.attention(q, n, i32(torch, far), c, max(new), with_lse=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    check_on_gpu(cache, q, lens, table, new, *got, range(0, 150, 9))


def test_more_runs_than_workgroups():
    """300 sequences of 8 key heads in three runs each: workgroups take several."""
    torch, B = lib()
    lens = [1100 + 3 * i % 400 for i in range(300)]
    cache, table = random_cache("float16", lens, 64, 8, 64, 370)
    q = make(torch, (300, 16, 64), torch.float16, 371)
    n, t = i32(torch, lens), i32(torch, table)
    out, lse = cache.attention(q, n, t, with_lse=True)
    check_on_gpu(cache, q, lens, table, [1] * 300, out, lse, range(0, 300, 23))
    for r in (0, 150, 299):
        one, one_lse = cache.attention(q[r:r + 1], n[r:r + 1], t[r:r + 1].contiguous(), with_lse=True)
        assert torch.equal(one, out[r:r + 1]) and torch.equal(one_lse, lse[r:r + 1])


@pytest.mark.parametrize("kind,n", [("wide", 65), ("wide", 130)] + [(k, n) for k in ("tokens", "guesses", "mixed")
                                                                    for n in (65, 129, 577, 1100)])
def test_waves_share_the_lengths_of_many_sequences(kind, n):
    """More sequences than a wave has lanes, split ones at the ends and between, in each kind of launch: the last lane's
    share, lanes without any, and results that are those of the sequence alone, bit for bit."""
    torch, B = lib()
    rng = np.random.default_rng(n)
    new = [int(x) for x in {"tokens": rng.choice([1], n), "guesses": rng.choice([0, 1, 3], n),
                            "mixed": rng.choice([0, 1, 1, 30], n), "wide": rng.choice([0, 1, 1, 3], n)}[kind]]
    lens = [x + int(y) for x, y in zip(new, rng.choice([0, 5, 90], n))]
    split = [0, 1, 63, 64, n // 2, n - 2, n - 1]
    for i, r in enumerate(split):
        new[r] = {"tokens": 1, "guesses": 1 + i % 3, "mixed": (1, 40, 200)[i % 3], "wide": 1 if i % 2 else 50 * n}[kind]
        lens[r] = new[r] + 1500 + 100 * i
    cache, table = random_cache("bfloat16", lens, 64, 2, 64, 380)
    q = make(torch, (sum(new), 16, 64), torch.bfloat16, 381)
    if kind == "wide":
        assert sum(new) * 16 >= 256 * 256 and sum(new) * 8 >= 1024 * n
    print("[shares] %s, %d sequences" % (kind, n), flush=True)
    t, c = i32(torch, table), cu(new)
    bounds = (None, None) if kind == "tokens" else (i32(torch, c), max(new))
    out, lse = cache.attention(q, i32(torch, lens), t, *bounds, max(lens), with_lse=True)
    some = sorted(set(split) | set(range(0, n, n // 12)))
    for r in some:
        a = slice(c[r], c[r + 1])
        if new[r]:
            one, one_lse = cache.attention(q[a], i32(torch, lens[r:r + 1]), t[r:r + 1].contiguous(), with_lse=True)
            assert torch.equal(one, out[a]) and torch.equal(one_lse, lse[a]), r
    check_on_gpu(cache, q, lens, table, new, out, lse, [r for r in some if 0 < new[r] <= 200])
