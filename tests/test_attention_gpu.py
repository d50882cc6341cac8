"""The language side's attention on the GPU against the float64 reference: packed prompts, the 8-bit cache's
append and rows (bit for bit), attention over the cache, and all of them as one chain.

Tolerances.  With u the element type's half step (bf16 2^-8, fp16 2^-11 relative), A = sum_j p_j |v_j| and scores
good to delta (fp32 sums of head_dim exact products: head_dim * 2^-24 * scale * |q| max |k| by Cauchy-Schwarz), the
result is off by at most u |out| for its own rounding, u A for that of the weights, 2 delta A and the hardware
exponential's 2^-21 A.  Weights are rounded to fp16 over the cache whatever the element type, and in fp16 a weight
below 2^-14 is rounded by up to 2^-25 instead.  The largest weight is 2^7 at least: 2^-32 sum |v|; over the cache it
is 2^15: 2^-40 of it times 127 or 448 steps of its block, for each token."""
import numpy as np
import pytest

from oracle import attention as O

pytestmark = pytest.mark.gpu

HALF = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


def lib():
    import torch
    from paper_2609_31551_amd import attention as A
    return torch, A


def f64(t):
    return t.detach().double().cpu().numpy()


def prompt_bounds(q, k, v, cu_q, cu_k, scale, causal, u):
    """Of out and lse, element by element."""
    size, _ = O.prompt_attention(q, k, np.abs(v), cu_q, cu_k, scale, causal)
    group = q.shape[1] // k.shape[1]
    delta, total, count = np.zeros(q.shape[:2]), np.zeros(q.shape), np.zeros(q.shape[:2])
    for r in range(len(cu_q) - 1):
        a, b = slice(cu_q[r], cu_q[r + 1]), slice(cu_k[r], cu_k[r + 1])
        if b.stop == b.start:
            continue
        for h in range(q.shape[1]):
            kk = k[b, h // group]
            delta[a, h] = q.shape[2] * 2.0 ** -24 * abs(scale) * np.linalg.norm(q[a, h], axis=1) * \
                np.linalg.norm(kk, axis=1).max()
            total[a, h] = np.abs(v[b, h // group]).sum(0)
            count[a, h] = b.stop - b.start
    return size, delta, total, count


def check(out, lse, ref, ref_lse, size, delta, total, count, u, sub):
    tol = u * (np.abs(ref) + size) + (2 * delta[..., None] + 2.0 ** -21) * size + sub * total + 2.0 ** -25
    bad = ~(np.abs(out - ref) <= tol)
    assert not bad.any(), "%d of %d outputs off, worst %.3g of its tolerance" % (
        bad.sum(), bad.size, np.nanmax(np.abs(out - ref) / tol))
    if lse is not None:
        np.testing.assert_array_equal(np.isneginf(lse), np.isneginf(ref_lse))
        seen = ~np.isneginf(ref_lse)
        ltol = delta + 2.0 ** -21 * (1 + np.abs(np.where(seen, ref_lse, 0))) + count * 2.0 ** -24
        assert (np.abs(lse - ref_lse)[seen] <= ltol[seen]).all()


def cu(lens):
    return [0] + list(np.cumsum(lens))


def make(torch, shape, dtype, seed, size=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (size * torch.randn(shape, generator=g, device="cuda")).to(dtype)


def run_prompt(q, k, v, cu_q, cu_k, causal, scale=None, check_bounds=True):
    torch, A = lib()
    s = q.shape[2] ** -0.5 if scale is None else scale
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    A.prompt_attention(q, k, v, cu_q, cu_k, causal=causal, scale=scale, out=out, lse=lse)
    torch.cuda.synchronize()
    cu_k = cu_q if cu_k is None else cu_k
    n = cu_q[-1]
    assert (out[n:] == 7.0).all() and (lse[n:] == 7.0).all()   # rows behind the last sequence
    if check_bounds:
        Q, K, V = f64(q)[:n], f64(k)[:cu_k[-1]], f64(v)[:cu_k[-1]]
        ref, ref_lse = O.prompt_attention(Q, K, V, cu_q, cu_k, s, causal)
        u = HALF[str(q.dtype)[6:]]
        size, delta, total, count = prompt_bounds(Q, K, V, cu_q, cu_k, s, causal, u)
        check(f64(out)[:n], f64(lse)[:n], ref, ref_lse, size, delta, total, count, u,
              2.0 ** -32 if q.dtype == torch.float16 else 0.0)
    return out, lse


LENS = {
    "small": ([1, 2, 31, 0, 32, 33], [1, 2, 31, 0, 32, 33]),
    "tiles": ([63, 64, 65, 127, 128, 129], [63, 64, 65, 127, 128, 129]),
    "behind": ([1, 40, 70, 128, 3], [200, 129, 70, 333, 64]),            # queries behind cached keys
    "few_keys": ([50, 5, 130, 3], [20, 0, 64, 1]),                       # first queries see nothing
    "long": ([300, 517], [700, 517]),
    "runs": ([5, 33, 0, 2, 129], [13000, 8193, 9000, 8192, 130]),        # few queries over keys in several runs
    "short_runs": ([1, 60, 128, 129, 40], [2047, 2048, 2049, 4100, 1100]),
}


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 4, 64), (6, 2, 128), (7, 1, 64), (5, 5, 128)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_prompt_attention(dtype, heads, kv_heads, dim, lens, causal):
    torch, _ = lib()
    a, b = LENS[lens]
    dt = getattr(torch, dtype)
    print("[prompt] %s %s" % (lens, dtype), flush=True)
    q = make(torch, (sum(a) + 3, heads, dim), dt, 1)
    k, v = make(torch, (sum(b) + 5, kv_heads, dim), dt, 2, 2.0), make(torch, (sum(b) + 5, kv_heads, dim), dt, 3)
    k[sum(b):], v[sum(b):], q[sum(a):] = float("nan"), float("nan"), float("nan")
    run_prompt(q, k, v, cu(a), cu(b), causal)


@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0, 1e-30])
def test_prompt_attention_scales(scale):
    torch, _ = lib()
    q, k, v = (make(torch, (260, 2, 64), torch.bfloat16, s) for s in (4, 5, 6))
    run_prompt(q, k, v, [0, 260], None, True, scale)


def test_prompt_attention_maximum_that_moves_from_tile_to_tile():
    torch, _ = lib()
    q, v = make(torch, (400, 2, 128), torch.float16, 7), make(torch, (400, 1, 128), torch.float16, 8)
    for order in (1, -1):
        k = make(torch, (400, 1, 128), torch.float16, 9) * 0.1
        k += (q[200:201, :1] * torch.linspace(-1, 1, 400, device="cuda")[::1, None, None]).half()
        run_prompt(q, torch.flip(k, (0,)).contiguous() if order < 0 else k, v, [0, 400], None, True, 0.5)


def test_prompt_attention_strides():
    torch, _ = lib()
    q, k, v = (make(torch, (333, h, 64), torch.bfloat16, 10 + h) for h in (6, 3, 2))
    k, v = k[:, :2], v                                                           # a slice of three heads
    want, want_lse = run_prompt(q, k.contiguous(), v, [0, 100, 333], None, True)
    fused = torch.cat([q, k, v], 1)                                             # one projection's rows
    got, lse = run_prompt(fused[:, :6], fused[:, 6:8], fused[:, 8:], [0, 100, 333], None, True)
    assert torch.equal(got, want) and torch.equal(lse, want_lse)
    by_head = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v)]   # heads outside rows
    _, A = lib()
    out = torch.empty_like(by_head[0])
    A.prompt_attention(*by_head, [0, 100, 333], out=out)
    assert torch.equal(out, want) and out.stride() == by_head[0].stride()
    one = k[:, :1].expand(-1, 2, -1)                                            # one head for all
    got, _ = run_prompt(q, one, v[:, :1].expand(-1, 2, -1), [0, 100, 333], None, True)
    again, _ = run_prompt(q, k[:, :1].contiguous(), v[:, :1].contiguous(), [0, 100, 333], None, True)
    assert torch.equal(got, again)


def test_prompt_attention_does_not_depend_on_the_batch():
    torch, A = lib()
    lens = [577, 1, 64, 300, 1201, 128, 90]
    c = cu(lens)
    q = make(torch, (c[-1], 8, 128), torch.bfloat16, 20)
    k, v = (make(torch, (c[-1], 2, 128), torch.bfloat16, s) for s in (21, 22))
    every, lse = A.prompt_attention(q, k, v, c, with_lse=True)
    for r, n in enumerate(lens):
        s = slice(c[r], c[r + 1])
        one, one_lse = A.prompt_attention(q[s], k[s], v[s], [0, n], with_lse=True)
        assert torch.equal(one, every[s]) and torch.equal(one_lse, lse[s])


def test_prompt_attention_of_a_large_launch_is_that_of_a_small_one():
    """The workgroup's size goes by the launch's work (here 256 queries, and 128 for one sequence), a query's
    arithmetic does not."""
    torch, A = lib()
    c = [0, 4000, 8000, 12000, 16100]
    q, k, v = (make(torch, (c[-1], h, 64), torch.bfloat16, 24 + h) for h in (16, 8, 8))
    every, lse = A.prompt_attention(q, k, v, c, with_lse=True)
    for r in (0, 3):
        s = slice(c[r], c[r + 1])
        one, one_lse = A.prompt_attention(q[s], k[s], v[s], [0, c[r + 1] - c[r]], with_lse=True)
        assert torch.equal(one, every[s]) and torch.equal(one_lse, lse[s])


def test_prompt_attention_of_many_sequences():
    """More query tiles than the work list holds, empty sequences among them."""
    torch, A = lib()
    lens = [1700 if i % 3 else 0 for i in range(64)]
    c = cu(lens)
    q, k, v = (make(torch, (c[-1], h, 64), torch.float16, 27 + h) for h in (2, 1, 1))
    every, lse = A.prompt_attention(q, k, v, c, with_lse=True)
    assert c[-1] > 768 * 64
    for r in (1, 32, 62):
        s = slice(c[r], c[r + 1])
        one, one_lse = A.prompt_attention(q[s], k[s], v[s], [0, lens[r]], with_lse=True)
        assert torch.equal(one, every[s]) and torch.equal(one_lse, lse[s])
    run_prompt(q[:c[2]], k[:c[2]], v[:c[2]], [0, 0, 200], [0, 0, 200], True)


def test_prompt_attention_runs_do_not_depend_on_the_batch():
    torch, A = lib()
    new, held = [100, 700, 40, 9], [13000, 300, 0, 8190]
    cq, ck = cu(new), cu([a + b for a, b in zip(new, held)])
    q = make(torch, (cq[-1], 4, 128), torch.bfloat16, 28)
    k, v = (make(torch, (ck[-1], 2, 128), torch.bfloat16, s) for s in (29, 30))
    every, lse = A.prompt_attention(q, k, v, cq, ck, with_lse=True)
    for r in range(4):
        s, t = slice(cq[r], cq[r + 1]), slice(ck[r], ck[r + 1])
        one, one_lse = A.prompt_attention(q[s], k[t], v[t], [0, new[r]], [0, new[r] + held[r]], with_lse=True)
        assert torch.equal(one, every[s]) and torch.equal(one_lse, lse[s])


@pytest.mark.parametrize("what", ["nan", "inf"])
def test_prompt_attention_hidden_tokens_in_runs(what):
    torch, A = lib()
    q = make(torch, (64, 2, 128), torch.float16, 33)
    k, v = make(torch, (9000, 1, 128), torch.float16, 34), make(torch, (9000, 1, 128), torch.float16, 35)
    want, want_lse = A.prompt_attention(q, k, v, [0, 64], [0, 9000], with_lse=True)
    k2, v2 = k.clone(), v.clone()
    k2[8980:, :, 3], v2[8980:, :, 5] = float(what), float(what)     # hidden from the first 44 queries
    got, lse = A.prompt_attention(q, k2, v2, [0, 64], [0, 9000], with_lse=True)
    assert (got[:44].float() - want[:44].float()).abs().max() <= 4 * HALF["float16"] * v.abs().max()
    assert (lse[:44] - want_lse[:44]).abs().max() <= 1e-4
    assert not torch.isfinite(got[44:, :, 5]).any()


@pytest.mark.parametrize("what", ["nan", "inf"])
def test_prompt_attention_hidden_tokens_may_hold_anything(what):
    """A later token's key and value never reach an earlier query, NaN and infinities included."""
    torch, A = lib()
    x = float(what)
    q = make(torch, (200, 4, 64), torch.bfloat16, 30)
    k, v = make(torch, (200, 2, 64), torch.bfloat16, 31), make(torch, (200, 2, 64), torch.bfloat16, 32)
    want, _ = A.prompt_attention(q, k, v, [0, 200])
    k2, v2 = k.clone(), v.clone()
    k2[150:, :, 3], v2[150:, :, 5] = x, x
    got, _ = A.prompt_attention(q, k2, v2, [0, 200])
    u = HALF["bfloat16"]
    assert (got[:150] - want[:150]).abs().max() <= 4 * u * v.abs().max()
    assert not torch.isfinite(got[150:, :, 5]).any()


def test_prompt_attention_long_sequence_against_float64_on_the_gpu():
    torch, A = lib()
    n, before = 5000, 1700
    q = make(torch, (n, 2, 128), torch.bfloat16, 40)
    k, v = (make(torch, (n + before, 1, 128), torch.bfloat16, s) for s in (41, 42))
    out, lse = A.prompt_attention(q, k, v, [0, n], [0, n + before], with_lse=True)
    K, V = k[:, 0].double(), v[:, 0].double()
    hidden = torch.arange(n + before, device="cuda")[None] > torch.arange(n, device="cuda")[:, None] + before
    for h in range(2):
        s = (q[:, h].double() @ K.t().contiguous() * 128 ** -0.5).masked_fill(hidden, -np.inf)
        p = torch.softmax(s, 1)
        ref, size = p @ V, p @ V.abs()
        u = HALF["bfloat16"]
        delta = 2.0 ** -14 * s[~hidden].abs().max()
        assert ((out[:, h].double() - ref).abs() <= u * (ref.abs() + size) + (2 * delta + 2.0 ** -20) * size).all()
        assert ((lse[:, h].double() - torch.logsumexp(s, 1)).abs() <= delta + n * 2.0 ** -24 + 2.0 ** -17).all()


def test_prompt_attention_keys_behind_four_gib():
    torch, A = lib()
    row = 1 << 22
    store = torch.empty(700 * row, dtype=torch.bfloat16, device="cuda")          # 5.9 GB, 8 MiB a row
    k = store.as_strided((700, 1, 64), (row, 64, 1))
    v = store.as_strided((700, 1, 64), (row, 64, 1), 64)
    k.copy_(make(torch, (700, 1, 64), torch.bfloat16, 50))
    v.copy_(make(torch, (700, 1, 64), torch.bfloat16, 51))
    q = make(torch, (130, 2, 64), torch.bfloat16, 52)
    got, _ = A.prompt_attention(q, k, v, [0, 130], [0, 700])
    want, _ = A.prompt_attention(q, k.contiguous(), v.contiguous(), [0, 130], [0, 700])
    assert torch.equal(got, want)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_small_weights_count(dtype, dim, causal):
    """4,095 keys of 2^-25.3 of the first key's weight each, whose value is 0: the result is made of them alone."""
    torch, _ = lib()
    n, dt = 4096, getattr(torch, dtype)
    k, v = torch.zeros(n, 1, dim, dtype=dt, device="cuda"), torch.ones(n, 1, dim, dtype=dt, device="cuda")
    k[0], v[0] = 16.0, 0.0
    q = torch.zeros(40, 1, dim, dtype=dt, device="cuda")
    q[:, :, 0] = 1.0
    run_prompt(q, k, v, [0, 40], [0, n], causal, scale=float(np.float32(25.3 * np.log(2.0) / 16)))


@pytest.mark.parametrize("causal", [True, False])
def test_large_values_do_not_overflow(causal):
    """Values up to 2^122: sums of 70 of them with weights of 1 at most are finite."""
    torch, _ = lib()
    q, k = make(torch, (70, 2, 64), torch.bfloat16, 60), make(torch, (70, 2, 64), torch.bfloat16, 61)
    v = torch.full((70, 2, 64), 2.0 ** 120, dtype=torch.bfloat16, device="cuda")
    v[:, :, ::2] *= -4.0
    run_prompt(q, k, v, [0, 70], None, causal)


@pytest.mark.parametrize("scale", [1e39, float("inf"), float("nan"), "x"])
def test_binding_refuses_scales_that_are_no_float32(scale):
    torch, A = lib()
    q = make(torch, (10, 2, 64), torch.bfloat16, 1)
    cache = A.Kv8Cache.empty(4, 2, 64, 16)
    pages, lens = torch.zeros(2, 2, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    for bad in (lambda: A.prompt_attention(q, q, q, [0, 10], scale=scale), lambda: cache.attention(q, lens, pages, scale=scale)):
        with pytest.raises((ValueError, RuntimeError)):
            bad()


def test_binding_refusals():
    torch, A = lib()
    q = make(torch, (10, 4, 64), torch.bfloat16, 1)
    k = make(torch, (10, 2, 64), torch.bfloat16, 2)
    for bad in (lambda: A.prompt_attention(q.float(), k.float(), k.float(), [0, 10]),
                lambda: A.prompt_attention(q, k.half(), k, [0, 10]),
                lambda: A.prompt_attention(q, k[:, :, :32], k, [0, 10]),
                lambda: A.prompt_attention(q[0], k, k, [0, 10]),
                lambda: A.prompt_attention(q, k, k, [0, 11]),
                lambda: A.prompt_attention(q, k, k, [0, 10], [0, 5, 10]),
                lambda: A.prompt_attention(q, k, k, [0, 10], [0, 12]),
                lambda: A.prompt_attention(q, k, k, [0, 6, 5]),
                lambda: A.prompt_attention(q, k, k, [0, 10], out=q[:9]),
                lambda: A.prompt_attention(q, k, k, [0, 10], lse=torch.empty(10, 4, device="cuda").half()),
                lambda: A.prompt_attention(q, k, k, list(range(11)) + [10] * 60),
                lambda: A.prompt_attention(q[:2], k.expand(-1, 2, -1), k, [0, 2], [0, 10],
                                           workspace=torch.zeros(8, device="cuda")),
                lambda: A.prompt_attention(q.transpose(1, 2), k, k, [0, 10])):
        with pytest.raises((ValueError, RuntimeError)):
            bad()
    cache = A.Kv8Cache.empty(4, 2, 64, 16)
    i32 = dict(dtype=torch.int32, device="cuda")
    pages, one, two = torch.zeros(2, 2, **i32), torch.zeros(1, **i32), torch.zeros(2, **i32)
    for bad in (lambda: cache.append(k, k, one, pages), lambda: cache.append(k, k, two, pages.long()),
                lambda: cache.append(k, k[:9], two, pages), lambda: cache.append(k, k, two, pages, max_new=4),
                lambda: cache.append(k.float(), k.float(), two, pages), lambda: cache.append(k, k, two.cpu(), pages),
                lambda: cache.append(k, k, two, pages, cu_new=two), lambda: cache.append(q, q, two, pages),
                lambda: cache.rows(pages, two, 4), lambda: cache.attention(q, one, pages),
                lambda: cache.attention(q[:9], two, pages), lambda: cache.attention(q[:, :3], two, pages),
                lambda: cache.attention(q, two, pages[0]),
                lambda: cache.attention(q, two, torch.zeros(2, 400, **i32),
                                        workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((ValueError, RuntimeError)):
            bad()


# ---- the 8-bit cache ---------------------------------------------------------------

FORMATS = ["int8", "e4m3"]


def kind(torch, form):
    return torch.int8 if form == "int8" else torch.float8_e4m3fn


def i32(torch, v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


class Both:
    """A cache on the GPU beside the reference's, its memory full of 0xff bytes (NaN in e4m3) at first."""

    def __init__(self, form, n_pages, kv_heads, page, dim):
        torch, A = lib()
        self.gpu = A.Kv8Cache.empty(n_pages, kv_heads, dim, page, kind(torch, form))
        for t in (self.gpu.k, self.gpu.v):
            t.view(torch.uint8).fill_(255)
        for t in (self.gpu.k_scale, self.gpu.v_scale):
            t.fill_(float("nan"))
        self.ref = O.Cache(n_pages, kv_heads, page, dim, form)

    def append(self, k, v, cu_new, held, table, uniform=None):
        torch, _ = lib()
        self.gpu.append(k, v, i32(torch, held), i32(torch, table), None if uniform else i32(torch, cu_new),
                        max_new=uniform or max(np.diff(cu_new)))
        for r in range(len(held)):
            a = slice(cu_new[r], cu_new[r + 1])
            self.ref.append(f64(k)[a], f64(v)[a], held[r], table[r])

    def check_rows(self, lens, table, dtype):
        torch, _ = lib()
        c = cu(lens)
        k, v = self.gpu.rows(i32(torch, table), i32(torch, c), c[-1] + 2, max_len=max(lens), dtype=dtype,
                             k=torch.full((c[-1] + 2, self.gpu.kv_heads, self.gpu.head_dim), 5.0, dtype=dtype, device="cuda"))
        assert (k[c[-1]:] == 5.0).all()
        for name, got in (("k", k), ("v", v)):
            want = np.concatenate([self.ref.rows(name, table[r], 0, n) for r, n in enumerate(lens)])
            want = torch.from_numpy(want).to(dtype).double().numpy()
            np.testing.assert_array_equal(f64(got)[:c[-1]], want)


def tables(rng, lens, page, spare=3, extra=0):
    need = [-(-n // page) for n in lens]
    order = rng.permutation(sum(need) + spare)
    table = np.full((len(lens), max(need) + extra), -1)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    return table, sum(need) + spare


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("page,heads,dim", [(16, 2, 64), (32, 1, 128), (64, 3, 128), (128, 1, 64), (64, 1, 64)])
def test_append_and_rows_bit_for_bit(form, dtype, page, heads, dim):
    torch, _ = lib()
    dt = getattr(torch, dtype)
    rng = np.random.default_rng(3)
    print("[kv8] append %s %s page %d" % (form, dtype, page), flush=True)
    steps = [[1, 0, page, 2 * page + 5, 37, 3], [1, 1, 1, 1, 1, 1], [page - 1, 70, 5, 0, page, 2], [1, 1, 1, 1, 1, 1]]
    total = np.sum(steps, 0)
    table, n_pages = tables(rng, total, page)
    both = Both(form, n_pages, heads, page, dim)
    held = np.zeros(6, int)
    for i, new in enumerate(steps):
        c = cu(new)
        size = [1.0, 30.0, 0.01, 3.0][i]   # the second step's tokens need larger scales
        k, v = make(torch, (c[-1], heads, dim), dt, 60 + i, size), make(torch, (c[-1], heads, dim), dt, 70 + i, size)
        both.append(k, v, c, list(held), table, uniform=1 if set(new) == {1} else None)
        held += new
        both.check_rows(list(held), table, dt)
    for name, got in (("k", both.gpu.k_scale), ("v", both.gpu.v_scale)):
        used = sorted(set(table[table >= 0]))
        np.testing.assert_array_equal(f64(got)[used], both.ref.scale[name][used])


@pytest.mark.parametrize("form", FORMATS)
def test_append_of_unusual_values(form):
    """Zeros, subnormals, the largest values, NaN and infinities, borders of the scale and ties."""
    torch, _ = lib()
    rows = 6 * 16
    for dt in (torch.bfloat16, torch.float16):
        top = torch.finfo(dt).max
        k, v = make(torch, (rows, 2, 64), dt, 80), make(torch, (rows, 2, 64), dt, 81)
        k[0:16] = 0.0
        v[0:16] = -0.0
        k[16:32] *= torch.finfo(dt).tiny * 0.01
        v[16:32, 0] = 2.0 ** -24 if dt == torch.float16 else 1e-39
        k[32:48, :, 5], k[40, :, 9], k[41, 0, 9], k[42, 1, 3] = 1.0, float("nan"), float("inf"), float("-inf")
        v[32:48] = float("nan")
        v[33:35, 1], v[33, 1, 5] = float("inf"), float("-inf")
        k[48:64] = torch.arange(64, device="cuda").to(dt) - 32.5          # ties
        k[48, :, 0] = 127.0
        v[48:64] = (torch.arange(64, device="cuda").float() / 16).to(dt)
        k[64:80, 0, 0], k[64:80, 1, 0], v[64:80, 0, 0], v[64:80, 1, 0] = 127.0, 127.5, 448.0, 450.0
        k[80:96, 0, 7], v[80:96, 1, 7] = top, -top
        both = Both(form, 8, 2, 16, 64)
        table = np.array([[3, 1, 7, 0, 2, 5]])
        both.append(k, v, [0, rows], [0], table)
        if dt == torch.bfloat16:
            both.check_rows([rows], table, dt)
        else:   # int8 may hold 65504 as 65536
            both.check_rows([80], table, dt)
        for name, got in (("k", both.gpu.k_scale), ("v", both.gpu.v_scale)):
            np.testing.assert_array_equal(f64(got)[table[0]], both.ref.scale[name][table[0]])


@pytest.mark.parametrize("form", FORMATS)
def test_append_drops_what_has_no_place(form):
    """Pages that are not held, sequences left out, tokens behind the table, rows outside the input."""
    torch, _ = lib()
    both = Both(form, 6, 1, 16, 64)
    before = both.gpu.k.view(torch.uint8).clone(), both.gpu.v.view(torch.uint8).clone()
    k, v = make(torch, (100, 1, 64), torch.float16, 90), make(torch, (100, 1, 64), torch.float16, 91)
    table = np.array([[0, -1, 2], [6, 3, 1 << 30], [4, 4, 4], [5, -1, -1]])
    held = i32(torch, [0, 10, -1, 8])
    both.gpu.append(k, v, held, i32(torch, table), i32(torch, [0, 40, 70, 80, 120]), max_new=60)
    for r, (h, a, n) in enumerate(((0, 0, 40), (10, 40, 30), (None, 70, 0), (8, 80, 20))):
        if h is not None:
            both.ref.append(f64(k)[a:a + n], f64(v)[a:a + n], h, list(table[r]))
    # page 3: the second sequence's tokens 16 ..; page 5: a page whose first 8 tokens were never written
    for page, lo, hi in ((0, 0, 16), (2, 0, 8), (3, 0, 16)):
        for name, codes in (("k", both.gpu.k), ("v", both.gpu.v.view(torch.uint8).transpose(2, 3).view(both.gpu.v.dtype))):
            np.testing.assert_array_equal(f64(codes.float())[page, :, lo:hi], both.ref.code[name][page, :, lo:hi])
    for page in (1, 4):
        assert torch.equal(both.gpu.k[page].view(torch.uint8), before[0][page])
        assert torch.equal(both.gpu.v[page].view(torch.uint8), before[1][page])
    assert (both.gpu.k.view(torch.uint8)[2, :, 8:] == 255).all()    # places that got no token
    # max_new cuts; no rows, no change
    both.gpu.append(k[:0], v[:0], held, i32(torch, table), i32(torch, [0, 0, 0, 0, 0]))


def test_rows_of_absent_pages_and_windows():
    torch, _ = lib()
    both = Both("int8", 5, 2, 16, 128)
    k, v = make(torch, (50, 2, 128), torch.bfloat16, 95), make(torch, (50, 2, 128), torch.bfloat16, 96)
    table = np.array([[4, 1, 0, 3]])
    both.append(k, v, [0, 50], [0], table)
    hole = np.array([[4, -1, 0, 3], [4, 1, 9, -7]])
    first, lens = [5, -3], [45, 60]
    a, b = both.gpu.rows(i32(torch, hole), i32(torch, cu(lens)), 105, first=i32(torch, first), dtype=torch.bfloat16)
    want = np.concatenate([both.ref.rows("k", hole[r], first[r], lens[r]) for r in range(2)])
    np.testing.assert_array_equal(f64(a), want)
    want = np.concatenate([both.ref.rows("v", hole[r], first[r], lens[r]) for r in range(2)])
    np.testing.assert_array_equal(f64(b), want)


def filled(form, lens, page, heads, dim, seed, extra=0):
    torch, _ = lib()
    rng = np.random.default_rng(seed)
    table, n_pages = tables(rng, lens, page, extra=extra)
    both = Both(form, n_pages, heads, page, dim)
    c = cu(lens)
    k, v = make(torch, (c[-1], heads, dim), torch.bfloat16, seed, 1.5), make(torch, (c[-1], heads, dim), torch.bfloat16, seed + 1)
    v *= torch.exp2(torch.arange(c[-1], device="cuda") // page % 5 - 2.0).to(v.dtype)[:, None, None]   # scales differ
    both.append(k, v, c, [0] * len(lens), table)
    return both, table


def check_decode(both, q, lens, table, new, scale, causal, out, lse):
    c, u = cu(new), HALF[str(q.dtype)[6:]]
    Q = f64(q)
    for r, n in enumerate(lens):
        a = slice(c[r], c[r + 1])
        ref, ref_lse = both.ref.attention(Q[a], n, table[r], scale, causal)
        k, v = both.ref.rows("k", table[r], 0, n), both.ref.rows("v", table[r], 0, n)
        absolute = O.Cache.__new__(O.Cache)
        absolute.page, absolute.form, absolute.scale = both.ref.page, both.ref.form, both.ref.scale
        absolute.code = {"k": both.ref.code["k"], "v": np.abs(both.ref.code["v"])}
        size, _ = absolute.attention(Q[a], n, table[r], scale, causal)
        group = q.shape[1] // k.shape[1]
        kn = np.linalg.norm(k, axis=2).max(0, initial=0.0)
        delta = (q.shape[2] + 2) * 2.0 ** -24 * scale * np.linalg.norm(Q[a], axis=2) * np.repeat(kn, group)[None]
        # the largest weight times its block's largest value, p <= 1 of the sum
        pages = np.array([p if 0 <= p < both.ref.scale["v"].shape[0] else 0 for p in table[r][:-(-n // both.ref.page)]], int)
        vs = both.ref.scale["v"][pages].max(0, initial=0.0) * O.MOST[both.ref.form]
        total = (n * np.repeat(vs, group))[None, :, None] * np.ones(ref.shape)
        # weights are rounded to fp16 (2^-11) whatever the element type
        tol_u = 2.0 ** -11
        got = f64(out)[a]
        tol = u * np.abs(ref) + tol_u * size + (2 * delta[..., None] + 2.0 ** -21) * size + 2.0 ** -40 * total + 2.0 ** -25
        bad = ~(np.abs(got - ref) <= tol)
        assert not bad.any(), "sequence %d: %d of %d off, worst %.3g of its tolerance" % (
            r, bad.sum(), bad.size, np.nanmax(np.abs(got - ref) / tol))
        if lse is not None:
            L = f64(lse)[a]
            np.testing.assert_array_equal(np.isneginf(L), np.isneginf(ref_lse))
            seen = ~np.isneginf(ref_lse)
            ltol = delta + 2.0 ** -21 * (1 + np.abs(np.where(seen, ref_lse, 0))) + n * 2.0 ** -24
            assert (np.abs(L - ref_lse)[seen] <= ltol[seen]).all()


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("page,heads,kv_heads,dim", [(16, 4, 4, 64), (64, 14, 2, 128), (32, 20, 1, 64), (128, 8, 1, 128)])
def test_decode(form, dtype, page, heads, kv_heads, dim):
    torch, _ = lib()
    lens = [1, 15, 16, 17, 64, 65, 255, 256, 257, 700, 1024, 1025, 2300]
    print("[kv8] decode %s %s page %d" % (form, dtype, page), flush=True)
    both, table = filled(form, lens, page, kv_heads, dim, 100)
    q = make(torch, (len(lens), heads, dim), getattr(torch, dtype), 5)
    out, lse = both.gpu.attention(q, i32(torch, lens), i32(torch, table), with_lse=True)
    check_decode(both, q, lens, table, [1] * len(lens), dim ** -0.5, True, out, lse)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("dtype,heads,kv_heads,dim", [("bfloat16", 7, 1, 128), ("float16", 4, 2, 64)])
def test_decode_several_queries(dtype, heads, kv_heads, dim, form, causal):
    """Ragged numbers of queries, none and more than the tokens among them, lengths past a split."""
    torch, _ = lib()
    new, lens = [3, 0, 17, 5, 1, 40, 9], [1300, 20, 17, 3, 0, 2600, 1025]
    both, table = filled(form, lens, 16, kv_heads, dim, 110)
    c = cu(new)
    q = make(torch, (c[-1] + 2, heads, dim), getattr(torch, dtype), 6)
    out = torch.full(q.shape, 9.0, dtype=q.dtype, device="cuda")
    out, lse = both.gpu.attention(q, i32(torch, lens), i32(torch, table), cu_q=i32(torch, c), max_q=40, causal=causal,
                                  scale=0.2, out=out, with_lse=True)
    assert (out[c[-1]:] == 9.0).all()
    check_decode(both, q, lens, table, new, 0.2, causal, out, lse)


@pytest.mark.parametrize("form", FORMATS)
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("page,causal", [(16, True), (128, False)])
def test_decode_full_batch(form, dtype, page, causal):
    """Several queries of so many sequences that a workgroup takes two row tiles: right, and each as when alone."""
    torch, _ = lib()
    rng = np.random.default_rng(7)
    lens = [0, 1, 2, 1025, 2100, 17, 1, 1500] + [int(n) for n in rng.integers(1, 400, 56)]
    new = [3, 9, 2, 9, 5, 0, 1, 8] + [int(n) for n in rng.integers(0, 10, 56)]
    both, table = filled(form, lens, page, 8, 128, 120)
    c = cu(new)
    q = make(torch, (c[-1], 32, 128), getattr(torch, dtype), 8)
    out, lse = both.gpu.attention(q, i32(torch, lens), i32(torch, table), cu_q=i32(torch, c), max_q=9, causal=causal,
                                  with_lse=True)
    check_decode(both, q[:c[12]], lens[:12], table, new[:12], 128 ** -0.5, causal, out, lse)
    for r, n in enumerate(new):
        if n:
            rows = slice(c[r], c[r + 1])
            alone, alone_lse = both.gpu.attention(q[rows], i32(torch, lens[r:r + 1]), i32(torch, table[r:r + 1]),
                                                  causal=causal, with_lse=True)
            assert torch.equal(out[rows], alone) and torch.equal(lse[rows], alone_lse), "sequence %d" % r


@pytest.mark.parametrize("form", FORMATS)
def test_decode_small_weights_count(form):
    """As above, over the cache: 1,023 tokens of 2^-25.3 of the first's weight each, in the first's runs of tiles."""
    torch, A = lib()
    both = Both(form, 64, 1, 16, 128)
    k, v = torch.zeros(1024, 1, 128, device="cuda").bfloat16(), torch.ones(1024, 1, 128, device="cuda").bfloat16()
    k[0], v[0] = 16.0, 0.0
    table = np.arange(64)[None]
    both.append(k, v, [0, 1024], [0], table)
    q = torch.zeros(1, 2, 128, device="cuda").bfloat16()
    q[:, 0, 0] = 1.0                       # the other head's scores are all 0
    scale = float(np.float32(25.3 * np.log(2.0) / 16))
    out, lse = both.gpu.attention(q, i32(torch, [1024]), i32(torch, table), scale=scale, with_lse=True)
    check_decode(both, q, [1024], table, [1], scale, True, out, lse)


def test_decode_over_absent_pages():
    torch, _ = lib()
    lens = [100, 330, 64]
    both, table = filled("e4m3", lens, 16, 2, 64, 120)
    table[0, 2], table[1, :17], table[1, 20], table[2, :] = -1, 1 << 20, -5, -1
    q = make(torch, (3, 4, 64), torch.float16, 7)
    out, lse = both.gpu.attention(q, i32(torch, lens), i32(torch, table), with_lse=True)
    assert (out[2] == 0).all() and torch.isneginf(lse[2]).all()
    check_decode(both, q, lens, table, [1, 1, 1], 0.125, True, out, lse)


@pytest.mark.parametrize("form", FORMATS)
def test_decode_with_scales_far_apart(form):
    """Blocks of zeros, tiny and huge values beside each other: every token's weight counts in the sum, and the
    result is good to the largest contribution."""
    torch, _ = lib()
    page, lens = 16, [8 * 16 + 5]
    rng = np.random.default_rng(8)
    table, n_pages = tables(rng, lens, page)
    both = Both(form, n_pages, 1, page, 64)
    k, v = make(torch, (lens[0], 1, 64), torch.bfloat16, 130), make(torch, (lens[0], 1, 64), torch.bfloat16, 131)
    for i, size in enumerate([0.0, 1e-30, 1.0, 0.0, 1e20, 1e-5, 0.0, 3e4, 1.0]):
        v[i * page:(i + 1) * page] *= size
    k[4 * page:5 * page] -= 20.0 * 8      # the huge one weighs little
    both.append(k, v, [0, lens[0]], [0], table)
    q = torch.ones(1, 2, 64, dtype=torch.bfloat16, device="cuda") * 0.05
    for n in (3 * page, 4 * page, lens[0]):
        out, lse = both.gpu.attention(q, i32(torch, [n]), i32(torch, table), with_lse=True)
        check_decode(both, q, [n], table, [1], 0.125, True, out, lse)


@pytest.mark.parametrize("size", [1e-38, 1e-20, 1e20, 1e30])
def test_decode_with_small_and_large_queries(size):
    """Queries' sizes across bf16's range, the scale bringing the scores back."""
    torch, _ = lib()
    both, table = filled("int8", [300], 32, 1, 64, 140)
    q = make(torch, (1, 3, 64), torch.bfloat16, 9, size)
    scale = min(0.2 / size, 1e37)
    out, lse = both.gpu.attention(q, i32(torch, [300]), i32(torch, table), scale=scale, with_lse=True)
    check_decode(both, q, [300], table, [1], float(np.float32(scale)), True, out, lse)


def test_decode_does_not_depend_on_the_batch_or_its_bounds():
    torch, _ = lib()
    lens = [700, 5, 1300, 256, 3000]
    both, table = filled("int8", lens, 64, 2, 128, 150, extra=9)
    q = make(torch, (5, 8, 128), torch.bfloat16, 10)
    every, lse = both.gpu.attention(q, i32(torch, lens), i32(torch, table), with_lse=True)
    for r, n in enumerate(lens):
        for more in (dict(), dict(max_len=n), dict(cu_q=i32(torch, [0, 1]), max_q=7)):
            one, one_lse = both.gpu.attention(q[r:r + 1], i32(torch, [n]), i32(torch, table[r:r + 1]), with_lse=True, **more)
            assert torch.equal(one[0], every[r]) and torch.equal(one_lse[0], lse[r])


def test_decode_lengths_are_cut_to_the_table():
    torch, _ = lib()
    both, table = filled("int8", [64, 64], 32, 1, 64, 160)
    q = make(torch, (2, 2, 64), torch.float16, 11)
    t = i32(torch, table)
    want, _ = both.gpu.attention(q, i32(torch, [64, 0]), t)
    got, _ = both.gpu.attention(q, i32(torch, [1 << 30, -7]), t)
    assert torch.equal(got, want) and (got[1] == 0).all()


def test_cache_behind_four_gib():
    torch, A = lib()
    page, dim, heads = 64, 128, 8
    n_pages = (5 << 30) // (page * dim * heads)                 # 5 GiB of keys, 5 of values
    cache = A.Kv8Cache.empty(n_pages, heads, dim, page)
    small = A.Kv8Cache.empty(8, heads, dim, page)
    k, v = (make(torch, (500, heads, dim), torch.bfloat16, s) for s in (170, 171))
    q = make(torch, (1, 16, dim), torch.bfloat16, 172)
    far = i32(torch, [[n_pages - 1 - i for i in range(8)]])
    near = i32(torch, [list(range(8))])
    zero, held = i32(torch, [0]), i32(torch, [500])
    got = []
    for c, t in ((cache, far), (small, near)):
        c.append(k, v, zero, t)
        got.append(c.rows(t, i32(torch, [0, 500]), 500) + c.attention(q, held, t, with_lse=True))
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_bounds_that_are_smaller_than_the_batch():
    """Tokens beyond max_new are dropped, rows beyond max_rows not written, queries beyond max_q not computed and
    tokens beyond max_len not seen."""
    torch, A = lib()
    both = Both("int8", 8, 1, 16, 64)
    table = np.array([[1, 2, 3], [5, 6, 7]])
    k, v = make(torch, (60, 1, 64), torch.float16, 240), make(torch, (60, 1, 64), torch.float16, 241)
    both.gpu.append(k, v, i32(torch, [0, 3]), i32(torch, table), i32(torch, [0, 20, 60]), max_new=25)
    both.ref.append(f64(k)[:20], f64(v)[:20], 0, table[0])
    both.ref.append(f64(k)[20:45], f64(v)[20:45], 3, table[1])
    assert (both.gpu.k.view(torch.uint8)[6, :, 12:] == 255).all() and (both.gpu.k.view(torch.uint8)[7] == 255).all()
    got = torch.full((48, 1, 64), 5.0, dtype=torch.float16, device="cuda")
    both.gpu.rows(i32(torch, table), i32(torch, [0, 20, 48]), 48, max_len=7, dtype=torch.float16, k=got)
    for r, a in ((0, 0), (1, 20)):
        if r == 0:
            np.testing.assert_array_equal(f64(got)[a:a + 7], both.ref.rows("k", table[r], 0, 7))
        assert (got[a + 7:a + 20] == 5.0).all()
    q = make(torch, (5, 2, 64), torch.float16, 242)
    out = torch.full(q.shape, 9.0, dtype=q.dtype, device="cuda")
    both.gpu.attention(q, i32(torch, [20, 0]), i32(torch, table), cu_q=i32(torch, [0, 4, 5]), max_q=2, max_len=11,
                       causal=False, out=out)
    assert (out[2:4] == 9.0).all() and (out[4] == 0).all()
    want, _ = both.gpu.attention(q[:2], i32(torch, [11]), i32(torch, table[:1]), causal=False)
    assert torch.equal(out[:2], want)


def test_pages_shared_for_reading():
    torch, A = lib()
    both, table = filled("e4m3", [100, 40], 16, 2, 64, 250)
    shared = table.copy()
    shared[1, :2] = table[0, :2]                       # the second sequence starts with the first one's pages
    q = make(torch, (2, 4, 64), torch.bfloat16, 251)
    out, lse = both.gpu.attention(q, i32(torch, [100, 40]), i32(torch, shared), with_lse=True)
    check_decode(both, q, [100, 40], shared, [1, 1], 0.125, True, out, lse)
    both.check_rows([100, 40], shared, torch.bfloat16)


def test_rows_of_keys_or_values_alone():
    import ctypes
    torch, A = lib()
    both, table = filled("int8", [50], 32, 2, 128, 260)
    t, c = i32(torch, table), i32(torch, [0, 50])
    want = both.gpu.rows(t, c, 50)
    s = A.Strides(256, 128)
    for i in range(2):
        got = torch.zeros_like(want[0])
        ptr = [None, None]
        ptr[i] = got.data_ptr()
        assert A.LIB.eas_kv8_rows(both.gpu._c, A.EAS_BF16, t.data_ptr(), t.shape[1], 1, c.data_ptr(), None, 50, 50, ptr[0],
                                  s, ptr[1], s, torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(got, want[i])


def test_empty_batches():
    torch, A = lib()
    q, k = make(torch, (4, 2, 64), torch.bfloat16, 270), make(torch, (0, 1, 64), torch.bfloat16, 271)
    out, lse = A.prompt_attention(q, k, k, [0, 4], [0, 0], with_lse=True)
    assert (out == 0).all() and torch.isneginf(lse).all()
    for cu_q in ([0], [0, 0]):
        out, lse = A.prompt_attention(q[:0], k, k, cu_q, with_lse=True)
        assert out.shape == (0, 2, 64) and lse.shape == (0, 2)
    cache = A.Kv8Cache.empty(2, 1, 64, 16)
    none, pages = i32(torch, []), torch.zeros((0, 3), dtype=torch.int32, device="cuda")
    cache.append(k, k, none, pages)
    assert cache.attention(q[:0], none, pages)[0].shape == (0, 2, 64)
    assert cache.rows(pages, i32(torch, [0]), 0)[0].shape == (0, 1, 64)
    torch.cuda.synchronize()


# ---- streams, graphs, and the chain ---------------------------------------------------

def test_other_stream():
    torch, A = lib()
    s = torch.cuda.Stream()
    q, k, v = (make(torch, (600, h, 64), torch.bfloat16, 180 + h) for h in (4, 2, 2))
    both, table = filled("int8", [600], 64, 2, 64, 190)
    want = A.prompt_attention(q, k, v, [0, 600], with_lse=True), both.gpu.attention(
        q[:1], i32(torch, [600]), i32(torch, table), with_lse=True)
    t, n = i32(torch, table), i32(torch, [600])
    torch.cuda.synchronize()
    for _ in range(3):
        got = A.prompt_attention(q, k, v, [0, 600], with_lse=True, stream=s), both.gpu.attention(
            q[:1], n, t, with_lse=True, stream=s)
        s.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_calls_with_runs_on_two_streams_at_once():
    """Their workspaces are their own: calls that overlap give what they give alone."""
    torch, A = lib()
    both, table = filled("e4m3", [5000, 3100], 64, 2, 128, 195)
    table, lens = i32(torch, table), i32(torch, [5000, 3100])
    q = make(torch, (40, 8, 128), torch.bfloat16, 196)
    k, v = make(torch, (6000, 2, 128), torch.bfloat16, 197), make(torch, (6000, 2, 128), torch.bfloat16, 198)

    def calls(x, stream=None):
        return (*A.prompt_attention(x, k, v, [0, 40], [0, 6000], with_lse=True, stream=stream),
                *both.gpu.attention(x[:6], lens, table, with_lse=True, stream=stream))
    queries = [q, q.flip(0).contiguous()]
    want = [calls(x) for x in queries]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i in range(2):
            got[i].append(calls(queries[i], streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for one in got[i]:
            assert all(torch.equal(x, y) for x, y in zip(one, want[i]))


@pytest.mark.parametrize("form", FORMATS)
def test_decoding_steps_in_a_graph(form):
    """One step -- append, attention, lengths moved on -- captured once and replayed: every replay equals the same
    step run eagerly on another cache, with eager work and synchronizations between."""
    torch, A = lib()
    lens = [250, 31, 700]
    caches, tabs = [], []
    for _ in range(2):
        both, table = filled(form, lens, 32, 2, 128, 200, extra=3)
        for r in range(3):   # room for the new tokens
            need = -(-lens[r] // 32)
            table[r, need:need + 3] = [-1] * 3
        caches.append(both.gpu)
        tabs.append(table)
    spare = [p for p in range(caches[0].n_pages) if p not in set(tabs[0][tabs[0] >= 0])]
    for t in tabs:
        for r in range(3):
            t[r, -(-lens[r] // 32)] = spare[r]
    state = []
    for c, t in zip(caches, tabs):
        state.append(dict(c=c, t=i32(torch, t), held=i32(torch, lens), lens=i32(torch, lens) + 1,
                          k=make(torch, (3, 2, 128), torch.bfloat16, 0), v=make(torch, (3, 2, 128), torch.bfloat16, 0),
                          q=make(torch, (3, 6, 128), torch.bfloat16, 0)))

    def step(s):
        s["c"].append(s["k"], s["v"], s["held"], s["t"])
        out = s["c"].attention(s["q"], s["lens"], s["t"], with_lse=True)
        s["held"].add_(1)
        s["lens"].add_(1)
        return out

    fixed, eager = state
    warm = torch.cuda.Stream()
    saved = {n: fixed[n].clone() for n in ("held", "lens")}
    codes = [x.clone() for x in (fixed["c"].k.view(torch.uint8), fixed["c"].v.view(torch.uint8), fixed["c"].k_scale, fixed["c"].v_scale)]
    warm.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(warm):
        step(fixed)
    torch.cuda.current_stream().wait_stream(warm)
    for n, x in saved.items():
        fixed[n].copy_(x)
    for x, y in zip((fixed["c"].k.view(torch.uint8), fixed["c"].v.view(torch.uint8), fixed["c"].k_scale, fixed["c"].v_scale), codes):
        x.copy_(y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(fixed)
    for n, x in saved.items():
        fixed[n].copy_(x)
    for i in range(6):
        for n, seed in (("k", 300 + i), ("v", 310 + i), ("q", 320 + i)):
            x = make(torch, state[0][n].shape, torch.bfloat16, seed, 1.0 + i)
            fixed[n].copy_(x)
            eager[n].copy_(x)
        graph.replay()
        want = step(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(captured, want)), "replay %d" % i
        assert torch.equal(fixed["c"].k.view(torch.uint8)[fixed["t"][fixed["t"] >= 0].long()],
                           eager["c"].k.view(torch.uint8)[fixed["t"][fixed["t"] >= 0].long()])


def test_prompt_in_a_graph():
    torch, A = lib()
    q, k, v = (make(torch, (300, h, 64), torch.float16, 210 + h) for h in (4, 2, 2))
    A.prompt_attention(q, k, v, [0, 120, 300], with_lse=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = A.prompt_attention(q, k, v, [0, 120, 300], with_lse=True)
    for i in range(4):
        q.copy_(make(torch, q.shape, torch.float16, 400 + i))
        graph.replay()
        want, want_lse = A.prompt_attention(q, k, v, [0, 120, 300], with_lse=True)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("form", FORMATS)
def test_encode_prefill_decode_chain(form):
    """The stages in a row: images encoded into envelopes, their rows projected to queries, keys and values;
    the prompts in two chunks (prompt attention; append; the cached first chunk taken back as rows and attended to
    with the second); then three decoding steps over the cache."""
    torch, A = lib()
    from _harness import gpu_encode
    from paper_2609_31551_amd import configs as C
    from paper_2609_31551_amd import router as R
    from paper_2609_31551_amd import synth
    p = C.with_layers(C.QWEN_IMAGE, 1)
    items = synth.make_items(p, 3, 0, shapes=[(2, 224, 308), (2, 392, 224), (2, 56, 56)])
    enc = gpu_encode(p, items, synth.make_weights(p, 0), out_dtype="bf16")
    rows = np.diff(enc["cu_out"])
    _, _, req = R.envelope_plan([0, 0, 0], 1, rows)
    emb = torch.from_numpy(enc["out"]).cuda().bfloat16()
    env = torch.empty_like(emb)
    R.envelope_gather(emb, enc["cu_out"], req, env)
    heads, kv_heads, dim = 4, 2, 64
    x = torch.nn.functional.layer_norm(env.float(), (env.shape[1],))
    proj = make(torch, (env.shape[1], (heads + 2 * kv_heads) * dim), torch.float32, 220, env.shape[1] ** -0.5)
    qkv = (x @ proj).bfloat16().view(-1, heads + 2 * kv_heads, dim)
    c = list(enc["cu_out"])
    lens = [int(n) for n in rows]
    half = [n // 2 for n in lens]
    steps = 3
    rng = np.random.default_rng(0)
    table, n_pages = tables(rng, [n + steps for n in lens], 16)
    both, t = Both(form, n_pages, kv_heads, 16, dim), i32(torch, table)

    def take(a, b):   # rows a[r] .. b[r] of each request
        return qkv[torch.cat([torch.arange(c[r] + a[r], c[r] + b[r], device="cuda") for r in range(3)])]

    def split(z):
        return z[:, :heads], z[:, heads:heads + kv_heads], z[:, heads + kv_heads:]

    q, k, v = split(take([0] * 3, half))
    run_prompt(q, k, v, cu(half), None, True)
    both.append(k, v, cu(half), [0] * 3, table)
    held_k, held_v = both.gpu.rows(t, i32(torch, cu(half)), sum(half))
    both.check_rows(half, table, torch.bfloat16)
    q, k, v = split(take(half, lens))
    rest = [n - h for n, h in zip(lens, half)]
    ch, cr = cu(half), cu(rest)
    kk = torch.cat([z for r in range(3) for z in (held_k[ch[r]:ch[r + 1]], k[cr[r]:cr[r + 1]])])
    vv = torch.cat([z for r in range(3) for z in (held_v[ch[r]:ch[r + 1]], v[cr[r]:cr[r + 1]])])
    run_prompt(q, kk, vv, cu(rest), cu(lens), True)
    both.append(k, v, cu(rest), half, table)
    for i in range(steps):
        new = make(torch, (3, heads + 2 * kv_heads, dim), torch.bfloat16, 230 + i)
        q, k, v = split(new)
        held = [n + i for n in lens]
        both.append(k, v, [0, 1, 2, 3], held, table, uniform=1)
        now = [n + 1 for n in held]
        out, lse = both.gpu.attention(q, i32(torch, now), t, with_lse=True)
        check_decode(both, q, now, table, [1] * 3, dim ** -0.5, True, out, lse)
