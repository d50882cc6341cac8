"""Prompts in pieces on the GPU against the float64 reference: rotary positions, the paged 16-bit cache's append, the
attention of new tokens over it, and all of them as one chain.

Tolerances.  Rotation: a turn is good to 2^-26 of a whole one (32 bits of it, rounded to a float of an eighth of a turn
at most), 2^-23.3 radians; the series and fp32's own steps add less than 2^-23; with the products' rounding the two sums
are off by at most 2^-21.5 (|x| + |y|), and rounded by half a step u of the element type (2^-25 absolute below fp16's
normal range).  What passes is equal.  Attention: as derived in test_attention_gpu.py, whose check() is taken here;
weights are rounded to the element type, fp16's lifted as in prompt attention."""
import numpy as np
import pytest

from oracle import paged as OP
from test_attention_gpu import HALF, check, cu, f64, make

pytestmark = pytest.mark.gpu

DTYPES = ["bfloat16", "float16"]


def lib():
    import torch
    from paper_2609_31551_amd import paged as B
    return torch, B


def i32(torch, x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def plan_of(B, sections, theta=10000.0, per_axis=False, adjacent=False):
    """The plan, and its frequencies and axes for the reference."""
    n = sum(sections)
    axis = [a for a, m in enumerate(sections) for _ in range(m)]
    freqs = [theta ** (-j / m) for m in sections for j in range(m)] if per_axis else [theta ** (-i / n) for i in range(n)]
    return B.Rotary.sections(sections, theta, per_axis=per_axis, adjacent=adjacent), (freqs, axis, adjacent)


def check_rotated(got, x, positions, ref, u, inverse=False):
    """got and x: GPU tensors."""
    freqs, axis, adjacent = ref
    X = f64(x)
    want = OP.rotate(X, positions, freqs, axis, adjacent, inverse)
    n = len(freqs)
    size = np.zeros(X.shape)
    first = np.arange(n) * 2 if adjacent else np.arange(n)
    second = first + 1 if adjacent else first + n
    size[..., first] = size[..., second] = np.abs(X[..., first]) + np.abs(X[..., second])
    tol = np.where(size > 0, 2.0 ** -21.5 * size + u * np.abs(want) * (1 + 2.0 ** -20) + 2.0 ** -25, 0.0)
    bad = ~(np.abs(f64(got) - want) <= tol)
    assert not bad.any(), "%d of %d off, worst %.3g of its tolerance" % (
        bad.sum(), bad.size, np.nanmax(np.abs(f64(got) - want) / np.maximum(tol, 1e-300)))
    assert (f64(got)[..., 2 * n:] == X[..., 2 * n:]).all()


# ---- rotary rows ----------------------------------------------------------------------

SECTIONS = [((32,), 64), ((8, 12, 12), 64), ((16, 24, 24), 128), ((0, 32, 32), 128), ((8, 16, 16), 80), ((4, 2, 1, 1), 64),
            ((8,), 16), ((24, 40), 256), ((128,), 256), ((40, 16), 112)]


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("sections,dim", SECTIONS, ids=str)
@pytest.mark.parametrize("dtype", DTYPES)
def test_rotary_rows(dtype, sections, dim, adjacent):
    torch, B = lib()
    dt, u = getattr(torch, dtype), HALF[dtype]
    rng = np.random.default_rng(dim)
    rot, ref = plan_of(B, sections, 5e5, per_axis=len(sections) == 2, adjacent=adjacent)
    for rows, heads, kv_heads in ((1, 1, 1), (7, 5, 1), (65, 28, 4), (300, 3, 2)):
        print("[rotary] %s %s %s rows %d" % (dtype, sections, adjacent, rows), flush=True)
        q, k = make(torch, (rows, heads, dim), dt, 1), make(torch, (rows, kv_heads, dim), dt, 2, 5.0)
        pos = rng.integers(-100, 40000, (len(sections), rows))
        pos[:, 0] = 0
        q2, k2 = rot.rows(q, i32(torch, pos), k)
        check_rotated(q2, q, pos, ref, u)
        check_rotated(k2, k, pos, ref, u)
        back, none = rot.rows(q, i32(torch, pos), inverse=True)
        check_rotated(back, q, pos, ref, u, inverse=True)
        assert none is None
        alone, _ = rot.rows(q, i32(torch, pos[:1]).expand(len(sections), rows) if len(sections) > 1 else i32(torch, pos))
        same, _ = rot.rows(q, i32(torch, pos[0]))
        assert torch.equal(alone, same)


def test_rotary_of_many_rows_is_that_of_few():
    """Launches of several rows a workgroup: bit for bit those of one."""
    torch, B = lib()
    rot, ref = plan_of(B, (16, 24, 24), 1e6)
    rows = 9001
    q, k = make(torch, (rows, 6, 128), torch.bfloat16, 3), make(torch, (rows, 2, 128), torch.bfloat16, 4)
    pos = np.random.default_rng(0).integers(0, 1 << 20, (3, rows))
    q2, k2 = rot.rows(q, i32(torch, pos), k)
    for a in (0, 500, 8990):
        s = slice(a, min(a + 40, rows))
        check_rotated(q2[s], q[s], pos[:, s], ref, 2.0 ** -8)
        q1, k1 = rot.rows(q[s], i32(torch, pos[:, s]), k[s])
        assert torch.equal(q1, q2[s]) and torch.equal(k1, k2[s])


def test_rotary_at_far_positions():
    torch, B = lib()
    rot, ref = plan_of(B, (16, 16), 1e4)
    pos = np.array([[0, 1, -1, 131072, 1 << 20, (1 << 31) - 1, -(1 << 31), 12345678],
                    [7, 1 << 30, -5, 99999, 0, -(1 << 31), (1 << 31) - 1, 777777777]])
    q = make(torch, (8, 4, 64), torch.float16, 5)
    check_rotated(rot.rows(q, i32(torch, pos))[0], q, pos, ref, 2.0 ** -11)


def test_rotary_strides_and_in_place():
    torch, B = lib()
    rot, ref = plan_of(B, (8, 12, 12), 1e4)
    pos = np.random.default_rng(1).integers(0, 3000, (3, 77))
    qkv = make(torch, (77, 10, 64), torch.bfloat16, 6)          # six query heads, two of keys, two of values
    want_q, want_k = rot.rows(qkv[:, :6].contiguous(), i32(torch, pos), qkv[:, 6:8].contiguous())
    wide = i32(torch, np.concatenate([pos, pos], 1))
    q, k = rot.rows(qkv[:, :6], wide[:, 77:], qkv[:, 6:8])      # positions with an axis stride of their own
    assert torch.equal(q, want_q) and torch.equal(k, want_k)
    by_head = torch.empty((6, 77, 64), dtype=q.dtype, device="cuda").transpose(0, 1)
    q, _ = rot.rows(qkv[:, :6], i32(torch, pos), q_out=by_head)
    assert q is by_head and torch.equal(q, want_q)
    one = qkv[:1, :1].expand(77, 6, 64)                         # the same row and head for all
    assert torch.equal(rot.rows(one, i32(torch, pos), q_out=torch.empty_like(want_q))[0],
                       rot.rows(one.contiguous(), i32(torch, pos))[0])
    whole = qkv.clone()
    q, k = rot.rows(whole[:, :6], i32(torch, pos), whole[:, 6:8], q_out=whole[:, :6], k_out=whole[:, 6:8])
    assert torch.equal(whole[:, :6], want_q) and torch.equal(whole[:, 6:8], want_k)
    assert torch.equal(whole[:, 8:], qkv[:, 8:])


def test_rotary_gradient():
    """The inverse of the outputs' gradients: against the reference's transposed rotation, and against differences of a
    weighted sum of the rotated rows."""
    torch, B = lib()
    rot, (freqs, axis, adjacent) = plan_of(B, (8, 4, 4), 1e3, adjacent=True)
    pos = np.random.default_rng(2).integers(0, 500, (3, 9))
    x, w = make(torch, (9, 2, 64), torch.float16, 7), make(torch, (9, 2, 64), torch.float16, 8)
    got, _ = rot.rows(w, i32(torch, pos), inverse=True)
    check_rotated(got, w, pos, (freqs, axis, adjacent), 2.0 ** -11, inverse=True)
    X, W, G = f64(x), f64(w), f64(got)
    rng = np.random.default_rng(3)
    for _ in range(5):   # the map is linear: a difference of 1 is exact
        step = rng.normal(size=X.shape)
        diff = (W * (OP.rotate(X + step, pos, freqs, axis, adjacent) - OP.rotate(X, pos, freqs, axis, adjacent))).sum()
        slack = (np.abs(step) * (2.0 ** -11 * np.abs(G) + 2.0 ** -20 * np.abs(W).max())).sum() + 1e-9
        assert abs((G * step).sum() - diff) <= slack


def test_rotary_refusals():
    torch, B = lib()
    rot = B.Rotary.sections((16, 16))
    q, pos = make(torch, (5, 2, 64), torch.bfloat16, 9), i32(torch, np.zeros((2, 5)))
    for bad in (dict(positions=pos[:, :4]), dict(positions=pos.long()), dict(positions=pos.t().contiguous().t()),
                dict(positions=pos.cpu()), dict(positions=i32(torch, np.zeros((3, 5)))), dict(q=q[:, :, :48]),
                dict(q=q.float()), dict(q=q.cpu()), dict(k=q[:4]), dict(k=q.half()), dict(q_out=q[:4]),
                dict(k_out=q), dict(q=q[..., ::2])):
        args = dict(dict(q=q, positions=pos), **bad)
        with pytest.raises((ValueError, RuntimeError)):
            rot.rows(**args)
    torch.cuda.synchronize()


# ---- append ---------------------------------------------------------------------------

def pages_of(lens, page, seed, extra=0, slack=0):
    """A page table for sequences of `lens` tokens, shuffled, -1 where none is needed, and the number of pages."""
    need = [-(-n // page) + slack for n in lens]
    order = np.random.default_rng(seed).permutation(sum(need) + extra)
    table = np.full((len(lens), max(max(need), 1)), -1, np.int64)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    return table, max(sum(need) + extra, 1)


class Both:
    """The cache on the GPU and the reference, both full of 9."""

    def __init__(self, dtype, n_pages, heads, page, dim):
        torch, B = lib()
        self.gpu = B.Kv16Cache.empty(n_pages, heads, dim, page, getattr(torch, dtype))
        self.gpu.k.fill_(9.0)
        self.gpu.v.fill_(9.0)
        self.ref = OP.Cache(n_pages, heads, page, dim, 9.0)

    def check_values(self):
        np.testing.assert_array_equal(f64(self.gpu.v), self.ref.v)

    def check_keys(self):
        np.testing.assert_array_equal(f64(self.gpu.k), self.ref.k)


@pytest.mark.parametrize("rotated", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page,heads,kv_heads,dim", [(16, 4, 2, 64), (32, 7, 1, 128), (64, 12, 3, 128), (128, 1, 1, 64)])
def test_append(dtype, page, heads, kv_heads, dim, rotated):
    torch, B = lib()
    dt = getattr(torch, dtype)
    rot, ref = plan_of(B, (8, 12, 12), 1e4, adjacent=page == 32)
    held = [0, 5, 16, 33, 200, 1, 0]
    both = None
    for step, new in enumerate(([3, 1, 70, 0, 57, 128, 1], [1] * 7)):
        total = [a + b for a, b in zip(held, new)]
        if both is None:
            table, n_pages = pages_of([n + 1 for n in total], page, 3, extra=2)
            both = Both(dtype, n_pages, kv_heads, page, dim)
        rows = sum(new)
        k, v, q = (make(torch, (rows, h, dim), dt, 10 * step + h, 2.0) for h in (kv_heads, kv_heads, heads))
        pos = np.random.default_rng(step).integers(0, 9000, (3, rows))
        where = dict(cu_new=i32(torch, cu(new)), max_new=max(new)) if step == 0 else {}
        more = dict(rotary=rot, positions=i32(torch, pos), q=q) if rotated else {}
        print("[append] %s page %d step %d" % (dtype, page, step), flush=True)
        out = both.gpu.append(k, v, i32(torch, held), i32(torch, table), **where, **more)
        if rotated:
            turned_q, turned_k = rot.rows(q, i32(torch, pos), k)       # the same arithmetic, bit for bit
            assert torch.equal(out, turned_q)
            check_rotated(turned_k, k, pos, ref, HALF[dtype])
        else:
            assert out is None
            turned_k = k
        c = cu(new)
        for r in range(len(new)):
            both.ref.append(f64(turned_k)[c[r]:c[r + 1]], f64(v)[c[r]:c[r + 1]], held[r], table[r])
        both.check_keys()
        both.check_values()
        held = total


def test_append_at_the_places_of_tokens():
    """Without positions a token's place turns it, on all axes; a batch of more than 64 sequences."""
    torch, B = lib()
    rot, ref = plan_of(B, (8, 12, 12), 1e4)
    rng = np.random.default_rng(4)
    held, new = rng.integers(0, 90, 150), rng.integers(0, 4, 150)
    table, n_pages = pages_of(held + new, 16, 5)
    k, v, q = (make(torch, (int(new.sum()), h, 64), torch.float16, 20 + h) for h in (2, 3, 4))
    v = v[:, :2]
    place = np.concatenate([np.arange(a, a + b) for a, b in zip(held, new)])
    want = []
    for positions in (None, i32(torch, place), i32(torch, np.stack([place] * 3))):
        both = Both("float16", n_pages, 2, 16, 64)
        out = both.gpu.append(k, v, i32(torch, held), i32(torch, table), cu_new=i32(torch, cu(new)), max_new=3, rotary=rot,
                              positions=positions, q=q)
        want.append((out, both.gpu.k, both.gpu.v))
    check_rotated(want[0][0], q, np.stack([place] * 3), ref, 2.0 ** -11)
    for other in want[1:]:
        assert all(torch.equal(a, b) for a, b in zip(want[0], other))


@pytest.mark.parametrize("n,most", [(1, 9), (63, 2), (64, 1), (65, 3), (130, 1), (4096, 1), (4097, 4), (9000, 2)])
def test_append_finds_the_sequence_of_a_row(n, most):
    """Batches of few and of many sequences, runs of empty ones among them, at the ends too: every row in its place."""
    torch, B = lib()
    rot, _ = plan_of(B, (32,), 1e4)
    rng = np.random.default_rng(n)
    for case, new in enumerate((rng.integers(0, most + 1, n), np.where(rng.random(n) < 0.02, most, 0),
                                np.where(np.arange(n) == n // 2, most, 0))):
        rows = int(new.sum())
        if rows == 0:
            continue
        print("[sequence of a row] %d sequences, case %d, %d rows" % (n, case, rows), flush=True)
        held, pages = rng.integers(0, 16 - most, n), rng.permutation(n)
        cache = B.Kv16Cache.empty(n, 1, 64, 16)
        cache.k.zero_(), cache.v.zero_()
        k, v, q = (make(torch, (rows, 1, 64), torch.bfloat16, 50 + i) for i in range(3))
        out = cache.append(k, v, i32(torch, held), i32(torch, pages[:, None]), cu_new=i32(torch, cu(new)), max_new=most,
                           rotary=rot, q=q)
        seq = np.repeat(np.arange(n), new)
        place = np.concatenate([np.arange(a, a + b) for a, b in zip(held, new)])
        turned_q, turned_k = rot.rows(q, i32(torch, place), k)
        assert torch.equal(out, turned_q)
        want_k, want_v = torch.zeros_like(cache.k), torch.zeros_like(cache.v)
        at = i32(torch, pages[seq]).long(), i32(torch, place).long()
        want_k[at[0], 0, at[1]], want_v[at[0], 0, at[1]] = turned_k[:, 0], v[:, 0]
        assert torch.equal(cache.k, want_k) and torch.equal(cache.v, want_v)


def test_append_drops_what_has_no_place():
    torch, B = lib()
    rot, _ = plan_of(B, (32,), 1e4)
    both = Both("bfloat16", 6, 1, 16, 64)
    # pages that are not held, lengths at the table's end, a sequence left out, rows of no sequence
    table = np.array([[0, -1, 1], [2, 6, 3], [4, 5, -7], [1, 1, 1]])
    held, new = [10, 10, 40, -3], [30, 30, 20, 5]
    c = [2] + [2 + x for x in np.cumsum(new)]                      # rows 0, 1 and those behind belong to none
    rows = c[-1] + 3
    k, v, q = (make(torch, (rows, 1, 64), torch.bfloat16, s) for s in (30, 31, 32))
    q_out = torch.full_like(q, 5.0)
    out = both.gpu.append(k, v, i32(torch, held), i32(torch, table), cu_new=i32(torch, c), max_new=25, rotary=rot, q=q,
                          q_out=q_out)
    assert out is q_out
    place = np.zeros(rows, np.int64)
    mine = np.zeros(rows, bool)
    for r in range(3):
        n = min(new[r], 25)
        place[c[r]:c[r] + n], mine[c[r]:c[r] + n] = np.arange(held[r], held[r] + n), True
    turned_q, turned_k = rot.rows(q, i32(torch, place), k)
    assert (out[~mine] == 5.0).all() and torch.equal(out[mine], turned_q[mine])
    for r in range(3):
        s = slice(c[r], c[r] + min(new[r], 25))
        both.ref.append(f64(turned_k)[s], f64(v)[s], held[r], table[r])
    both.check_keys()
    both.check_values()
    # prefix sums beyond the rows, and the same number for all with sequences that have none
    both.gpu.append(k[:4], v[:4], i32(torch, [0, 0]), i32(torch, table[:2]), cu_new=i32(torch, [0, 2, 1 << 30]), max_new=9)
    both.ref.append(f64(k)[:2], f64(v)[:2], 0, table[0])
    both.ref.append(f64(k)[2:4], f64(v)[2:4], 0, table[1])
    both.check_keys()


def test_append_refusals():
    torch, B = lib()
    rot = B.Rotary.sections((32,))
    c = B.Kv16Cache.empty(4, 2, 64, 16)
    x, h, t = make(torch, (3, 2, 64), torch.bfloat16, 40), i32(torch, [0, 0, 0]), i32(torch, [[0], [1], [2]])
    for bad in (dict(k=x.half()), dict(v=x[:2]), dict(k=x[:, :1]), dict(held=h[:2]), dict(held=h.long()), dict(pages=t.long()),
                dict(pages=t[0]), dict(max_new=2), dict(q=x), dict(positions=h), dict(rotary=rot, q=x[:2]),
                dict(rotary=rot, q_out=x), dict(rotary=rot, q=x.half()), dict(rotary=rot, positions=i32(torch, [0, 0])),
                dict(rotary=B.Rotary.sections((64,))), dict(cu_new=i32(torch, [0, 3]))):
        with pytest.raises((ValueError, RuntimeError)):
            c.append(**dict(dict(k=x, v=x, held=h, pages=t), **bad))
    torch.cuda.synchronize()


# ---- attention ------------------------------------------------------------------------

def filled(dtype, lens, page, heads, dim, seed, **more):
    """A cache with `lens` tokens of each sequence in it, and NaN wherever no token is."""
    torch, B = lib()
    table, n_pages = pages_of(lens, page, seed, **more)
    both = Both(dtype, n_pages, heads, page, dim)
    for x in (both.gpu.k, both.gpu.v):
        x.fill_(float("nan"))
    both.ref.k[:], both.ref.v[:] = np.nan, np.nan
    k, v = (make(torch, (sum(lens), heads, dim), getattr(torch, dtype), seed + i, 2.0 - i) for i in (0, 1))
    both.gpu.append(k, v, i32(torch, [0] * len(lens)), i32(torch, table), cu_new=i32(torch, cu(lens)), max_new=max(lens))
    c = cu(lens)
    K, V = f64(k), f64(v)
    for r in range(len(lens)):
        both.ref.append(K[c[r]:c[r + 1]], V[c[r]:c[r + 1]], 0, table[r])
    return both, table


def check_attention(both, q, lens, table, new, scale, causal, out, lse, only=None):
    """Every sequence's rows against the reference; lse a tensor."""
    c, dim = cu(new), q.shape[2]
    dtype = str(q.dtype)[6:]
    Q, O, L = f64(q), f64(out), f64(lse)
    group = q.shape[1] // both.ref.k.shape[1]
    for r in range(len(lens)) if only is None else only:
        a = slice(c[r], c[r + 1])
        if new[r] == 0:
            continue
        ref, ref_lse, size = both.ref.attention(Q[a], lens[r], table[r], scale, causal)
        held = [p for p in table[r][:-(-lens[r] // both.ref.page)] if 0 <= p < both.ref.k.shape[0]]
        k = np.nan_to_num(both.ref.k[held]).reshape(len(held), both.ref.k.shape[1], both.ref.page, dim)
        v = np.abs(np.nan_to_num(both.ref.v[held]))
        total = np.repeat(v.sum((0, 2)), group, 0)[None] if held else np.zeros((1, q.shape[1], dim))
        top = np.repeat(np.linalg.norm(k, axis=3).max((0, 2)), group, 0)[None] if held else np.zeros((1, q.shape[1]))
        delta = dim * 2.0 ** -24 * abs(scale) * np.linalg.norm(Q[a], axis=2) * top
        check(O[a], L[a], ref, ref_lse, size, delta, total, np.full(delta.shape, lens[r]), HALF[dtype],
              2.0 ** -32 if dtype == "float16" else 0.0)


def attend(both, q, lens, table, new, causal=True, scale=None, **more):
    torch, B = lib()
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    both.gpu.attention(q, i32(torch, lens), i32(torch, table), cu_q=i32(torch, cu(new)), max_q=max(new), causal=causal,
                       scale=scale, out=out, lse=lse, **more)
    torch.cuda.synchronize()
    n = sum(new)
    assert (out[n:] == 7.0).all() and (lse[n:] == 7.0).all()
    return out, lse


NEW = {
    "tokens": ([1, 1, 1, 1, 1, 1], [1, 2, 33, 64, 300, 129]),
    "few": ([2, 5, 3, 9, 0, 4], [2, 100, 33, 9, 50, 515]),
    "chunks": ([63, 64, 65, 127, 128, 130], [63, 200, 65, 128, 129, 333]),
    "mixed": ([1, 140, 1, 31, 7, 1], [400, 140, 1, 100, 64, 77]),
    "more_than_held": ([30, 9, 70, 3], [20, 0, 64, 1]),                     # first queries see nothing
    "runs": ([1, 5, 150, 1, 33], [5000, 2100, 2600, 90, 1300]),
}


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("new", list(NEW))
@pytest.mark.parametrize("page,heads,kv_heads,dim", [(16, 4, 4, 64), (64, 14, 2, 128), (32, 20, 1, 64), (128, 5, 5, 128)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_attention(dtype, page, heads, kv_heads, dim, new, causal):
    torch, B = lib()
    new, lens = NEW[new]
    print("[attention] %s %s page %d heads %d" % (dtype, new, page, heads), flush=True)
    both, table = filled(dtype, lens, page, kv_heads, dim, 50, extra=1)
    q = make(torch, (sum(new) + 2, heads, dim), getattr(torch, dtype), 60)
    q[sum(new):] = float("nan")
    out, lse = attend(both, q, lens, table, new, causal, max_len=max(lens))
    check_attention(both, q, lens, table, new, dim ** -0.5, causal, out, lse)


@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0, 1e-30])
@pytest.mark.parametrize("new", [[1, 1], [100, 60]])
def test_attention_scales(new, scale):
    torch, _ = lib()
    both, table = filled("bfloat16", [260, 70], 32, 2, 64, 70)
    q = make(torch, (sum(new), 4, 64), torch.bfloat16, 71)
    out, lse = attend(both, q, [260, 70], table, new, scale=scale)
    check_attention(both, q, [260, 70], table, new, float(np.float32(scale)), True, out, lse)


def test_attention_without_prefix_sums_and_with_strides():
    torch, B = lib()
    lens = [130, 5, 600]
    both, table = filled("float16", lens, 16, 2, 128, 80)
    for each in (1, 4, 70):
        lens2 = [max(n, each) for n in lens] if each < 5 else [130, 70, 600]
        if each == 70:
            both, table = filled("float16", lens2, 16, 2, 128, 81)
        q = make(torch, (3 * each, 6, 128), torch.float16, 82)
        want = both.gpu.attention(q, i32(torch, lens2), i32(torch, table), cu_q=i32(torch, cu([each] * 3)), max_q=each,
                                  with_lse=True)
        check_attention(both, q, lens2, table, [each] * 3, 128 ** -0.5, True, *want)
        fused = torch.cat([q, q], 1)
        by_head = torch.empty((6, 3 * each, 128), dtype=q.dtype, device="cuda").transpose(0, 1)
        for args in (dict(q=q), dict(q=fused[:, 6:]), dict(q=q, out=by_head), dict(q=q, max_q=each)):
            got = both.gpu.attention(lens=i32(torch, lens2), pages=i32(torch, table), with_lse=True, **args)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_attention_does_not_depend_on_the_batch_or_its_bounds():
    torch, _ = lib()
    lens, new = [700, 5, 1300, 256, 3000, 4100, 900], [1, 5, 40, 200, 1, 130, 2]
    both, table = filled("bfloat16", lens, 64, 2, 128, 90, extra=9)
    q = make(torch, (sum(new), 8, 128), torch.bfloat16, 91)
    every, lse = attend(both, q, lens, table, new)
    c = cu(new)
    for r, n in enumerate(lens):
        a = slice(c[r], c[r + 1])
        t, l = i32(torch, table[r:r + 1]), i32(torch, [n])
        for more in (dict(), dict(max_len=n), dict(cu_q=i32(torch, [0, new[r]]), max_q=new[r] + 300)):
            one, one_lse = both.gpu.attention(q[a], l, t, with_lse=True, **more)
            assert torch.equal(one, every[a]) and torch.equal(one_lse, lse[a]), (r, list(more))
        # other pages
        order = np.random.default_rng(r).permutation(both.gpu.n_pages)
        other, _ = filled("bfloat16", [1], 64, 2, 128, 0, extra=both.gpu.n_pages - 1)
        other.gpu.k[torch.tensor(order, device="cuda")], other.gpu.v[torch.tensor(order, device="cuda")] = both.gpu.k, both.gpu.v
        moved = np.where(table[r:r + 1] >= 0, order[np.maximum(table[r:r + 1], 0)], -1)
        one, _ = other.gpu.attention(q[a], l, i32(torch, moved))
        assert torch.equal(one, every[a]), r


@pytest.mark.parametrize("new", [1, 6, 150])
@pytest.mark.parametrize("page", [16, 64])
def test_attention_over_absent_pages(page, new):
    torch, B = lib()
    lens = [1000, 150 + new, 2000]
    both, table = filled("bfloat16", lens, page, 2, 64, 100)
    q = make(torch, (3 * new, 6, 64), torch.bfloat16, 101)
    gone = table.copy()
    gone[0, 1::3], gone[1, :], gone[2, :20] = -1, 1 << 30, -2
    gone[2, 5] = table[2, 5]
    for causal in (True, False):
        out, lse = attend(both, q, lens, gone, [new] * 3, causal)
        check_attention(both, q, lens, gone, [new] * 3, 0.125, causal, out, lse)
        assert (out[new:2 * new] == 0).all() and torch.isneginf(lse[new:2 * new]).all()


@pytest.mark.parametrize("what", ["nan", "inf", "-inf"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new,length,at", [(4, 40, 38), (9, 700, 695), (33, 33, 20), (200, 200, 130), (129, 700, 600),
                                           (64, 2500, 2440), (300, 130, 90), (40, 4200, 4170)])
def test_hidden_tokens_may_hold_anything(dtype, new, length, at, what):
    """The tokens from `at` on hold NaN or infinities: earlier queries are right, later ones' dimension is not finite."""
    torch, _ = lib()
    both, table = filled(dtype, [length], 32, 2, 128, 110)
    q = make(torch, (new, 4, 128), getattr(torch, dtype), 111)
    first = at - (length - new)
    clean = filled(dtype, [length], 32, 2, 128, 110)[0]
    for t in range(at, length):
        both.gpu.k[int(table[0, t // 32]), :, t % 32, 3] = float(what)
        both.gpu.v[int(table[0, t // 32]), :, t % 32, 5] = float(what)
    out, lse = attend(both, q, [length], table, [new])
    Q, ref = f64(q), clean.ref
    want, want_lse, size = ref.attention(Q, length, table[0], 128 ** -0.5, True)
    K = ref.k[table[0]].transpose(1, 0, 2, 3).reshape(2, -1, 128)[:, :length]
    V = np.abs(ref.v[table[0]].transpose(1, 0, 2, 3).reshape(2, -1, 128)[:, :length])
    top, total = np.repeat(np.linalg.norm(K, axis=2).max(1), 2)[None], np.repeat(V.sum(1), 2, 0)[None]
    delta = 128 * 2.0 ** -24 * 128 ** -0.5 * np.linalg.norm(Q, axis=2) * top
    s = slice(0, first)
    check(f64(out)[s], f64(lse)[s], want[s], want_lse[s], size[s], delta[s], np.broadcast_to(total, size.shape)[s],
          np.full(delta.shape, length)[s], HALF[dtype], 2.0 ** -32 if dtype == "float16" else 0.0)
    if what != "-inf":   # a score of -inf weighs nothing
        assert not torch.isfinite(out[first:, :, 5]).any()


@pytest.mark.parametrize("new", [1, 70])
def test_infinite_scores(new):
    """Keys whose scores are all -inf weigh nothing, wherever they stand; +inf makes a query's result NaN."""
    torch, _ = lib()
    for length, gone in ((300, slice(0, 200)), (300, slice(100, 229)), (3000, slice(0, 2500))):
        both, table = filled("bfloat16", [length], 16, 1, 64, 120)
        q = make(torch, (new, 2, 64), torch.bfloat16, 121).abs()
        ids = np.arange(length)[gone]
        pages, slots = torch.tensor(table[0][ids // 16], device="cuda"), torch.tensor(ids % 16, device="cuda")
        both.gpu.k[pages, :, slots, 7] = -float("inf")
        out, lse = attend(both, q, [length], table, [new])
        kept = np.delete(np.arange(length), ids)
        Q = f64(q)
        k = np.stack([both.ref.k[table[0][t // 16], :, t % 16] for t in kept])
        v = np.stack([both.ref.v[table[0][t // 16], :, t % 16] for t in kept])
        from oracle import attention as O
        for h in range(2):
            sees = O.visible(new, length, True)[:, kept]
            want, want_lse = O.attention(Q[:, h], k[:, 0], v[:, 0], 0.125, sees)
            some = ~np.isneginf(want_lse)
            np.testing.assert_allclose(f64(out)[:, h], want, atol=0.05, rtol=0.02)   # bf16: 2^-8 of sums of |v| up to 6
            np.testing.assert_array_equal(np.isneginf(f64(lse)[:, h]), ~some)
            np.testing.assert_allclose(f64(lse)[some, h], want_lse[some], atol=2e-4, rtol=1e-5)
        both.gpu.k[int(table[0, 0]), :, 0, 7] = float("inf")
        out, lse = attend(both, q, [length], table, [new])
        assert torch.isnan(out).all() and torch.isnan(lse).all()


@pytest.mark.parametrize("new", [1, 60])
@pytest.mark.parametrize("dtype", DTYPES)
def test_small_weights_count(dtype, new):
    """4,095 tokens of 2^-25.3 of the first one's weight each, whose value is 0."""
    torch, B = lib()
    n, dt = 4096, getattr(torch, dtype)
    cache = B.Kv16Cache.empty(n // 64, 1, 64, 64, dt)
    cache.k.zero_()
    cache.v.fill_(1.0)
    cache.k[0, 0, 0], cache.v[0, 0, 0] = 16.0, 0.0
    q = torch.zeros(new, 1, 64, dtype=dt, device="cuda")
    q[:, :, 0] = 1.0
    scale = float(np.float32(25.3 * np.log(2.0) / 16))
    out, _ = cache.attention(q, i32(torch, [n]), i32(torch, [np.arange(n // 64)]), scale=scale)
    small = 2.0 ** -25.3
    want = (n - new + np.arange(new)) * small / (1 + (n - new + np.arange(new)) * small)
    err = np.abs(f64(out)[:, 0] - want[:, None])
    # two half steps, the exponentials, and 2^-32 of each value's weight of the largest
    tol = (2 * HALF[dtype] + 2.0 ** -17) * want + (n * 2.0 ** -32 if dtype == "float16" else 0)
    assert (err <= tol[:, None]).all()


def test_bounds_that_are_smaller_than_the_batch():
    torch, B = lib()
    both, table = filled("float16", [40, 30], 16, 1, 64, 130)
    q = make(torch, (45, 2, 64), torch.float16, 131)
    for top in (2, 20):
        out = torch.full(q.shape, 9.0, dtype=q.dtype, device="cuda")
        both.gpu.attention(q, i32(torch, [20, 0]), i32(torch, table), cu_q=i32(torch, [0, 40, 45]), max_q=top, max_len=11,
                           causal=False, out=out)
        assert (out[top:40] == 9.0).all() and (out[40:40 + min(top, 5)] == 0).all()
        want, _ = attend(both, q[:40], [11], table[:1], [40], causal=False)
        np.testing.assert_allclose(f64(out[:top]), f64(want[:top]), atol=2e-2)
    # queries left out leave the others' places as they are
    full, _ = attend(both, q[:38], [40, 30], table, [30, 8])
    out = torch.full(q.shape, 9.0, dtype=q.dtype, device="cuda")
    both.gpu.attention(q[:33], i32(torch, [40, 30]), i32(torch, table), cu_q=i32(torch, [0, 30, 38]), max_q=9, out=out[:33])
    np.testing.assert_allclose(f64(out[:9]), f64(full[:9]), atol=2e-2)
    np.testing.assert_allclose(f64(out[30:33]), f64(full[30:33]), atol=2e-2)
    assert (out[9:30] == 9.0).all() and (out[33:] == 9.0).all()


def test_lengths_are_cut_to_the_table():
    torch, _ = lib()
    both, table = filled("bfloat16", [64, 64, 64], 32, 1, 64, 140)
    q = make(torch, (3, 2, 64), torch.bfloat16, 141)
    want, _ = both.gpu.attention(q, i32(torch, [64, 0, 64]), i32(torch, table))
    got, _ = both.gpu.attention(q, i32(torch, [1 << 30, -7, (1 << 31) - 1]), i32(torch, table))
    assert torch.equal(got, want) and (got[1] == 0).all()


def test_pages_shared_for_reading():
    torch, B = lib()
    both, table = filled("bfloat16", [100, 40], 16, 2, 64, 150)
    shared = table.copy()
    shared[1, :2] = table[0, :2]                       # the second sequence starts with the first one's pages
    q = make(torch, (2, 4, 64), torch.bfloat16, 151)
    out, lse = attend(both, q, [100, 40], shared, [1, 1])
    check_attention(both, q, [100, 40], shared, [1, 1], 0.125, True, out, lse)


def test_many_sequences():
    """More than a wave holds, of mixed kinds, some empty."""
    torch, _ = lib()
    rng = np.random.default_rng(160)
    new = [int(x) for x in rng.choice([0, 1, 1, 1, 2, 7, 40, 90], 200)]
    lens = [n + int(x) for n, x in zip(new, rng.integers(0, 70, 200))]
    both, table = filled("bfloat16", [max(n, 1) for n in lens], 16, 1, 64, 161)
    q = make(torch, (sum(new), 3, 64), torch.bfloat16, 162)
    out, lse = attend(both, q, lens, table, new)
    check_attention(both, q, lens, table, new, 0.125, True, out, lse)


def test_cache_behind_four_gib():
    torch, B = lib()
    page, dim, heads = 64, 128, 8
    n_pages = (5 << 30) // (page * dim * heads * 2)             # 5 GiB of keys, 5 of values
    cache, small = B.Kv16Cache.empty(n_pages, heads, dim, page), B.Kv16Cache.empty(8, heads, dim, page)
    k, v = (make(torch, (500, heads, dim), torch.bfloat16, s) for s in (170, 171))
    far, near = i32(torch, [[n_pages - 1 - i for i in range(8)]]), i32(torch, [list(range(8))])
    rot = B.Rotary.sections((16, 24, 24))
    for new in (1, 90):
        q = make(torch, (new, 16, dim), torch.bfloat16, 172)
        got = []
        for c, t in ((cache, far), (small, near)):
            c.append(k, v, i32(torch, [0]), t, rotary=rot)
            got.append(c.attention(q, i32(torch, [500]), t, with_lse=True))
        assert all(torch.equal(a, b) for a, b in zip(*got))


def test_empty_batches():
    torch, B = lib()
    cache = B.Kv16Cache.empty(2, 1, 64, 16)
    k = make(torch, (0, 1, 64), torch.bfloat16, 180)
    none, pages = i32(torch, []), torch.zeros((0, 3), dtype=torch.int32, device="cuda")
    rot = B.Rotary.sections((32,))
    assert cache.append(k, k, none, pages, rotary=rot, q=k).shape == (0, 1, 64)
    assert cache.attention(k, none, pages)[0].shape == (0, 1, 64)
    assert rot.rows(k, i32(torch, []), k)[1].shape == (0, 1, 64)
    q = make(torch, (1, 1, 64), torch.bfloat16, 181)
    out, lse = cache.attention(q, i32(torch, [0]), i32(torch, [[0]]), with_lse=True)
    assert (out == 0).all() and torch.isneginf(lse).all()


def test_attention_refusals():
    torch, B = lib()
    c = B.Kv16Cache.empty(4, 2, 64, 16)
    q, n, t = make(torch, (3, 4, 64), torch.bfloat16, 190), i32(torch, [1, 1, 1]), i32(torch, [[0], [1], [2]])
    for bad in (dict(q=q.half()), dict(q=q[:, :3]), dict(q=q[..., :32]), dict(lens=n[:2]), dict(lens=n.cpu()),
                dict(pages=t[0]), dict(pages=t.cpu()), dict(max_q=2), dict(cu_q=i32(torch, [0, 1, 3])), dict(out=q[:2]),
                dict(out=q.half()), dict(lse=n), dict(scale=float("nan")), dict(workspace=n)):
        with pytest.raises((ValueError, RuntimeError)):
            c.attention(**dict(dict(q=q, lens=n, pages=t), **bad))
    torch.cuda.synchronize()


# ---- streams, graphs, and the chain ---------------------------------------------------

def test_calls_on_two_streams_at_once():
    """Their workspaces are their own: calls that overlap give what they give alone."""
    torch, B = lib()
    lens, new = [5000, 3100, 900], [200, 1, 6]
    both, table = filled("bfloat16", lens, 64, 2, 128, 195)
    table, n, c = i32(torch, table), i32(torch, lens), i32(torch, cu(new))
    q = make(torch, (207, 8, 128), torch.bfloat16, 196)
    rot, pos = B.Rotary.sections((16, 24, 24)), i32(torch, np.arange(207))

    def calls(x, stream=None):
        x, _ = rot.rows(x, pos, stream=stream)
        return both.gpu.attention(x, n, table, cu_q=c, max_q=200, with_lse=True, stream=stream)
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


def test_a_step_in_a_graph():
    """Chunks and single tokens: append with rotation, attention, lengths moved on, captured once and replayed; every
    replay equals the same step run eagerly on another cache, with eager work and synchronizations between."""
    torch, B = lib()
    lens, new = [1250, 31, 700], [1, 40, 1]
    rot = B.Rotary.sections((16, 24, 24), 1e6)
    rows, state = sum(new), []
    for _ in range(2):
        both, table = filled("bfloat16", lens, 32, 2, 128, 200, slack=8)
        state.append(dict(c=both.gpu, t=i32(torch, table), held=i32(torch, lens), lens=i32(torch, lens) + i32(torch, new),
                          cu=i32(torch, cu(new)), pos=i32(torch, np.zeros((3, rows))),
                          **{x: make(torch, (rows, h, 128), torch.bfloat16, 0) for x, h in (("k", 2), ("v", 2), ("q", 6))}))

    def step(s):
        q = s["c"].append(s["k"], s["v"], s["held"], s["t"], s["cu"], max(new), rotary=rot, positions=s["pos"], q=s["q"])
        out = s["c"].attention(q, s["lens"], s["t"], s["cu"], max(new), with_lse=True)
        s["held"].add_(i32_new)
        s["lens"].add_(i32_new)
        return (q,) + out

    i32_new = i32(torch, new)
    fixed, eager = state
    saved = {n: fixed[n].clone() for n in ("held", "lens")}
    pages = fixed["c"].k.clone(), fixed["c"].v.clone()
    warm = torch.cuda.Stream()
    warm.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(warm):
        step(fixed)
    torch.cuda.current_stream().wait_stream(warm)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(fixed)
    for n, x in saved.items():
        fixed[n].copy_(x)
    fixed["c"].k.copy_(pages[0])
    fixed["c"].v.copy_(pages[1])
    for i in range(6):
        for n, seed in (("k", 300 + i), ("v", 310 + i), ("q", 320 + i)):
            x = make(torch, fixed[n].shape, torch.bfloat16, seed, 1.0 + i)
            fixed[n].copy_(x)
            eager[n].copy_(x)
        for s in state:
            s["pos"].add_(i + 3)
        graph.replay()
        want = step(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(captured, want)), "replay %d" % i
        held = fixed["t"][fixed["t"] >= 0].long()
        for x, y in ((fixed["c"].k, eager["c"].k), (fixed["c"].v, eager["c"].v)):
            assert torch.equal(x[held].view(torch.int16), y[held].view(torch.int16))


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_prompt_in_chunks_is_the_prompt_at_once(dtype):
    """A prompt's rotated chunks, appended and attended to one by one, beside another request's single tokens: every row
    is prompt attention's over the rotated rows, to both ways' bounds."""
    torch, B = lib()
    from paper_2609_31551_amd import attention as A
    from test_attention_gpu import prompt_bounds
    from oracle import attention as O
    dt = getattr(torch, dtype)
    total, other = 700, 90
    rot, ref = plan_of(B, (16, 24, 24), 1e4)
    rng = np.random.default_rng(5)
    pos = rng.integers(0, 2000, (3, total))
    q, k, v = (make(torch, (total, h, 128), dt, 210 + i) for i, h in enumerate((8, 2, 2)))
    q1, k1, v1 = (make(torch, (other, h, 128), dt, 220 + i) for i, h in enumerate((8, 2, 2)))
    both, table = filled(dtype, [total, other], 32, 2, 128, 230)
    both.gpu.k.fill_(float("nan"))
    both.gpu.v.fill_(float("nan"))
    t, outs, at = i32(torch, table), [], 0
    for step, n in enumerate((1, 130, 64, 257, 5, 243)):
        held = i32(torch, [at, step])
        new = [n, 1]
        rows = torch.cat([q[at:at + n], q1[step:step + 1]]), torch.cat([k[at:at + n], k1[step:step + 1]]), \
            torch.cat([v[at:at + n], v1[step:step + 1]])
        p = i32(torch, np.concatenate([pos[:, at:at + n], np.full((3, 1), step)], 1))
        c = i32(torch, cu(new))
        turned = both.gpu.append(rows[1], rows[2], held, t, c, n, rotary=rot, positions=p, q=rows[0])
        out, lse = both.gpu.attention(turned, held + i32(torch, new), t, c, n, max_len=at + n, with_lse=True)
        outs.append((out[:n], lse[:n]))
        at += n
    assert at == total
    out, lse = (torch.cat(x) for x in zip(*outs))
    rq, rk = rot.rows(q, i32(torch, pos), k)
    once, once_lse = A.prompt_attention(rq, rk, v, [0, total], with_lse=True)
    Q, K, V, c = f64(rq), f64(rk), f64(v), [0, total]
    want, want_lse = O.prompt_attention(Q, K, V, c, c, 128 ** -0.5, True)
    bounds = prompt_bounds(Q, K, V, c, c, 128 ** -0.5, True, HALF[dtype])
    for x, y in ((out, lse), (once, once_lse)):
        check(f64(x), f64(y), want, want_lse, *bounds, HALF[dtype], 2.0 ** -32 if dtype == "float16" else 0.0)
