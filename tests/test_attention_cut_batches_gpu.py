"""The cache's calls with bounds and prefix sums that do not fit: what is left out is what the header says, and the
rest is as if nothing had been."""
import numpy as np
import pytest

from test_attention_gpu import Both, check_decode, f64, filled, i32, lib, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [True, False])
def test_queries_that_are_left_out_leave_the_others_as_they_are(causal):
    """Queries beyond max_q and rows outside [0, n_rows) are not computed; the others see the same tokens."""
    torch, A = lib()
    lens = [40, 7, 300]
    both, table = filled("int8", lens, 16, 2, 64, 300)
    t, n = i32(torch, table), i32(torch, lens)
    q = make(torch, (18, 4, 64), torch.bfloat16, 1)
    want, want_lse = both.gpu.attention(q, n, t, cu_q=i32(torch, [0, 6, 9, 18]), max_q=9, causal=causal, with_lse=True)
    check_decode(both, q, lens, table, [6, 3, 9], 64 ** -0.5, causal, want, want_lse)
    out, lse = torch.full_like(q, 9.0), torch.full((18, 4), 9.0, device="cuda")
    both.gpu.attention(q, n, t, cu_q=i32(torch, [0, 6, 9, 18]), max_q=4, causal=causal, out=out, lse=lse)
    for a, b in ((0, 4), (6, 9), (9, 13)):
        assert torch.equal(out[a:b], want[a:b]) and torch.equal(lse[a:b], want_lse[a:b])
    for a, b in ((4, 6), (13, 18)):
        assert (out[a:b] == 9.0).all() and (lse[a:b] == 9.0).all()
    # the same batch two rows lower, of which a call gets 14: rows -2, -1 and 14, 15 do not exist
    out, lse = torch.full_like(q[2:16], 9.0), torch.full((14, 4), 9.0, device="cuda")
    both.gpu.attention(q[2:16].contiguous(), n, t, cu_q=i32(torch, [-2, 4, 7, 16]), max_q=9, causal=causal, out=out, lse=lse)
    assert torch.equal(out, want[2:16]) and torch.equal(lse, want_lse[2:16])


def test_tokens_beyond_max_len_are_not_seen():
    """Query i sees token j <= i + lens[r] - Lq, and of these those below max_len."""
    torch, A = lib()
    both, table = filled("e4m3", [40], 16, 1, 64, 310)
    t = i32(torch, table)
    q = make(torch, (6, 2, 64), torch.float16, 2)
    got = both.gpu.attention(q, i32(torch, [40]), t, max_len=30, with_lse=True)          # all see 30 or more
    want = both.gpu.attention(q, i32(torch, [30]), t, causal=False, with_lse=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    got = both.gpu.attention(q, i32(torch, [40]), t, max_len=37, with_lse=True)          # the first three see 35 .. 37
    want = both.gpu.attention(q[:3], i32(torch, [37]), t, with_lse=True)
    assert all(torch.equal(a[:3], b) for a, b in zip(got, want))


@pytest.mark.parametrize("form", ["int8", "e4m3"])
@pytest.mark.parametrize("page,lo,hi", [(16, -3, 30), (16, -20, 30), (64, -2, 2)])
def test_append_drops_rows_before_the_first(form, page, lo, hi):
    """A sequence that begins before row 0: its tokens of rows 0 .. are stored at their places."""
    torch, A = lib()
    both = Both(form, 8, 2, page, 64)
    for x in (both.gpu.k, both.gpu.v):
        x.view(torch.uint8).fill_(0)
    both.gpu.k_scale.zero_(), both.gpu.v_scale.zero_()
    k, v = make(torch, (hi, 2, 64), torch.bfloat16, 3), make(torch, (hi, 2, 64), torch.bfloat16, 4)
    table = np.array([[2, 5, 1, 7]])
    both.gpu.append(k, v, i32(torch, [1]), i32(torch, table), i32(torch, [lo, hi]), max_new=hi - lo)
    both.ref.append(f64(k), f64(v), 1 - lo, list(table[0]))
    both.check_rows([1 - lo + hi], table, torch.bfloat16)


def test_rows_of_sequences_that_begin_before_the_first_row():
    """And bounds far above the batch's: every row there is, is written, and no other."""
    torch, A = lib()
    both, table = filled("int8", [200, 90], 32, 2, 64, 330)
    t, first = i32(torch, table), i32(torch, [10, 3])
    want = both.gpu.rows(t, i32(torch, [0, 150, 230]), 230, first=first)
    for most in (230, 100000, 1 << 30):
        got = [torch.full((140, 2, 64), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        both.gpu.rows(t, i32(torch, [-70, 80, 160]), 140, first=first, max_len=most, k=got[0], v=got[1])
        for a, b in zip(got, want):
            assert torch.equal(a, b[70:210])
    got = torch.full((140, 2, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    both.gpu.rows(t, i32(torch, [-70, 80, 160]), 140, first=first, max_len=100, k=got)
    assert torch.equal(got[:30], want[0][70:100]) and (got[30:80] == 5.0).all() and torch.equal(got[80:], want[0][150:210])
