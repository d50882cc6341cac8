"""Bounds of a batch that are larger than 32 bits hold, and negative ones, through the binding."""
import pytest

from test_attention_gpu import filled, i32, lib, make

pytestmark = pytest.mark.gpu


def test_counts_beyond_32_bits():
    """"All of them", written as a large number."""
    torch, A = lib()
    both, table = filled("int8", [50, 20], 16, 1, 64, 320)
    t, c, n = i32(torch, table), i32(torch, [0, 50, 70]), i32(torch, [50, 20])
    want = both.gpu.rows(t, c, 70)
    for most in (1 << 32, (1 << 32) + 3, 1 << 63):
        got = both.gpu.rows(t, c, 70, max_len=most, k=torch.full_like(want[0], 5.0), v=torch.full_like(want[1], 5.0))
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    q = make(torch, (5, 2, 64), torch.bfloat16, 5)
    cq = i32(torch, [0, 3, 5])
    want, _ = both.gpu.attention(q, n, t, cu_q=cq, max_q=3)
    got, _ = both.gpu.attention(q, n, t, cu_q=cq, max_q=1 << 32, max_len=1 << 40, out=torch.full_like(q, 9.0))
    assert torch.equal(got, want)
    other, _ = filled("int8", [50, 20], 16, 1, 64, 320)
    k, v = make(torch, (6, 1, 64), torch.bfloat16, 6), make(torch, (6, 1, 64), torch.bfloat16, 7)
    for b, most in ((both, 4), (other, 1 << 32)):
        b.gpu.append(k, v, n, t, i32(torch, [0, 4, 6]), max_new=most)
    assert torch.equal(both.gpu.k[t[t >= 0].long()], other.gpu.k[t[t >= 0].long()])
    for bad in (lambda: both.gpu.rows(t, c, 70, max_len=-(1 << 32)), lambda: both.gpu.append(k, v, n, t, cq, max_new=-1),
                lambda: both.gpu.attention(q, n, t, cu_q=cq, max_q=-(1 << 32)),
                lambda: both.gpu.attention(q, n, t, max_len=-(1 << 32), cu_q=cq)):
        with pytest.raises((ValueError, RuntimeError)):
            bad()
    wide = q[:1].expand((1 << 32) + 5, -1, -1)             # more rows than the calls count
    kw = k[:1].expand((1 << 32) + 6, -1, -1)
    for bad in (lambda: both.gpu.attention(wide, n, t, cu_q=cq, max_q=3, out=wide), lambda: both.gpu.append(kw, kw, n, t, cq, max_new=4)):
        with pytest.raises(ValueError):
            bad()
