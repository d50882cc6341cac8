"""What a query sees of NaN makes its result NaN, causal or not, and nobody else's."""
import pytest

from test_attention_gpu import HALF, lib, make

pytestmark = pytest.mark.gpu

NAN = float("nan")


def both(q, k, v, causal, cu_k=None):
    torch, A = lib()
    n = q.shape[0]
    return A.prompt_attention(q, k, v, [0, n], [0, k.shape[0]], causal=causal, with_lse=True)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,dim,lq,lk", [("bfloat16", 64, 200, 200), ("float16", 128, 70, 9000), ("bfloat16", 128, 300, 700)])
def test_nan_in_one_query(dtype, dim, lq, lk, causal):
    torch, _ = lib()
    dt = getattr(torch, dtype)
    q, k, v = make(torch, (lq, 2, dim), dt, 1), make(torch, (lk, 1, dim), dt, 2), make(torch, (lk, 1, dim), dt, 3)
    want, want_lse = both(q, k, v, causal)
    q2 = q.clone()
    q2[41, :, 7] = NAN
    got, lse = both(q2, k, v, causal)
    assert torch.isnan(got[41]).all() and torch.isnan(lse[41]).all()
    others = [i for i in range(lq) if i != 41]
    tol = 4 * HALF[dtype] * float(v.abs().max())     # a row that is taken another way is rounded otherwise
    assert (got[others] - want[others]).abs().max() <= tol and (lse[others] - want_lse[others]).abs().max() <= 1e-4
    if not causal:
        assert torch.equal(got[others], want[others]) and torch.equal(lse[others], want_lse[others])


@pytest.mark.parametrize("where", ["key", "value"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,dim,lq,lk,at", [("bfloat16", 64, 200, 200, 130), ("float16", 128, 200, 200, 0),
                                                ("bfloat16", 128, 64, 9000, 8970), ("float16", 64, 64, 9000, 1500)])
def test_nan_in_one_token(dtype, dim, lq, lk, at, causal, where):
    torch, _ = lib()
    dt = getattr(torch, dtype)
    q, k, v = make(torch, (lq, 4, dim), dt, 4), make(torch, (lk, 2, dim), dt, 5), make(torch, (lk, 2, dim), dt, 6)
    want, want_lse = both(q, k, v, causal)
    (k if where == "key" else v)[at, :, 9] = NAN
    got, lse = both(q, k, v, causal)
    first = max(0, at - (lk - lq)) if causal else 0       # the first query that sees it
    tol = 4 * HALF[dtype] * float(v[torch.isfinite(v)].abs().max())
    assert (got[:first] - want[:first]).abs().max() <= tol if first else True
    assert (lse[:first] - want_lse[:first]).abs().max() <= 1e-4 if first else True
    if where == "key":
        assert torch.isnan(got[first:]).all() and torch.isnan(lse[first:]).all()
    else:
        assert torch.isnan(got[first:, :, 9]).all()
        rest = [d for d in range(dim) if d != 9]
        assert (got[first:][:, :, rest] - want[first:][:, :, rest]).abs().max() <= tol
        assert (lse[first:] - want_lse[first:]).abs().max() <= 1e-4
