"""A sequence whose keys are split into runs gives the same bits alone, where a workgroup takes 128 of its queries, and
in a batch that gives a workgroup 256: the runs' borders come from its keys alone."""
import pytest

from test_attention_gpu import cu, lib, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,dim,lq,lk", [("bfloat16", 128, 512, 8704), ("bfloat16", 128, 512, 9512),
                                             ("float16", 64, 512, 16448), ("float16", 128, 300, 8900)])
def test_runs_do_not_depend_on_the_workgroups_size(dtype, dim, lq, lk, causal):
    torch, A = lib()
    n, heads = 8, 32
    dt = getattr(torch, dtype)
    # 256 queries a workgroup need two workgroups a CU of them; alone a sequence has fewer
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    assert n * -(-lq // 256) * heads >= 2 * cus > -(-lq // 256) * heads
    cq, ck = cu([lq] * n), cu([lk] * n)
    q = make(torch, (cq[-1], heads, dim), dt, 1)
    k, v = make(torch, (ck[-1], 8, dim), dt, 2), make(torch, (ck[-1], 8, dim), dt, 3)
    every, lse = A.prompt_attention(q, k, v, cq, ck, causal=causal, with_lse=True)
    for r in range(n):
        a, b = slice(cq[r], cq[r + 1]), slice(ck[r], ck[r + 1])
        one, one_lse = A.prompt_attention(q[a], k[b], v[b], [0, lq], [0, lk], causal=causal, with_lse=True)
        assert torch.equal(one, every[a]) and torch.equal(one_lse, lse[a]), "sequence %d" % r
