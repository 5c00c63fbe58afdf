"""A decode step of group rollouts whose batch has drained: the operators take no rows and no sequences."""
import pytest
import torch

from gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pat():
    import paper_2605_23945_amd as p
    p.load_library()
    return p


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("groups", [0, 3])
def test_a_step_without_sequences(pat, groups, dtype):
    hq, hkv, d, P, H = 4, 2, 64, 16, 256
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)      # noqa: E731
    k = torch.full((3, hkv, P, d), 2.0, dtype=torch.bfloat16, device=DEV)
    v, table, cs = k.clone(), i(0, 2), pat.pat_op_rope_table(32, d, device=DEV)
    w = pat.pat_op_f8_pack_weight(torch.ones((hq + 2 * hkv) * d, H, device=DEV))
    qkv = pat.pat_op_f8_gemm(*w, (hq + 2 * hkv) * d, torch.empty(0, H, dtype=dtype, device=DEV))
    q = torch.empty(0, hq, d, dtype=dtype, device=DEV)
    pat.pat_op_kv_append(qkv, i(0), i(0), cs, k, v, table, q)
    plan = pat.pat_op_attn_plan(i(0), i(groups + 1), i(groups), 32, hq, hkv, d)
    for out in (pat.pat_op_attn_shared(q, k, v, table, plan), pat.pat_op_attn_shared(q, k, v, table, plan, q)):
        assert out.shape == (0, hq, d) and out.dtype == dtype
    assert pat.pat_op_attn_plan(i(0), i(groups + 1), i(groups), 32, hq, hkv, d, plan=plan) is plan
    torch.cuda.synchronize()
    assert bool((k == 2).all()) and bool((v == 2).all())


def test_what_a_step_without_sequences_still_refuses(pat):
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)      # noqa: E731
    plan = pat.pat_op_attn_plan(i(0), i(1), i(0), 32, 4, 2, 64)
    k = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16, device=DEV)
    q = torch.empty(0, 4, 64, device=DEV)
    for call in (lambda: pat.pat_op_attn_plan(i(0), i(2), i(0), 32, 4, 2, 64), lambda: pat.pat_op_attn_plan(i(0), i(1), i(0), 32, 3, 2, 64),
                 lambda: pat.pat_op_attn_plan(i(1), i(1), i(0), 32, 4, 2, 64), lambda: pat.pat_op_attn_plan(i(1), i(2), i(1), 32, 4, 2, 64, plan=plan),
                 lambda: pat.pat_op_attn_shared(torch.empty(1, 4, 64, device=DEV), k, k, i(1, 2), plan), lambda: pat.pat_op_attn_shared(q, k, k, i(1, 2), plan),
                 lambda: pat.pat_op_attn_shared(q, k, k, i(0, 2), plan, q.to(torch.bfloat16)), lambda: pat.pat_op_attn_shared(q.to(torch.float16), k, k, i(0, 2), plan)):
        with pytest.raises(pat.PatError):
            call()
