"""The operators of include/pat_operators.h together, as a decode layer of group rollouts calls them: prompts appended once per group, then per step the
8-bit QKV product, rotation and append, the plan, the attention over shared prefixes and the 8-bit output product onto the residual.  Each
operator is held to the plain implementation on what it was really given; nothing waits between them."""
import numpy as np
import pytest
import torch

from gpu_util import DEV
from operator_refs import attend, check, eight_bit, project, rotate

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pat():
    import paper_2605_23945_amd as p
    p.load_library()
    return p


def _i32(a):
    return torch.as_tensor(np.asarray(a), dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hq,hkv,d,P,H", [(4, 4, 64, 16, 256), (8, 1, 128, 64, 320)])
def test_layer_of_grouped_answers(pat, hq, hkv, d, P, H, dtype):
    g = torch.Generator().manual_seed(hq)
    prompts, answers, steps = [37, 70], [3, 2], 4
    start, n = [0, 3, 5], 5
    of = [0, 0, 0, 1, 1]
    width = (hq + 2 * hkv) * d
    wqkv, wo = (torch.randn(*s, generator=g).mul(0.05).to(torch.bfloat16) for s in ((width, H), (H, hq * d)))
    pq, po = pat.pat_op_f8_pack_weight(wqkv.to(DEV)), pat.pat_op_f8_pack_weight(wo.to(DEV))
    wq8, wo8 = eight_bit(wqkv, 128), eight_bit(wo, 128)
    cs = pat.pat_op_rope_table(256, d, device=DEV)
    # pages: a prompt's whole pages shared, its last part copied to each answer
    per = -(-(max(prompts) + steps) // P)
    order, at = np.random.default_rng(1).permutation(n * per + 8), 0
    table = np.zeros((n, per), np.int64)
    for s in range(n):
        whole = prompts[of[s]] // P
        for p in range(per):
            if p < whole and s not in start:
                table[s, p] = table[start[of[s]], p]
            else:
                table[s, p] = order[at]
                at += 1
    k = torch.full((len(order), hkv, P, d), float("nan"), dtype=torch.bfloat16, device=DEV)
    v = k.clone()
    dtab = _i32(table)
    # the prompts, once per group, through its first answer's row
    x = torch.randn(sum(prompts), H, generator=g).to(dtype)
    seq = np.repeat([start[0], start[1]], prompts)
    pos = np.concatenate([np.arange(p) for p in prompts])
    qkv = pat.pat_op_f8_gemm(*pq, width, x.to(DEV))
    q = torch.empty(len(pos), hq, d, dtype=dtype, device=DEV)
    pat.pat_op_kv_append(qkv, _i32(seq), _i32(pos), cs, k, v, dtab, q)
    for s in range(n):
        if s not in start and prompts[of[s]] % P:
            src, dst = table[start[of[s]], prompts[of[s]] // P], table[s, prompts[of[s]] // P]
            k[dst], v[dst] = k[src], v[src]
    kv_len = _i32([prompts[o] for o in of])
    residual = torch.randn(n, H, generator=g).to(dtype).to(DEV)
    plan = None
    kept = []
    for step in range(steps):
        xin = residual.clone()
        qkv = pat.pat_op_f8_gemm(*pq, width, residual)
        q = torch.empty(n, hq, d, dtype=dtype, device=DEV)
        pat.pat_op_kv_append(qkv, _i32(range(n)), kv_len, cs, k, v, dtab, q)
        kv_len = kv_len + 1
        plan = pat.pat_op_attn_plan(kv_len, _i32(start), _i32(prompts), 256, hq, hkv, d, plan=plan)
        o = pat.pat_op_attn_shared(q, k, v, dtab, plan)
        pat.pat_op_f8_gemm(*po, H, o.view(n, hq * d), residual, mode=1)
        kept.append((xin, qkv, q, o, residual.clone(), k.clone(), v.clone()))
    for step, (xin, qkv, q, o, out, k, v) in enumerate(kept):
        ref, allow = project(eight_bit(xin.cpu(), 1), wq8)
        check(qkv, ref, allow)
        h = qkv.cpu().double().view(n, -1, d)
        pos = torch.tensor([prompts[i] + step for i in of])
        r, mag = rotate(h, pos)
        check(q, r[:, :hq], mag[:, :hq] * 6 * 2.0 ** -24)
        for s in range(n):
            at = torch.arange(int(pos[s]) + 1)
            page = torch.as_tensor(table[s])[at // P]
            ks, vs = (t.cpu()[page, :, at % P] for t in (k, v))
            check(ks[-1], r[s, hq:hq + hkv], mag[s, hq:hq + hkv] * 6 * 2.0 ** -24)
            assert torch.equal(vs[-1], h[s, hq + hkv:].to(torch.bfloat16))
            ref, allow = attend(q[s].cpu(), ks, vs)
            check(o[s], ref, allow)
        ref, allow = project(eight_bit(o.cpu().view(n, -1), 1), wo8)
        x0 = xin.cpu().double()
        check(out, ref + x0, allow + 2.0 ** -23 * (ref.abs() + x0.abs()))


def test_the_binding_refuses_other_forms(pat):
    f = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device=DEV)      # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)                     # noqa: E731
    k = f(2, 2, 16, 64, dtype=torch.bfloat16)
    cs, table = f(8, 32, 2), i(1, 2)
    good = dict(qkv=f(1, 6 * 64), seq=i(1), pos=i(1), cos_sin=cs, k_pages=k, v_pages=k.clone(), page_table=table, q_out=f(1, 2, 64))
    pat.pat_op_kv_append(**good)
    for bad in (dict(qkv=f(1, 5 * 64)), dict(qkv=f(2, 6 * 64)), dict(seq=i(2)), dict(pos=i(1).long()), dict(cos_sin=f(8, 64, 2)), dict(k_pages=k.float()), dict(v_pages=k.transpose(1, 2)),
                dict(page_table=table.long()), dict(q_out=f(1, 2, 64, dtype=torch.bfloat16)), dict(q_out=f(1, 2, 128)[..., ::2]), dict(gq=f(64, dtype=torch.bfloat16)),
                dict(qkv=f(1, 6 * 64 + 1)[:, 1:]), dict(skipped=i(2)), dict(qkv=f(1, 6 * 64).cpu())):
        with pytest.raises(pat.PatError):
            pat.pat_op_kv_append(**{**good, **bad})
    plan = pat.pat_op_attn_plan(i(1), torch.tensor([0, 1], dtype=torch.int32, device=DEV), i(1), 32, 2, 2, 64)
    for args in ((f(1, 4, 64), k, k, table), (f(2, 2, 64), k, k, i(2, 2)), (f(1, 2, 64), k, k, i(2, 2)), (f(1, 2, 64, dtype=torch.float16), k, k, table)):
        with pytest.raises(pat.PatError):
            pat.pat_op_attn_shared(*args, plan)
    with pytest.raises(pat.PatError):
        pat.pat_op_attn_plan(i(3), i(3), i(2), 32, 2, 2, 64, plan=plan)
    with pytest.raises(pat.PatError):
        pat.pat_op_attn_plan(i(3), i(2), i(2), 32, 2, 2, 64)
    pw = pat.pat_op_f8_pack_weight(f(32, 64))
    for kw in (dict(n=48, x=f(2, 64)), dict(n=32, x=f(2, 256)), dict(n=32, x=f(2, 64), y=f(2, 33)), dict(n=32, x=f(2, 64), y=f(2, 32, dtype=torch.float16)), dict(n=32, x=f(2, 64), mode=1),
               dict(n=32, x=f(64, 2).t()), dict(n=32, x=f(1, 64).expand(3, 64)), dict(n=32, x=f(2, 64), y=f(1, 32).expand(2, 32))):
        with pytest.raises(pat.PatError):
            pat.pat_op_f8_gemm(*pw, **kw)
