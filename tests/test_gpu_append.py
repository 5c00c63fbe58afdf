"""Rotation and append to the paged cache (pat_op_kv_append, pat_op_rope_table) against a plain implementation in 64 bits."""
import numpy as np
import pytest
import torch

from gpu_util import DEV
from operator_refs import angles, check, rms, rotate

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module")
def pat():
    import paper_2605_23945_amd as p
    p.load_library()
    return p


def _table(n_seqs, tokens, P, seed, spare=2):
    """A page table of distinct pages in random order."""
    per = -(-tokens // P)
    order = np.random.default_rng(seed).permutation(n_seqs * per + spare)
    return torch.as_tensor(order[:n_seqs * per].reshape(n_seqs, per).astype(np.int32)), n_seqs * per + spare


def _case(pat, hq, hkv, d, P, seq, pos, dtype, norm, n_seqs, n_pos, pad=0, inplace=False, seed=0):
    g = torch.Generator().manual_seed(seed)
    rows, width = len(seq), (hq + 2 * hkv) * d
    x = torch.randn(rows, width, generator=g).to(dtype)
    gq, gk = ((1 + 0.1 * torch.randn(d, generator=g)).to(torch.bfloat16) for _ in range(2))
    table, n_pages = _table(n_seqs, n_pos, P, seed)
    pools = [torch.randn(n_pages, hkv, P, d, generator=g).to(torch.bfloat16) for _ in range(2)]
    buf = torch.full((rows, width + pad), 3.0, dtype=dtype, device=DEV)
    qkv = buf[:, :width]
    qkv.copy_(x)
    q = qkv[:, :hq * d].unflatten(1, (hq, d)) if inplace else torch.full((rows, hq, d), 7.0, dtype=dtype, device=DEV)
    k, v = (t.to(DEV) for t in pools)
    skipped = torch.zeros(1, dtype=torch.int32, device=DEV)
    seq, pos = torch.as_tensor(seq, dtype=torch.int32), torch.as_tensor(pos, dtype=torch.int32)
    cs = pat.pat_op_rope_table(n_pos, d, 10000.0, DEV)
    pat.pat_op_kv_append(qkv, seq.to(DEV), pos.to(DEV), cs, k, v, table.to(DEV), q, gq.to(DEV) if norm else None, gk.to(DEV) if norm else None, EPS, skipped)
    # the plain form
    ok = (seq >= 0) & (seq < n_seqs) & (pos >= 0) & (pos < n_pos)
    h = x.double().view(rows, hq + 2 * hkv, d)
    hn = h.clone()
    if norm:
        hn[:, :hq], hn[:, hq:hq + hkv] = rms(h[:, :hq], gq.double(), EPS), rms(h[:, hq:hq + hkv], gk.double(), EPS)
    r, mag = rotate(hn, pos)
    # per element: the table's and the products' roundings (4 of |a| + |b|), the norm's sum over d, its root, division and two products
    allow = mag * (6 + ((d + 8) if norm else 0)) * 2.0 ** -24
    ref_k, ref_v = (t.double() for t in pools)
    al_k, al_v = torch.zeros_like(ref_k), torch.zeros_like(ref_v)
    touched = torch.zeros(n_pages, P, dtype=torch.bool)
    for i in range(rows):
        if not ok[i]:
            continue
        p, o = int(table[seq[i], pos[i] // P]), int(pos[i]) % P
        ref_k[p, :, o], al_k[p, :, o] = r[i, hq:hq + hkv], allow[i, hq:hq + hkv]
        ref_v[p, :, o] = h[i, hq + hkv:]
        touched[p, o] = True
    want_q = torch.where(ok[:, None, None], r[:, :hq], x.double().view(rows, -1, d)[:, :hq] if inplace else torch.tensor(7.0).double())
    check(q, want_q, torch.where(ok[:, None, None], allow[:, :hq], 0.0))
    check(k, ref_k, al_k)
    check(v, ref_v, al_v)
    keep = ~touched[:, None, :, None].expand_as(ref_k)
    assert torch.equal(k.cpu()[keep], pools[0][keep]) and torch.equal(v.cpu()[keep], pools[1][keep])       # bit for bit
    if pad:
        assert bool((buf[:, width:] == 3.0).all())
    assert int(skipped) == int(((seq >= 0) & ~ok).sum())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("hq,hkv,d,P", [(4, 4, 64, 16), (8, 1, 128, 64), (3, 1, 128, 32), (5, 5, 64, 128), (1, 1, 128, 16)])
def test_decode_rows(pat, hq, hkv, d, P, norm, dtype):
    n = 7
    pos = [0, 1, P - 1, P, 2 * P + 3, 299, 150]
    _case(pat, hq, hkv, d, P, list(range(n)), pos, dtype, norm, n, 300, seed=hq + d)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_prompt_rows_in_any_order(pat, dtype):
    seq = np.repeat([2, 0, 1], [37, 1, 66])
    pos = np.concatenate([np.arange(37)[::-1], [5], np.arange(10, 76)])
    _case(pat, 4, 2, 64, 16, seq, pos, dtype, True, 3, 80, seed=3)


@pytest.mark.parametrize("rows", [1, 2])
def test_few_rows_and_far_positions(pat, rows):
    """At position 131071 an fp32 angle would be off by 2^-8: the table's is not."""
    _case(pat, 2, 1, 128, 128, [0, 1][:rows], [131071, 99999][:rows], torch.float32, False, 2, 131072, seed=9)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_padding_and_rows_out_of_range_write_nothing(pat, dtype):
    seq = [0, -1, 1, 5, 1, 0, -7, 1]
    pos = [3, 4, -1, 2, 64, 63, 10 ** 6, 2 ** 30]
    _case(pat, 4, 4, 64, 16, seq, pos, dtype, False, 2, 64, seed=5)
    _case(pat, 4, 4, 64, 16, seq, pos, dtype, False, 2, 64, inplace=True, seed=5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_with_a_stride_and_in_place(pat, dtype):
    _case(pat, 8, 2, 64, 32, [0, 1, 2], [9, 8, 7], dtype, True, 3, 40, pad=8, inplace=True, seed=6)


def test_bad_page_is_skipped(pat):
    d, P = 64, 16
    table = torch.tensor([[0, 99], [-1, 1]], dtype=torch.int32, device=DEV)
    k = torch.zeros(2, 1, P, d, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    qkv = torch.ones(4, 3 * d, device=DEV)
    q = torch.zeros(4, 1, d, device=DEV)
    skipped = torch.zeros(1, dtype=torch.int32, device=DEV)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)      # noqa: E731
    pat.pat_op_kv_append(qkv, i32([0, 0, 1, 1]), i32([2, 17, 3, 18]), pat.pat_op_rope_table(32, d), k, v, table, q, skipped=skipped)
    assert int(skipped) == 2
    assert bool((v[0, 0, 2] == 1).all()) and bool((v[1, 0, 2] == 1).all()) and float(v.float().sum()) == 2 * d
    assert bool((q[1] == 0).all()) and bool((q[2] == 0).all()) and bool((q[0] != 0).any()) and bool((q[3] != 0).any())


def test_no_rows(pat):
    d = 64
    k = torch.zeros(1, 1, 16, d, dtype=torch.bfloat16, device=DEV)
    e = torch.empty(0, dtype=torch.int32, device=DEV)
    pat.pat_op_kv_append(torch.empty(0, 3 * d, device=DEV), e, e, pat.pat_op_rope_table(4, d), k, k.clone(), torch.zeros(1, 1, dtype=torch.int32, device=DEV),
                         torch.empty(0, 1, d, device=DEV))
    assert float(k.float().abs().sum()) == 0


def test_the_table_is_the_rounded_exact_one(pat):
    """fp32 cos and sin: half a step, and a 64-bit sine of an angle up to 5e4 that is itself off by a few 2^-53 of the angle."""
    cs = pat.pat_op_rope_table(50000, 128, 10000.0, DEV).cpu().double()
    a = angles(50000, 128)
    for got, ref in ((cs[..., 0], a.cos()), (cs[..., 1], a.sin())):
        assert bool(((got - ref).abs() <= 2.0 ** -24 * ref.abs() + 50000 * 2.0 ** -50).all())


def test_append_writes_what_the_decoder_reads(pat):
    """The pool of one layer in the decoder's own layout: rows appended here are what pat_kv_read gives there."""
    import pat_inputs as pi
    from gpu_util import make_decoder
    shard = pi.CONFIGS["tiny_tp1"]["shard"]
    dec = make_decoder(shard, 2, 64, 256, 16)
    dec.pat_decode_admit([0, 1], [1, 2], [20, 33], [5, 5])
    pages, _ = dec.pat_get_pages()
    hkv, d, P = shard.hkv, shard.head_dim, 16
    base = (dec._kv.data_ptr() + 255) // 256 * 256 - dec._kv.data_ptr()
    pool = dec._kv[base:base + dec.req.kv_bytes].view(torch.bfloat16).view(shard.n_layers, 2, dec.req.n_pages, hkv, P, d)
    seq = np.repeat([0, 1], [20, 33]).astype(np.int32)
    pos = np.concatenate([np.arange(20), np.arange(33)]).astype(np.int32)
    qkv = torch.randn(53, (shard.hq + 2 * hkv) * d, device=DEV)
    q = torch.empty(53, shard.hq, d, device=DEV)
    pat.pat_op_kv_append(qkv, torch.as_tensor(seq, device=DEV), torch.as_tensor(pos, device=DEV), pat.pat_op_rope_table(64, d), pool[1, 0], pool[1, 1],
                         torch.as_tensor(np.ascontiguousarray(pages), device=DEV), q)
    h = qkv.double().cpu().view(53, -1, d)
    r, mag = rotate(h, torch.as_tensor(pos))
    for s in range(2):
        at = torch.as_tensor(seq == s)
        k, v = dec.pat_kv_read(s, 1, int(at.sum()))
        check(k, r[at][:, shard.hq:shard.hq + hkv], mag[at][:, shard.hq:shard.hq + hkv] * 6 * 2.0 ** -24)
        assert torch.equal(v.cpu(), h[at][:, shard.hq + hkv:].to(torch.bfloat16))
    dec.close()
