"""The operators of include/pat_operators.h on torch tensors: arguments checked, then the library's kernels on the current stream of
the tensors' device.  There is no fallback: a missing library raises, as does every argument the kernels do not take.
"""
from __future__ import annotations

import torch

from .binding import PAT_EINVAL, PatError, load_library

_TYPE = {torch.float32: 0, torch.bfloat16: 1}
PAT_ATTN_MAX_SEQS = 2048
# the current device, and a device's current stream as a number: torch's own short cuts where it has them, two microseconds of eleven on a small call
_current = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _need(ok, what):
    if not ok:
        raise PatError(PAT_EINVAL, what)


def _one_device(t, *others):
    """The device of all these tensors (None: left out)."""
    dev = t.device
    for o in others:
        if o is not None and o.device != dev:
            _need(False, "tensors on one GPU are needed")
    if dev.type != "cuda":
        _need(False, "tensors on one GPU are needed")
    return dev


_functions = {}


def _call(dev, name, *args):
    """The library's call with its device the current one, on that device's current stream."""
    fn, at = _functions.get(name), dev.index
    if fn is None:
        fn = _functions[name] = getattr(load_library(), name)
    if _current() != at:
        with torch.cuda.device(at):
            rc = fn(*args, _stream(at))
    else:
        rc = fn(*args, _stream(at))
    if rc:
        raise PatError(rc, name)


def _cache(k, v):
    """[n_pages, heads, tokens of a page, features] of the two pools."""
    shape = k.shape
    _need(k.dtype is torch.bfloat16 and v.dtype is torch.bfloat16 and len(shape) == 4 and shape == v.shape and k.is_contiguous() and v.is_contiguous(),
          "k and v pools: contiguous bf16 [n_pages, n_kv_heads, page_tokens, head_dim]")
    return shape


def _table(t):
    shape = t.shape
    _need(t.dtype is torch.int32 and len(shape) == 2 and t.is_contiguous(), "page_table: contiguous int32 [sequences, max_pages]")
    return shape


def _list(t, n, what):
    if t.dtype is not torch.int32 or t.shape != (n,) or not t.is_contiguous():
        _need(False, f"{what}: contiguous int32 [{n}]")
    return t.data_ptr()


def _rows(t, heads, d, what):
    """Elements from row to row of [rows, heads, d] whose rows are dense."""
    rows, strides = t.shape[0], t.stride()
    if t.shape != (rows, heads, d) or t.dtype not in _TYPE or strides[2] != 1 or (heads > 1 and strides[1] != d):
        _need(False, f"{what}: fp32 or bf16 [rows, {heads}, {d}], rows dense")
    return strides[0] if rows > 1 else heads * d


def pat_op_rope_table(n_pos, head_dim, base=10000.0, device="cuda:0"):
    """fp32 [n_pos, head_dim / 2, 2]: cos and sin of every position's angles."""
    with torch.cuda.device(device):
        cs = torch.empty(n_pos, head_dim // 2, 2, dtype=torch.float32, device="cuda")
        _call(cs.device, "pat_op_rope_table", n_pos, head_dim, base, cs.data_ptr())
    return cs


def pat_op_kv_append(qkv, seq, pos, cos_sin, k_pages, v_pages, page_table, q_out, gq=None, gk=None, eps=1e-6, skipped=None):
    """Rotates (and with gains normalises) the q heads of qkv [rows, (hq + 2 hkv) d] into q_out [rows, hq, d], and appends its k and v heads to the
    pages of sequence seq[i] at position pos[i] (both int32 [rows]); seq[i] < 0 is a row of padding.  skipped: NULL or int32 [1], raised by
    the rows that name no place of the cache.  Returns q_out."""
    n_pages, hkv, P, d = _cache(k_pages, v_pages)
    dev = _one_device(qkv, seq, pos, cos_sin, k_pages, v_pages, page_table, q_out, gq, gk, skipped)
    n_seqs, max_pages = _table(page_table)
    _need(qkv.dim() == 2 and qkv.dtype in _TYPE and qkv.stride(1) == 1 and q_out.dim() == 3 and q_out.dtype == qkv.dtype and q_out.shape[0] == qkv.shape[0],
          "qkv [rows, (hq + 2 hkv) d] and q_out [rows, hq, d]: fp32 or bf16 of one type, rows dense")
    (rows, width), hq, n_pos = qkv.shape, q_out.shape[1], cos_sin.shape[0]
    if width != (hq + 2 * hkv) * d:
        _need(False, f"qkv: {(hq + 2 * hkv) * d} features a row for {hq} q and {hkv} k and v heads, not {width}")
    _need(cos_sin.dtype is torch.float32 and cos_sin.is_contiguous() and cos_sin.shape == (n_pos, d // 2, 2), "cos_sin: contiguous fp32 [positions, d / 2, 2]")
    _need((gq is None) == (gk is None), "gq and gk: both or neither")
    if gq is not None:
        _need(all(g.dtype is torch.bfloat16 and g.is_contiguous() and g.shape == (d,) for g in (gq, gk)), "gq, gk: contiguous bf16 [d]")
    _need(skipped is None or (skipped.dtype is torch.int32 and skipped.numel() == 1), "skipped: int32 [1]")
    ld = qkv.stride(0) if rows > 1 else width
    _call(dev, "pat_op_kv_append", qkv.data_ptr(), _TYPE[qkv.dtype], ld, rows, hq, hkv, d, _list(seq, rows, "seq"), _list(pos, rows, "pos"),
          cos_sin.data_ptr(), n_pos, gq.data_ptr() if gq is not None else None, gk.data_ptr() if gk is not None else None, eps,
          k_pages.data_ptr(), v_pages.data_ptr(), n_pages, P, page_table.data_ptr(), n_seqs, max_pages, q_out.data_ptr(), _rows(q_out, hq, d, "q_out"),
          skipped.data_ptr() if skipped is not None else None)
    return q_out


class AttnPlan:
    """How a step's attention is cut: made by pat_op_attn_plan, read by the pat_op_attn_shared of every layer."""
    __slots__ = ("buf", "n_seqs", "hq", "hkv", "d", "scratch_bytes")

    def __init__(self, buf, n_seqs, hq, hkv, d, scratch_bytes):
        self.buf, self.n_seqs, self.hq, self.hkv, self.d, self.scratch_bytes = buf, n_seqs, hq, hkv, d, scratch_bytes


def pat_op_attn_plan(kv_len, group_start, shared_len, max_len, n_q_heads, n_kv_heads, head_dim, plan=None):
    """The plan of one step for sequences of kv_len[s] <= max_len cached tokens (int32 [n]), of which group_start[g] .. group_start[g + 1] - 1 share
    their first shared_len[g] tokens (int32 [groups + 1] and [groups]).  plan: one to write anew (of as many sequences and the same heads), as a
    captured graph does.  No sequences (a drained step): a plan by which the attention does nothing."""
    n, ng = kv_len.shape[0], shared_len.shape[0]
    dev = _one_device(kv_len, group_start, shared_len)
    _need(n <= PAT_ATTN_MAX_SEQS and ng <= PAT_ATTN_MAX_SEQS and (n == 0 or ng > 0), f"up to {PAT_ATTN_MAX_SEQS} sequences and groups, a group at least for any sequence")
    if plan is None:
        lib, most = load_library(), max(n, 1)
        nbytes, scratch = lib.pat_op_attn_plan_bytes(most, n_q_heads, n_kv_heads), lib.pat_op_attn_scratch_bytes(most, n_q_heads, n_kv_heads, head_dim)
        _need(nbytes > 0 and scratch > 0, f"{n_q_heads} query heads on {n_kv_heads} KV heads of {head_dim} features")
        plan = AttnPlan(torch.empty(nbytes if n else 0, dtype=torch.uint8, device=dev), n, n_q_heads, n_kv_heads, head_dim, scratch)
    _need((plan.n_seqs, plan.hq, plan.hkv, plan.d, plan.buf.device) == (n, n_q_heads, n_kv_heads, head_dim, dev), "plan: made for other sequences or heads, or on another device")
    if n == 0:
        for t, size, what in ((kv_len, 0, "kv_len"), (group_start, ng + 1, "group_start"), (shared_len, ng, "shared_len")):
            _list(t, size, what)
        return plan
    _call(dev, "pat_op_attn_plan", _list(kv_len, n, "kv_len"), _list(group_start, ng + 1, "group_start"), _list(shared_len, ng, "shared_len"), n, ng,
          max_len, n_q_heads, n_kv_heads, plan.buf.data_ptr())
    return plan


def pat_op_attn_shared(q, k_pages, v_pages, page_table, plan, out=None):
    """out [n, hq, d] = attention of one query token per sequence, q [n, hq, d], over the paged cache as the plan cuts it."""
    n_pages, hkv, P, d = _cache(k_pages, v_pages)
    dev = _one_device(q, k_pages, v_pages, page_table, out, plan.buf)
    n_seqs, max_pages = _table(page_table)
    n, hq = plan.n_seqs, plan.hq
    _need(plan.hkv == hkv and plan.d == d and n_seqs == n and q.shape[0] == n, "the plan is for other sequences or heads")
    ldq = _rows(q, hq, d, "q")
    if out is None:
        out = torch.empty(n, hq, d, dtype=q.dtype, device=dev)
    _need(out.dtype == q.dtype and out.shape[0] == n, "out: of q's type and rows")
    if n == 0:
        _rows(out, hq, d, "out")
        return out
    scratch = torch.empty(plan.scratch_bytes, dtype=torch.uint8, device=dev)
    _call(dev, "pat_op_attn_shared", q.data_ptr(), _TYPE[q.dtype], ldq, n, hq, hkv, d, k_pages.data_ptr(), v_pages.data_ptr(), n_pages, P,
          page_table.data_ptr(), max_pages, plan.buf.data_ptr(), out.data_ptr(), _rows(out, hq, d, "out"), scratch.data_ptr())
    return out


def pat_op_f8_pack_weight(w):
    """w [n, k] fp32 or bf16 -> (packed, scales): its 8-bit form, uint8 tensors as pat_op_f8_gemm reads them."""
    _need(w.dim() == 2 and w.dtype in _TYPE and (w.stride(1) == 1 or w.shape[1] == 1), "w: fp32 or bf16 [n, k], rows dense")
    n, k = w.shape
    dev, lib = _one_device(w), load_library()
    nbytes, sbytes = lib.pat_op_f8_weight_bytes(n, k), lib.pat_op_f8_scale_bytes(n, k)
    _need(nbytes > 0, f"n = {n}, k = {k}")
    packed, scales = (torch.empty(b, dtype=torch.uint8, device=dev) for b in (nbytes, sbytes))
    _call(dev, "pat_op_f8_pack_weight", w.data_ptr(), _TYPE[w.dtype], w.stride(0) if n > 1 else k, n, k, packed.data_ptr(), scales.data_ptr())
    return packed, scales


def pat_op_f8_gemm(packed, scales, n, x, y=None, mode=0, y_dtype=None):
    """y [m, n] = (mode 0) or += (mode 1) x W^T for x [m, k] and the packed W [n, k]; y's type is x's unless y or y_dtype says otherwise."""
    _need(x.dim() == 2 and x.dtype in _TYPE and (x.stride(1) == 1 or x.shape[1] == 1), "x: fp32 or bf16 [m, k], rows dense")
    m, k = x.shape
    dev, lib = _one_device(x, packed, scales, y), load_library()
    if packed.dtype is not torch.uint8 or scales.dtype is not torch.uint8 or packed.numel() != lib.pat_op_f8_weight_bytes(n, k) or scales.numel() != lib.pat_op_f8_scale_bytes(n, k) \
            or not packed.is_contiguous() or not scales.is_contiguous():
        _need(False, f"packed weight and scales of a [{n}, {k}] matrix are needed")
    if y is None:
        _need(mode == 0, "mode 1 adds to a given y")
        y = torch.empty(m, n, dtype=y_dtype or x.dtype, device=dev)
    if y.dtype not in _TYPE or y.shape != (m, n) or (y.stride(1) != 1 and n > 1):
        _need(False, f"y: fp32 or bf16 [{m}, {n}], rows dense")
    nbytes = lib.pat_op_f8_gemm_scratch_bytes(n, k, m)
    _need(nbytes >= 0, "x: more rows than a call takes")
    scratch = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=dev)
    _call(dev, "pat_op_f8_gemm", packed.data_ptr(), scales.data_ptr(), n, k, x.data_ptr(), _TYPE[x.dtype], x.stride(0) if m > 1 else k, m, y.data_ptr(),
          _TYPE[y.dtype], y.stride(0) if m > 1 else n, mode, scratch.data_ptr())
    return y
