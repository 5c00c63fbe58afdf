"""The operators of a decode layer that answers one prompt several times, on 8-bit weights: what is measured of them.

Three operators, each through the public binding (`paper_2605_23945_amd.pat_op_*`):

- "append":  the rows of a QKV projection are rotated at their positions (after a per-head RMSNorm of q and k in the model
             family that has it); q goes out, k and v are appended to their sequences' pages;
- "attend":  one query token per sequence over its paged cache, where the sequences of a group (several answers to one
             prompt) share the pages of a long prefix, which is read once for all of them;
- "project": y = x W^T, W held in 8-bit floating point with a power-of-two scale per block of 128 x 128, x brought to the
             same form on the way with a scale per row and block of 128.

Head layouts and widths are those of the tensor-parallel shards that this repository measures elsewhere.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda:0"

# (query heads, KV heads, features of a head) of the shards
HEADS = {"tiny_tp1": (4, 4, 64), "7b_tp1": (32, 32, 128), "7b_tp4": (8, 8, 128), "13b_tp2": (20, 20, 128), "70b_tp8": (8, 1, 128),
         "70b_tp1": (64, 8, 128)}
ROPE_BASE, EPS = 10000.0, 1e-6
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # The new token of one last sequence on a narrow shard: a launch and nothing else.
        dict(name="append_7b_tp4_b1", kind="append", heads="7b_tp4", seqs=1, new=1, ctx=2047, page=64, norm=False, dtype="bf16"),
        # A decode step of the full 7B batch, activations in fp32 as the projections leave them.
        dict(name="append_7b_tp1_b256", kind="append", heads="7b_tp1", seqs=256, new=1, ctx=620, page=64, norm=False, dtype="fp32"),
        # Ragged prompts prefilled together, the model family that normalises q and k per head, short pages.
        dict(name="append_13b_tp2_prompts", kind="append", heads="13b_tp2", seqs=9, new=1219, ctx=0, page=16, norm=True, dtype="bf16"),
        # Three answers to a short question, the smallest heads.
        dict(name="attend_tiny", kind="attend", heads="tiny_tp1", groups=1, members=3, prefix=41, suffix=9, page=16, dtype="bf16"),
        # Eight answers to one prompt on a narrow shard.
        dict(name="attend_7b_tp4_1x8", kind="attend", heads="7b_tp4", groups=1, members=8, prefix=701, suffix=150, page=64, dtype="bf16"),
        # Grouped queries, one KV head, ragged groups with the long prompts of that shard's workload, activations in fp32.
        dict(name="attend_70b_tp8_16x8", kind="attend", heads="70b_tp8", groups=16, members=8, prefix=2100, suffix=611, page=64, dtype="fp32"),
        # Many answers to one long document.
        dict(name="attend_13b_tp2_1x64", kind="attend", heads="13b_tp2", groups=1, members=64, prefix=8190, suffix=333, page=128, dtype="bf16"),
        # The full 7B batch as 16 prompts of 16 answers in the middle of their generation.
        dict(name="attend_7b_tp1_16x16", kind="attend", heads="7b_tp1", groups=16, members=16, prefix=576, suffix=450, page=64, dtype="bf16"),
        # One sequence's QKV projection: the weights' bytes are all there is.
        dict(name="project_7b_tp1_qkv_b1", kind="project", n=12288, k=4096, m=1, dtype="bf16"),
        # A draining batch's down projection, activations in fp32.
        dict(name="project_13b_tp2_down_b27", kind="project", n=5120, k=6912, m=27, dtype="fp32"),
        # A full batch's gate and up projections.
        dict(name="project_7b_tp1_gateup_b251", kind="project", n=22016, k=4096, m=251, dtype="bf16"),
        # Prompts prefilled together on the grouped-query shard: the matrix product bounds it.
        dict(name="project_70b_tp8_gateup_m5003", kind="project", n=7168, k=8192, m=5003, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("append", "attend", "project"))
    dtype = rng.choice(("bf16", "bf16", "fp32"))
    if kind == "project":
        n, k = _log_int(rng, 200, 22016), _log_int(rng, 256, 11008)
        if rng.random() < 0.6:                               # most widths are multiples of 16 and of 128, the others anything
            n, k = max(16, n // 16 * 16), max(128, k // 128 * 128)
        m = _log_int(rng, 1, max(2, min(5003, int(2.8e11 / (n * k)))))
        return dict(kind=kind, n=n, k=k, m=m, dtype=dtype)
    heads = rng.choice(tuple(HEADS))
    hq, hkv, d = HEADS[heads]
    page = rng.choice((16, 32, 64, 64, 128))
    if kind == "append":
        tokens = 8e7 / ((hq + 2 * hkv) * d)                # rows of a call at the most
        if rng.random() < 0.5:
            return dict(kind=kind, heads=heads, seqs=_log_int(rng, 1, 256), new=1, ctx=_log_int(rng, 1, 4000), page=page, norm=rng.random() < 0.3, dtype=dtype)
        seqs = _log_int(rng, 1, 16)
        return dict(kind=kind, heads=heads, seqs=seqs, new=_log_int(rng, 2, min(4000, int(tokens / seqs))), ctx=rng.choice((0, 0, _log_int(rng, 1, 4000))),
                    page=page, norm=rng.random() < 0.3, dtype=dtype)
    members = _log_int(rng, 1, 64)
    groups = _log_int(rng, 1, max(1, 256 // members))
    tokens = 1.2e9 / (hkv * d * 4)                           # cached tokens of a call at the most, the prefixes' counted once
    prefix = _log_int(rng, 1, max(2, min(16000, int(0.5 * tokens / groups))))
    suffix = _log_int(rng, 1, max(2, min(2000, int(0.5 * tokens / (groups * members)))))
    if members * groups * hq * (1.5 * prefix + 1.5 * suffix) > 3.5e7:      # scores of a call
        prefix, suffix = min(prefix, 576), min(suffix, 450)
    return dict(kind=kind, heads=heads, groups=groups, members=members, prefix=prefix, suffix=suffix, page=page, dtype=dtype)


# ---- lengths: by the case alone ------------------------------------------------------------------------------

def _spread(n, mean):
    """n numbers of at least 1 spread evenly over [mean / 2, 3 mean / 2], large and small ones in turn."""
    v = [max(1, int(mean * (0.5 + (i + 0.5) / n))) for i in range(n)]
    return [v[i // 2] if i % 2 == 0 else v[n - 1 - i // 2] for i in range(n)]


def _groups(case):
    """(members of each group, shared tokens of each group, cached tokens of each sequence)."""
    members = _spread(case["groups"], case["members"])
    shared = _spread(case["groups"], case["prefix"])[::-1]
    suffix = _spread(sum(members), case["suffix"])
    of = [g for g, n in enumerate(members) for _ in range(n)]
    return members, shared, [shared[g] + u for g, u in zip(of, suffix)]


def _rows(case):
    """(sequence, position) of each row of an append: the new tokens of each sequence behind its cached ones."""
    seqs = case["seqs"]
    new = [1] * seqs if case["new"] == 1 else _spread(seqs, case["new"])
    old = [0] * seqs if case["ctx"] == 0 else _spread(seqs, case["ctx"])[::-1]
    seq = np.repeat(np.arange(seqs, dtype=np.int32), new)
    pos = np.concatenate([np.arange(o, o + n, dtype=np.int32) for o, n in zip(old, new)])
    return seq, pos, [o + n for o, n in zip(old, new)]


# ---- inputs ---------------------------------------------------------------------------------------------------

def _normal(g, shape, dtype, std=1.0, mean=0.0):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(mean, std, generator=g).to(dtype)


def _cache(g, shape):
    return torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.0, generator=g)


def _int(a):
    return torch.as_tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def _angles(n_pos, d):
    """Angles of the rotation in 64 bits: position times base^(-2 j / d)."""
    j = torch.arange(d // 2, dtype=torch.float64, device=DEV)
    return torch.arange(n_pos, dtype=torch.float64, device=DEV)[:, None] * torch.pow(torch.tensor(ROPE_BASE, dtype=torch.float64, device=DEV), -2.0 * j / d)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rng = np.random.default_rng(seed)
    dtype = DTYPES[case["dtype"]]
    st = dict(kind=case["kind"], dtype=dtype)
    if case["kind"] == "project":
        # activations with a few strong channels; the weights' 8-bit form is laid out once
        n, k, m = case["n"], case["k"], case["m"]
        x = torch.empty(m, k, device=DEV).normal_(0.0, 1.0, generator=g)
        x *= 1 + 15 * (torch.empty(k, device=DEV).uniform_(0, 1, generator=g) < 0.01)
        w = _normal(g, (n, k), torch.bfloat16, 0.02)
        st.update(x=x.to(dtype), y=torch.empty(m, n, dtype=dtype, device=DEV), n=n)
        if own:
            import paper_2605_23945_amd as pat
            st.update(pat=pat, w=pat.pat_op_f8_pack_weight(w))
        else:
            st.update(w=_eight_bit(w.float(), 128).to(torch.bfloat16))      # exact: 4 significant bits
        return st
    hq, hkv, d = HEADS[case["heads"]]
    P = case["page"]
    st.update(hq=hq, hkv=hkv, d=d, P=P)
    if case["kind"] == "append":
        seq, pos, total = _rows(case)
        pages = [-(-t // P) for t in total]
        n_pages, max_pages = sum(pages) + 3, max(pages)
        order = rng.permutation(n_pages)
        table = np.zeros((case["seqs"], max_pages), np.int32)
        at = 0
        for s, n in enumerate(pages):
            table[s, :n] = order[at:at + n]
            at += n
        ang = _angles(max(total), d)
        st.update(seq=_int(seq), pos=_int(pos), table=_int(table), cs=torch.stack([ang.cos(), ang.sin()], -1).float().contiguous(),
                  qkv=_normal(g, (len(seq), (hq + 2 * hkv) * d), dtype), k=_cache(g, (n_pages, hkv, P, d)), v=_cache(g, (n_pages, hkv, P, d)),
                  q=torch.empty(len(seq), hq, d, dtype=dtype, device=DEV), norm=case["norm"])
        st["gq"], st["gk"] = (_normal(g, (d,), torch.bfloat16, 0.1, 1.0) for _ in range(2)) if case["norm"] else (None, None)
        if own:
            import paper_2605_23945_amd as pat
            st.update(pat=pat)
        return st
    members, shared, total = _groups(case)
    start = np.concatenate([[0], np.cumsum(members)])
    whole = [s // P for s in shared]                         # pages that a group shares
    max_pages = max(-(-t // P) for t in total)
    n_pages = sum(whole) + sum(-(-t // P) - whole[g] for g, n in enumerate(members) for t in total[start[g]:start[g + 1]])
    order = rng.permutation(n_pages)
    table = np.zeros((len(total), max_pages), np.int32)
    at = 0
    first, copies = [], []                                   # a prefix that ends inside a page: each sequence has its copy of that page's beginning
    for g_, n in enumerate(members):
        table[start[g_]:start[g_ + 1], :whole[g_]] = order[at:at + whole[g_]]
        at += whole[g_]
        for s in range(start[g_], start[g_ + 1]):
            rest = -(-total[s] // P) - whole[g_]
            table[s, whole[g_]:whole[g_] + rest] = order[at:at + rest]
            at += rest
            first.append(table[start[g_], whole[g_]])
            copies.append(table[s, whole[g_]])
    kv = []
    for _ in range(2):
        pool = _cache(g, (n_pages, hkv, P, d))
        cut = torch.arange(P, device=DEV)[None, :] < _int([s % P for s, n in zip(shared, members) for _ in range(n)])[:, None]
        src, dst = _int(first).long(), _int(copies).long()
        pool[dst] = torch.where(cut[:, None, :, None], pool[src], pool[dst])
        kv.append(pool)
    st.update(q=_normal(g, (len(total), hq, d), dtype, 2.0), k=kv[0], v=kv[1], table=_int(table), kv_len=_int(total), start=_int(start),
              shared=_int(shared), most=max(members), max_shared=max(shared), max_len=max(total), out=torch.empty(len(total), hq, d, dtype=dtype, device=DEV),
              max_suffix=max(t - s for t, s in zip(total, [s for s, n in zip(shared, members) for _ in range(n)])))
    if own:                                                  # a step's plan serves the attention of all layers
        import paper_2605_23945_amd as pat
        st.update(pat=pat, plan=pat.pat_op_attn_plan(st["kv_len"], st["start"], st["shared"], st["max_len"], hq, hkv, d))
    return st


# ---- the plain forms ------------------------------------------------------------------------------------------

def _two_to(e):
    """2^e in fp32 by its bits: pow() of the device is a step off at some of them."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _eight_bit(x, rows):
    """The values that x [m, k] has in 8 bits (4 exponent, 3 mantissa bits) with a power-of-two scale per `rows` rows and 128 columns: the
    smallest under which no element is above 448."""
    m, k = x.shape
    mb, kb = -(-m // rows), -(-k // 128)
    p = torch.zeros(mb * rows, kb * 128, device=x.device)
    p[:m, :k] = x
    p = p.view(mb, rows, kb, 128)
    f, e = torch.frexp(p.abs().amax((1, 3), keepdim=True))   # amax = f 2^e; 448 = 0.875 * 2^9
    e = torch.where(f == 0, 0, torch.where(f <= 0.875, e - 9, e - 8))
    q = (p * _two_to(-e)).to(torch.float8_e4m3fn).float()
    return (q * _two_to(e)).reshape(mb * rows, kb * 128)[:m, :k]


def _project(st):
    y = _eight_bit(st["x"].float(), 1) @ st["w"].float().t()
    return y.to(st["dtype"])


def _turn(x, gain, cos, sin, norm):
    """x [rows, heads, d] normalised (where the model does) and rotated: features j and j + d / 2 are a pair."""
    if norm:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.float()
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)


def _append(st):
    hq, hkv, d, P, dtype = st["hq"], st["hkv"], st["d"], st["P"], st["dtype"]
    q, k, v = st["qkv"].float().view(-1, hq + 2 * hkv, d).split([hq, hkv, hkv], 1)
    pos = st["pos"].long()
    cs = st["cs"][pos][:, None]
    page = st["table"][st["seq"].long(), pos // P].long()
    st["k"][page, :, pos % P] = _turn(k, st["gk"], cs[..., 0], cs[..., 1], st["norm"]).to(torch.bfloat16)
    st["v"][page, :, pos % P] = v.to(torch.bfloat16)
    return _turn(q, st["gq"], cs[..., 0], cs[..., 1], st["norm"]).to(dtype), st["k"], st["v"]


def _attend(st):
    hq, hkv, d, P = st["hq"], st["hkv"], st["d"], st["P"]
    n, groups, G = st["q"].shape[0], st["shared"].shape[0], hq // hkv
    start, table = st["start"].long(), st["table"].long()
    member = start[:-1, None] + torch.arange(st["most"], device=DEV)                       # [group, member]
    there = member < start[1:, None]
    member = member.clamp(max=n - 1)
    group = torch.searchsorted(start, torch.arange(n, device=DEV), right=True) - 1         # of each sequence
    place = torch.arange(n, device=DEV) - start[group]
    q = st["q"].float().view(n, hkv, G, d) * (1.0 / math.sqrt(d))
    # the prefix, once for the group's sequences
    at = torch.arange(st["max_shared"], device=DEV)
    page = table[start[:-1]][:, at // P]
    kp, vp = (t[page, :, at % P].permute(0, 2, 1, 3).float().contiguous() for t in (st["k"], st["v"]))            # [group, hkv, token, d]
    qg = q[member].permute(0, 2, 1, 3, 4).reshape(groups, hkv, -1, d)
    sp = (qg @ kp.transpose(2, 3).contiguous()).view(groups, hkv, st["most"], G, -1)
    sp = sp.masked_fill(at >= st["shared"][:, None, None, None, None], -math.inf)[group, :, place]                # [sequence, hkv, G, token]
    # each sequence's own tokens
    own_at = st["shared"][group, None].long() + torch.arange(st["max_suffix"], device=DEV)
    inside = own_at < st["kv_len"][:, None]
    own_at = own_at.clamp(max=st["table"].shape[1] * P - 1)
    page = torch.gather(table, 1, own_at // P)
    ks, vs = (t[page, :, own_at % P].permute(0, 2, 1, 3).float().contiguous() for t in (st["k"], st["v"]))
    ss = (q @ ks.transpose(2, 3).contiguous()).masked_fill(~inside[:, None, None], -math.inf)
    s = torch.cat([sp, ss], -1)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    pp, ps = p.split([st["max_shared"], st["max_suffix"]], -1)
    o = (pp[member] * there[:, :, None, None, None]).permute(0, 2, 1, 3, 4).reshape(groups, hkv, -1, st["max_shared"]) @ vp
    o = o.view(groups, hkv, st["most"], G, d)[group, :, place] + ps @ vs
    return o.reshape(n, hq, d).to(st["dtype"])


def run(st):
    kind = st["kind"]
    if own:
        pat = st["pat"]
        if kind == "append":
            pat.pat_op_kv_append(st["qkv"], st["seq"], st["pos"], st["cs"], st["k"], st["v"], st["table"], st["q"], st["gq"], st["gk"], EPS)
            return st["q"], st["k"], st["v"]
        if kind == "attend":
            return pat.pat_op_attn_shared(st["q"], st["k"], st["v"], st["table"], st["plan"], st["out"])
        return pat.pat_op_f8_gemm(*st["w"], st["n"], st["x"], st["y"])
    return {"append": _append, "attend": _attend, "project": _project}[kind](st)


# ---- from the definitions, in 64 bits ---------------------------------------------------------------------------

def _exact_eight_bit(x, rows):
    """As the definition of the 8-bit form has it: the block's scale, then each element to the nearest of the format's values, ties to even."""
    x = x.double()
    m, k = x.shape
    row, col = torch.arange(m, device=x.device) // rows, torch.arange(k, device=x.device) // 128
    top = torch.zeros(-(-m // rows), k, dtype=torch.float64, device=x.device).index_reduce_(0, row, x.abs(), "amax")
    top = torch.zeros(top.shape[0], -(-k // 128), dtype=torch.float64, device=x.device).index_reduce_(1, col, top, "amax")
    two_to = lambda e: ((e.long() + 1023) << 52).view(torch.float64)      # noqa: E731
    e = torch.ceil(torch.log2((top / 448.0).clamp(min=2.0 ** -200)))      # then to the right side of the border, where the logarithm is not exact
    e = torch.where(two_to(e - 1) * 448.0 >= top, e - 1, e)
    e = torch.where(two_to(e) * 448.0 < top, e + 1, e)
    scale = torch.where(top == 0, 1.0, two_to(e))[row][:, col]
    u = x / scale
    f = torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6)))
    f = torch.where(two_to(f) > u.abs().clamp(min=2.0 ** -6), f - 1, f)
    step = two_to(f) * 0.125
    return torch.round(u / step) * step * scale


def exact(case, seed):
    global own
    was, own = own, False
    st = prepare(case, seed)
    own = was
    if case["kind"] == "project":
        return _exact_eight_bit(st["x"], 1) @ st["w"].double().t()
    hq, hkv, d, P = st["hq"], st["hkv"], st["d"], st["P"]
    if case["kind"] == "append":
        x = st["qkv"].double().view(-1, hq + 2 * hkv, d).clone()
        pos = st["pos"].long()
        a = _angles(int(pos.max()) + 1, d)[pos]
        turn = torch.polar(torch.ones_like(a), a)[:, None]   # the rotation as a product of complex numbers
        for heads, gain in ((slice(0, hq), st["gq"]), (slice(hq, hq + hkv), st["gk"])):
            t = x[:, heads]
            if case["norm"]:
                t = t / (t.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt() * gain.double()
            z = torch.complex(t[..., :d // 2].contiguous(), t[..., d // 2:].contiguous()) * turn
            x[:, heads] = torch.cat([z.real, z.imag], -1)
        page = st["table"][st["seq"].long(), pos // P].long()
        k, v = st["k"].double(), st["v"].double()
        k[page, :, pos % P], v[page, :, pos % P] = x[:, hq:hq + hkv], x[:, hq + hkv:]
        return x[:, :hq], k, v
    lens, out = st["kv_len"].tolist(), []
    for s, n in enumerate(lens):                             # a sequence's whole cache through its own table row
        at = torch.arange(n, device=DEV)
        page = st["table"][s].long()[at // P]
        k, v = (t[page, :, at % P].double().repeat_interleave(hq // hkv, 1) for t in (st["k"], st["v"]))      # [token, hq, d]
        w = torch.softmax((k * st["q"][s].double()).sum(-1) / math.sqrt(d), 0)
        out.append((w[..., None] * v).sum(0))
    return torch.stack(out)


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "project":
        n, k, m = case["n"], case["k"], case["m"]
        return {"bytes": float(n * k + n * k / 16384 + m * k * size + m * n * size), "flops": 2.0 * n * k * m}
    hq, hkv, d = HEADS[case["heads"]]
    if case["kind"] == "append":
        seq, pos, total = _rows(case)
        rows = len(seq)
        table = len(np.unique(pos)) * d * 4
        return {"bytes": float(rows * ((2 * hq + 2 * hkv) * d * size + 4 * hkv * d + 12) + table), "flops": float(rows * (hq + hkv) * d * (7 if case["norm"] else 3))}
    members, shared, total = _groups(case)
    own_tokens = sum(total) - sum(n * s for n, s in zip(members, shared))
    return {"bytes": float((sum(shared) + own_tokens) * hkv * d * 4 + 2 * len(total) * hq * d * size), "flops": 4.0 * sum(total) * hq * d}
