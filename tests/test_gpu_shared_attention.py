"""Decode attention over shared prefixes (pat_op_attn_plan, pat_op_attn_shared) against a plain implementation in 64 bits."""
import numpy as np
import pytest
import torch

from gpu_util import DEV
from operator_refs import attend, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pat():
    import paper_2605_23945_amd as p
    p.load_library()
    return p


def _i32(a, dev=DEV):
    return torch.as_tensor(np.asarray(a), dtype=torch.int32, device=dev)


class Batch:
    """groups: [(shared tokens, [cached tokens of each sequence])]; pages in random order, those of a prefix shared, a page that it fills in part
    copied; everything else in the pools is `junk`."""

    def __init__(self, groups, hq, hkv, d, P, dtype, seed=0, junk=float("nan"), peak=1.0):
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.lens = [n for _, seqs in groups for n in seqs]
        self.shared = [s for s, _ in groups]
        self.start = np.concatenate([[0], np.cumsum([len(seqs) for _, seqs in groups])])
        self.hq, self.hkv, self.d, self.P, self.dtype = hq, hkv, d, P, dtype
        per = max(1, -(-max(self.lens + [1]) // P))
        total = sum(-(-n // P) + 1 for n in self.lens) + sum(max(0, s) // P for s in self.shared) + 1
        order, at = rng.permutation(total), 0
        self.table = np.full((len(self.lens), per), -1, np.int64)
        k, v = (torch.full((total, hkv, P, d), junk, dtype=torch.bfloat16) for _ in range(2))
        self.kv = []
        self.q = (torch.randn(len(self.lens), hq, d, generator=g) * peak).to(dtype)
        s = 0
        for shared, seqs in groups:
            sh = max(0, shared)
            prefix = torch.randn(2, sh, hkv, d, generator=g).to(torch.bfloat16)
            whole = order[at:at + sh // P]
            at += sh // P
            for n in seqs:
                own = torch.randn(2, n, hkv, d, generator=g).to(torch.bfloat16)
                if n >= sh:                                    # a shorter sequence has a cache of its own
                    own[:, :sh] = prefix
                    self.table[s, :len(whole)] = whole
                for p in range(-(-n // P)):
                    if self.table[s, p] < 0:
                        self.table[s, p] = order[at]
                        at += 1
                    part = own[:, p * P:(p + 1) * P]
                    k[self.table[s, p], :, :part.shape[1]] = part[0].transpose(0, 1)
                    v[self.table[s, p], :, :part.shape[1]] = part[1].transpose(0, 1)
                self.kv.append(own)
                s += 1
        self.k, self.v = k.to(DEV), v.to(DEV)

    def run(self, pat, max_len=None, q=None, out=None, table=None):
        plan = pat.pat_op_attn_plan(_i32(self.lens), _i32(self.start), _i32(self.shared), max_len or max(self.lens + [1]), self.hq, self.hkv, self.d)
        return pat.pat_op_attn_shared(self.q.to(DEV) if q is None else q, self.k, self.v, _i32(self.table) if table is None else table, plan, out)

    def check(self, got, rows=None):
        for s in range(len(self.lens)) if rows is None else rows:
            ref, allow = attend(self.q[s], self.kv[s][0], self.kv[s][1])
            check(got[s], ref, allow)


HEADS = [(4, 4, 64), (8, 1, 128), (4, 4, 128), (6, 2, 64), (5, 1, 128), (40, 1, 64), (2, 1, 128), (8, 8, 128)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_head_layouts(pat, hq, hkv, d, dtype):
    b = Batch([(41, [50, 43, 60]), (0, [7]), (33, [33, 34])], hq, hkv, d, 16, dtype, seed=hq)
    b.check(b.run(pat))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("shared", [1, 15, 16, 31, 32, 33, 64, 127, 128, 129, 200])
def test_prefixes_that_end_anywhere(pat, P, shared, dtype):
    b = Batch([(shared, [shared, shared + 1, shared + 130, shared + 17])], 4, 4, 64, P, dtype, seed=shared + P)
    b.check(b.run(pat))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hq,hkv", [(8, 8), (8, 1)])
def test_lengths_from_nothing_on(pat, hq, hkv, dtype):
    """Empty slots, single tokens, sequences shorter than their group's prefix, groups that share nothing or are empty."""
    b = Batch([(20, [0, 25, 19, 21, 1, 40]), (-3, [2, 0]), (10, []), (50, [50]), (64, [3, 64, 64]), (9, [0, 0])], hq, hkv, 128, 16, dtype, seed=4)
    got = b.run(pat, max_len=100)
    b.check(got)
    assert bool((got[0] == 0).all()) and bool((got[7] == 0).all())


@pytest.mark.parametrize("members", [1, 2, 3, 8, 16, 17, 33, 100])
def test_members(pat, members):
    """Row blocks of every fill, one and several of them."""
    for hq, hkv in ((4, 4), (8, 1)):
        b = Batch([(77, [77 + 3 * i % 50 for i in range(members)])], hq, hkv, 64, 32, torch.bfloat16, seed=members)
        b.check(b.run(pat), rows=sorted({0, members // 2, members - 1, min(16, members - 1), min(31, members - 1)}))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hq,hkv,shared,own", [(8, 8, 5000, 900), (8, 1, 9000, 2500), (2, 2, 20000, 7000)])
def test_long_contexts_in_chunks(pat, hq, hkv, shared, own, dtype):
    b = Batch([(shared, [shared + own, shared + 1, shared + own // 2]), (0, [own])], hq, hkv, 128, 64, dtype, seed=7)
    b.check(b.run(pat))


def test_the_widest_plan(pat):
    """2048 sequences: the planning workgroup's last thread, chunks as long as its room for parts asks for."""
    groups = [(40 + i % 30, [40 + i % 30 + (7 * j) % 23 for j in range(1 + i % 4)]) for i in range(819)]
    n = sum(len(s) for _, s in groups)
    groups.append((0, [3] * (2048 - n)))
    b = Batch(groups, 4, 4, 64, 16, torch.bfloat16, seed=1)
    got = b.run(pat)
    b.check(got, rows=list(range(0, 2048, 37)) + [2047])


def test_more_keys_than_a_look_up_of_pages_holds(pat):
    """One head and 2000 short sequences leave a long one few chunks: a wave walks more than 32 tiles, and looks its pages up anew."""
    b = Batch([(0, [30000])] + [(0, [1])] * 2000 + [(12000, [12000, 12001])], 1, 1, 64, 16, torch.bfloat16, seed=2)
    got = b.run(pat)
    b.check(got, rows=[0, 1, 2000, 2001, 2002])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strong_scores_and_infinite_ones(pat, dtype):
    """Peaked rows; keys whose scores overflow to -infinity have no weight."""
    b = Batch([(60, [70, 65])], 4, 4, 64, 16, dtype, seed=5, peak=12.0)
    b.check(b.run(pat))
    big = 2.0 ** 120
    for t in (3, 62):                                          # a shared and an own key of sequence 0
        b.kv[0][0][t] = -torch.sign(b.q[0].float()).to(torch.bfloat16) * big
        b.k[b.table[0, t // 16], :, t % 16] = b.kv[0][0][t].to(DEV)
    b.q[0] = b.q[0].float().sign().mul(2.0 ** 10).to(dtype)
    got = b.run(pat)
    ref, _ = attend(b.q[0], b.kv[0][0], b.kv[0][1])
    keep = [t for t in range(70) if t not in (3, 62)]
    ref2, allow = attend(b.q[0], b.kv[0][0][keep], b.kv[0][1][keep])
    assert torch.allclose(ref, ref2)
    check(got[0], ref2, allow)


def test_values_behind_a_sequence_do_not_count(pat):
    """NaN and infinities in every place of the pools that no sequence holds, and behind a shorter sequence of a group."""
    for junk in (float("nan"), float("inf"), torch.finfo(torch.bfloat16).min):
        b = Batch([(37, [37, 40, 55, 36, 12])], 4, 4, 64, 16, torch.float32, seed=6, junk=junk)
        b.check(b.run(pat))


def test_strided_rows(pat):
    b = Batch([(20, [30, 25, 21])], 4, 4, 64, 16, torch.bfloat16, seed=8)
    wide = torch.zeros(3, 12, 64, dtype=torch.bfloat16, device=DEV)
    wide[:, :4] = b.q.to(DEV)
    out = torch.full((3, 6, 64), 5.0, dtype=torch.bfloat16, device=DEV)
    got = b.run(pat, q=wide[:, :4], out=out[:, 1:5])
    b.check(got)
    assert bool((out[:, 0] == 5).all()) and bool((out[:, 5] == 5).all())


def test_same_call_twice_is_the_same_bits(pat):
    b = Batch([(700, [720 + i for i in range(20)])], 8, 2, 128, 64, torch.float32, seed=9)
    assert torch.equal(b.run(pat), b.run(pat))


def test_impossible_lengths_groups_and_pages_give_nan(pat):
    b = Batch([(20, [30, 25, 21])], 4, 4, 64, 16, torch.float32, seed=10)
    got = b.run(pat, max_len=28)                               # sequence 0 is longer than the plan may have them
    assert bool(got[0].isnan().all())
    b.check(got, rows=[1, 2])
    lens = b.lens
    b.lens = [30, -5, 21]
    got = b.run(pat, max_len=40)
    assert bool(got[1].isnan().all())
    b.check(got, rows=[0, 2])
    b.lens = lens
    for start in ([0, 2], [1, 3], [0, 4]):
        keep, b.start = b.start, np.asarray(start)
        assert bool(b.run(pat).isnan().all())
        b.start = keep
    t = b.table.copy()
    t[1, 1] = 10 ** 6                                          # sequence 1's own page; the prefix is read through sequence 0's row
    got = b.run(pat, table=_i32(t))
    assert bool(got[1].isnan().all())
    b.check(got, rows=[0, 2])
    got = b.run(pat, table=_i32(b.table[:, :1]))               # tables too short for the lengths: no sequence has all of its pages
    assert bool(got.isnan().all())
    plan = pat.pat_op_attn_plan(_i32([5, 5, 5]), _i32([0, 3]), _i32([0]), 5, 8, 8, 64)
    plan.hq, plan.hkv = 4, 4                                   # a plan made for other heads
    assert bool(pat.pat_op_attn_shared(b.q.to(DEV), b.k, b.v, _i32(b.table), plan).isnan().all())


def test_a_plan_made_for_fewer_sequences_gives_nan(pat):
    plan = pat.pat_op_attn_plan(_i32([5]), _i32([0, 1]), _i32([0]), 5, 4, 4, 64)
    wide = pat.pat_op_attn_plan(_i32([5] * 2048), _i32([0, 2048]), _i32([0]), 5, 4, 4, 64)
    wide.buf = plan.buf
    k = torch.zeros(1, 4, 16, 64, dtype=torch.bfloat16, device=DEV)
    got = pat.pat_op_attn_shared(torch.ones(2048, 4, 64, device=DEV), k, k.clone(), _i32([[0]] * 2048), wide)
    assert bool(got.isnan().all())


@pytest.mark.parametrize("hq,hkv", [(4, 4), (130, 1)])
def test_lengths_far_beyond_the_table(pat, hq, hkv):
    """The longest length a plan takes, with pages for a few tokens: no number for those, at once, and the others' results as they are."""
    b = Batch([(20, [30, 25]), (0, [40]), (5, [9, 21])], hq, hkv, 64, 16, torch.bfloat16)
    top = 1 << 30
    for lens, shared, good in (([30, 25, top, 9, 21], [20, 0, 5], [0, 1, 3, 4]), ([top, top, 40, 9, 21], [top, 0, 5], [2, 3, 4]), ([top, top - 1, top, top, top], [20, 0, 5], [])):
        plan = pat.pat_op_attn_plan(_i32(lens), _i32(b.start), _i32(shared), top, hq, hkv, 64)
        got = pat.pat_op_attn_shared(b.q.to(DEV), b.k, b.v, _i32(b.table), plan)
        b.check(got, rows=good)
        assert bool(got[[s for s in range(5) if s not in good]].isnan().all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_out_in_place_of_q(pat, dtype):
    b = Batch([(41, [50, 43, 60]), (0, [7])], 8, 2, 128, 16, dtype)
    q = b.q.to(DEV)
    b.check(b.run(pat, q=q, out=q))


def test_captured_step_follows_the_lengths(pat):
    """Plan and attention in one graph: replays with grown lengths, other work between them, each against the eager result."""
    b = Batch([(60, [75 + i for i in range(6)]), (0, [20])], 8, 2, 64, 16, torch.bfloat16, seed=11)
    kv_len, start, shared, table, q = _i32([n - 4 for n in b.lens]), _i32(b.start), _i32(b.shared), _i32(b.table), b.q.to(DEV)
    plan = pat.pat_op_attn_plan(kv_len, start, shared, 100, 8, 2, 64)
    out = torch.empty(7, 8, 64, dtype=torch.bfloat16, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        pat.pat_op_attn_shared(q, b.k, b.v, table, plan, out)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        pat.pat_op_attn_plan(kv_len, start, shared, 100, 8, 2, 64, plan=plan)
        pat.pat_op_attn_shared(q, b.k, b.v, table, plan, out)
    for step in range(4):
        kv_len.copy_(_i32([n - 3 + step for n in b.lens]))
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        junk = torch.randn(1 << 20, device=DEV).sum()          # the program's own work between replays
        for s in range(7):
            n = b.lens[s] - 3 + step
            ref, allow = attend(b.q[s], b.kv[s][0][:n], b.kv[s][1][:n])
            check(out[s], ref, allow)
        assert bool(torch.isfinite(junk))


def test_two_streams_at_once(pat):
    bs = [Batch([(300 + i, [320 + i, 330 + i, 310 + i])], 8, 2, 64, 32, torch.bfloat16, seed=20 + i) for i in range(2)]
    ins = [(b.q.to(DEV), _i32(b.table), pat.pat_op_attn_plan(_i32(b.lens), _i32(b.start), _i32(b.shared), 400, 8, 2, 64)) for b in bs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in bs], [[], []]
    for _ in range(10):
        for i, (b, st, (q, t, plan)) in enumerate(zip(bs, streams, ins)):
            with torch.cuda.stream(st):
                got[i].append(pat.pat_op_attn_shared(q, b.k, b.v, t, plan))
    torch.cuda.synchronize()
    for b, outs in zip(bs, got):
        b.check(outs[0])
        assert all(torch.equal(outs[0], o) for o in outs)


def test_pages_beyond_two_gib(pat):
    """A pool of more than 2^31 bytes and elements: the last pages' offsets pass 32 bits."""
    hkv, P, d = 8, 128, 128
    n_pages = (1 << 31) // (hkv * P * d) + 3
    k = torch.empty(n_pages, hkv, P, d, dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    g = torch.Generator().manual_seed(3)
    own = torch.randn(2, 200, hkv, d, generator=g).to(torch.bfloat16)
    table = [n_pages - 1, n_pages - 2]
    for p, page in enumerate(table):
        part = own[:, p * P:(p + 1) * P]
        k[page, :, :part.shape[1]] = part[0].transpose(0, 1).to(DEV)
        v[page, :, :part.shape[1]] = part[1].transpose(0, 1).to(DEV)
    q = torch.randn(2, 8, d, generator=g).to(torch.bfloat16)
    plan = pat.pat_op_attn_plan(_i32([200, 150]), _i32([0, 2]), _i32([140]), 256, 8, hkv, d)
    got = pat.pat_op_attn_shared(q.to(DEV), k, v, _i32([table, table]), plan)
    for s, n in enumerate((200, 150)):
        ref, allow = attend(q[s], own[0][:n], own[1][:n])
        check(got[s], ref, allow)
    # and the append writes there
    qkv = torch.randn(1, 3 * hkv * d, generator=g).to(torch.bfloat16).to(DEV)
    pat.pat_op_kv_append(qkv, _i32([0]), _i32([201]), pat.pat_op_rope_table(256, d), k, v, _i32([table, table]), torch.empty(1, hkv, d, dtype=torch.bfloat16, device=DEV))
    assert torch.equal(v[n_pages - 2, :, 201 - P].reshape(-1), qkv[0, 2 * hkv * d:])
