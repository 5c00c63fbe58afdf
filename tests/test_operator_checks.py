"""The checks of operator_probes.py refuse results that lack a piece of the data, planted in the reference here: needs no GPU."""
import pytest
import torch

import operator_probes as probes


@pytest.mark.parametrize("k", [1111, 9800, 28672])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_block_of_columns_too_few_or_too_many_is_seen(k, dtype):
    x, w = probes.integers(3, k, 1), probes.integers(40, k, 2)
    ref = probes.project(x, w)
    assert probes.project_ok(ref.to(dtype), ref)
    for block in (0, k // 256, (k - 1) // 128 - 1):
        at = slice(block * 128, block * 128 + 128)
        piece = probes.project(x[:, at], w[:, at])
        assert not probes.project_ok((ref - piece).to(dtype), ref)
        assert not probes.project_ok((ref + piece).to(dtype), ref)


def test_a_column_too_few_is_seen_in_fp32():
    x, w = probes.integers(3, 28672, 1), probes.integers(40, 28672, 2)
    ref = probes.project(x, w)
    assert not probes.project_ok((ref - probes.project(x[:, 5:6], w[:, 5:6])).float(), ref)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,d", [(41, 64), (7000, 128), (30000, 64)])
def test_a_tile_of_keys_too_few_or_too_many_is_seen(n, d, dtype):
    c = probes.Cache([(n // 2, [n])], 1, d, 16, 3)
    v = c.kv[0][1]
    ref = probes.mean(v, 2)
    assert probes.mean_ok(ref.to(dtype), ref)
    for t in (0, n // 64 * 32, (n - 1) // 32 * 32):
        cut = torch.cat([v[:t], v[t + 32:]])
        assert not probes.mean_ok(probes.mean(cut, 2).to(dtype), ref)
        twice = torch.cat([v, v[t:t + 32]])
        assert not probes.mean_ok(probes.mean(twice, 2).to(dtype), ref)


def test_the_cache_holds_what_its_sequences_hold():
    c = probes.Cache([(37, [37, 50, 64]), (0, [1])], 2, 64, 16, 4)
    for s, n in enumerate(c.lens):
        at = torch.arange(n)
        page = torch.as_tensor(c.table[s])[at // 16]
        assert torch.equal(c.k[page, :, at % 16], c.kv[s][0]) and torch.equal(c.v[page, :, at % 16], c.kv[s][1])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_value_from_the_next_place_is_seen(dtype):
    c = probes.Cache([(0, [3000])], 1, 64, 16, 5)
    k, v = c.kv[0]
    at = [0, 31, 32, 2999]
    assert probes.alone(k, at, 4)
    q = probes.peaked(k, at, 4)
    p = torch.softmax((q.double() @ k[:, 0].double().t()) / 8, -1)
    out = p @ v[:, 0].double()
    assert probes.peak_ok(out.to(dtype), v, at)
    assert not probes.peak_ok(out.to(dtype), v, [1, 31, 32, 2999])


def test_weights_and_queries_of_fewer_terms_are_seen():
    """Cut off after two bf16 terms, where fp32 results are promised three."""
    cut = lambda x, bits: (x.float().view(torch.int32) & -(1 << bits)).view(torch.float32).double()      # noqa: E731
    two = lambda x: cut(x, 16) + cut(x.double() - cut(x, 16), 16)      # noqa: E731
    q = probes.queries(64, 64, 1)[:, 0]
    n, score = 500, q.double() / 8
    p = torch.exp(-score)
    assert probes.weights_ok((n * p / (1 + n * p)).float(), n, score)
    assert not probes.weights_ok((n * two(p) / (1 + n * p)).float(), n, score)
    assert probes.queries_ok(torch.sigmoid(-score).float(), score)
    assert not probes.queries_ok(torch.sigmoid(-two(q) / 8).float(), score)
