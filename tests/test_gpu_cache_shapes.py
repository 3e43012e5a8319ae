"""Attention over the packed cache, and its append: prompts of some hundred queries, coefficients at addresses of 4 bytes."""
import pytest
import torch

from test_gpu_cache import amq, close, expected, filled, tables  # noqa: F401

pytestmark = pytest.mark.gpu


def shifted(t):
    """The same contiguous tensor, 4 bytes behind a boundary of 16."""
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
    flat[1:] = t.flatten()
    return flat[1:].view(t.shape)


@pytest.mark.parametrize("lengths,room,heads,group,d,k", [([300, 299, 3, 0], 19, 2, 4, 128, 4), ([300, 2000, 301], 200, 1, 4, 128, 4), ([700], 44, 3, 1, 100, 3),
                                                          ([450, 1], 300, 2, 3, 64, 2)])
def test_prompts(amq, lengths, room, heads, group, d, k):  # noqa: F811
    """As many queries as the first sequence has tokens: the causal edge passes through every tile, and the shorter sequences' first queries see nothing."""
    gen = torch.Generator(device="cuda").manual_seed(lengths[0])
    small, pages = tables(gen, len(lengths), lengths, 16)
    table = torch.full((len(lengths), max(room, small.shape[1])), -1, dtype=torch.int32, device="cuda")
    table[:, :small.shape[1]] = small
    cache = filled(amq, gen, pages, 16, heads, d, k)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    q_len = lengths[0]
    q = torch.randn((len(lengths), q_len, heads * group, d), device="cuda", generator=gen)
    got = amq.cache_attention(q, cache, table, n, 0.1)
    close(got, expected(amq, q, cache, table, n, 0.1))
    for b, m in enumerate(lengths):
        assert (got[b, :max(q_len - m, 0)] == 0).all()


@pytest.mark.parametrize("k", [1, 2, 3, 4])
@pytest.mark.parametrize("which", [(1,), (3,), (1, 3)])
def test_coefficients_at_any_address(amq, k, which):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(k)
    lengths = [1500, 40, 333]
    table, pages = tables(gen, 3, lengths, 16)
    cache = list(filled(amq, gen, pages, 16, 4, 128, k))
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    q = torch.randn((3, 1, 8, 128), device="cuda", generator=gen)
    want = amq.cache_attention(q, cache, table, n, 0.1)
    rows = [t[:2, :3].reshape(3, 2, *t.shape[2:]).contiguous() for t in cache]
    after = [t.clone() for t in cache]
    amq.cache_append(*rows, after, table, n, 128)
    for i in which:
        cache[i] = shifted(cache[i])
    assert torch.equal(amq.cache_attention(q, cache, table, n, 0.1), want)
    amq.cache_append(rows[0], shifted(rows[1]), rows[2], rows[3], cache, table, n, 128)
    for g, w in zip(cache, after):
        assert torch.equal(g, w)
