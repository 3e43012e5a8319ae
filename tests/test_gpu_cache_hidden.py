"""Attention over the packed cache: what a query does not see leaves its result alone, bit for bit."""
import pytest
import torch

from test_gpu_cache import amq, close, expected, filled, tables  # noqa: F401

pytestmark = pytest.mark.gpu


# lengths, room of the table, heads, group, d, k, q_len: whole sequences by twelve and by four warps, shares with one and with two row tiles
CASES = [([45, 7], 64, 2, 4, 128, 4, 3), ([33], 48, 1, 1, 64, 2, 2), ([300, 64, 41], 512, 16, 4, 128, 4, 6), ([1500, 65], 4096, 2, 3, 100, 3, 3), ([2500], 4096, 1, 8, 128, 4, 2),
         ([2100, 2081], 4096, 2, 2, 128, 1, 40), ([600, 90], 4096, 1, 4, 128, 2, 4)]


@pytest.mark.parametrize("value", [1e3, 1e6, 1e10, -1e30, 3e38, float("nan"), float("inf")])
@pytest.mark.parametrize("lengths,room,heads,group,d,k,q_len", CASES)
def test_later_tokens_do_not_count(amq, lengths, room, heads, group, d, k, q_len, value):  # noqa: F811
    """The coefficients of the newest token of each sequence, which only the last of its queries sees, at any size."""
    gen = torch.Generator(device="cuda").manual_seed(len(lengths) + d + k)
    small, pages = tables(gen, len(lengths), lengths, 16)
    table = torch.full((len(lengths), room // 16), -1, dtype=torch.int32, device="cuda")
    table[:, :small.shape[1]] = small
    cache = filled(amq, gen, pages, 16, heads, d, k)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    q = torch.randn((len(lengths), q_len, heads * group, d), device="cuda", generator=gen)
    want = expected(amq, q, cache, table, n, 0.1)
    before = amq.cache_attention(q, cache, table, n, 0.1)
    close(before, want)
    for part in (3, 1):
        for b, m in enumerate(lengths):
            cache[part][table[b, (m - 1) // 16].long(), (m - 1) % 16] = value
        after = amq.cache_attention(q, cache, table, n, 0.1)
        assert torch.equal(after[:, :-1], before[:, :-1])


@pytest.mark.parametrize("k", [1, 2, 3, 4])
def test_every_query_sees_its_own_last_token(amq, k):  # noqa: F811
    """Coefficients that grow a hundredfold from token to token: each query's result lies by its own largest."""
    gen = torch.Generator(device="cuda").manual_seed(k)
    q_len = 6
    table, pages = tables(gen, 1, [40], 16)
    cache = filled(amq, gen, pages, 16, 2, 128, k)
    for i in range(q_len):
        t = 40 - q_len + i
        cache[3][table[0, t // 16].long(), t % 16] *= 100.0 ** (i + 1)
    n = torch.tensor([40], dtype=torch.int32, device="cuda")
    q = torch.randn((1, q_len, 8, 128), device="cuda", generator=gen)
    close(amq.cache_attention(q, cache, table, n, 0.1), expected(amq, q, cache, table, n, 0.1))
