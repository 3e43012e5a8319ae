"""Attention over the packed cache: every digit of its fixed-point numbers counts.

Queries, and weights times coefficients, are four signed digits of 8 bits each.  Terms of 23-bit integers cancel here up to a few units, and so that the upper two
digits of the terms are alike: what is left comes from the lower two digits alone, and everything after is small integers, exact in fp32.  A digit lost, doubled
or weighted wrongly is an error of a score's or a result's own size."""
import pytest
import torch

from test_gpu_cache import amq, values  # noqa: F401

pytestmark = pytest.mark.gpu


def integer(rng, position, difference):
    """An integer of [2^22, 2^23) that is held times 2^(7 - position), such that it and it less `difference` agree in the upper two digits (the number plus 0x80808080
    has the digits, plus 128, as its bytes)."""
    shift = 7 - position
    while True:
        q = int(torch.randint(1 << 22, 1 << 23, (1,), generator=rng))
        if (((q << shift) + 0x8080) & 0xffff) >= difference << shift:
            return q


def table_of(pages, room):
    t = torch.full((1, room), -1, dtype=torch.int32, device="cuda")
    t[0, :pages] = torch.arange(pages, dtype=torch.int32, device="cuda")
    return t


@pytest.mark.parametrize("room", [3, 256])                 # whole sequences, shares
@pytest.mark.parametrize("group", [1, 3, 8, 64])
def test_digits_of_queries(amq, group, room):  # noqa: F811
    """Two elements Q and -(Q - delta) at places of one bit position, whose bits are alike in every token: a score is +-delta times the scale, exact but for its own
    rounding and the exponential's: a weight is within 2^-21 of itself, and a sum of 48 of them and the quotient within as much again."""
    rng = torch.Generator().manual_seed(group)
    d, length, page, heads = 128, 47, 16, 64 // group if group in (1, 8, 64) else 8
    rows = heads * group
    bits = torch.rand((length, heads, d), generator=rng) < 0.5
    q = torch.zeros((1, 1, rows, d))
    for row in range(rows):
        head = row // group
        position = row % 8
        words = torch.randperm(16, generator=rng)[:2]      # (a byte of the plane each)
        a, b = (int(w) * 8 + position for w in words)
        if group == 1:                                      # (the rows of a head share its planes, so only a row of its own may choose)
            bits[:, head, b] = bits[:, head, a]
        else:
            a, b = row % group % 64 // 8 * 16 + position, row % group % 64 // 8 * 16 + 8 + position
            bits[:, head, b] = bits[:, head, a]
        delta = int(torch.randint(1, 40, (1,), generator=rng))
        value = integer(rng, position, delta)
        q[0, 0, row, a], q[0, 0, row, b] = value, -(value - delta)
    cache = amq.new_cache(3, page, heads, d, 1)
    planes = torch.zeros((3 * page, heads, 1, d))
    planes[:length, :, 0] = bits.float() - 0.5
    cache[0].copy_(amq.pack(planes.view(-1, 1, d).cuda()).view_as(cache[0]))
    cache[2].copy_(amq.pack(torch.randn((3 * page * heads, 1, d), generator=rng).cuda()).view_as(cache[2]))
    cache[1].fill_(1.0)
    cache[3].fill_(1.0)
    n = torch.tensor([length], dtype=torch.int32, device="cuda")
    q = q.cuda()
    got = amq.cache_attention(q, cache, table_of(3, room), n, 1 / 16)
    k, v = values(amq, cache[0], cache[1], d).flatten(0, 1)[:length], values(amq, cache[2], cache[3], d).flatten(0, 1)[:length]
    s = torch.einsum("hgd,thd->hgt", q[0, 0].double().view(heads, group, d), k) / 16
    want = torch.einsum("hgt,thd->hgd", torch.softmax(s, -1), v).view(1, 1, rows, d)
    assert ((got.double() - want).abs() <= 2.0 ** -19).all()


@pytest.mark.parametrize("room", [3, 256])
@pytest.mark.parametrize("q_len", [1, 8])
@pytest.mark.parametrize("k", [1, 2, 3, 4])
def test_digits_of_values(amq, k, q_len, room):  # noqa: F811
    """Coefficients A and -(A - delta) with planes alike, of one token (k > 1) or of two (k = 1), under a scale of 0, which weighs all tokens alike: what is left is the
    mean of +-delta, a small integer over the number of tokens.  Its sums are exact; the quotient and the joins of twelve warps or shares are rounded, in fp32,
    16 times at most."""
    rng = torch.Generator().manual_seed(10 * k + q_len)
    d, length, page, heads, group = 128, 48, 16, 2, 4
    if k == 1:
        q_len = 1                                           # (an odd number of tokens would leave half a pair)
    cache = amq.new_cache(3, page, heads, d, k)
    planes = torch.randn((length, heads, k, d), generator=rng)
    coeffs = torch.zeros((length, heads, k))
    for t in range(length):
        for h in range(heads):
            for i in range(0, k - 1, 2) if k > 1 else range(1):
                delta = int(torch.randint(1, 40, (1,), generator=rng))
                value = integer(rng, 0, delta)
                if k > 1:
                    coeffs[t, h, i], coeffs[t, h, i + 1] = value, -(value - delta)
                    planes[t, h, i + 1] = planes[t, h, i]
                elif t % 2 == 0:
                    coeffs[t, h, 0], coeffs[t + 1, h, 0] = value, -(value - delta)
                    planes[t + 1, h] = planes[t, h]
    cache[0].copy_(amq.pack(torch.randn((length * heads, k, d), generator=rng).cuda()).view_as(cache[0]))
    cache[1].fill_(0.5)
    cache[2].copy_(amq.pack(planes.view(-1, k, d).cuda()).view_as(cache[2]))
    cache[3].copy_(coeffs.cuda().view_as(cache[3]))
    n = torch.tensor([length], dtype=torch.int32, device="cuda")
    q = torch.randn((1, q_len, heads * group, d), generator=rng).cuda()
    got = amq.cache_attention(q, cache, table_of(3, room), n, 0.0).view(q_len, heads, group, d).double()
    v = values(amq, cache[2], cache[3], d).flatten(0, 1)
    for i in range(q_len):
        seen = length - q_len + 1 + i
        want = v[:seen].mean(0)[:, None].expand(heads, group, d)
        size = v[:seen].abs().mean(0)[:, None]
        assert ((got[i] - want).abs() <= 16 * 2.0 ** -24 * size).all()
