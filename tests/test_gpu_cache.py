"""The paged cache in packed planes: writing of rows, and attention over it, against their definitions in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def amq():
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    from paper_1802_00150_b200 import amq as binding
    return binding


def filled(amq, gen, pages, page_size, heads, d, k):
    """A cache of random planes and coefficients (all its pages, those of no sequence too)."""
    cache = amq.new_cache(pages, page_size, heads, d, k)
    for codes, coeffs in (cache[:2], cache[2:]):
        codes.copy_(amq.pack(torch.randn((pages * page_size * heads, k, d), device="cuda", generator=gen)).view_as(codes))
        coeffs.copy_(torch.randn(coeffs.shape, device="cuda", generator=gen) * 0.2 + 0.4)
    return cache


def values(amq, codes, coeffs, d):
    """What the rows stand for, in double."""
    k, wpr = codes.shape[-2:]
    rows = codes.reshape(-1, k, wpr)
    bits = (rows[..., None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
    signs = bits.flatten(2)[:, :, :d].double() * 2 - 1
    return (signs * coeffs.reshape(-1, k, 1).double()).sum(1).view(*codes.shape[:-2], d)


def expected(amq, q, cache, table, lengths, scale):
    """(result, allowed error).  q enters as fixed-point numbers of 23 bits or more relative to a query's largest element and p to the largest of 32 tokens, so
    a score is off by 2^-22 (and its fp32 roundings) of scale * sum_i |a_i| * d * max|q|, a weight by that and 2^-22; a weight's error counts twice
    (in the sum and in the normalisation)."""
    batch, q_len, q_heads, d = q.shape
    pages, page_size, heads = cache[0].shape[:3]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    allowed = torch.zeros((batch, q_len, q_heads, 1), dtype=torch.float64, device="cuda")
    k, v = values(amq, cache[0], cache[1], d).flatten(0, 1), values(amq, cache[2], cache[3], d).flatten(0, 1)
    for b in range(batch):
        n = min(max(int(lengths[b]), 0), table.shape[1] * page_size)
        for i in range(q_len):
            t = torch.arange(max(n - q_len + 1 + i, 0), device="cuda")
            page = table[b].long()[t // page_size]
            slot = (page * page_size + t % page_size)[(page >= 0) & (page < pages)]
            if not len(slot):
                continue
            x = q[b, i].double().view(heads, -1, d)
            s = torch.einsum("hgd,thd->hgt", x, k[slot]) * scale
            p = torch.softmax(s, -1)
            out[b, i] = torch.einsum("hgt,thd->hgd", p, v[slot]).reshape(q_heads, d)
            a = cache[1].flatten(0, 1)[slot].double().abs().sum(-1).amax(0)                             # (heads,)
            size = cache[3].flatten(0, 1)[slot].double().abs().sum(-1).amax(0)[:, None]
            off = abs(scale) * a[:, None] * d * x.abs().amax(-1)                                        # (heads, group)
            allowed[b, i] = (8 * 2.0 ** -22 * (1 + off) * size).reshape(q_heads, 1)
    return out, allowed


def tables(gen, batch, lengths, page_size, spare=2):
    """Pages of the sequences in random order; entries behind a sequence's pages are never read and hold anything."""
    need = [-(-n // page_size) for n in lengths]
    pages = sum(need) + spare
    order = torch.randperm(pages, generator=gen, device="cuda", dtype=torch.int32)
    table = torch.full((batch, max(max(need), 1)), 1 << 30, dtype=torch.int32, device="cuda")
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    return table, pages


def close(got, want):
    ref, allowed = want
    assert ((got.double() - ref).abs() <= allowed).all(), float(((got.double() - ref).abs() / allowed.clamp(min=1e-30)).max())


CASES = [  # lengths, page size, heads, group, d, k, q_len
    ([1], 1, 1, 1, 1, 1, 1), ([300], 16, 8, 1, 64, 4, 1), ([5, 0, 33, 64], 16, 2, 4, 128, 4, 1), ([31, 32, 33, 7, 8, 9], 16, 1, 2, 100, 3, 1),
    ([1500, 1, 700], 1, 5, 3, 100, 3, 3), ([129, 1000], 64, 3, 8, 128, 4, 1), ([2, 5, 1, 0], 4, 2, 5, 127, 2, 4), ([4000], 16, 2, 4, 128, 4, 1),
    ([20000], 64, 1, 1, 128, 4, 1), ([9000], 7, 2, 8, 80, 2, 2), ([400, 399], 16, 16, 1, 128, 1, 1), ([260], 256, 2, 2, 33, 4, 6),
    ([40], 16, 1, 1, 128, 4, 40), ([70000], 64, 1, 8, 128, 3, 1), ([50] * 90, 16, 2, 4, 64, 4, 1), ([3000], 1000, 4, 4, 128, 2, 1),
    # sequences without tokens between others, more than a warp of them; more blocks than CTAs fit the GPU
    ([0, 0, 700, 0, 1, 0, 900] + [0] * 40 + [33, 0, 64] * 10 + [0, 5], 16, 2, 4, 64, 4, 1), ([600, 40], 16, 16, 4, 128, 2, 40),
    ([0] * 70 + [2000], 32, 1, 8, 128, 1, 1), ([513] * 40, 1, 4, 1, 128, 4, 1),
    ([1500, 3, 0, 2040] + [70] * 60, 16, 16, 1, 64, 2, 1), ([1025, 2048, 1, 31] * 4, 16, 64, 2, 40, 1, 2),
]


@pytest.mark.parametrize("lengths,page_size,heads,group,d,k,q_len", CASES)
def test_attention(amq, lengths, page_size, heads, group, d, k, q_len):
    gen = torch.Generator(device="cuda").manual_seed(len(lengths) + d + k)
    table, pages = tables(gen, len(lengths), lengths, page_size)
    cache = filled(amq, gen, pages, page_size, heads, d, k)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    q = torch.randn((len(lengths), q_len, heads * group, d), device="cuda", generator=gen)
    scale = 1 / math.sqrt(d)
    want = expected(amq, q, cache, table, n, scale)
    close(amq.cache_attention(q, cache, table, n, scale), want)
    # views: heads in front of tokens, rows of a wider table, a workspace and a result of the caller's
    other = q.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    wide = torch.full((len(lengths), table.shape[1] + 3), -7, dtype=torch.int32, device="cuda")
    wide[:, 1:1 + table.shape[1]] = table
    ws = amq.new_cache_attention_workspace(len(lengths), q_len, heads * group, heads, d, table.shape[1] * page_size)
    out = torch.full(q.shape, float("nan"), device="cuda")
    again = amq.cache_attention(other, cache, wide[:, 1:1 + table.shape[1]], n, scale, ws, out)
    assert again is out
    close(out, want)
    assert torch.equal(out, amq.cache_attention(q, cache, table, n, scale))     # (bit for bit)


@pytest.mark.parametrize("factor", [1e-30, 1e-3, 30.0, 1e4])
def test_sizes_of_queries(amq, factor):
    """Scores from nothing to one token taking all the weight: the scale goes against the queries' size."""
    gen = torch.Generator(device="cuda").manual_seed(20)
    table, pages = tables(gen, 2, [500, 77], 16)
    cache = filled(amq, gen, pages, 16, 2, 128, 4)
    n = torch.tensor([500, 77], dtype=torch.int32, device="cuda")
    q = torch.randn((2, 1, 8, 128), device="cuda", generator=gen) * factor
    for scale in (0.1 / factor, 0.0, -0.05 / factor):
        close(amq.cache_attention(q, cache, table, n, scale), expected(amq, q, cache, table, n, scale))
    q[0, 0, 3] = 0
    close(amq.cache_attention(q, cache, table, n, 0.1), expected(amq, q, cache, table, n, 0.1) if factor < 1 else expected(amq, q, cache, table, n, 0.1))


def test_one_long_outlier(amq):
    """A query with one element far above the others, coefficients of very different size, zero and negative coefficients."""
    gen = torch.Generator(device="cuda").manual_seed(21)
    table, pages = tables(gen, 1, [333], 16)
    cache = filled(amq, gen, pages, 16, 2, 64, 4)
    cache[1].mul_(torch.tensor([1.0, -0.1, 1e-3, 0.0], device="cuda"))
    cache[3].mul_(torch.tensor([0.0, 1e-4, -1.0, 3.0], device="cuda"))
    cache[3][:, ::3] *= 1e-5
    n = torch.tensor([333], dtype=torch.int32, device="cuda")
    q = torch.randn((1, 1, 6, 64), device="cuda", generator=gen)
    q[..., 5] = 100.0
    close(amq.cache_attention(q, cache, table, n, 0.125), expected(amq, q, cache, table, n, 0.125))


def test_pages_that_are_none_and_lengths_outside(amq):
    gen = torch.Generator(device="cuda").manual_seed(22)
    lengths = [200, 100, 90, 64]
    table, pages = tables(gen, 4, lengths, 16)
    cache = filled(amq, gen, pages, 16, 2, 128, 4)
    table[0, 3] = -1
    table[0, 0] = pages
    table[1, :] = -1                                        # no token left
    table[2, 5] = 2 ** 31 - 1                               # the page that the length ends in
    q = torch.randn((4, 2, 4, 128), device="cuda", generator=gen)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    want = expected(amq, q, cache, table, n, 0.1)
    got = amq.cache_attention(q, cache, table, n, 0.1)
    close(got, want)
    assert (got[1] == 0).all()
    table, pages = tables(gen, 4, [64, 64, 64, 64], 16)
    n = torch.tensor([-5, 0, 2 ** 31 - 1, 1], dtype=torch.int32, device="cuda")        # behind the table: cut there
    want = expected(amq, q, cache, table, n, 0.1)
    got = amq.cache_attention(q, cache, table, n, 0.1)
    close(got, want)
    assert (got[0] == 0).all() and (got[1] == 0).all() and (got[3, 0] == 0).all()


def test_nothing_hidden_counts(amq):
    """NaN and infinities in coefficients that no query sees; a query of NaN answers NaN, and only where it is one."""
    gen = torch.Generator(device="cuda").manual_seed(23)
    lengths = [45, 46, 1]
    table, pages = tables(gen, 3, lengths, 16)
    cache = filled(amq, gen, pages, 16, 2, 128, 4)
    q = torch.randn((3, 1, 4, 128), device="cuda", generator=gen)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    want = expected(amq, q, cache, table, n, 0.1)
    seen = torch.zeros((pages, 16), dtype=torch.bool, device="cuda")
    for b, m in enumerate(lengths):
        t = torch.arange(m, device="cuda")
        seen[table[b].long()[t // 16], t % 16] = True
    for coeffs, bad in ((cache[1], float("nan")), (cache[3], float("inf"))):
        coeffs[~seen] = bad
    for codes in (cache[0], cache[2]):
        codes[~seen] = -1
    close(amq.cache_attention(q, cache, table, n, 0.1), want)
    q[1, 0, 2, 7] = float("nan")
    q[1, 0, 3, 9] = float("inf")
    got = amq.cache_attention(q, cache, table, n, 0.1)
    assert torch.isnan(got[1, 0, 2:]).all() and not torch.isnan(got[1, 0, :2]).any() and not torch.isnan(got[0]).any() and not torch.isnan(got[2]).any()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("part", [1, 3])
def test_coefficients_that_are_none(amq, part, value):
    """A coefficient that is NaN or infinite counts for the queries that see its token, of a few drafted ones the later, and for no other."""
    gen = torch.Generator(device="cuda").manual_seed(27)
    table, pages = tables(gen, 2, [600, 100], 16)
    cache = filled(amq, gen, pages, 16, 2, 128, 4)
    n = torch.tensor([600, 100], dtype=torch.int32, device="cuda")
    q = torch.randn((2, 3, 4, 128), device="cuda", generator=gen)
    want = expected(amq, q, cache, table, n, 0.1)
    last = int(table[0, 599 // 16])                         # the newest token of the first sequence, one head of two
    cache[part][last, 599 % 16, 1, 2] = value
    got = amq.cache_attention(q, cache, table, n, 0.1)
    assert torch.isnan(got[0, 2, 2:]).all()
    got[0, 2, 2:], want[0][0, 2, 2:] = 0, 0
    close(got, want)


def test_a_cache_beyond_32_bit_offsets(amq):
    """Rows behind 2^31 words and 2^32 bytes of codes: a page near the end of a large cache."""
    heads, d, k, page_size = 16, 128, 4, 256
    pages = (5 << 30) // (page_size * heads * k * 16)
    gen = torch.Generator(device="cuda").manual_seed(24)
    cache = amq.new_cache(pages, page_size, heads, d, k)
    small = filled(amq, gen, 2, page_size, heads, d, k)
    for big, part in zip(cache, small):
        big[pages - 1], big[3] = part[0], part[1]
    n = torch.tensor([500], dtype=torch.int32, device="cuda")
    q = torch.randn((1, 1, 16, 128), device="cuda", generator=gen)
    here = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda")
    want = expected(amq, q, small, here, n, 0.1)
    there = torch.tensor([[pages - 1, 3]], dtype=torch.int32, device="cuda")
    close(amq.cache_attention(q, cache, there, n, 0.1), want)
    rows = [t[:1, :1].contiguous() for t in small]         # one token of one sequence
    amq.cache_append(rows[0], rows[1], rows[2], rows[3], cache, there, torch.tensor([200], dtype=torch.int32, device="cuda"), d)
    for big, row in zip(cache, rows):
        assert torch.equal(big[pages - 1, 199], row[0, 0])


@pytest.mark.parametrize("k,group", [(1, 8), (4, 4), (2, 3)])
@pytest.mark.parametrize("lengths", [[40, 0, 3], [1, 0, 0], [0, 0, 0], [130, 2000, 17], [2049, 1, 4096]])
def test_a_table_with_room_for_more(amq, lengths, k, group):
    """Lengths far below what the table has room for: fewer shares than CTAs, and no share without tokens."""
    gen = torch.Generator(device="cuda").manual_seed(26)
    small, pages = tables(gen, 3, [max(n, 1) for n in lengths], 16)
    cache = filled(amq, gen, pages, 16, 2, 128, k)
    table = torch.full((3, 512), -1, dtype=torch.int32, device="cuda")
    table[:, :small.shape[1]] = small
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    q = torch.randn((3, 1, 2 * group, 128), device="cuda", generator=gen)
    want = expected(amq, q, cache, table, n, 0.1)
    ws = torch.full((amq.cache_attention_workspace_bytes(3, 1, 2 * group, 2, 128, 8192),), 255, dtype=torch.uint8, device="cuda")     # (NaN, should it be read)
    close(amq.cache_attention(q, cache, table, n, 0.1, ws), want)


@pytest.mark.parametrize("batch,heads,group,q_len,most,none", [(150, 8, 4, 2, 200, 0.4), (90, 2, 3, 1, 1200, 0.1), (700, 1, 1, 1, 40, 0.0), (140, 8, 1, 1, 700, 0.9),
                                                               (5, 32, 4, 48, 300, 0.4), (75, 8, 4, 1, 2500, 0.2)])
def test_more_sequences_than_shares(amq, batch, heads, group, q_len, most, none):
    """Sequences without tokens among many, one to several in a share, and head counts that leave the line of tokens whole."""
    gen = torch.Generator(device="cuda").manual_seed(batch)
    n = torch.randint(1, most, (batch,), device="cuda", generator=gen, dtype=torch.int32)
    n[torch.rand((batch,), device="cuda", generator=gen) < none] = 0
    small, pages = tables(gen, batch, n.tolist(), 16)
    cache = filled(amq, gen, pages, 16, heads, 64, 2)
    table = torch.full((batch, 160), -1, dtype=torch.int32, device="cuda")
    table[:, :small.shape[1]] = small
    q = torch.randn((batch, q_len, heads * group, 64), device="cuda", generator=gen)
    want = expected(amq, q, cache, table, n, 0.1)
    out = torch.full(q.shape, float("nan"), device="cuda")
    bytes_ = amq.cache_attention_workspace_bytes(batch, q_len, heads * group, heads, 64, 160 * 16)
    assert bytes_
    ws = torch.full((bytes_,), 255, dtype=torch.uint8, device="cuda")           # (NaN, should it be read)
    close(amq.cache_attention(q, cache, table, n, 0.1, ws, out), want)


def test_attention_in_a_graph_and_on_another_stream(amq):
    gen = torch.Generator(device="cuda").manual_seed(25)
    lengths = [3000, 17]
    table, pages = tables(gen, 2, lengths, 16)
    cache = filled(amq, gen, pages, 16, 2, 128, 4)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    q = torch.randn((2, 1, 8, 128), device="cuda", generator=gen)
    want = expected(amq, q, cache, table, n, 0.1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = amq.cache_attention(q, cache, table, n, 0.1)
    torch.cuda.current_stream().wait_stream(side)
    close(got, want)
    ws = amq.new_cache_attention_workspace(2, 1, 8, 2, 128, table.shape[1] * 16)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = amq.cache_attention(q, cache, table, n, 0.1, ws)
    q.copy_(torch.randn(q.shape, device="cuda", generator=gen))
    n.copy_(torch.tensor([1234, 16], dtype=torch.int32, device="cuda"))
    ws.fill_(255)                                           # (a workspace's contents are nobody's)
    want = expected(amq, q, cache, table, n, 0.1)
    graph.replay()
    close(got, want)


@pytest.mark.parametrize("batch,count,page_size,heads,d,k", [(1, 1, 1, 1, 1, 1), (3, 1, 16, 8, 128, 4), (2, 40, 16, 5, 100, 3), (4, 7, 4, 2, 64, 2), (1, 700, 64, 16, 128, 4)])
def test_append(amq, batch, count, page_size, heads, d, k):
    gen = torch.Generator(device="cuda").manual_seed(30 + count)
    lengths = [count + 11 * b for b in range(batch)]
    lengths[-1] = max(1, count // 2)                        # fewer tokens than rows: the first rows are nobody's
    table, pages = tables(gen, batch, lengths, page_size)
    cache = filled(amq, gen, pages, page_size, heads, d, k)
    if batch > 2:
        table[1, (lengths[1] - 1) // page_size] = -3        # no page
    new = []
    for _ in range(2):
        x = torch.randn((batch * count * heads, d), device="cuda", generator=gen)
        codes, coeffs = amq.quantize(x, k, 2)
        new += [codes.view(batch, count, heads, k, -1), coeffs.view(batch, count, heads, k)]
    want = [t.clone() for t in cache]
    for b in range(batch):
        for i in range(count):
            t = lengths[b] - count + i
            if t >= 0 and 0 <= int(table[b, t // page_size]) < pages:
                for w, x in zip(want, new):
                    w[int(table[b, t // page_size]), t % page_size] = x[b, i]
    amq.cache_append(*new, cache, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), d)
    for g, w in zip(cache, want):
        assert torch.equal(g, w)


def test_append_outside_the_table(amq):
    gen = torch.Generator(device="cuda").manual_seed(31)
    cache = filled(amq, gen, 3, 4, 2, 128, 2)
    before = [t.clone() for t in cache]
    new = [t[:1, :2].repeat(3, 1, *([1] * (t.dim() - 2))).contiguous() for t in cache]
    table = torch.tensor([[0, 1]] * 3, dtype=torch.int32, device="cuda")
    amq.cache_append(*new, cache, table, torch.tensor([-1, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda"), 128)
    for g, w in zip(cache, before):
        assert torch.equal(g, w)


def test_refused_tensors(amq):
    cache = amq.new_cache(4, 16, 2, 128, 4)
    table, n = torch.zeros((1, 4), dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    q = torch.zeros((1, 1, 4, 128), device="cuda")
    amq.cache_attention(q, cache, table, n, 0.1)
    bad = [(q.double(), cache, table, n), (q[0], cache, table, n), (q.cpu(), cache, table, n), (torch.zeros((1, 1, 4, 256), device="cuda"), cache, table, n),
           (torch.zeros((1, 1, 128, 4), device="cuda").transpose(2, 3), cache, table, n), (q, cache, table.long(), n), (q, cache, table[0], n),
           (q, cache, table, n.long()), (q, cache, table, torch.ones(2, dtype=torch.int32, device="cuda")), (q, (cache[0], cache[1], cache[2], cache[3][:1]), table, n),
           (torch.zeros((2, 1, 4, 128), device="cuda"), cache, table, n), (q, tuple(t.cpu() for t in cache), table, n)]
    for args in bad:
        with pytest.raises(TypeError):
            amq.cache_attention(*args, 0.1)
    with pytest.raises(TypeError):
        amq.cache_attention(q, cache, table, n, 0.1, None, torch.zeros((1, 1, 4, 64), device="cuda"))
    with pytest.raises(amq.AmqError):                       # three query heads over two
        amq.cache_attention(q[:, :, :3], cache, table, n, 0.1)
    rows = [torch.zeros((1, 1, 2, 4, 4), dtype=torch.int32, device="cuda"), torch.zeros((1, 1, 2, 4), device="cuda")] * 2
    amq.cache_append(*rows, cache, table, n, 128)
    with pytest.raises(TypeError):
        amq.cache_append(rows[0][:, :, :1], rows[1], rows[2], rows[3], cache, table, n, 128)
    with pytest.raises(TypeError):
        amq.cache_append(rows[0], rows[1][:, :, :1], rows[2], rows[3], cache, table, n, 128)
