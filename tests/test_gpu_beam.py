"""Beam search's choice and the reordering of states against their definitions in 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def amq():
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    from paper_1802_00150_b200 import amq as binding
    return binding


def expected(logits, scores, finished, eos):
    """The definition, in double: all pairs' scores, a stable descending order.  (A library's sum over a row may depend on where the row starts, so that
    equal rows differ by 1e-15: scores are rounded to 1e-11, far above that and far below what fp32 logits near a maximum differ by.)"""
    batch, beams = scores.shape
    vocab = logits.shape[1]
    z = logits.double()
    good = ~torch.isnan(z).any(1) & ~torch.isposinf(z).any(1) & ~torch.isneginf(z).all(1)
    safe = torch.where(good[:, None], z, 0.0)
    logp = torch.where(good[:, None], safe - torch.logsumexp(safe, 1, keepdim=True), -torch.inf)
    if finished is not None:
        done = finished.view(-1, 1) != 0
        logp = torch.where(done, torch.where(torch.arange(vocab, device="cuda") == eos, 0.0, -torch.inf).double(), logp)
    base = torch.where(torch.isfinite(scores), scores.double(), -torch.inf)
    total = ((base.view(-1, 1) + logp).view(batch, -1) * 1e11).round() / 1e11
    best, at = torch.sort(total, dim=1, descending=True, stable=True)
    best, at = best[:, :beams], at[:, :beams]
    parents, tokens = at // vocab, at % vocab
    ended = tokens == eos
    if finished is not None:
        ended |= torch.gather(finished, 1, parents) != 0
    return best, parents.int(), tokens.int(), ended.int()


def same(got, want):
    """Indices exactly; a score is rounded once, from a double that holds a log-sum-exp summed in fp32: within 2^-24 of itself and 2e-6."""
    for g, w in zip(got[1:], want[1:]):
        assert torch.equal(g, w)
    a, b = got[0].double(), want[0]
    gone = torch.isinf(b)
    assert torch.equal(gone, torch.isinf(a)) and (a[gone] < 0).all()
    assert ((a - b)[~gone].abs() <= 2.0 ** -24 * b[~gone].abs() + 2e-6).all()


@pytest.mark.parametrize("batch,beams,vocab", [(1, 1, 1), (1, 4, 1), (2, 3, 5), (1, 5, 9999), (3, 8, 42000), (7, 2, 100), (20, 10, 2047), (2, 16, 20001),
                                               (1, 32, 50000), (300, 4, 333), (2, 32, 31), (1, 1, 200000), (5, 7, 2049),
                                               (14, 5, 700), (15, 5, 700), (33, 8, 9000), (34, 8, 9000), (66, 4, 26000), (67, 4, 26000), (67, 9, 3), (70, 32, 2000)])
def test_choice(amq, batch, beams, vocab):
    gen = torch.Generator(device="cuda").manual_seed(batch + beams + vocab)
    logits = torch.randn((batch * beams, vocab), device="cuda", generator=gen) * 2.5
    scores = -20 * torch.rand((batch, beams), device="cuda", generator=gen)
    eos = vocab // 3
    finished = (torch.rand((batch, beams), device="cuda", generator=gen) < 0.2).int()
    same(amq.beam_select(logits, scores), expected(logits, scores, None, -1))
    same(amq.beam_select(logits, scores, finished, eos), expected(logits, scores, finished, eos))
    same(amq.beam_select(logits, scores, None, eos), expected(logits, scores, None, eos))


@pytest.mark.parametrize("offset,spare", [(0, 0), (1, 0), (2, 3), (3, 14)])
def test_rows_at_any_offset(amq, offset, spare):
    gen = torch.Generator(device="cuda").manual_seed(4)
    wide = torch.randn((12, offset + 4097 + spare), device="cuda", generator=gen)
    scores = -torch.rand((3, 4), device="cuda", generator=gen)
    logits = wide[:, offset:offset + 4097]
    same(amq.beam_select(logits, scores), expected(logits, scores, None, -1))


@pytest.mark.parametrize("beams,vocab", [(4, 3000), (8, 40), (32, 9000), (5, 9999)])
def test_equal_logits_go_to_the_first(amq, beams, vocab):
    """All logits alike (more ties than a slice's list holds), equal rows and equal scores: the lowest pairs."""
    scores = torch.full((2, beams), -1.0, device="cuda")
    logits = torch.zeros((2 * beams, vocab), device="cuda")
    same(amq.beam_select(logits, scores), expected(logits, scores, None, -1))
    # a few values over and over
    gen = torch.Generator(device="cuda").manual_seed(5)
    row = torch.randint(0, 3, (2, 1, vocab), device="cuda", generator=gen).float()
    logits = row.expand(2, beams, vocab).reshape(2 * beams, vocab).contiguous()
    same(amq.beam_select(logits, scores), expected(logits, scores, None, -1))
    # Ascending and descending rows: beams whose scores are equal as numbers, but not as sums in one order.  A log-sum-exp in fp32 is off by up to 2e-6:
    # the weighted mean of |x| 2^-24 (at most log(vocab) 2^-24 = 7e-7) for the argument's rounding, 2^-22 for exp itself, and 17 additions of 2^-24
    # (8 in a thread, 5 across a warp, 3 across its chunks) = 1e-6.  So the parents may change places here; the scores and, parent by parent, the tokens may not.
    up = torch.arange(vocab, device="cuda").float() / 100
    logits = torch.stack([up, up.flip(0)] * beams)
    got, want = amq.beam_select(logits, scores), expected(logits, scores, None, -1)
    assert ((got[0].double() - want[0]).abs() <= 2.0 ** -24 * want[0].abs() + 2e-6).all()
    assert torch.equal(got[1].sort(1).values, torch.arange(beams, device="cuda", dtype=torch.int32).expand(2, beams))     # each beam's best token
    row = got[1] + beams * torch.arange(2, device="cuda", dtype=torch.int32)[:, None]
    assert torch.equal(got[2], torch.where(row % 2 == 0, vocab - 1, 0).int())


@pytest.mark.parametrize("batch,beams,vocab", [(1, 8, 128000), (16, 20, 42000), (38, 32, 9999), (2, 12, 300000), (40, 6, 1000), (40, 9, 1000), (3, 4, 100001),
                                               (1, 32, 260)])
def test_order_within_a_row(amq, batch, beams, vocab):
    """Rows of any order: the largest last (every piece passes what the one before it left as a bound), first, in a few places of many, all but a few -inf."""
    gen = torch.Generator(device="cuda").manual_seed(batch * beams + vocab)
    logits = torch.randn((batch * beams, vocab), device="cuda", generator=gen) * 2.5
    scores = -20 * torch.rand((batch, beams), device="cuda", generator=gen)
    up = torch.sort(logits, dim=1).values
    for z in (up, up.flip(1).contiguous(), torch.cat((up[:, vocab // 3:], up[:, :vocab // 3]), 1).contiguous(), torch.where(logits > 0, logits.round(), 0.0),
              torch.where(logits > 9, logits, -torch.inf), torch.where(logits > 9, 0.0, logits.clamp(max=-0.0))):
        same(amq.beam_select(z, scores), expected(z, scores, None, -1))


def test_zeros_of_either_sign_are_alike(amq):
    logits = torch.full((4, 5000), -3.0, device="cuda")
    logits[:, 7::11] = -0.0
    logits[:, 4::23] = 0.0
    scores = torch.tensor([[-1.0, -2.0, -3.0, -4.0]], device="cuda")
    same(amq.beam_select(logits, scores), expected(logits, scores, None, -1))


def test_masked_tokens_and_dead_beams(amq):
    gen = torch.Generator(device="cuda").manual_seed(6)
    batch, beams, vocab, eos = 6, 4, 700, 9
    logits = torch.randn((batch, beams, vocab), device="cuda", generator=gen)
    scores = -torch.rand((batch, beams), device="cuda", generator=gen)
    finished = torch.zeros((batch, beams), dtype=torch.int32, device="cuda")
    inf = float("inf")
    logits[0, :, 5:] = -inf                                 # five tokens left
    logits[1, 1] = -inf                                     # a beam without a continuation
    logits[1, 2, 100] = float("nan")
    logits[1, 3, 100] = inf
    scores[2, 1:] = -inf                                    # the first step: one beam counts
    logits[3] = -inf                                        # nothing at all
    logits[4] = -inf
    logits[4, 2, 17] = 0.5                                  # a single pair
    scores[4, 0] = float("nan")
    scores[4, 1] = inf
    finished[5] = 1                                         # all ended
    logits[5] = float("nan")                                # (not read)
    logits = logits.view(batch * beams, vocab)
    same(amq.beam_select(logits, scores, finished, eos), expected(logits, scores, finished, eos))
    # type's lowest value as a mask
    logits = torch.randn((8, vocab), device="cuda", generator=gen)
    logits[:, ::2] = torch.finfo(torch.float32).min
    same(amq.beam_select(logits, scores[:2], None, -1), expected(logits, scores[:2], None, -1))


def test_one_beam_is_greedy(amq):
    gen = torch.Generator(device="cuda").manual_seed(7)
    logits = torch.randn((9, 10000), device="cuda", generator=gen)
    scores, parents, tokens, _ = amq.beam_select(logits, torch.zeros((9, 1), device="cuda"))
    logp, arg = amq.log_softmax_argmax(logits)
    assert torch.equal(tokens.view(-1), arg) and (parents == 0).all()
    assert (scores.view(-1) - logp.amax(1)).abs().max() <= 4e-6


def test_choice_over_its_own_scores(amq):
    """The C call may write the scores and flags over those it reads."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    logits = torch.randn((12, 5000), device="cuda", generator=gen)
    scores = -torch.rand((3, 4), device="cuda", generator=gen)
    finished = torch.zeros((3, 4), dtype=torch.int32, device="cuda")
    want = expected(logits, scores, finished, 3)
    parents, tokens = torch.empty_like(finished), torch.empty_like(finished)
    amq._check(amq._native.amq_beam_select(logits, 5000, 5000, scores, finished, 3, 3, 4, scores, parents, tokens, finished))
    same((scores, parents, tokens, finished), want)


def test_choice_repeats_in_a_graph_and_on_another_stream(amq):
    gen = torch.Generator(device="cuda").manual_seed(9)
    logits = torch.randn((64, 9999), device="cuda", generator=gen)
    scores = -torch.rand((16, 4), device="cuda", generator=gen)
    want = expected(logits, scores, None, -1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = amq.beam_select(logits, scores)
    torch.cuda.current_stream().wait_stream(side)
    same(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = amq.beam_select(logits, scores)
    logits.copy_(torch.randn((64, 9999), device="cuda", generator=gen))
    graph.replay()
    same(got, expected(logits, scores, None, -1))


def gathered(t, parents):
    return t[torch.arange(t.shape[0], device="cuda")[:, None], parents.long().clamp(0, t.shape[1] - 1)]


@pytest.mark.parametrize("batch,beams", [(1, 1), (1, 4), (3, 5), (2, 8), (5, 16), (2, 32), (256, 2)])
def test_reordering(amq, batch, beams):
    gen = torch.Generator(device="cuda").manual_seed(batch * beams)
    parents = torch.randint(-2, beams + 2, (batch, beams), device="cuda", generator=gen, dtype=torch.int32)      # (outside: clamped)
    states = [torch.randn((batch, beams, 1024), device="cuda", generator=gen), torch.randn((batch, beams, 7, 3), device="cuda", generator=gen),
              torch.randint(0, 99, (batch, beams, 30), device="cuda", generator=gen, dtype=torch.int32),
              torch.randn((batch, beams, 9), device="cuda", generator=gen, dtype=torch.float64),
              torch.randn((batch, beams, 66), device="cuda", generator=gen).half(), torch.empty((batch, beams, 0), device="cuda")]
    want = [gathered(t, parents) for t in states]
    out = amq.beam_reorder(states, parents, [torch.empty_like(t) for t in states])
    for g, w in zip(out, want):
        assert torch.equal(g, w)
    assert amq.beam_reorder(states, parents) is states
    for g, w in zip(states, want):
        assert torch.equal(g, w)
    wide = [torch.randn((batch, beams, 256), device="cuda", generator=gen)]     # all rows in 16-byte words
    want = gathered(wide[0], parents)
    amq.beam_reorder(wide, parents)
    assert torch.equal(wide[0], want)


def test_reordering_of_views(amq):
    """The used part of wider rows, in place and into another stride: what lies between the rows stays."""
    gen = torch.Generator(device="cuda").manual_seed(10)
    parents = torch.tensor([[1, 1, 0], [2, 0, 2]], dtype=torch.int32, device="cuda")
    wide = torch.randn((2, 3, 20), device="cuda", generator=gen)
    before, used = wide.clone(), wide[:, :, 3:14]
    out = torch.zeros((2, 3, 13), device="cuda")
    amq.beam_reorder([used], parents, [out[:, :, 1:12]])
    assert torch.equal(out[:, :, 1:12], gathered(before[:, :, 3:14], parents)) and (out[:, :, 0] == 0).all() and (out[:, :, 12] == 0).all()
    amq.beam_reorder([used], parents)
    assert torch.equal(used, gathered(before[:, :, 3:14], parents))
    assert torch.equal(wide[:, :, :3], before[:, :, :3]) and torch.equal(wide[:, :, 14:], before[:, :, 14:])


def test_refused_tensors(amq):
    parents = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    good = torch.zeros((2, 3, 8), device="cuda")
    for states, out in (([good.cpu()], None), ([torch.zeros((3, 2, 8), device="cuda")], None), ([good.transpose(1, 2).contiguous().transpose(1, 2)], None),
                        ([torch.zeros((3, 2, 8), device="cuda").transpose(0, 1)], None), ([good], [good.double()]), ([good], []), (good[0, 0, 0], None)):
        with pytest.raises(TypeError):
            amq.beam_reorder(states, parents, out)
    with pytest.raises(TypeError):
        amq.beam_reorder([good], parents.long())
    with pytest.raises(amq.AmqError):
        amq.beam_reorder([good] * 9, parents)
    with pytest.raises(amq.AmqError):                       # rows of three bytes
        amq.beam_reorder([torch.zeros((2, 3, 3), dtype=torch.uint8, device="cuda")], parents)
    logits, scores = torch.zeros((6, 50), device="cuda"), torch.zeros((2, 3), device="cuda")
    for bad in (logits[:5], logits.double(), logits.cpu(), torch.zeros((50, 6), device="cuda").T):
        with pytest.raises(TypeError):
            amq.beam_select(bad, scores)
    with pytest.raises(TypeError):
        amq.beam_select(logits, scores, torch.zeros((3, 2), dtype=torch.int32, device="cuda"), 1)
    with pytest.raises(TypeError):
        amq.beam_select(logits, scores, torch.zeros((2, 3), dtype=torch.int64, device="cuda"), 1)
    with pytest.raises(amq.AmqError):
        amq.beam_select(logits, scores, torch.zeros((2, 3), dtype=torch.int32, device="cuda"), -1)
    with pytest.raises(amq.AmqError):
        amq.beam_select(torch.zeros((66, 50), device="cuda"), torch.zeros((2, 33), device="cuda"))
