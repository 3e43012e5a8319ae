"""Beam search's choice at the ends of what it accepts: logits at the ends of fp32, scores that do not tell
logits apart, vocabularies up to 2^31."""
import math

import pytest
import torch

from test_gpu_beam import amq  # noqa: F401

pytestmark = pytest.mark.gpu


def test_the_largest_vocabulary(amq):  # noqa: F811
    """2^31 - 2 tokens, one beam and (half as many) two: the best are the row's first and last tokens, all others are -inf (ten billion bytes of them)."""
    most = 2 ** 31 - 2
    logits = torch.full((most,), -math.inf, device="cuda")
    at = [0, 1, most // 2 - 1, most // 2, most - 2, most - 1]
    for value, place in enumerate(at):
        logits[place] = float(value)
    for beams in (1, 2):
        vocab = most // beams
        rows = logits[:beams * vocab].view(beams, vocab)
        scores = torch.zeros((1, beams), device="cuda")
        got, parents, tokens, _ = amq.beam_select(rows, scores)
        best = []
        for b in range(beams):
            here = [(float(v), p - b * vocab) for v, p in enumerate(at) if b * vocab <= p < (b + 1) * vocab]
            lse = math.log(sum(math.exp(v) for v, _ in here))
            best += [(v - lse, b, t) for v, t in here]
        best = sorted(best, reverse=True)[:beams]
        # (two beams: 0, 1, 2 and 3, 4, 5, whose best scores are one number, -log(1 + 1/e + 1/e^2); as sums of fp32 exponentials they differ by some 2^-24, so
        # the beams may change places: every score is each beam's best, parent by parent the tokens are right)
        assert sorted(parents[0].tolist()) == sorted(b for _, b, _ in best)
        assert sorted(zip(parents[0].tolist(), tokens[0].tolist())) == sorted((b, t) for _, b, t in best)
        assert max(abs(g - w) for g, (w, _, _) in zip(got[0].tolist(), best)) <= 1e-6
    # more ties than a list holds, at the end of the row: the first of them
    logits[most - 1000:] = 9.0
    got, _, tokens, _ = amq.beam_select(logits.view(1, most), torch.zeros((1, 1), device="cuda"))
    assert tokens.item() == most - 1000


LOWEST = torch.finfo(torch.float32).min


@pytest.mark.parametrize("batch,vocab", [(1, 7), (1, 9999), (20, 3001), (70, 20000)])
def test_logits_at_the_ends_of_fp32(amq, batch, vocab):  # noqa: F811
    """Finite logits of any size have a log-sum-exp: rows of the type's lowest value alone (every token masked with it), of values whose product with log2(e) is
    beyond fp32, with a few such values among others.  Against the definition in double, summed relative to the row's largest."""
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    beams = 6
    z = torch.randn((batch, beams, vocab), device="cuda", generator=gen) * 2.5
    scores = -20 * torch.rand((batch, beams), device="cuda", generator=gen)
    z[:, 1] = LOWEST                                        # -log(vocab) each
    z[:, 2] = -3e38
    z[:, 2, 5] = LOWEST                                     # (nothing beside the others)
    z[:, 3, 3] = 3e38                                       # the one continuation with a probability
    z[:, 4] = LOWEST
    z[:, 4, 6] = 2.5e38
    z[:, 4, 2] = 2.5e38                                     # two of them
    z[:, 5, ::2] = LOWEST                                   # an ordinary mask
    scores[:, 1] = -0.5 + math.log(vocab)                   # (so that the first tokens of the row are chosen)
    scores[:, 2] = -0.6 + math.log(vocab)
    d = z.double()
    top = d.amax(2, keepdim=True)
    total = scores.double()[..., None] + (d - top - torch.log(torch.exp(d - top).sum(2, keepdim=True)))
    # (a library's sum over a row of equal numbers is off by 1e-15; far below what other candidates differ by)
    total = (total.view(batch, -1).clamp(min=-1e20) * 1e10).round() / 1e10
    best, at = torch.sort(total, dim=1, descending=True, stable=True)
    got, parents, tokens, _ = amq.beam_select(z.view(batch * beams, vocab), scores)
    assert torch.equal(parents.long(), at[:, :beams] // vocab) and torch.equal(tokens.long(), at[:, :beams] % vocab)
    assert ((got.double() - best[:, :beams]).abs() <= 2.0 ** -24 * best[:, :beams].abs() + 3e-6).all()


def test_a_single_beam_of_lowest_values(amq):  # noqa: F811
    """A uniform row, whatever its value: the first token, at -log(vocab)."""
    for value in (LOWEST, -1.0, 0.0, 3.4e38):
        got, parents, tokens, _ = amq.beam_select(torch.full((1, 4096), value, device="cuda"), torch.zeros((1, 1), device="cuda"))
        assert parents.item() == 0 and tokens.item() == 0 and abs(got.item() + math.log(4096)) <= 2.0 ** -20


@pytest.mark.parametrize("batch", [1, 40])
@pytest.mark.parametrize("score", [-1e9, -1e15, 0.0])
def test_scores_that_do_not_tell_logits_apart(amq, batch, score):  # noqa: F811
    """One beam's continuations rank as its logits do, equal ones by the smaller token, wherever in the row they lie, and beams of one score by the smaller
    beam: logits a step of fp32 apart (6e-8) under a score whose double has steps of 1.2e-7, 0.125 or, for 0, steps that tell them apart."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    beams, vocab = 8, 6000
    z = torch.zeros((batch, beams, vocab), device="cuda")
    base = 0.75 * torch.ones(40, device="cuda")
    steps = torch.randint(0, 9, (40,), device="cuda", generator=gen)        # (values again and again)
    near = base + steps * 2.0 ** -24
    for b in range(batch):
        z[b, :, torch.randperm(vocab, device="cuda", generator=gen)[:40]] = near        # (all beams' rows alike)
    scores = torch.full((batch, beams), score, device="cuda")
    live = torch.arange(beams, device="cuda") < 2
    scores[:, ~live] = -torch.inf
    got, parents, tokens, _ = amq.beam_select(z.view(batch * beams, vocab), scores)
    for b in range(batch):
        row = z[b, 0].double()
        order = torch.sort(row, descending=True, stable=True).indices[:beams].tolist()
        if score == 0.0:                                    # the two beams' pairs of one logit side by side
            place = {t: i for i, t in enumerate(order)}
            want = sorted(((-row[t].item(), q, place[t], t) for q in range(2) for t in order))[:beams]
            want = [(q, t) for _, q, _, t in want]
        elif score == -1e15:                                # nothing but the beam's logits tells: the first beam's best
            want = [(0, t) for t in order]
        else:                                               # which logits share a score hangs on the log-sum-exp; the order of each beam's does not
            chosen = list(zip(parents[b].tolist(), tokens[b].tolist()))
            for q in range(2):
                mine = [t for p, t in chosen if p == q]
                assert mine == order[:len(mine)]
            assert chosen[0] == (0, order[0]) and all(p < 2 for p, _ in chosen)
            continue
        assert list(zip(parents[b].tolist(), tokens[b].tolist())) == want


@pytest.mark.parametrize("batch,beams,vocab", [(1, 8, 300000), (1, 1, 2000000), (16, 2, 300000), (1, 6, 9999)])
def test_long_rows_of_equal_terms(amq, batch, beams, vocab):  # noqa: F811
    """A few logits (one of 61, so that every thread meets some) above many equal ones, whose exponentials a running sum in fp32 would all round one way (4e-6 at 300000 tokens, 1.4e-5 at 2000000).  Here: an
    exponential is within 2^-22 of itself, its exponent |d| off by 2^-23 |d| (two roundings); a piece's words are summed with 13 roundings, a warp's shares with six
    and the store one: 20 2^-24.  The weighted mean of |d| is below log(vocab)."""
    bound = 2.0 ** -22 + 2.0 ** -23 * math.log(vocab) + 20 * 2.0 ** -24
    for d in torch.linspace(0.6, 8.2, 9).tolist():
        logits = torch.full((batch * beams, vocab), 1.5 - d, device="cuda")
        logits[:, ::61] = 1.5
        got, _, tokens, _ = amq.beam_select(logits, torch.zeros((batch, beams), device="cuda"))
        z = logits[0].double()
        want = -(math.log(float(torch.exp(z - 1.5).sum())))
        assert (tokens[:, 0] == 0).all()
        assert (got[:, 0].double() - want).abs().max() <= bound + 2.0 ** -24 * abs(want)


@pytest.mark.parametrize("batch", [1, 20, 70])
@pytest.mark.parametrize("beams", [1, 4, 8, 9, 12, 20, 32])
def test_few_tokens_above_the_lowest_value(amq, batch, beams):  # noqa: F811
    """Tokens masked with the type's lowest value, up to all but a few of a row: the unmasked ones are found whatever their number, by that of the beams or below."""
    gen = torch.Generator(device="cuda").manual_seed(beams)
    for vocab in (31, 147, 402, 581, 3000):
        for kept in (0.5, 0.1, 0.02):
            z = torch.randn((batch * beams, vocab), device="cuda", generator=gen) * 2.5
            z = torch.where(torch.rand(z.shape, device="cuda", generator=gen) < kept, z, LOWEST)
            z[:, 3] = 1.0                                   # (one at least)
            scores = -20 * torch.rand((batch, beams), device="cuda", generator=gen)
            d = z.double()
            top = d.amax(1, keepdim=True)
            total = (d - top - torch.log(torch.exp(d - top).sum(1, keepdim=True))).view(batch, beams, vocab) + scores.double()[..., None]
            best = torch.sort(total.view(batch, -1), dim=1, descending=True, stable=True)
            got, parents, tokens, _ = amq.beam_select(z, scores)
            assert ((got.double() - best.values[:, :beams]).abs() <= 2.0 ** -24 * best.values[:, :beams].abs() + 3e-6).all()
            real = best.values[:, :beams] > -1e30           # (those of the lowest value differ by nothing that a double holds)
            assert torch.equal((parents.long() * vocab + tokens)[real], best.indices[:, :beams][real])
