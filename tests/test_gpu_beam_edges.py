"""Beam search's choice at the ends of what it accepts: vocabularies up to 2^31."""
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
