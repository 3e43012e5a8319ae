"""The operators as a decoder uses them: products, the paged cache and attention over it, feed-forward products with their activation and residual, the output layer,
beam search's choice, and the reordering of token histories and block tables behind it; step after step, eagerly and as a replayed graph."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BATCH, BEAMS, VOCAB, WIDTH, HEADS, KV_HEADS, D, FF, BITS, STEPS, EOS = 3, 4, 300, 256, 4, 2, 64, 384, 3, 12, 7
ROWS = BATCH * BEAMS


@pytest.fixture(scope="module")
def amq():
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    from paper_1802_00150_b200 import amq as binding
    return binding


class Decoder:
    """One layer.  A page holds one token, so that a row of the block table is a beam's past, and reordering beams is reordering rows."""

    def __init__(self, amq, seed):
        self.amq = amq
        gen = torch.Generator(device="cuda").manual_seed(seed)
        weights = lambda m, n: amq.quantize(torch.randn((m, n), device="cuda", generator=gen) / math.sqrt(n), BITS, 2)  # noqa: E731
        self.qkv, self.o = weights((HEADS + 2 * KV_HEADS) * D, WIDTH), weights(WIDTH, HEADS * D)
        self.up, self.down, self.out, self.embedding = weights(FF, WIDTH), weights(WIDTH, FF), weights(VOCAB, WIDTH), weights(VOCAB, WIDTH)
        self.bias = torch.randn(FF, device="cuda", generator=gen) * 0.1
        self.cache = amq.new_cache(ROWS * STEPS, 1, KV_HEADS, D, 4)
        self.table = torch.full((BATCH, BEAMS, STEPS), -1, dtype=torch.int32, device="cuda")
        self.history = torch.zeros((BATCH, BEAMS, STEPS + 1), dtype=torch.int32, device="cuda")
        self.lengths = torch.zeros(ROWS, dtype=torch.int32, device="cuda")
        self.position = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.scores = torch.full((BATCH, BEAMS), -math.inf, device="cuda")
        self.scores[:, 0] = 0.0
        self.finished = torch.zeros((BATCH, BEAMS), dtype=torch.int32, device="cuda")
        self.tokens = torch.randint(VOCAB, (BATCH, 1), device="cuda", generator=gen, dtype=torch.int32).expand(BATCH, BEAMS).contiguous()
        self.seen = {}

    def quantized(self, x):
        return self.amq.quantize(x, BITS, 2)

    def step(self):
        amq = self.amq
        self.history.scatter_(2, self.position.expand(BATCH, BEAMS, 1), self.tokens[..., None])
        pages = (self.position * ROWS + torch.arange(ROWS, device="cuda")).to(torch.int32).view(BATCH, BEAMS, 1)
        self.table.scatter_(2, self.position.expand(BATCH, BEAMS, 1), pages)
        self.lengths.add_(1)
        codes, beta = amq.embedding_rows(*self.embedding, WIDTH, self.tokens.view(-1))
        x = amq.unpack(codes, beta, WIDTH)
        qkv = amq.binary_gemm(*self.qkv, codes, beta, WIDTH)
        q = qkv[:, :HEADS * D].view(ROWS, 1, HEADS, D)
        k = qkv[:, HEADS * D:(HEADS + KV_HEADS) * D].reshape(ROWS * KV_HEADS, D)
        v = qkv[:, (HEADS + KV_HEADS) * D:].reshape(ROWS * KV_HEADS, D)
        new = []
        for rows in (k, v):
            c, a = amq.quantize(rows, 4, 2)
            new += [c.view(ROWS, 1, KV_HEADS, 4, -1), a.view(ROWS, 1, KV_HEADS, 4)]
        table = self.table.view(ROWS, STEPS)
        amq.cache_append(*new, self.cache, table, self.lengths, D)
        attended = amq.cache_attention(q, self.cache, table, self.lengths, 1 / math.sqrt(D))
        h = amq.binary_gemm_act(*self.o, *self.quantized(attended.view(ROWS, HEADS * D)), HEADS * D, residual=x)
        inner = amq.binary_gemm_act(*self.up, *self.quantized(h), WIDTH, bias=self.bias, activation=amq.ACT_GELU)
        y = amq.binary_gemm_act(*self.down, *self.quantized(inner), FF, residual=h)
        logits = amq.binary_gemm(*self.out, *self.quantized(y), WIDTH)
        scores, parents, tokens, finished = amq.beam_select(logits, self.scores, self.finished, EOS)
        self.seen = {"x": x, "q": q, "new": new, "attended": attended, "h": h, "inner": inner, "y": y, "logits": logits, "before": (self.scores.clone(), self.finished.clone()),
                     "table": self.table.clone(), "choice": (scores, parents, tokens, finished)}
        amq.beam_reorder([self.history, self.table], parents)
        self.scores.copy_(scores)
        self.finished.copy_(finished)
        self.tokens.copy_(tokens)
        self.position.add_(1)


def dense(amq, planes, n):
    return amq.unpack(*planes, n).double()


def test_a_step_is_its_parts(amq):
    """Every stage against its definition in 64 bits on what the stage in front has left (a quantizer on slightly different numbers may choose other bits): products of
    sums of up to 384 terms and at most 12 roundings each, relative to the sums of absolute terms; attention and choice as in their own tests."""
    model = Decoder(amq, 1)
    past = []                                           # (k rows, v rows) of each step
    for t in range(STEPS):
        model.step()
        s = model.seen
        past.append([c.clone() for c in s["new"]])

        def product(planes, n, x, bias=None):
            w, xq = dense(amq, planes, n), dense(amq, model.quantized(x), n)
            size = xq.abs() @ w.abs().T + (0 if bias is None else bias.double().abs())
            return xq @ w.T + (0 if bias is None else bias.double()), 64 * 2.0 ** -24 * size

        ref, off = product(model.o, HEADS * D, s["attended"].view(ROWS, HEADS * D))
        assert ((s["h"].double() - (ref + s["x"].double())).abs() <= off + 2.0 ** -22 * s["x"].double().abs()).all()
        ref, off = product(model.up, WIDTH, s["h"], model.bias)
        assert ((s["inner"].double() - 0.5 * ref * torch.erfc(-ref / math.sqrt(2))).abs() <= 1.2 * off + 2.0 ** -21 * ref.abs()).all()
        ref, off = product(model.down, FF, s["inner"])
        assert ((s["y"].double() - (ref + s["h"].double())).abs() <= off + 2.0 ** -22 * s["h"].double().abs()).all()
        # attention: the rows that a beam's own past has put into the cache, found through its table
        for row in range(ROWS):
            pages = s["table"].view(ROWS, STEPS)[row, :t + 1].long()
            assert torch.equal(pages // ROWS, torch.arange(t + 1, device="cuda"))           # one token of every step so far
            for part in range(4):
                want = torch.stack([past[int(page) // ROWS][part][int(page) % ROWS, 0] for page in pages])
                assert torch.equal(model.cache[part][pages, 0], want)
            keys = amq.unpack(model.cache[0][pages, 0].view(-1, 4, 4).contiguous(), model.cache[1][pages, 0].view(-1, 4).contiguous(), D).double().view(t + 1, KV_HEADS, D)
            values = amq.unpack(model.cache[2][pages, 0].view(-1, 4, 4).contiguous(), model.cache[3][pages, 0].view(-1, 4).contiguous(), D).double().view(t + 1, KV_HEADS, D)
            q = s["q"][row, 0].double().view(KV_HEADS, HEADS // KV_HEADS, D)
            p = torch.softmax(torch.einsum("hgd,thd->hgt", q, keys) / math.sqrt(D), -1)
            ref = torch.einsum("hgt,thd->hgd", p, values).reshape(HEADS, D)
            size = model.cache[3][pages, 0].abs().sum(-1).max().double()
            reach = model.cache[1][pages, 0].abs().sum(-1).max().double() * D * q.abs().max() / math.sqrt(D)
            assert ((s["attended"][row, 0].double() - ref).abs() <= 8 * 2.0 ** -22 * (1 + reach) * size).all()
        # choice
        scores, finished = s["before"]
        logp = torch.log_softmax(s["logits"].double(), 1).view(BATCH, BEAMS, VOCAB)
        only = torch.full((VOCAB,), -math.inf, dtype=torch.float64, device="cuda")
        only[EOS] = 0
        total = (torch.where(finished[..., None] != 0, only, logp) + scores.double()[..., None]).view(BATCH, -1)
        best, at = torch.sort(total, dim=1, descending=True, stable=True)
        assert torch.equal(s["choice"][1].long(), at[:, :BEAMS] // VOCAB) and torch.equal(s["choice"][2].long(), at[:, :BEAMS] % VOCAB)
        assert (s["choice"][0].double() - best[:, :BEAMS]).abs().max() <= 1e-5
    # what the beams carry: every history leads to its beam's last choice
    assert torch.equal(model.lengths, torch.full_like(model.lengths, STEPS))
    assert (model.history[:, :, 0] == model.history[:, :1, 0]).all()


def test_steps_as_a_replayed_graph(amq):
    """The same steps captured once and replayed give the same tokens, scores and cache, bit for bit."""
    eager, captured = Decoder(amq, 2), Decoder(amq, 2)
    for _ in range(STEPS):
        eager.step()
    warm = Decoder(amq, 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        warm.step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.step()
    for _ in range(STEPS):
        graph.replay()
    for name in ("history", "table", "scores", "finished", "tokens", "lengths"):
        assert torch.equal(getattr(eager, name), getattr(captured, name)), name
    for a, b in zip(eager.cache, captured.cache):
        assert torch.equal(a, b)
