"""What a quantized language model does between its products and around them, as cases that can be timed and compared: the packed
product with its bias, activation and residual; keys and values written into a paged cache that holds them in packed planes;
attention over that cache; beam search's choice of continuations and the reordering of the states behind it.

Sizes are those of the library's own workloads (hidden 650, 1024, 2048, vocabularies 9999, 10000 and 42000) or generic ones.
Planes and coefficients are greedy codes of Gaussian rows; a case's inputs follow from the seed alone.
"""
import math

import torch

own = False                 # True: the framework's kernels; False: the same in elementary operations

NONE, RELU, GELU, SILU, TANH, SIGMOID = range(6)


def listed():
    return [
        # a feed-forward layer's first product for one token: latency
        {"name": "product_4096x1024_b1_gelu", "op": "product", "m": 4096, "n": 1024, "batch": 1, "k_w": 2, "k_a": 2, "act": GELU, "residual": False},
        # the product back onto the residual stream for a batch of 512 vectors
        {"name": "product_2048x8192_b512", "op": "product", "m": 2048, "n": 8192, "batch": 512, "k_w": 3, "k_a": 2, "act": SILU, "residual": True},
        # 64 streams, each adding its newest token to the cache
        {"name": "append_b64_one", "op": "append", "batch": 64, "new": 1, "heads": 8, "d": 128, "k": 4, "page": 16, "tokens": 2048},
        # four prompts going into the cache at once, ragged
        {"name": "append_b4_prompts", "op": "append", "batch": 4, "new": 2000, "heads": 8, "d": 128, "k": 4, "page": 64, "tokens": 4096},
        # one stream with a short past: latency
        {"name": "attention_b1_300", "op": "attention", "batch": 1, "q_len": 1, "heads": 8, "group": 1, "d": 64, "k": 4, "page": 16, "tokens": 300},
        # a serving batch, four query heads to a key head, ragged lengths
        {"name": "attention_b64_4096", "op": "attention", "batch": 64, "q_len": 1, "heads": 8, "group": 4, "d": 128, "k": 4, "page": 16, "tokens": 4096},
        # one long document
        {"name": "attention_b1_65000", "op": "attention", "batch": 1, "q_len": 1, "heads": 8, "group": 8, "d": 128, "k": 4, "page": 64, "tokens": 65000},
        # a few drafted tokens checked at once: odd head size, three bits, a page to a token
        {"name": "attention_b20_draft", "op": "attention", "batch": 20, "q_len": 3, "heads": 5, "group": 3, "d": 100, "k": 3, "page": 1, "tokens": 1500},
        # one stream's five beams over the ragged vocabulary
        {"name": "select_b1k5_9999", "op": "select", "batch": 1, "beams": 5, "vocab": 9999},
        # 64 streams of eight beams over the largest vocabulary
        {"name": "select_b64k8_42000", "op": "select", "batch": 64, "beams": 8, "vocab": 42000},
        # h and c of one layer behind four beams: latency
        {"name": "reorder_b1k4_1024x2", "op": "reorder", "batch": 1, "beams": 4, "row": 1024, "states": 2},
        # h and c of two layers behind a serving batch
        {"name": "reorder_b256k8_2048x4", "op": "reorder", "batch": 256, "beams": 8, "row": 2048, "states": 4},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# widths: one in two a multiple of 64 as most models have it, the others whatever comes
def _width(rng, lo, hi):
    v = _log_int(rng, lo, hi)
    return max(lo, v // 64 * 64) if rng.random() < 0.5 else v


def draw(rng):
    ops = ["product", "product", "append", "attention", "attention", "attention", "select", "select", "reorder"]
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0), _size(c))
    while True:
        op = rng.choice(ops)
        if op == "product":
            c = {"m": _width(rng, 64, 42000), "n": _width(rng, 64, 8192), "batch": rng.choice([1, _log_int(rng, 1, 1024)]),
                 "k_w": rng.choice([1, 2, 2, 3, 4]), "k_a": rng.choice([1, 2, 2, 3, 4]), "act": rng.randrange(6), "residual": rng.random() < 0.5}
        elif op == "append":
            new = rng.choice([1, _log_int(rng, 1, 4096)])
            c = {"batch": _log_int(rng, 1, 256), "new": new, "heads": rng.choice([1, 2, 4, 5, 8, 16]), "d": rng.choice([64, 80, 100, 128]),
                 "k": rng.choice([2, 3, 4, 4]), "page": rng.choice([1, 16, 16, 64]), "tokens": new + _log_int(rng, 1, 1024)}
        elif op == "attention":
            c = {"batch": rng.choice([1, _log_int(rng, 1, 128)]), "q_len": rng.choice([1, 1, 1, rng.randint(2, 6)]),
                 "heads": rng.choice([1, 2, 4, 5, 8, 16]), "group": rng.choice([1, 2, 3, 4, 4, 8]), "d": rng.choice([64, 80, 100, 128, 128]),
                 "k": rng.choice([1, 2, 3, 4, 4, 4]), "page": rng.choice([1, 16, 16, 64]), "tokens": _log_int(rng, 1, 65000)}
        elif op == "select":
            c = {"batch": rng.choice([1, _log_int(rng, 1, 256)]), "beams": rng.choice([1, 2, 3, 4, 5, 8, 10, 16]), "vocab": _log_int(rng, 100, 50000)}
        else:
            c = {"batch": _log_int(rng, 1, 256), "beams": rng.choice([2, 3, 4, 5, 8, 16]), "row": _width(rng, 100, 4096), "states": rng.randint(1, 4)}
        c["op"] = op
        if _size(c) <= most[op]:
            return c


def _size(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------


def _wpr(n):
    return 4 * ((n + 127) // 128)                   # 32-bit words of a packed plane


def _row_bytes(n, k):
    return k * ((n + 7) // 8 + 4)                   # planes and coefficients of one row


def _lengths(case):
    """Tokens of each sequence: from a quarter of the longest up, the newest ones counted."""
    b, longest, new = case["batch"], case["tokens"], case.get("new", case.get("q_len", 1))
    return [max(min(new, longest), longest - (i * 7 % b) * (longest - longest // 4) // b) for i in range(b)]


def work(case):
    """Every input read once, every output written once; a product counts as the dense one it stands for."""
    op = case["op"]
    if op == "product":
        m, n, batch = case["m"], case["n"], case["batch"]
        return {"bytes": m * _row_bytes(n, case["k_w"]) + batch * _row_bytes(n, case["k_a"]) + 4 * m + 4 * batch * m * (2 if case["residual"] else 1),
                "flops": 2 * batch * m * n}
    if op == "append":
        rows = 2 * case["batch"] * case["new"] * case["heads"]
        return {"bytes": 2 * rows * _row_bytes(case["d"], case["k"]), "flops": 0}
    if op == "attention":
        heads, group, d, q_len, total = case["heads"], case["group"], case["d"], case["q_len"], sum(_lengths(case))
        return {"bytes": 2 * total * heads * _row_bytes(d, case["k"]) + 8 * case["batch"] * q_len * heads * group * d + 4 * (total // case["page"]),
                "flops": 4 * total * heads * group * q_len * d}
    if op == "select":
        rows = case["batch"] * case["beams"]
        return {"bytes": 4 * rows * case["vocab"] + 9 * rows + 13 * rows, "flops": 3 * rows * case["vocab"]}
    return {"bytes": 8 * case["batch"] * case["beams"] * case["row"] * case["states"] + 4 * case["batch"] * case["beams"], "flops": 0}


# ---- inputs ---------------------------------------------------------------------------------------------------------


def _normal(gen, *shape, std=1.0):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=gen)


def _greedy(x, k):
    """Rows in k planes, each the signs of what the planes before it leave and their mean size: codes (rows, k, words), coeffs (rows, k)."""
    rows, n = x.shape
    words = _wpr(n)
    codes = torch.empty((rows, k, words), dtype=torch.int32, device=x.device)
    coeffs = torch.empty((rows, k), device=x.device)
    weight = 1 << torch.arange(32, device=x.device)
    for at in range(0, rows, 1 << 18):
        r = x[at:at + (1 << 18)].clone()
        for i in range(k):
            bits = r >= 0
            a = r.abs().mean(1)
            r = r - torch.where(bits, a[:, None], -a[:, None])
            full = torch.zeros((r.shape[0], words * 32), dtype=torch.bool, device=x.device)
            full[:, :n] = bits
            w = (full.view(-1, words, 32) * weight).sum(2)
            codes[at:at + (1 << 18), i] = torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)
            coeffs[at:at + (1 << 18), i] = a
    return codes, coeffs


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    s = {"case": case}
    if op == "product":
        m, n, batch = case["m"], case["n"], case["batch"]
        s["W"] = _greedy(_normal(gen, m, n, std=1.0 / math.sqrt(n)), case["k_w"])
        s["x"] = _greedy(_normal(gen, batch, n), case["k_a"])
        s["bias"] = _normal(gen, m, std=0.1)
        s["residual"] = _normal(gen, batch, m) if case["residual"] else None
    elif op in ("append", "attention"):
        batch, heads, d, k, page = case["batch"], case["heads"], case["d"], case["k"], case["page"]
        lengths = _lengths(case)
        most = -(-max(lengths) // page)
        pages = sum(-(-n // page) for n in lengths) + 3
        # the pages of all sequences, in an order that a program has after a while of allocating and freeing
        order = torch.randperm(pages, device="cuda", generator=gen, dtype=torch.int32)
        table = torch.full((batch, most), -1, dtype=torch.int32)
        at = 0
        for i, n in enumerate(lengths):
            need = -(-n // page)
            table[i, :need] = torch.arange(at, at + need, dtype=torch.int32)
            at += need
        table = table.cuda()
        s["table"] = torch.where(table >= 0, order[table.clamp(min=0).long()], table)
        s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        if op == "append":
            new = case["new"]
            s["new"] = []
            s["cache"] = []
            for _ in range(2):
                codes, coeffs = _greedy(_normal(gen, batch * new * heads, d), k)
                s["new"] += [codes.view(batch, new, heads, k, -1), coeffs.view(batch, new, heads, k)]
                s["cache"] += [torch.zeros((pages, page, heads, k, _wpr(d)), dtype=torch.int32, device="cuda"),
                               torch.zeros((pages, page, heads, k), device="cuda")]
        else:
            s["cache"] = []
            for _ in range(2):
                codes, coeffs = _greedy(_normal(gen, pages * page * heads, d), k)
                s["cache"] += [codes.view(pages, page, heads, k, -1), coeffs.view(pages, page, heads, k)]
            s["q"] = _normal(gen, batch, case["q_len"], heads * case["group"], d)
            s["scale"] = 1.0 / math.sqrt(d)
    elif op == "select":
        batch, beams, vocab = case["batch"], case["beams"], case["vocab"]
        s["logits"] = _normal(gen, batch * beams, vocab, std=2.5)
        s["scores"] = torch.empty((batch, beams), device="cuda").uniform_(-20.0, -5.0, generator=gen)
        s["finished"] = (torch.empty((batch, beams), device="cuda").uniform_(generator=gen) < 0.125).to(torch.int32)
        s["finished"][:, 0] = 0
        s["eos"] = 2
    else:
        batch, beams, row = case["batch"], case["beams"], case["row"]
        s["states"] = [_normal(gen, batch, beams, row) for _ in range(case["states"])]
        s["out"] = [torch.empty_like(t) for t in s["states"]]
        s["parents"] = torch.randint(beams, (batch, beams), device="cuda", generator=gen, dtype=torch.int32)
    return s


# ---- the operators in their plain form ------------------------------------------------------------------------------


def _values(codes, coeffs, n):
    """What packed rows stand for: (..., n) fp32."""
    bits = (codes[..., None] >> torch.arange(32, dtype=torch.int32, device=codes.device)) & 1
    signs = bits.flatten(-2)[..., :n].to(torch.float32) * 2 - 1
    return (signs * coeffs[..., None]).sum(-2)


def _activate(v, act):
    if act == RELU:
        return v.clamp(min=0)
    if act == GELU:
        return 0.5 * v * torch.erfc(v * -math.sqrt(0.5))
    if act == SILU:
        return v / (1 + torch.exp(-v))
    if act == TANH:
        return torch.tanh(v)
    if act == SIGMOID:
        return 1 / (1 + torch.exp(-v))
    return v


def _plain_product(s):
    c = s["case"]
    y = _activate(_values(*s["x"], c["n"]) @ _values(*s["W"], c["n"]).T + s["bias"], c["act"])
    return y if s["residual"] is None else y + s["residual"]


def _plain_append(s):
    table, page, new = s["table"].long(), s["case"]["page"], s["case"]["new"]
    at = s["lengths"].long()[:, None] - new + torch.arange(new, device="cuda")
    kept = at >= 0
    at = at.clamp(min=0)
    slot = (torch.gather(table, 1, at // page) * page + at % page)[kept]
    kc, ka, vc, va = s["new"]
    kcache, kcoef, vcache, vcoef = s["cache"]
    kcache.flatten(0, 1)[slot] = kc[kept]
    kcoef.flatten(0, 1)[slot] = ka[kept]
    vcache.flatten(0, 1)[slot] = vc[kept]
    vcoef.flatten(0, 1)[slot] = va[kept]
    return s["cache"]


def _plain_attention(s):
    c = s["case"]
    batch, q_len, heads, group, d = c["batch"], c["q_len"], c["heads"], c["group"], c["d"]
    kcache, kcoef, vcache, vcoef = s["cache"]
    table = s["table"].clamp(min=0).long()
    k = _values(kcache[table], kcoef[table], d).flatten(1, 2)               # (batch, tokens, heads, d)
    v = _values(vcache[table], vcoef[table], d).flatten(1, 2)
    q = s["q"].view(batch, q_len, heads, group, d).permute(0, 2, 3, 1, 4).reshape(batch, heads, group * q_len, d)
    scores = (q @ k.permute(0, 2, 3, 1)) * s["scale"]                       # (batch, heads, group * q_len, tokens)
    seen = s["lengths"].long()[:, None] - q_len + 1 + torch.arange(q_len, device="cuda")
    hidden = torch.arange(k.shape[1], device="cuda") >= seen[..., None]     # (batch, q_len, tokens)
    scores = scores.view(batch, heads, group, q_len, -1).masked_fill(hidden[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    out = (p.flatten(2, 3) @ v.permute(0, 2, 1, 3)).view(batch, heads, group, q_len, d) / total.clamp(min=1e-30)
    return out.permute(0, 3, 1, 2, 4).reshape(batch, q_len, heads * group, d)


def _plain_select(s):
    c = s["case"]
    batch, beams, vocab = c["batch"], c["beams"], c["vocab"]
    z = s["logits"].double()                # beams are compared unrounded: candidates of two beams may lie within fp32 rounding
    top = z.amax(1, keepdim=True)
    logp = z - (top + torch.log(torch.exp(z - top).sum(1, keepdim=True)))
    done = s["finished"].view(-1, 1) != 0
    only = torch.where(torch.arange(vocab, device="cuda") == s["eos"], 0.0, -math.inf).double()
    total = (torch.where(done, only, logp) + s["scores"].double().view(-1, 1)).view(batch, beams * vocab)
    best, at = torch.topk(total, beams, dim=1)
    # among equal totals the lowest place first
    at, order = torch.sort(at, dim=1)
    best, again = torch.sort(torch.gather(best, 1, order), dim=1, descending=True, stable=True)
    at = torch.gather(at, 1, again)
    parents, tokens = at // vocab, at % vocab
    ended = (torch.gather(s["finished"], 1, parents) != 0) | (tokens == s["eos"])
    return best.float(), parents.to(torch.int32), tokens.to(torch.int32), ended.to(torch.int32)


def _plain_reorder(s):
    batch, beams = s["parents"].shape
    rows = (torch.arange(batch, device="cuda")[:, None] * beams + s["parents"]).view(-1).long()
    return [t.flatten(0, 1)[rows].view_as(t) for t in s["states"]]


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"product": _plain_product, "append": _plain_append, "attention": _plain_attention, "select": _plain_select,
                "reorder": _plain_reorder}[op](s)
    from paper_1802_00150_b200 import amq
    c = s["case"]
    if op == "product":
        return amq.binary_gemm_act(*s["W"], *s["x"], c["n"], bias=s["bias"], activation=c["act"], residual=s["residual"])
    if op == "append":
        amq.cache_append(*s["new"], s["cache"], s["table"], s["lengths"], c["d"])
        return s["cache"]
    if op == "attention":
        return amq.cache_attention(s["q"], s["cache"], s["table"], s["lengths"], s["scale"])
    if op == "select":
        return amq.beam_select(s["logits"], s["scores"], s["finished"], s["eos"])
    return amq.beam_reorder(s["states"], s["parents"], s["out"])


# ---- the operators from their definitions, in 64 bits ------------------------------------------------------------------


def _dense(codes, coeffs, n):
    out = 0
    for i in range(codes.shape[-2]):
        word = codes[..., i, :].long()
        plane = torch.stack([(word >> j) & 1 for j in range(32)], dim=-1).flatten(-2)[..., :n]
        out = out + coeffs[..., i, None].double() * (2 * plane - 1)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "product":
        W, x, n = s["W"], s["x"], case["n"]
        y = torch.empty((case["batch"], case["m"]), dtype=torch.float64, device="cuda")
        dx = _dense(*x, n)
        for at in range(0, case["m"], 4096):
            y[:, at:at + 4096] = dx @ _dense(W[0][at:at + 4096], W[1][at:at + 4096], n).T
        y += s["bias"].double()
        act = case["act"]
        if act == RELU:
            y = torch.maximum(y, torch.zeros_like(y))
        elif act == GELU:
            y = y * torch.special.ndtr(y)
        elif act == SILU:
            y = y * torch.special.expit(y)
        elif act == TANH:
            y = torch.tanh(y)
        elif act == SIGMOID:
            y = torch.special.expit(y)
        return y if s["residual"] is None else y + s["residual"].double()
    if op == "append":
        return None
    if op == "attention":
        batch, q_len, heads, group, d, page = (case[k] for k in ("batch", "q_len", "heads", "group", "d", "page"))
        out = torch.zeros((batch, q_len, heads * group, d), dtype=torch.float64, device="cuda")
        for b, n in enumerate(_lengths(case)):
            pages = s["table"][b, :-(-n // page)].long()
            kc, ka, vc, va = (t[pages].flatten(0, 1)[:n] for t in s["cache"])
            k, v = _dense(kc, ka, d), _dense(vc, va, d)
            for i in range(q_len):
                seen = n - q_len + 1 + i
                if seen <= 0:
                    continue
                q = s["q"][b, i].double().view(heads, group, d)
                a = torch.einsum("hgd,thd->hgt", q, k[:seen]) * s["scale"]
                out[b, i] = torch.einsum("hgt,thd->hgd", torch.softmax(a, -1), v[:seen]).reshape(heads * group, d)
        return out
    if op == "select":
        batch, beams, vocab = case["batch"], case["beams"], case["vocab"]
        best = torch.empty((batch, beams), dtype=torch.float64, device="cuda")
        for b in range(batch):
            z = torch.log_softmax(s["logits"][b * beams:(b + 1) * beams].double(), 1)
            for i in range(beams):
                if s["finished"][b, i]:
                    z[i] = -math.inf
                    z[i, s["eos"]] = 0.0
            best[b] = torch.sort((z + s["scores"][b].double()[:, None]).flatten(), descending=True).values[:beams]
        return best, None, None, None
    rows = torch.arange(case["batch"], device="cuda")[:, None]
    return [t.double()[rows, s["parents"].long()] for t in s["states"]]
