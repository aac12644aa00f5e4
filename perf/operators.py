"""Timed cases of the last stage's answer: the operators between a model's hidden
rows and the tokens that it adds to its requests.

  linear   product of activation rows with weights in 8-bit integers, a scale
           for each row (token) and each column (channel)
  probs    logits -> probabilities at each row's own temperature
  verify   drafted tokens against the target's probabilities, from given
           random numbers, and the token that follows the accepted ones

A case is one call through ``int8`` or ``speculate``. Sizes are those of the
repository's model shapes and vocabulary (``synth``, ``bench.py``), of its decode
batches and prefill chunks, and odd ones between. Inputs are synthetic:
activations N(0, 1) with a few large columns, weights whose 8-bit values are those
of a normal draw, logits 3.5 N(0, 1), a draft model whose logits are the target's
plus N(0, 0.5^2), drafted tokens drawn from it.

Fields of a case (plain values):
  op               "linear" | "probs" | "verify"
  m, n, k          linear: rows, output columns, depth
  dtype, out       type of the input rows (probabilities) and of the result:
                   "bf16" or "f32"
  rows, vocab      probs: rows; verify: see seqs
  greedy, masked   probs: every so-many-th row has temperature 0 (0: none); the share
                   of tokens with a logit of -infinity
  seqs, most       verify: sequences and the most drafts of one; drafts are 0 .. most
                   in number where ragged, else most
  ragged, known    verify: whether draft probabilities are given (else the drafts were
                   chosen outright, as by a table look-up)
"""

from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
VOCAB = 128256


def _linear(name, m, n, k, dtype="bf16", out="bf16"):
    c = {"op": "linear", "m": m, "n": n, "k": k, "dtype": dtype, "out": out}
    return dict(c, name=name) if name else c


def _probs(name, rows, vocab, dtype="f32", out="f32", greedy=0, masked=0.0):
    c = {"op": "probs", "rows": rows, "vocab": vocab, "dtype": dtype, "out": out,
         "greedy": greedy, "masked": masked}
    return dict(c, name=name) if name else c


def _verify(name, seqs, most, vocab, dtype="f32", ragged=False, known=True):
    c = {"op": "verify", "seqs": seqs, "most": most, "vocab": vocab, "dtype": dtype,
         "ragged": ragged, "known": known}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token through the QKV projection of the two-layer test model: the
        # smallest product there is (latency and launches)
        _linear("linear tiny 1", 1, 512, 256),
        # one interactive request, down projection of the 70B shape
        _linear("linear l70 down 1", 1, 8192, 28672),
        # a decode batch of 64, LM head of the 70B shape: logits in 32 bits
        _linear("linear l70 head 64", 64, VOCAB, 8192, out="f32"),
        # a decode batch of 150 with draft tokens, QKV projection of the 32B shape
        _linear("linear q32 qkv 150", 150, 10240, 5120),
        # odd sizes in 32 bits, as a model is checked with
        _linear("linear odd f32", 613, 1277, 2503, dtype="f32", out="f32"),
        # a prefill chunk of 2048 tokens, gate-up projection of the 70B shape
        _linear("linear l70 gate-up 2048", 2048, 57344, 8192),
        # the next token of one request of a small model
        _probs("probs 1", 1, 1024),
        # 64 requests with 4 drafts each, all their rows
        _probs("probs 320", 320, VOCAB, greedy=5),
        # a vocabulary of odd size, logits and probabilities in 16 bits, a grammar that
        # rules out most tokens
        _probs("probs odd bf16", 37, 32003, dtype="bf16", out="bf16", greedy=4, masked=0.9),
        # one interactive request with 4 drafts
        _verify("verify 1", 1, 4, VOCAB),
        # a batch of 64 whose drafts come from a table look-up
        _verify("verify 64 look-up", 64, 5, VOCAB, ragged=True, known=False),
        # the largest batch, up to 7 drafts each from a draft model
        _verify("verify 256", 256, 7, VOCAB, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "probs", "verify"])
    if kind == "linear":
        m, n, k = _log(rng, 1, 3000), _log(rng, 33, 57344), _log(rng, 65, 28672)
        if rng.random() < 0.5:  # most products of a model are multiples of 128
            n, k = (n + 127) // 128 * 128, (k + 127) // 128 * 128
        while m * n * k > 2048 * 57344 * 8192:
            m = (m + 1) // 2
        return _linear(None, m, n, k, rng.choice(["bf16", "bf16", "f32"]),
                       rng.choice(["bf16", "f32"]))
    if kind == "probs":
        return _probs(None, _log(rng, 1, 500), _log(rng, 500, 160000), rng.choice(["bf16", "f32"]),
                      rng.choice(["bf16", "f32", "f32"]), rng.choice([0, 3, 7]),
                      rng.choice([0.0, 0.0, 0.5, 0.99]))
    return _verify(None, _log(rng, 1, 256), rng.randint(1, 8), _log(rng, 500, 128256),
                   rng.choice(["bf16", "f32", "f32"]), rng.random() < 0.6, rng.random() < 0.7)


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 11)
    return g


def _inputs(case, seed):
    """The call's inputs, whoever computes it."""
    g = _generator(seed)
    dev = "cuda"
    if case["op"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        x = torch.randn((m, k), generator=g, device=dev)
        big = torch.randint(0, k, (max(1, k // 500),), generator=g, device=dev)
        x[:, big] *= 12.0
        wq = torch.empty((n, k), dtype=torch.int8, device=dev)
        for r in range(0, n, 16384):
            part = torch.randn((min(16384, n - r), k), generator=g, device=dev)
            wq[r:r + 16384] = (part * 29.0).round_().clamp_(-127, 127).to(torch.int8)
        ws = torch.empty(n, device=dev).uniform_(5e-4, 9e-4, generator=g)
        return {"x": x.to(TYPES[case["dtype"]]), "wq": wq, "ws": ws}
    if case["op"] == "probs":
        rows, vocab = case["rows"], case["vocab"]
        logits = torch.randn((rows, vocab), generator=g, device=dev).mul_(3.5)
        if case["masked"]:
            out = torch.rand((rows, vocab), generator=g, device=dev) < case["masked"]
            out[:, vocab // 2] = False
            logits.masked_fill_(out, -math.inf)
        t = torch.empty(rows, device=dev).uniform_(0.5, 1.2, generator=g)
        if case["greedy"]:
            t[case["greedy"] - 1::case["greedy"]] = 0.0
        return {"logits": logits.to(TYPES[case["dtype"]]), "temperature": t}
    seqs, most, vocab = case["seqs"], case["most"], case["vocab"]
    counts = torch.full((seqs,), most, dtype=torch.int64, device=dev)
    if case["ragged"]:
        counts = torch.randint(0, most + 1, (seqs,), generator=g, device=dev)
        counts[0] = most
    starts = torch.zeros(seqs + 1, dtype=torch.int64, device=dev)
    starts[1:] = counts.cumsum(0)
    n = int(starts[-1])
    logits = torch.randn((n + seqs, vocab), generator=g, device=dev).mul_(3.5)
    # the target's row that each drafted token is held against
    seq = torch.repeat_interleave(torch.arange(seqs, device=dev), counts)
    at = torch.arange(n, device=dev) + seq
    noise = torch.randn((n, vocab), generator=g, device=dev).mul_(0.5)
    q = torch.softmax(noise.add_(logits[at]), 1)
    p = torch.softmax(logits, 1)
    if case["known"]:
        drafts = torch.multinomial(q, 1, generator=g).view(-1)
    else:
        drafts = torch.multinomial(p[at], 1, generator=g).view(-1)
        # every fourth look-up names a token at random
        drafts[::4] = torch.randint(0, vocab, drafts[::4].shape, generator=g, device=dev)
    td = TYPES[case["dtype"]]
    return {"p": p.to(td), "q": q.to(td) if case["known"] else None, "drafts": drafts.int(),
            "starts": starts.int(), "most": most,
            "accept_u": torch.rand(n, generator=g, device=dev),
            "sample_u": torch.rand(seqs, generator=g, device=dev)}


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if own and case["op"] == "linear":  # a model's weights are packed when they are loaded
        from paper_2606_18600_amd import int8
        s["w"] = int8.pack_weight(s["wq"], s["ws"])
        del s["wq"]
    return s


def run(state):
    op = state["case"]["op"]
    if op == "linear":
        return _run_linear(state)
    if op == "probs":
        return _run_probs(state)
    return _run_verify(state)


def _run_linear(s):
    td = TYPES[s["case"]["out"]]
    if own:
        from paper_2606_18600_amd import int8
        return int8.linear(s["x"], s["w"], dtype=td)
    x = s["x"].float()
    scale = (x.abs().amax(1) / 127.0).clamp_min(2.0 ** -120)
    q = torch.round(x * (1.0 / scale)[:, None])
    acc = q @ s["wq"].float().t()
    return (acc * (scale[:, None] * s["ws"])).to(td)


def _run_probs(s):
    td = TYPES[s["case"]["out"]]
    if own:
        from paper_2606_18600_amd import speculate
        return speculate.token_probs(s["logits"], s["temperature"], dtype=td)
    x, t = s["logits"].float(), s["temperature"]
    top, at = x.max(1)
    e = torch.exp((x - top[:, None]) * (1.0 / torch.where(t > 0, t, 1.0))[:, None])
    e = e / e.sum(1, keepdim=True)
    at = (x == top[:, None]).to(torch.uint8).argmax(1)  # the lowest index of the largest logit
    tokens = torch.arange(x.shape[1], device=x.device)
    return torch.where((t > 0)[:, None], e, (tokens == at[:, None]).float()).to(td)


def _run_verify(s):
    if own:
        from paper_2606_18600_amd import speculate
        return speculate.verify_drafts(s["p"], s["q"], s["drafts"], s["starts"], s["most"],
                                       s["accept_u"], s["sample_u"])
    p, q, starts, most = s["p"], s["q"], s["starts"].long(), s["most"]
    seqs = starts.numel() - 1
    first, count = starts[:-1], starts[1:] - starts[:-1]
    j = torch.arange(most, device=p.device)
    there = j < count[:, None]
    at = torch.where(there, first[:, None] + j, 0)       # drafted rows [seqs, most]
    target = at + torch.arange(seqs, device=p.device)[:, None]
    token = s["drafts"].long()[at]
    pd = p[torch.where(there, target, 0), token].double()
    qd = torch.ones_like(pd) if q is None else q[at, token].double()
    yes = there & (s["accept_u"][at].double() * qd < pd)
    n = yes.long().cumprod(1).sum(1)
    stopped = n < count
    weight = p[first + torch.arange(seqs, device=p.device) + n].double()
    row = torch.where(stopped, first + n, 0)
    if q is None:
        refused = s["drafts"].long()[row]
        tokens = torch.arange(p.shape[1], device=p.device)
        left = weight.masked_fill((tokens == refused[:, None]) & stopped[:, None], 0.0)
    else:
        left = (weight - torch.where(stopped[:, None], q[row].double(), 0.0)).clamp_min(0.0)
    left = torch.where(left.sum(1, keepdim=True) > 0, left, weight)
    run_sum = left.cumsum(1)
    want = s["sample_u"].double()[:, None] * run_sum[:, -1:]
    new = (run_sum <= want).sum(1)
    out = torch.where(j < n[:, None], token, -1)
    out = torch.cat([out, torch.full_like(out[:, :1], -1)], 1).scatter(1, n[:, None], new[:, None])
    return n.int(), out.int()


def work(case):
    size = {"bf16": 2, "f32": 4}
    if case["op"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": n * k + 4 * n + m * k * size[case["dtype"]] + m * n * size[case["out"]],
                "flops": 2 * m * n * k}
    if case["op"] == "probs":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * (size[case["dtype"]] + size[case["out"]]) + 4 * case["rows"],
                "flops": 4 * n}
    # one row of the target's probabilities for each sequence and, where a draft
    # was refused (a fifth of them are), the row that it was drawn from
    most = case["most"]
    refused = sum(1 - 0.8 ** j for j in range(most + 1)) / (most + 1) if case["ragged"] else \
        1 - 0.8 ** most
    rows = case["seqs"] * (1 + (refused if case["known"] else 0))
    return {"bytes": rows * case["vocab"] * size[case["dtype"]] + 24 * case["seqs"] * (most + 1),
            "flops": 3 * rows * case["vocab"]}


def exact(case, seed):
    """linear and probs in 64 bits; the tokens of verify are whole numbers."""
    if case["op"] == "verify":
        return None
    s = _inputs(case, seed)
    if case["op"] == "probs":
        x = s["logits"].double()
        t = s["temperature"].double()[:, None]
        soft = torch.softmax(x / torch.where(t == 0, torch.ones_like(t), t), dim=-1)
        best = torch.zeros_like(x)
        width = x.shape[1]
        order = torch.arange(width, 0, -1, device=x.device)
        lead = torch.where(x == x.amax(-1, keepdim=True), order, 0).amax(-1)
        best[torch.arange(x.shape[0], device=x.device), width - lead] = 1.0
        return torch.where(t == 0, best, soft)
    # An 8-bit value is defined by its rounding in 32 bits (a scale is stored in 32 bits);
    # everything after it is exact in 64.
    x = s["x"].to(torch.float32)
    largest = torch.maximum(x.max(dim=1).values, -x.min(dim=1).values)
    scale = torch.clamp(largest / 127.0, min=2.0 ** -120)
    levels = (x * torch.reciprocal(scale).unsqueeze(1)).round().double()
    cols = []
    for part, ws in zip(s["wq"].split(16384), s["ws"].split(16384)):
        sums = torch.mm(levels, part.double().t().contiguous())
        cols.append(sums * ws.double() * scale.double().unsqueeze(1))
    return torch.cat(cols, dim=1)
