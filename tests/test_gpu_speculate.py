"""Token probabilities and draft verification on the GPU against their
definitions in 64 bits, and the whole answer of a last stage: LM head in 8 bits,
probabilities, verification."""

from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2606_18600_amd import int8, speculate, synth
from paper_2606_18600_amd.harness import DeviceStage, upload_weights

pytestmark = pytest.mark.gpu

TD = {"f32": torch.float32, "bf16": torch.bfloat16}
INF = float("inf")


# ---- probabilities ---------------------------------------------------------
def _probs_reference(logits, temperature):
    x = logits.detach().double().cpu().numpy()
    t = np.ones(len(x)) if temperature is None else temperature.double().cpu().numpy()
    out = np.zeros_like(x)
    arg = np.zeros_like(x)
    for r, row in enumerate(x):
        if np.isnan(row).any() or (row == INF).any():
            out[r] = np.nan
        elif (row == -INF).all():
            pass
        elif not t[r] > 2.0 ** -100:
            out[r, row.argmax()] = 1.0
        else:
            arg[r] = (row - row.max()) / min(t[r], 2.0 ** 100)
            e = np.exp(arg[r])
            out[r] = e / e.sum()
    return out, arg


def _probs_close(y, logits, temperature, out):
    """A value's relative error: the exponent's argument takes a difference, a factor
    of two roundings and a product, so 4 * 2^-24 of its size, the exponential 2^-23,
    the sum at most 96 additions in a row and the terms' own errors, whose mean
    weighted argument is at most ln(vocab), the reciprocal and the product 2^-23; bf16
    2^-8 more. Below 2^-125 a value may be flushed to 0."""
    ref, arg = _probs_reference(logits, temperature)
    got = y.detach().double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    vocab = ref.shape[1]
    size = np.where(np.isfinite(arg), np.abs(arg), 0.0)
    rel = 2.0 ** -24 * (4 * size + 4 * np.log(vocab) + 112)
    if out == "bf16":
        rel = rel + 2.0 ** -8 * (1 + rel)
    bad = np.abs(got - ref) - rel * ref - 2.0 ** -125
    assert np.nanmax(bad) <= 0, np.nanmax(np.abs(got - ref) / (ref + 2.0 ** -125))


def _logits(seed, rows, vocab, dtype="f32", scale=4.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (scale * torch.randn((rows, vocab), generator=g, device="cuda")).to(TD[dtype])


@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (2, 7), (5, 63), (1, 1000), (7, 1024),
                                        (2, 4097), (33, 8191), (4, 8192), (3, 8193), (2, 32003),
                                        (300, 515), (1, 65537), (2, 128256), (270, 16400),
                                        (260, 50001), (1, 300001), (128, 32769), (130, 65535),
                                        (129, 65537), (140, 98304), (128, 98305), (131, 131072),
                                        (128, 131073)])
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"),
                                       ("bf16", "bf16")])
def test_token_probs(rows, vocab, dtype, out):
    x = _logits(rows + vocab, rows, vocab, dtype)
    t = torch.linspace(0.3, 2.0, rows, device="cuda")
    t[rows // 2] = 0.0
    for temperature in (None, t):
        y = speculate.token_probs(x, temperature, dtype=TD[out])
        assert y.dtype == TD[out] and y.shape == x.shape
        _probs_close(y, x, temperature, out)


@pytest.mark.parametrize("vocab", [40, 5000, 8192, 20011, 128256])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masks_infinities_and_greedy_ties(vocab, dtype):
    """Rows of masked tokens, masks of the type's lowest value, whole pieces of a row
    masked, rows of nothing, ties of the largest logit, NaN and +infinity."""
    x = _logits(vocab, 12, vocab, dtype)
    low = torch.finfo(TD[dtype]).min
    x[0, ::2] = -INF
    x[1, :] = -INF
    x[2, :] = -INF
    x[2, vocab - 1] = low                      # one token left, of the lowest value
    x[3, :] = low                              # all equal: uniform
    x[4, : vocab - 3] = low
    x[5, : vocab // 2] = -INF                  # leading pieces empty
    x[6, vocab // 2:] = -INF
    x[7, vocab // 3], x[8, vocab // 2] = float("nan"), INF
    x[9, 5], x[9, vocab - 1], x[9, vocab // 2] = 90.0, 90.0, 90.0
    x[10, :] = 0.0
    x[11] = x[11].clamp(max=0.0)
    x[11, vocab - 2:] = 60.0
    t = torch.full((12,), 0.8, device="cuda")
    for temperature in (None, t, t * 0, -t, t * float("nan"), t * 1e-31, t * 1e-25, t * 1e35):
        _probs_close(speculate.token_probs(x, temperature), x, temperature, "f32")
    greedy = speculate.token_probs(x, t * 0)
    assert greedy[9, 5] == 1 and greedy[10, 0] == 1 and greedy[11, vocab - 2] == 1
    assert (greedy[1] == 0).all() and greedy.nansum(1)[[0, 2, 3, 4, 5, 6]].eq(1).all()


@pytest.mark.parametrize("rows,vocab", [(128, 50003), (150, 128256)])
def test_masks_in_many_long_rows(rows, vocab):
    """The same where one block holds a row."""
    x = _logits(vocab, rows, vocab)
    low = torch.finfo(torch.float32).min
    x[0, ::2], x[1, :], x[2, :], x[3, :] = -INF, -INF, -INF, low
    x[2, vocab - 1] = low
    x[5, : vocab // 2], x[6, 17:] = -INF, -INF
    x[7, vocab // 3], x[8, vocab - 1] = float("nan"), INF
    x[9, 5], x[9, vocab - 1], x[9, vocab // 2] = 90.0, 90.0, 90.0
    x[10, :] = 0.0
    x[11, vocab - 2:] = 60.0
    t = torch.full((rows,), 0.8, device="cuda")
    for temperature in (None, t, t * 0):
        _probs_close(speculate.token_probs(x, temperature), x, temperature, "f32")
    wide = torch.full((rows, vocab + 7), -3.0, device="cuda")
    wide[:, 3:3 + vocab] = x
    y = speculate.token_probs(x, t)
    z = speculate.token_probs(wide[:, 3:3 + vocab], t, out=wide[:, 3:3 + vocab])
    assert torch.equal(y.nan_to_num(2.0), z.nan_to_num(2.0))
    assert (wide[:, :3] == -3).all() and (wide[:, 3 + vocab:] == -3).all()


@pytest.mark.parametrize("vocab", [300, 8195, 40000])
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
def test_probs_strides_and_in_place(vocab, dtype, out):
    wide = _logits(3, 6, vocab + 11, dtype)
    x = wide[:, 3:3 + vocab]
    t = torch.full((6,), 0.7, device="cuda")
    y = speculate.token_probs(x, t, dtype=TD[out])
    _probs_close(y, x, t, out)
    big = torch.full((6, vocab + 5), -3.0, dtype=TD[out], device="cuda")
    z = speculate.token_probs(x.contiguous(), t, out=big[:, 1:1 + vocab])
    assert torch.equal(z, y) and (big[:, 0] == -3).all() and (big[:, 1 + vocab:] == -3).all()
    if dtype == out:
        before = wide.clone()
        assert torch.equal(speculate.token_probs(x, t, out=x), y) and torch.equal(x, y)
        assert torch.equal(wide[:, :3], before[:, :3])
        assert torch.equal(wide[:, 3 + vocab:], before[:, 3 + vocab:])


def test_probs_of_very_many_rows():
    """More rows than one launch takes, of lengths for each kernel."""
    for rows, vocab, dtype in ((65536 * 3, 2, "f32"), (70001, 40, "bf16"), (65600, 8200, "bf16")):
        x = _logits(rows, rows, vocab, dtype)
        t = torch.linspace(0.5, 2.0, rows, device="cuda")
        y = speculate.token_probs(x, t)
        some = torch.tensor([0, 1, 65534, 65535, 65536, rows - 1], device="cuda")
        _probs_close(y[some], x[some], t[some], "f32")
    y = speculate.token_probs(torch.zeros((1 << 24) + 3, 1, device="cuda"))
    assert bool((y == 1).all())


@pytest.mark.parametrize("vocab", [3, 700, 20000, 70000])
@pytest.mark.parametrize("rows", [18, 130])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_offsets_beyond_32_bits(vocab, rows, dtype):
    """Rows far apart: elements past 2^32 of the logits and the probabilities."""
    ld = (1 << 32) // (rows - 2) // 64 * 64
    x, y = (torch.empty(ld * (rows - 1) + vocab, dtype=TD[dtype], device="cuda")
            .as_strided((rows, vocab), (ld, 1)) for _ in range(2))
    x.copy_(_logits(vocab, rows, vocab, dtype))
    speculate.token_probs(x, out=y)
    _probs_close(y, x, None, dtype)
    args = _drafts(vocab, [1] * (rows // 2), vocab, dtype)
    x.copy_(args["p"])
    y[:rows // 2].copy_(args["q"])
    _check(args, p=x, q=y[:rows // 2])


def test_probs_shapes():
    x = _logits(5, 24, 700)
    y = speculate.token_probs(x)
    assert torch.equal(speculate.token_probs(x.view(2, 3, 4, 700)), y.view(2, 3, 4, 700))
    assert torch.equal(speculate.token_probs(x[3]), y[3])
    assert speculate.token_probs(x[:0]).shape == (0, 700)
    assert torch.equal(speculate.token_probs(x.t().contiguous().t()), y)
    # more rows than a launch's grid takes in one dimension
    many = _logits(6, 70000, 9)
    _probs_close(speculate.token_probs(many), many, None, "f32")


# ---- verification ----------------------------------------------------------
def _verify_reference(p, q, drafts, starts, most, accept_u, sample_u):
    p = p.detach().double().cpu().numpy()
    q = None if q is None else q.detach().double().cpu().numpy()
    drafts, starts = drafts.cpu().numpy(), starts.cpu().numpy()
    au, su = accept_u.double().cpu().numpy(), sample_u.double().cpu().numpy()
    n_all, vocab = len(drafts), p.shape[1]

    def positive(w):
        return np.where(np.isfinite(w) & (w > 0), w, 0.0)
    counts, tokens = [], []
    for i in range(len(su)):
        s0 = min(max(int(starts[i]), 0), n_all)
        s1 = min(max(int(starts[i + 1]), s0), n_all)
        k = min(s1 - s0, most)
        n = 0
        while n < k:
            d = int(drafts[s0 + n])
            if not 0 <= d < vocab:
                break
            qd = 1.0 if q is None else q[s0 + n, d]
            if not au[s0 + n] * qd < p[s0 + i + n, d]:
                break
            n += 1
        w = positive(p[s0 + i + n])
        left = w.copy()
        if n < k:
            if q is None:
                if 0 <= drafts[s0 + n] < vocab:
                    left[drafts[s0 + n]] = 0
            else:
                with np.errstate(invalid="ignore"):
                    left = positive(w - q[s0 + n])
        if left.sum() > 0:
            w = left
        new = -1
        if w.sum() > 0:
            c = np.cumsum(w)
            over = np.nonzero((c > su[i] * c[-1]) & (w > 0))[0]
            new = int(over[0]) if len(over) else int(np.nonzero(w)[0][-1])
        counts.append(n)
        tokens.append([int(t) for t in drafts[s0:s0 + n]] + [new] + [-1] * (most - n))
    return counts, tokens


def _check(args, **changes):
    a = dict(args, **changes)
    n, tokens = speculate.verify_drafts(a["p"], a["q"], a["drafts"], a["starts"], a["most"], a["au"],
                                        a["su"])
    want_n, want = _verify_reference(a["p"], a["q"], a["drafts"], a["starts"], a["most"], a["au"],
                                     a["su"])
    assert n.dtype == tokens.dtype == torch.int32
    assert n.tolist() == want_n
    assert tokens.tolist() == want
    return n, tokens


def _drafts(seed, counts, vocab, dtype="f32", known=True, scale=3.0, noise=0.6):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    counts = torch.tensor(counts, dtype=torch.int64)
    seqs, n = len(counts), int(counts.sum())
    starts = torch.zeros(seqs + 1, dtype=torch.int64)
    starts[1:] = counts.cumsum(0)
    at = torch.arange(n) + torch.repeat_interleave(torch.arange(seqs), counts)
    x = scale * torch.randn((n + seqs, vocab), generator=g, device="cuda")
    p = torch.softmax(x, 1)
    q = torch.softmax(x[at.cuda()] + noise * torch.randn((n, vocab), generator=g, device="cuda"), 1)
    source = q if known else p[at.cuda()]
    drafts = torch.multinomial(source, 1, generator=g).view(-1) if n else torch.zeros(0, device="cuda")
    return {"p": p.to(TD[dtype]), "q": q.to(TD[dtype]) if known else None, "drafts": drafts.int(),
            "starts": starts.int().cuda(), "most": int(counts.max()),
            "au": torch.rand(n, generator=g, device="cuda"),
            "su": torch.rand(seqs, generator=g, device="cuda")}


@pytest.mark.parametrize("counts,vocab", [
    ([0], 1), ([1], 1), ([3], 2), ([4], 1000), ([0, 0, 0], 1023), ([1, 0, 5, 2], 1024),
    ([2, 7, 0, 3, 1], 1025), ([4] * 40, 4099), ([3, 0, 8], 32003), ([5], 128256),
    ([6, 6, 1, 0, 2], 128256), ([2] * 300, 530), ([70, 0, 130], 600), ([1] * 3, 200003),
])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("known", [True, False])
def test_verify(counts, vocab, dtype, known):
    args = _drafts(sum(counts) + vocab, counts, vocab, dtype, known)
    _check(args)
    seqs = len(counts)
    for u in (0.0, 1.0 - 2.0 ** -24):   # all accepted where anything allows it, and few
        au = torch.full_like(args["au"], u)
        _check(args, au=au, su=torch.full((seqs,), u, device="cuda"))
    _check(args, most=args["most"] + 3)
    _check(args, most=max(0, args["most"] - 1))


def test_identical_distributions_accept_everything():
    args = _drafts(5, [6] * 20, 3001)
    at = torch.arange(120, device="cuda") + torch.arange(20, device="cuda").repeat_interleave(6)
    n, _ = _check(args, q=args["p"][at])
    assert (n == 6).all()


@pytest.mark.parametrize("vocab", [50, 9000])
def test_greedy_target(vocab):
    """A target at temperature 0: a draft is accepted if it is the largest logit, else
    that token takes its place."""
    args = _drafts(9, [4] * 30, vocab, scale=1.0)
    logits = _logits(10, 150, vocab)
    p = speculate.token_probs(logits, torch.zeros(150, device="cuda"))
    best = p.argmax(1)
    at = torch.arange(120, device="cuda") + torch.arange(30, device="cuda").repeat_interleave(4)
    drafts = args["drafts"].clone()
    good = torch.rand(120, device="cuda") < 0.7
    drafts[good] = best[at].int()[good]
    for q in (args["q"], None):
        n, tokens = _check(args, p=p, q=q, drafts=drafts)
        last = tokens.gather(1, n.long()[:, None])[:, 0]
        assert torch.equal(last.long(), best[torch.arange(30, device="cuda") * 5 + n])


def test_empty_and_strange_rows():
    """Target rows of zeros, with NaN, infinities and negative values, that the
    draft's cover entirely; drafts outside the vocabulary."""
    args = _drafts(13, [3] * 12, 2500)
    p, q, d = args["p"].clone(), args["q"].clone(), args["drafts"].clone()
    p[0:4] = 0                       # sequence 0: nothing to draw from
    p[4:8, ::3] = float("nan")       # 1
    p[8:12, 7] = INF                 # 2
    p[12:16, 5:900] = -1.0           # 3
    p[16:20] = q[12:15].min() / 4    # 4: below the draft's everywhere
    q[12:15] = 1.0
    p[20:24] = 0
    p[20:24, 2499] = 1e-30           # 5: one tiny weight in the last place
    d[18], d[22], d[25] = -1, 2500, 2 ** 31 - 1
    q[27:30] = float("nan")          # 9
    for draft in (q, None):
        n, tokens = _check(args, p=p, q=draft, drafts=d)
        assert tokens[0].tolist() == [-1] * 4 and n[6] == 0 and n[7] <= 1
    _check(args, su=torch.full((12,), float("nan"), device="cuda"))
    _check(args, su=torch.full((12,), 1.5, device="cuda"))
    _check(args, su=torch.full((12,), -1.0, device="cuda"))


@pytest.mark.parametrize("seqs", [3, 200])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nothing_left_of_long_rows(seqs, dtype):
    """Rows longer than one block sums at once, drawn by two launches or by whole rows:
    target rows of zeros, below the draft's everywhere, with infinities, and with all
    their weight in the last token."""
    vocab = 70001
    args = _drafts(43, [1] * seqs, vocab, dtype)
    p, q, d = args["p"], args["q"], args["drafts"]
    p[0:2] = 0
    p[2], p[3] = q[1] / 4, 0
    q[1] = 1.0
    p[4:6, 60000], p[4:6, 3] = INF, float("nan")
    d[2] = 60000
    if seqs > 3:
        p[6:8] = 0
        p[6:8, vocab - 1] = 1e-30
        d[3] = 0
    for draft in (q, None):
        for u in (0.0, 0.7, 1.0 - 2.0 ** -24):
            _, tokens = _check(args, p=p, q=draft, drafts=d,
                               au=torch.full((seqs,), 0.9999, device="cuda"),
                               su=torch.full((seqs,), u, device="cuda"))
            assert tokens[0].tolist() == [-1, -1]


@pytest.mark.parametrize("starts", [[-5, 3, 2, 9, 400], [0, 0, 0, 0, 0], [9, 9, 9, 9, 9],
                                    [400, -400, 400, -400, 400], [3, 1, 8, 8, 2]])
def test_offsets_out_of_range_are_clamped(starts):
    args = _drafts(17, [2, 3, 0, 4], 700)
    s = torch.tensor(starts, dtype=torch.int32, device="cuda")
    for known in (True, False):
        _check(args, starts=s, q=args["q"] if known else None)


@pytest.mark.parametrize("vocab", [65, 1031, 20000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_verify_strides(vocab, dtype):
    """Rows inside wider ones, at any address of their type; the values around them
    are large and must not be drawn."""
    args = _drafts(19, [3, 0, 5, 2], vocab, dtype)
    wide = {}
    for name, pad in (("p", 3), ("q", 5)):
        t = args[name]
        big = torch.full((t.shape[0], vocab + 9), 50.0, dtype=t.dtype, device="cuda")
        big[:, pad:pad + vocab] = t
        wide[name] = big[:, pad:pad + vocab]
    a = _check(args)
    b = _check(args, **wide)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_draws_follow_the_weights():
    """Of 4096 evenly spaced random numbers each token of the residual gets its
    share, to one in either direction."""
    vocab, seqs = 3000, 4096
    g = torch.Generator(device="cuda")
    g.manual_seed(23)
    w = torch.rand(vocab, generator=g, device="cuda") ** 8
    w[::5] = 0
    p = (w / w.sum()).expand(seqs, vocab).contiguous()
    su = (torch.arange(seqs, device="cuda") + 0.5) / seqs
    z = torch.zeros(0, device="cuda")
    n, tokens = speculate.verify_drafts(p, None, z.int(), torch.zeros(seqs + 1, device="cuda").int(),
                                        0, z, su)
    got = torch.bincount(tokens[:, 0].long(), minlength=vocab).double().cpu()
    want = p[0].double().cpu() / p[0].double().cpu().sum() * seqs
    assert (n == 0).all() and ((got - want).abs() <= 1 + 1e-6).all()
    assert (tokens[1:, 0] >= tokens[:-1, 0]).all()


def test_no_sequences():
    args = _drafts(29, [2, 1], 100)
    n, tokens = speculate.verify_drafts(args["p"][:0], args["q"][:0], args["drafts"][:0],
                                        args["starts"][:1], 3, args["au"][:0], args["su"][:0])
    assert n.shape == (0,) and tokens.shape == (0, 4)


# ---- together --------------------------------------------------------------
def _answer(st, gain, head, hidden, temperature, args):
    logits = st.lm_head(gain, head, hidden, stream=torch.cuda.current_stream().cuda_stream)
    probs = speculate.token_probs(logits, temperature, out=logits)
    return (probs,) + speculate.verify_drafts(probs, args["q"], args["drafts"], args["starts"],
                                              args["most"], args["au"], args["su"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [1000, 20003])
def test_answer_of_a_last_stage(dtype, vocab):
    """Hidden rows -> LM head in 8 bits -> probabilities -> verified tokens, eager and
    captured; every replay on other hidden rows and random numbers, with eager calls
    between them."""
    shape, counts = synth.TINY, [4, 0, 2, 5, 1, 3]
    rows = sum(counts) + len(counts)
    args = _drafts(31, counts, vocab)
    g = torch.Generator(device="cuda")
    g.manual_seed(37)
    gain = torch.ones(shape.hidden, device="cuda").to(TD[dtype])
    head = int8.quantize(torch.randn((vocab, shape.hidden), generator=g, device="cuda") / 6)
    hidden = torch.randn((rows, shape.hidden), generator=g, device="cuda").to(TD[dtype])
    temperature = torch.full((rows,), 0.9, device="cuda")
    temperature[::4] = 0
    layer = [upload_weights(synth.host_layer_weights(shape, 1, 0), dtype)]
    st = DeviceStage(shape, dtype, 0, layer, 8, 64, 8)
    try:
        logits = st.lm_head(gain, head, hidden)
        torch.cuda.synchronize()
        probs, n, tokens = _answer(st, gain, head, hidden, temperature, args)
        _probs_close(probs, logits, temperature, "f32")
        want_n, want = _verify_reference(probs, args["q"], args["drafts"], args["starts"],
                                         args["most"], args["au"], args["su"])
        assert n.tolist() == want_n and tokens.tolist() == want
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            captured = _answer(st, gain, head, hidden, temperature, args)
        for _ in range(4):
            hidden.copy_(torch.randn(hidden.shape, generator=g, device="cuda"))
            args["au"].copy_(torch.rand(args["au"].shape, generator=g, device="cuda"))
            args["su"].copy_(torch.rand(args["su"].shape, generator=g, device="cuda"))
            graph.replay()
            torch.cuda.synchronize()
            eager = _answer(st, gain, head, hidden, temperature, args)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(captured, eager))
    finally:
        st.close()


def test_two_streams():
    cases = [_drafts(41 + i, [3, 1, 4] * (1 + 20 * i), 6000 + 7 * i) for i in range(2)]

    def call(a):
        probs = speculate.token_probs(a["p"].log())
        return (probs,) + speculate.verify_drafts(probs, a["q"], a["drafts"], a["starts"], a["most"],
                                                  a["au"], a["su"])
    want = [call(a) for a in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[], []]
    for _ in range(4):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(call(cases[i]))
    torch.cuda.synchronize()
    for w, results in zip(want, got):
        for r in results:
            assert all(torch.equal(a, b) for a, b in zip(w, r))
