"""Embedding lookup, its gradient, log-probabilities from logits and their gradient on the GPU against the fp64 oracle.

Tolerances, derived before the first run.  u = 2^-24 is half an fp32 step.
  lse      sum of exponentials: each has the error of ex2 (2^-22), of its argument (2 roundings of |t| <= range) and of
           the sums (a thread adds about vocab / threads terms, then a tree): lse_tol below, plus one rounding of lse.
  entropy  the same errors, weighted with |t|.
  gradient p inherits the error of its exponent, (|z| + |lse|) u each, and of exp (2^-21); the result is rounded once to
           its type (eps / 2).
  embed_bwd  k additions: k u sum |dout|, one rounding for the scale."""
import numpy as np
import pytest
import torch

from oracle import vocab_oracle as vo

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def B():
    from paper_2605_16154_b200 import binding
    return binding


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def placed(t, gap=0, shift=0):
    """The same matrix with `gap` extra elements between its rows, starting `shift` elements into its allocation."""
    n, c = t.shape
    flat = torch.full((shift + n * (c + gap) + 8,), 777.0, dtype=t.dtype, device=t.device)
    view = flat[shift:shift + n * (c + gap)].view(n, c + gap)[:, :c]
    view.copy_(t)
    return view


def host(t):
    return t.detach().double().cpu().numpy()


# ---- embedding --------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,d,gap,shift", [(1, 1, 1, 0, 0), (1, 50, 2048, 0, 0), (64, 1003, 40, 0, 0), (333, 77, 129, 3, 1), (5000, 300, 8, 8, 8),
                                                 (700, 512, 1024, 0, 0), (31, 9, 4097, 0, 1), (2, 5, 16384, 0, 0)])
def test_embed_rounds_the_scaled_row_once(kind, n, vocab, d, gap, shift):
    g = gen(n + d)
    table = placed((torch.randn(vocab, d, generator=g, device="cuda") * 0.02).to(TYPES[kind]), gap, shift)
    tok = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    if n > 4:
        tok[1], tok[3] = -1, vocab                               # padded; outside
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for scale in (1.0, 0.37):
        out = B().grpo_embed(table, tok, scale, status=status)
        want = (table[tok.long().clamp(0, vocab - 1)].float() * scale).to(TYPES[kind])
        want[(tok < 0) | (tok >= vocab)] = 0
        assert torch.equal(out, want)
    assert int(status) == (32 if n > 4 else 0)


def test_embed_writes_nothing_beside_its_rows():
    table = torch.randn(20, 24, device="cuda").bfloat16()
    tok = torch.arange(6, dtype=torch.int32, device="cuda")
    buf = torch.full((8, 40), 5.0, dtype=torch.bfloat16, device="cuda")
    B().grpo_embed(table, tok, out=buf[1:7, 8:32])
    assert torch.equal(buf[1:7, 8:32], table[:6])
    buf[1:7, 8:32] = 5.0
    assert bool((buf == 5.0).all())


def check_embed_grad(grad, dout, tok, vocab, scale, before=None):
    want = vo.embed_bwd(host(dout), tok.cpu().numpy(), vocab, scale)
    live = (tok >= 0) & (tok < vocab)
    mass = vo.embed_bwd(np.abs(host(dout)), tok.cpu().numpy(), vocab, abs(scale))
    k = np.bincount(tok[live].cpu().numpy().astype(np.int64), minlength=vocab)[:, None]
    start = 0.0 if before is None else host(before)
    tol = (k + 2) * U * mass + 2 * U * np.abs(start + want)
    assert np.all(np.abs(host(grad) - start - want) <= tol)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,d,gap,shift", [(1, 1, 1, 0, 0), (1, 70001, 8, 0, 0), (997, 1003, 520, 0, 0), (64, 3, 129, 5, 1), (3000, 17, 72, 0, 0),
                                                 (8193, 255, 64, 0, 0), (20000, 256, 24, 8, 0), (20011, 65537, 33, 0, 0), (16, 2, 1024, 0, 0),
                                                 (40000, 70000, 16, 0, 8), (129, 40, 2056, 0, 0),
                                                 (270001, 70000, 8, 0, 0), (500, 4194400, 8, 0, 0), (1025, 4194400, 8, 0, 0),
                                                 (2048, 900, 16, 0, 0), (2049, 900, 16, 0, 0), (1030, 2097150, 8, 0, 0), (1024, 2097151, 8, 0, 0)])
def test_embed_gradient(kind, n, vocab, d, gap, shift):
    g = gen(n + vocab)
    dout = placed(torch.randn(n, d, generator=g, device="cuda").to(TYPES[kind]), gap, shift)
    u = torch.rand(n, generator=g, device="cuda")
    tok = (vocab * u ** 3).int().clamp_(0, vocab - 1)            # some tokens far more often than others
    if n > 10:
        tok[torch.rand(n, generator=g, device="cuda") < 0.2] = -1
        tok[7] = vocab + 3
    grad = B().grpo_embed_bwd(dout, tok, vocab, scale=1.5)
    check_embed_grad(grad, dout, tok, vocab, 1.5)
    again = B().grpo_embed_bwd(dout, tok, vocab, scale=1.5, grad=torch.full_like(grad, float("nan")))
    assert torch.equal(grad, again)                              # same bits, and every row is written
    more = B().grpo_embed_bwd(dout, tok, vocab, scale=1.5, grad=grad.clone(), accumulate=True)
    check_embed_grad(more, dout, tok, vocab, 1.5, before=grad)
    absent = torch.ones(vocab, dtype=torch.bool, device="cuda")
    absent[tok[(tok >= 0) & (tok < vocab)].long()] = False
    keep = torch.full_like(grad, 3.0)
    B().grpo_embed_bwd(dout, tok, vocab, scale=1.5, grad=keep, accumulate=True)
    assert bool((keep[absent] == 3.0).all())


@pytest.mark.parametrize("n", [15, 16, 17, 5000, 30000])
def test_embed_gradient_of_one_token_and_of_none(n):
    dout = torch.randn(n, 136, generator=gen(n), device="cuda")
    tok = torch.full((n,), 4, dtype=torch.int32, device="cuda")
    check_embed_grad(B().grpo_embed_bwd(dout, tok, 9), dout, tok, 9, 1.0)
    tok.fill_(-1)
    assert not B().grpo_embed_bwd(dout, tok, 9).any()
    assert not B().grpo_embed_bwd(dout[:0], tok[:0], 9).any()


# ---- log-probabilities ------------------------------------------------------------------------------------------
def logp_tolerances(z, temperature, lse):
    zt = np.where(np.isfinite(z), np.abs(z), 0.0) / temperature
    vocab = z.shape[1]
    spread = 2 * zt.max(-1) + 2                                  # |t| of any term
    threads = 32 if vocab <= 1024 else 256
    sums = (vocab / threads + 24) * U
    lse_tol = 2.0 ** -22 + 4 * U * spread + sums + 2 * U * (np.abs(lse) + spread)
    return lse_tol, lse_tol + 2 * U * spread, (spread + 2) * (2.0 ** -21 + 4 * U * spread + 2 * sums)


def close(got, want, tol):
    got, want = host(got), np.asarray(want)
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got)) and np.array_equal(np.isnan(want), np.isnan(got))
    tol = np.broadcast_to(tol, want.shape)
    bad = np.abs(got[fine] - want[fine]) > tol[fine]
    assert not bad.any(), (got[fine][bad][:4], want[fine][bad][:4], tol[fine][bad][:4])


def check_logp(logits, tok, temperature, top):
    z = host(logits)
    want = vo.token_logp(z, None if tok is None else tok.cpu().numpy(), temperature, top)
    logp, entropy, lse, top_id, top_logp = B().grpo_token_logp(logits, tok, temperature, top)
    lt, pt, et = logp_tolerances(z, temperature, np.where(np.isfinite(want["lse"]), want["lse"], 0))
    close(lse, want["lse"], lt)
    close(entropy, want["entropy"], et)
    if tok is not None:
        close(logp, want["logp"], pt)
    if top:
        assert np.array_equal(top_id.cpu().numpy(), want["top_id"])
        close(top_logp, want["top_logp"], pt[:, None])
    return want


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,gap,shift", [(1, 1, 0, 0), (3, 2, 0, 1), (9, 7, 0, 0), (40, 31, 1, 3), (17, 256, 0, 0), (8, 1000, 0, 5), (70, 1024, 0, 0),
                                               (33, 1025, 0, 0), (5, 4099, 6, 1), (700, 2050, 0, 0), (1, 5000, 3, 2), (2, 16390, 0, 0),
                                               (1, 130011, 0, 7), (3, 33000, 8, 0), (300, 4500, 0, 0)])
def test_logp(kind, n, vocab, gap, shift):
    g = gen(n * 31 + vocab)
    logits = placed((torch.randn(n, vocab, generator=g, device="cuda") * 3).to(TYPES[kind]), gap, shift)
    tok = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    if n > 4:
        tok[1], tok[n - 1] = -1, vocab + 1
    for temperature, top in ((1.0, 0), (0.7, min(5, vocab)), (2.5, min(16, vocab)), (1.0, 1)):
        check_logp(logits, tok, temperature, top)
    check_logp(logits, None, 1.0, min(2, vocab))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [13, 800, 1500, 6000, 40000])
def test_logp_of_unusual_rows(kind, vocab):
    """Sorted either way, all equal, few values left by a mask, none left, the type's lowest value, signed zeros, NaN, +inf."""
    t = TYPES[kind]
    low = torch.finfo(t).min
    ramp = torch.arange(vocab, device="cuda", dtype=torch.float32) * (20.0 / vocab)
    rows = [ramp, ramp.flip(0), torch.full_like(ramp, -2.5), torch.full_like(ramp, float("-inf")), torch.full_like(ramp, low)]
    few = torch.full_like(ramp, float("-inf"))
    few[[2, 5, vocab - 1]] = torch.tensor([1.0, 3.0, 1.0], device="cuda")
    lowest = torch.full_like(ramp, low)
    lowest[4:9] = torch.randn(5, generator=gen(1), device="cuda")
    zeros = torch.zeros_like(ramp)
    zeros[::3] = -0.0
    nan = torch.randn(vocab, generator=gen(2), device="cuda")
    nan[[3, vocab - 2]] = float("nan")
    inf = torch.randn(vocab, generator=gen(3), device="cuda")
    inf[[6, vocab - 3]] = float("inf")
    lone = torch.full_like(ramp, float("-inf"))
    lone[vocab // 2] = -7.0
    rows += [few, lowest, zeros, nan, inf, lone]
    logits = torch.stack(rows).to(t)
    tok = torch.tensor([0, 1, 2, 3, 4, 5, 6, 7, 8, 9, vocab // 2], dtype=torch.int32, device="cuda")
    with np.errstate(over="ignore", invalid="ignore"):
        finite = torch.where(logits.abs() > 1e30, torch.zeros_like(logits), logits)
        z = host(logits)
        for top in (0, 4, 13):
            want = vo.token_logp(z, tok.cpu().numpy(), 0.9, top)
            logp, entropy, lse, top_id, top_logp = B().grpo_token_logp(logits, tok, 0.9, top)
            lt, pt, et = logp_tolerances(host(finite), 0.9, 0.0)
            big = np.where(np.isfinite(want["lse"]), np.abs(want["lse"]), 0) * 4 * U + pt     # rows of the lowest value: |lse| is large
            close(lse, clip32(want["lse"]), big + lt)
            close(entropy, want["entropy"], et)
            if top:
                assert np.array_equal(top_id.cpu().numpy(), want["top_id"])


def clip32(x):
    """Values beyond fp32's range as the infinities they round to."""
    with np.errstate(invalid="ignore"):
        return np.where(np.abs(x) > 3.4028235e38, np.copysign(np.inf, x), x)


def check_logp_bwd(logits, tok, temperature, dlogp, dent, got, lse32, ent32):
    z = host(logits)
    want = vo.token_logp_bwd(z, tok.cpu().numpy(), host(dlogp), None if dent is None else host(dent), temperature)
    eps = torch.finfo(logits.dtype).eps / 2
    zt, lse = np.where(np.isfinite(z), z, 0.0) / temperature, np.where(np.isfinite(host(lse32)), host(lse32), 0.0)[:, None]
    lp = np.where(np.isfinite(z), zt - lse, -np.inf)
    p = np.exp(lp)
    h = 0.0 if dent is None else np.abs(host(dent))[:, None]
    inner = np.abs(host(dlogp))[:, None] + h * (np.where(np.isfinite(lp), np.abs(lp), 0) + np.abs(host(ent32))[:, None] + 1)
    rel = 4 * U * (np.abs(zt) + np.abs(lse) + 4) + 2.0 ** -21
    terms = (p * inner + np.where(np.arange(z.shape[1])[None] == tok.cpu().numpy()[:, None], np.abs(host(dlogp))[:, None], 0)) / temperature
    tol = rel * terms + eps * (np.abs(want) + rel * terms) + 2.0 ** -133        # the last: the smallest step of the type
    close(got, want, tol)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,gap,shift,gap2,shift2", [(1, 1, 0, 0, 0, 0), (3, 7, 0, 0, 0, 0), (11, 257, 1, 3, 1, 3), (11, 257, 1, 3, 0, 0), (4, 4099, 6, 1, 6, 1),
                                                          (6, 32000, 0, 0, 0, 0), (2, 9000, 0, 2, 8, 2)])
def test_logp_gradient(kind, n, vocab, gap, shift, gap2, shift2):
    g = gen(n * 7 + vocab)
    logits = placed((torch.randn(n, vocab, generator=g, device="cuda") * 3).to(TYPES[kind]), gap, shift)
    if vocab > 100:
        logits[::2, vocab // 2:vocab - 3] = float("-inf")
        logits[n - 1] = float("-inf")
    tok = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    if n > 2:
        tok[1], tok[2] = -1, vocab
    dlogp, dent = torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
    for temperature, de in ((1.0, None), (0.8, dent)):
        _, entropy, lse, _, _ = B().grpo_token_logp(logits, tok, temperature)
        out = placed(torch.full((n, vocab), 9.0, dtype=logits.dtype, device="cuda"), gap2, shift2)
        got = B().grpo_token_logp_bwd(logits, tok, lse, entropy, dlogp, de, temperature, dlogits=out)
        check_logp_bwd(logits, tok, temperature, dlogp, de, got, lse, entropy)
        work = placed(logits, gap, shift)
        B().grpo_token_logp_bwd(work, tok, lse, entropy, dlogp, de, temperature, dlogits=work)      # in place
        assert torch.equal(work, got)


def test_logp_gradient_against_differences():
    n, vocab, T = 4, 300, 1.3
    g = gen(8)
    z, tok = torch.randn(n, vocab, generator=g, device="cuda"), torch.tensor([5, 299, 0, 17], dtype=torch.int32, device="cuda")
    a, b = torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
    _, ent, lse, _, _ = B().grpo_token_logp(z, tok, T)
    grad = B().grpo_token_logp_bwd(z, tok, lse, ent, a, b, T)
    step = torch.randn(n, vocab, generator=g, device="cuda")

    def loss(q):
        lp, e, _, _, _ = B().grpo_token_logp(q, tok, T)
        return float((lp.double() * a.double() + e.double() * b.double()).sum())
    h = 1e-2
    num = (loss(z + h * step) - loss(z - h * step)) / (2 * h)
    # third-order term of the difference: h^2 times a bounded directional derivative; fp32 forward error over h
    assert num == pytest.approx(float((grad.double() * step.double()).sum()), abs=4 * (n * 6e-6 / h + 10 * h * h))


def test_refusals_of_the_binding():
    b = B()
    z, tok = torch.zeros(4, 32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    v = torch.zeros(4, device="cuda")
    bad = [lambda: b.grpo_token_logp(z.t(), tok), lambda: b.grpo_token_logp(z.half(), tok), lambda: b.grpo_token_logp(z, tok.long()),
           lambda: b.grpo_token_logp(z, tok[:3]), lambda: b.grpo_token_logp(z, tok.cpu()), lambda: b.grpo_token_logp(z, tok, 0.0),
           lambda: b.grpo_token_logp(z, tok, top=17), lambda: b.grpo_token_logp(z[:1].expand(4, 32), tok),
           lambda: b.grpo_token_logp_bwd(z, tok, v, None, v, v), lambda: b.grpo_token_logp_bwd(z, tok, v, v, v, dlogits=z.bfloat16()),
           lambda: b.grpo_token_logp_bwd(z, tok, v, v, None), lambda: b.grpo_embed(z, tok, out=z.bfloat16()),
           lambda: b.grpo_embed(z, tok, float("nan")), lambda: b.grpo_embed_bwd(z, tok, 5, accumulate=True),
           lambda: b.grpo_embed_bwd(z, tok, 5, grad=torch.zeros(5, 31, device="cuda")), lambda: b.grpo_embed_bwd(z, tok, 0),
           lambda: b.grpo_embed_bwd(z, tok, 5, workspace=torch.zeros(64, dtype=torch.uint8, device="cuda"))]
    for f in bad:
        with pytest.raises(b.PcmError):
            f()


def test_captured_calls_follow_their_inputs_on_another_stream():
    b, n, vocab, d = B(), 300, 5003, 64
    g = gen(12)
    table, z = torch.randn(vocab, d, generator=g, device="cuda").bfloat16(), torch.randn(n, vocab, generator=g, device="cuda")
    tok = torch.randint(-1, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    a = torch.randn(n, generator=g, device="cuda")

    def step():
        emb = b.grpo_embed(table, tok, 2.0)
        lp, ent, lse, ids, tl = b.grpo_token_logp(z, tok, 1.1, top=4)
        return emb, lp, ent, ids, tl, b.grpo_token_logp_bwd(z, tok, lse, ent, a, a, 1.1), b.grpo_embed_bwd(emb, tok, vocab, 2.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in (1, 2):
        z.copy_(torch.randn(n, vocab, generator=gen(seed), device="cuda"))
        tok.copy_(torch.randint(-1, vocab, (n,), generator=gen(seed), device="cuda", dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(held, step()):
            assert torch.equal(x, y)


# ---- many rows (a block of 128 threads each), far offsets, several streams --------------------------------------------
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,gap,shift", [(1025, 0, 0), (2603, 2, 3)])
def test_logp_of_many_rows(kind, vocab, gap, shift):
    n, g = 1300, gen(vocab)
    logits = (torch.randn(n, vocab, generator=g, device="cuda") * 3).to(TYPES[kind])
    low = torch.finfo(TYPES[kind]).min
    ramp = torch.arange(vocab, device="cuda", dtype=torch.float32) * (20.0 / vocab)
    for i, row in enumerate((ramp, ramp.flip(0), torch.full_like(ramp, 1.5), torch.full_like(ramp, float("-inf")), torch.full_like(ramp, -30.0))):
        logits[40 * i + 3] = row.to(logits.dtype)
    logits[500:520, 7:] = float("-inf")                          # fewer values than places
    logits[520, 9], logits[521, 11], logits[522, :5] = float("nan"), float("inf"), low
    logits = placed(logits, gap, shift)
    tok = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    tok[500:520] = torch.arange(20, device="cuda", dtype=torch.int32) % 7
    tok[600], tok[1299] = -5, vocab
    z = host(logits)
    want = vo.token_logp(z, tok.cpu().numpy(), 1.25, 16)
    finite = np.where(np.isfinite(z) & (np.abs(z) < 1e30), z, 0.0)
    lt, pt, et = logp_tolerances(finite, 1.25, np.where(np.isfinite(want["lse"]), want["lse"], 0))
    for top in (16, 3, 0):
        logp, entropy, lse, top_id, top_logp = B().grpo_token_logp(logits, tok, 1.25, top)
        close(lse, want["lse"], lt)
        close(entropy, want["entropy"], et)
        close(logp, clip32(want["logp"]), pt)
        if top:
            assert np.array_equal(top_id.cpu().numpy(), want["top_id"][:, :top])
            close(top_logp, clip32(want["top_logp"][:, :top]), pt[:, None] + 4 * U * np.abs(np.where(np.abs(want["top_logp"][:, :top]) < 1e38, want["top_logp"][:, :top], 0)))


def test_rows_far_apart():
    """Offsets that do not fit 32 bits: rows of logits, of an embedding table, of the gradient."""
    ld, vocab = 1_300_000_000, 5001
    buf = torch.empty(2 * ld + vocab, dtype=torch.bfloat16, device="cuda")
    logits = buf.as_strided((3, vocab), (ld, 1))
    logits.copy_(torch.randn(3, vocab, generator=gen(1), device="cuda"))
    tok = torch.tensor([5, 5000, 77], dtype=torch.int32, device="cuda")
    check_logp(logits, tok, 1.0, 4)
    a = torch.ones(3, device="cuda")
    _, ent, lse, _, _ = B().grpo_token_logp(logits, tok)
    near = B().grpo_token_logp_bwd(logits.contiguous(), tok, lse, ent, a, a)
    assert torch.equal(B().grpo_token_logp_bwd(logits, tok, lse, ent, a, a, dlogits=logits), near)
    del logits, buf
    vocab, d = 40000, 60000
    table = torch.empty(vocab, d, dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([0, 39999, 36000, 39999], dtype=torch.int32, device="cuda")
    table[[0, 36000, 39999]] = torch.randn(3, d, generator=gen(2), device="cuda").bfloat16()
    assert torch.equal(B().grpo_embed(table, rows), table[rows.long()])
    del table
    dout = torch.randn(4, d, generator=gen(3), device="cuda")
    grad = B().grpo_embed_bwd(dout, rows, vocab)
    assert torch.equal(grad[0], dout[0]) and torch.equal(grad[36000], dout[2]) and torch.allclose(grad[39999], dout[1] + dout[3])
    assert int(torch.count_nonzero(grad[1:36000])) == 0 and int(torch.count_nonzero(grad[36001:39999])) == 0


def test_calls_on_two_streams_at_once():
    b = B()
    work = []
    for k in range(2):
        g = gen(40 + k)
        z = torch.randn(900, 6000, generator=g, device="cuda").bfloat16()
        tok = torch.randint(0, 6000, (900,), generator=g, device="cuda", dtype=torch.int32)
        dout = torch.randn(900 * 20, 256, generator=g, device="cuda")
        long = torch.randint(0, 6000, (900 * 20,), generator=g, device="cuda", dtype=torch.int32)
        work.append((z, tok, dout, long))

    def step(z, tok, dout, long):
        lp, ent, lse, ids, tl = b.grpo_token_logp(z, tok, 1.0, 8)
        return lp, ids, tl, b.grpo_token_logp_bwd(z, tok, lse, ent, lp, ent), b.grpo_embed_bwd(dout, long, 6000)
    want = [step(*w) for w in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = []
        for s, w in zip(streams, work):
            with torch.cuda.stream(s):
                got.append(step(*w))
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert all(torch.equal(p, q) for p, q in zip(x, y))
