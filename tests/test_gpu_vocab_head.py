"""Log-probabilities from hidden states and head weight, their gradients, and the whole vocabulary path of a tied policy, on
the GPU against the fp64 oracle.

Tolerances, derived before the first run.  u = 2^-24.
  z        bf16 products are exact in fp32; the tensor core adds 16 of them at a time into an accumulator that it may
           truncate: (d / 16 + 2) 2^-23 sum |x w|.
  logp     z's error twice (its own and through lse), plus ex2 and sums as in the logits' own test.
  dx       d z is rounded to bf16 (half a step: with 8 significant bits 2^-8 of the value), the product adds vocab / 16
           truncations, the result is rounded (2^-8).
  dw       d z = hi + lo leaves 2^-8 of 2^-8, 2^-16 of each; pieces of 32 truncations; fp32 additions of the pieces.
  Either inherits the error of d z itself: p times the error of its exponent."""
import numpy as np
import pytest
import torch

from oracle import vocab_oracle as vo

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def B():
    from paper_2605_16154_b200 import binding
    return binding


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def host(t):
    return t.detach().double().cpu().numpy()


def wide(t, gap):
    """The same rows, `gap` elements of something else after each."""
    buf = torch.full((t.shape[0], t.shape[1] + gap), 333.0, dtype=t.dtype, device=t.device)
    buf[:, :t.shape[1]] = t
    return buf[:, :t.shape[1]]


def problem(n, d, vocab, gap=0, seed=0):
    g = gen(seed * 1000 + n + d + vocab)
    x = wide(torch.randn(n, d, generator=g, device="cuda").bfloat16(), gap)
    w = wide((torch.randn(vocab, d, generator=g, device="cuda") * (2.0 / d ** 0.5)).bfloat16(), gap)
    tok = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    if n > 6:
        tok[2], tok[n - 1], tok[5] = -1, vocab, -7
        x[2], x[5] = float("nan"), float("inf")                 # what padded rows hold does not matter
    dlogp, dent = torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda") * 0.1
    return x, w, tok, dlogp, dent


def finite(x, tok, vocab):
    x = host(x)
    x[~((tok >= 0) & (tok < vocab)).cpu().numpy()] = 0.0
    return x


def z_error(x, w, temperature):
    """Per row: bound of the error of any logit, over the temperature; range of the logits."""
    mass = np.abs(x) @ np.abs(w).T
    z = x @ w.T / temperature
    return (x.shape[1] / 16 + 2) * 2.0 ** -23 * mass.max(-1) / temperature, np.abs(z).max(-1)


SIZES = [(1, 8, 1, 0), (1, 64, 3, 0), (3, 72, 130, 8), (16, 2048, 4000, 0), (128, 64, 256, 0), (129, 64, 257, 0), (130, 200, 1000, 16),
         (300, 256, 5003, 0), (701, 1024, 515, 0), (257, 520, 1111, 8), (1, 1024, 50001, 0), (900, 96, 96, 0), (40, 640, 128, 0), (5, 2056, 700, 0), (150, 4096, 1500, 8)]


@pytest.mark.parametrize("n,d,vocab,gap", SIZES)
def test_head_logp(n, d, vocab, gap):
    x, w, tok, _, _ = problem(n, d, vocab, gap)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    xf, wf = finite(x, tok, vocab), host(w)
    for temperature in (1.0, 0.6):
        logp, entropy, lse = B().grpo_head_logp(x, w, tok, temperature, status=status)
        want = vo.head_logp(xf, wf, tok.cpu().numpy(), temperature)
        ze, rng = z_error(xf, wf, temperature)
        base = 2.0 ** -22 + 8 * U * (2 * rng + 2) + (vocab / 128 / 16 + 170) * U
        for got, name, tol in ((lse, "lse", ze + base), (logp, "logp", 2 * ze + base), (entropy, "entropy", (2 * rng + 3) * (ze + base))):
            assert np.all(np.abs(host(got) - want[name]) <= tol), (name, np.abs(host(got) - want[name]).max(), tol.max())
    assert int(status) == (32 if n > 6 else 0)


def check_grads(x, w, tok, lse, entropy, dlogp, dent, temperature, dx, dw, dw0=None):
    vocab = w.shape[0]
    xf, wf, t = finite(x, tok, vocab), host(w), tok.cpu().numpy()
    dent_h = None if dent is None else host(dent)
    dz = vo.token_logp_bwd(xf @ wf.T, t, host(dlogp), dent_h, temperature)
    ze, rng = z_error(xf, wf, temperature)
    lse_h, ent_h = host(lse), host(entropy)
    z = xf @ wf.T / temperature
    lp = z - lse_h[:, None]
    live = ((t >= 0) & (t < vocab))[:, None]
    p = np.where(live, np.exp(lp), 0.0)
    h = 0.0 if dent is None else np.abs(dent_h)[:, None]
    inner = np.abs(host(dlogp))[:, None] + h * (np.abs(lp) + np.abs(ent_h)[:, None] + 1)
    # lse comes from the forward call: its error is one more of z's kind
    rel = (2 * ze + 8 * U * (rng + np.abs(lse_h) + 4) + 2.0 ** -20)[:, None]
    edz = rel * p * inner / temperature + 2 * U * np.abs(dz)
    if dx is not None:
        want = dz @ wf
        mass = np.abs(dz) @ np.abs(wf)
        tol = (edz * (1 + 2.0 ** -8)) @ np.abs(wf) + (2.0 ** -8 + (vocab / 16 + 2) * 2.0 ** -23) * mass
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol) + 2.0 ** -133
        assert np.all(np.abs(host(dx) - want) <= tol), np.max(np.abs(host(dx) - want) - tol)
        assert not host(dx)[~live[:, 0]].any()
    if dw is not None:
        want = dz.T @ xf
        mass = np.abs(dz).T @ np.abs(xf)
        pieces = x.shape[0] / 256 + 4
        # the targets' part, summed by token in fp32: k additions of at most k rows, one product each
        tgt = np.where(live & (np.arange(vocab)[None] == t[:, None]), np.abs(dz), 0.0)
        most = np.bincount(t[live[:, 0]], minlength=vocab).max() if live.any() else 0
        tol = edz.T @ np.abs(xf) + (2.0 ** -16 + 34 * 2.0 ** -23 + 2 * pieces * U) * mass + (most + 4) * U * (tgt.T @ np.abs(xf))
        if dw0 is not None:
            want = want + host(dw0)
            tol = tol + 4 * U * np.abs(host(dw0))
        assert np.all(np.abs(host(dw) - want) <= tol + 1e-37), np.max(np.abs(host(dw) - want) - tol)
        if dw0 is None and np.linalg.norm(want):
            # without the worst case of every term: pieces 34 x 2^-23, remainder at most 2^-16, exponent a few 2^-20
            assert np.linalg.norm(host(dw) - want) <= 2e-5 * np.linalg.norm(want)


@pytest.mark.parametrize("n,d,vocab,gap", SIZES + [(5000, 64, 40, 0), (200, 64, 20000, 0)])
def test_head_gradients(n, d, vocab, gap):
    b = B()
    x, w, tok, dlogp, dent = problem(n, d, vocab, gap, seed=1)
    if n > 6:
        dlogp[2], dent[2] = float("nan"), float("inf")
    dl, de = dlogp.clone(), dent.clone()
    if n > 6:
        dl[2], de[2] = 0.0, 0.0                                  # the oracle leaves padded rows out; numpy's masks do not like NaN
    _, entropy, lse = b.grpo_head_logp(x, w, tok, 0.8)
    out = wide(torch.full((n, d), 4.0, device="cuda").bfloat16(), gap)
    dx, dw = b.grpo_head_logp_bwd(x, w, tok, lse, entropy, dlogp, dent, 0.8, dx=out)
    check_grads(x, w, tok, lse, entropy, dl, de, 0.8, dx, dw)
    dx2, dw2 = b.grpo_head_logp_bwd(x, w, tok, lse, entropy, dlogp, dent, 0.8, dw=torch.full_like(dw, float("nan")))
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)         # same bits
    if gap:
        assert bool((out._base[:, d:] == 333.0).all())
    only, none = b.grpo_head_logp_bwd(x, w, tok, lse, None, dlogp, None, 0.8, want_dw=False)
    assert none is None
    check_grads(x, w, tok, lse, entropy, dl, None, 0.8, only, None)
    before = torch.randn(vocab, d, generator=gen(3), device="cuda")
    none, dw3 = b.grpo_head_logp_bwd(x, w, tok, lse, entropy, dlogp, dent, 0.8, dw=before.clone(), accumulate=True, want_dx=False,
                                     chunk_rows=max(1, n // 3))
    assert none is None
    check_grads(x, w, tok, lse, entropy, dl, de, 0.8, None, dw3, dw0=before)
    if n > 3:
        dx4, _ = b.grpo_head_logp_bwd(x, w, tok, lse, entropy, dlogp, dent, 0.8, chunk_rows=n // 2 + 1)
        check_grads(x, w, tok, lse, entropy, dl, de, 0.8, dx4, None)


def test_no_rows():
    b = B()
    w = torch.randn(300, 64, device="cuda").bfloat16()
    x, tok, v = w[:0], torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, device="cuda")
    logp, entropy, lse = b.grpo_head_logp(x, w, tok)
    assert logp.numel() == 0
    dx, dw = b.grpo_head_logp_bwd(x, w, tok, lse, entropy, v, v, dw=torch.ones(300, 64, device="cuda"))
    assert dx.shape == (0, 64) and not dw.any()


def test_refusals_of_the_binding():
    b = B()
    x, w, tok, dlogp, dent = problem(8, 64, 100)
    _, ent, lse = b.grpo_head_logp(x, w, tok)
    bad = [lambda: b.grpo_head_logp(x.float(), w.float(), tok), lambda: b.grpo_head_logp(x[:, :60], w[:, :60], tok),
           lambda: b.grpo_head_logp(x, w[:, :56], tok), lambda: b.grpo_head_logp(x, w, tok.long()),
           lambda: b.grpo_head_logp(x, w, tok, -1.0), lambda: b.grpo_head_logp(x, w, None),
           lambda: b.grpo_head_logp(x, w, tok, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda")),
           lambda: b.grpo_head_logp(x.reshape(-1)[4:4 + 7 * 64].view(7, 64), w, tok[:7]),        # eight bytes into its allocation
           lambda: b.grpo_head_logp_bwd(x, w, tok, lse, None, dlogp, dent), lambda: b.grpo_head_logp_bwd(x, w, tok, lse, ent, dlogp, dent, accumulate=True),
           lambda: b.grpo_head_logp_bwd(x, w, tok, lse, ent, dlogp, dent, want_dx=False, want_dw=False),
           lambda: b.grpo_head_logp_bwd(x, w, tok, lse, ent, dlogp, dent, dx=torch.zeros(8, 64, device="cuda")),
           lambda: b.grpo_head_logp_bwd(x, w, tok, lse, ent, dlogp, dent, chunk_rows=-4)]
    for f in bad:
        with pytest.raises(b.PcmError):
            f()


def test_weight_gradient_is_as_exact_as_fp32_products():
    """Spread-out rows: a row's d z is its target's for the most part, which fp32 sums carry; the rest is cut to 16 bits."""
    b = B()
    x, w, tok, dlogp, dent = problem(700, 512, 4001, seed=6)
    dlogp[2] = dent[2] = 0.0
    _, entropy, lse = b.grpo_head_logp(x, w, tok)
    dx, dw = b.grpo_head_logp_bwd(x, w, tok, lse, entropy, dlogp, dent * 1e-2)
    xf, wf = finite(x, tok, 4001), host(w)
    want_dx, want = vo.head_logp_bwd(xf, wf, tok.cpu().numpy(), host(dlogp), host(dent) * 1e-2)
    dz = vo.token_logp_bwd(xf @ wf.T, tok.cpu().numpy(), host(dlogp), host(dent) * 1e-2)
    rest = dz.copy()
    rest[np.arange(700), np.clip(tok.cpu().numpy(), 0, 4000)] = 0.0
    share = np.linalg.norm(rest) / np.linalg.norm(dz)
    # remainder 2^-16 at most of the rest; p from fp32 exponents (2^-20); 34 truncations a piece and fp32 sums of the targets
    bound = share * (2.0 ** -16 + 2.0 ** -19) + 34 * 2.0 ** -23 * 0.5
    assert np.linalg.norm(host(dw) - want) <= bound * np.linalg.norm(want)
    # dx: its own rounding, 2^-8 of each element at most, spread evenly over half steps of 2^-9 to 2^-8 of the value (3^-1/2 of
    # it in the mean); the rest's rounding likewise, its errors independent of one another
    bound = 2.0 ** -8 * 3 ** -0.5 * (1 + 2 * share)
    assert np.linalg.norm(host(dx) - want_dx) <= bound * np.linalg.norm(want_dx)


def test_a_nan_in_a_live_row_reaches_its_gradient_and_no_other():
    b = B()
    x, w, tok, dlogp, dent = problem(5, 64, 300)
    x[2, 7] = float("nan")
    logp, entropy, lse = b.grpo_head_logp(x, w, tok)
    keep = torch.arange(5, device="cuda") != 2
    assert bool(torch.isnan(logp[2]) & torch.isnan(lse[2]) & torch.isnan(entropy[2])) and bool(torch.isfinite(logp[keep]).all())
    for de in (dent, None):
        dx, dw = b.grpo_head_logp_bwd(x, w, tok, lse, entropy, dlogp, de)
        assert bool(torch.isnan(dx[2]).all()) and bool(torch.isfinite(dx[keep]).all())
        assert bool(torch.isnan(dw).any())


def test_a_row_without_a_finite_logit_has_no_gradient():
    """lse = -inf, as a caller may hand in, with a valid token: nothing of the row reaches either gradient."""
    b = B()
    x, w, tok, dlogp, dent = problem(6, 64, 300)
    _, entropy, lse = b.grpo_head_logp(x, w, tok)
    lse[3] = float("-inf")
    x[3, 5] = float("inf")                                       # what its logits are made of does not matter
    dx, dw = b.grpo_head_logp_bwd(x, w, tok, lse, entropy, dlogp, dent)
    keep = torch.arange(6, device="cuda") != 3
    dx2, dw2 = b.grpo_head_logp_bwd(x[keep], w, tok[keep], lse[keep], entropy[keep], dlogp[keep], dent[keep])
    assert not dx[3].any() and torch.equal(dx[keep], dx2)
    assert torch.allclose(dw, dw2, rtol=1e-5, atol=1e-6)         # 0 x inf nowhere


def test_wide_hidden_states_keep_their_accuracy():
    """The tensor core truncates each of d / 16 additions; pieces of 1024 keep the drift of a wide sum at that of 64 additions:
    2 x 64 x 2^-24 = 7.6e-6 of a logit at the very most, typically a tenth, before it is averaged over the vocabulary."""
    b = B()
    x, w, tok, _, _ = problem(64, 4096, 3001, seed=4)
    logp, entropy, lse = b.grpo_head_logp(x, w, tok)
    want = vo.head_logp(finite(x, tok, 3001), host(w), tok.cpu().numpy())
    for got, name in ((logp, "logp"), (entropy, "entropy"), (lse, "lse")):
        assert np.linalg.norm(host(got) - want[name]) <= 2e-6 * np.linalg.norm(want[name]), name


def test_head_agrees_with_the_logits_path():
    b = B()
    x, w, tok, dlogp, dent = problem(64, 256, 700)
    keep = (tok >= 0) & (tok < 700)
    x[~keep] = 0
    w = torch.cat([w, w[:4]])                                     # 704 rows: what grpo_gemm's tensor-core kernel takes
    logits = b.grpo_gemm(x, True, w, True, 64, 704, 256, out_dtype=torch.float32)[:, :700]
    w = w[:700]
    lp, ent, lse, ids, _ = b.grpo_token_logp(logits, tok, 1.2, top=3)
    lp2, ent2, lse2 = b.grpo_head_logp(x, w, tok, 1.2)
    assert torch.allclose(lp, lp2, atol=2e-4) and torch.allclose(ent, ent2, atol=2e-3) and torch.allclose(lse, lse2, atol=2e-4)


def test_tied_policy_step_and_its_gradients():
    """tokens -> embedding -> RMS norm (torch) -> head over the same table -> clipped surrogate with entropy bonus -> gradient
    of the one table, both ends accumulated in fp32; against the same step in fp64 autograd."""
    b = B()
    n, vocab, d, T, scale = 400, 1013, 128, 1.1, 3.0
    g = gen(77)
    table = (torch.randn(vocab, d, generator=g, device="cuda") * 0.3).bfloat16()
    inp = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    tgt = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    tgt[::9] = -1
    inp[::9] = -1
    live = tgt >= 0
    adv = torch.randn(n, generator=g, device="cuda")
    count = int(live.sum())

    # the library's step
    h = b.grpo_embed(table, inp, scale)
    x = (h.float() * torch.rsqrt(h.float().square().mean(-1, keepdim=True) + 1e-5)).bfloat16()
    logp, entropy, lse = b.grpo_head_logp(x, table, tgt, T)
    old = logp + torch.randn(n, generator=g, device="cuda") * 0.05          # no ratio near the clip of 0.2
    ratio = (logp - old).exp()
    dlogp = torch.where(live, -adv * ratio / count, 0.0)
    dent = torch.full((n,), -1e-2 / count, device="cuda")
    grad = torch.zeros(vocab, d, device="cuda")
    dx, _ = b.grpo_head_logp_bwd(x, table, tgt, lse, entropy, dlogp, dent, T, dw=grad, accumulate=True)
    hd = h.double().requires_grad_()
    (hd * torch.rsqrt(hd.square().mean(-1, keepdim=True) + 1e-5)).backward(dx.double())
    dh = hd.grad.float()
    assert not dh[~live].any()
    b.grpo_embed_bwd(dh, inp, vocab, scale, grad=grad, accumulate=True)

    # the same in fp64 (from the same rounded activations, so that only the operators differ)
    tab = table.double().requires_grad_()
    emb = torch.where(live[:, None], tab[inp.clamp(min=0).long()], 0.0) * scale
    emb = emb + (h.double() - emb).detach()
    y = emb * torch.rsqrt(emb.square().mean(-1, keepdim=True) + 1e-5)
    y = y + (x.double() - y).detach()
    lp = torch.log_softmax(y @ tab.t() / T, -1)
    lt = lp.gather(1, tgt.clamp(min=0).long()[:, None])[:, 0]
    ent = -(lp.exp() * lp).sum(-1)
    r = (lt - old.double()).exp()
    loss = -(torch.minimum(r * adv.double(), r.clamp(0.5, 2.0) * adv.double()) * live).sum() / count - 1e-2 * (ent * live).sum() / count
    loss.backward()
    assert float((lt - logp.double())[live].abs().max()) < 1e-4
    # dx is rounded to bf16 twice (d z and the result, 2^-8 at most each)
    assert float((grad.double() - tab.grad).norm() / tab.grad.norm()) < 2.0 ** -7


def test_captured_calls_follow_their_inputs():
    b = B()
    x, w, tok, dlogp, dent = problem(333, 192, 2003)

    def step():
        logp, entropy, lse = b.grpo_head_logp(x, w, tok, 0.9)
        return (logp, entropy, lse) + b.grpo_head_logp_bwd(x, w, tok, lse, entropy, dlogp, dent, 0.9, chunk_rows=200)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in (5, 6):
        x.copy_(torch.randn(333, 192, generator=gen(seed), device="cuda"))
        tok.copy_(torch.randint(-1, 2003, (333,), generator=gen(seed), device="cuda", dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(held, step()):
            assert torch.equal(a, c)


def test_far_offsets_of_the_logit_gradient():
    """One chunk whose d z has more than 2^31 elements gives what small chunks give."""
    b = B()
    n, d, vocab = 18000, 64, 131072
    g = gen(9)
    x, w = torch.randn(n, d, generator=g, device="cuda").bfloat16(), (torch.randn(vocab, d, generator=g, device="cuda") * 0.2).bfloat16()
    tok = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    a = torch.randn(n, generator=g, device="cuda")
    _, ent, lse = b.grpo_head_logp(x, w, tok)
    dx, dw = b.grpo_head_logp_bwd(x, w, tok, lse, ent, a, None, chunk_rows=n)
    dx2, dw2 = b.grpo_head_logp_bwd(x, w, tok, lse, ent, a, None, chunk_rows=3000)
    # dx is summed over other splits of the vocabulary, so its fp32 value may fall on the other side of a bf16 rounding: one
    # step, 2^-7 of the value, at most
    assert float((dx.float() - dx2.float()).norm() / dx.float().norm()) < 2.0 ** -7
    # the pieces of dw are the same 512 rows only where chunks divide so: fp32 rounding of up to n / 512 additions
    assert float((dw - dw2).norm() / dw.norm()) < (n / 512) * U + 34 * 2.0 ** -23


def test_calls_on_two_streams_at_once():
    b = B()
    work = [problem(700, 256, 3000, seed=k) for k in (20, 21)]

    def step(x, w, tok, dlogp, dent):
        logp, ent, lse = b.grpo_head_logp(x, w, tok)
        return (logp, ent, lse) + b.grpo_head_logp_bwd(x, w, tok, lse, ent, dlogp, dent, chunk_rows=300)
    want = [step(*q) for q in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = []
        for s, q in zip(streams, work):
            with torch.cuda.stream(s):
                got.append(step(*q))
        torch.cuda.synchronize()
        for p, q in zip(got, want):
            assert all(torch.equal(u, v) for u, v in zip(p, q))


def test_calls_back_to_back_in_one_workspace():
    """Inputs written on the device right before each call, one workspace for all calls, nothing waited for in between: the
    kernels of a call overlap their launches, so each has to wait for what it reads and for what it overwrites."""
    b = B()
    n, d, vocab = 1500, 128, 2011
    problems = [problem(n, d, vocab, seed=k) for k in (30, 31, 32)]
    need = max(b.grpo_head_logp_bwd_workspace_bytes(n, d, vocab, 700), b.grpo_embed_workspace_bytes(n, vocab, d),
               b.grpo_head_logp_workspace_bytes(n, d, vocab)) + 256
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    x, w, tok, dlogp, dent = (torch.empty_like(t) for t in problems[0])

    def step(p, ws):
        for dst, src in zip((x, w, tok, dlogp, dent), p):
            dst.copy_(src)
        logp, ent, lse = b.grpo_head_logp(x, w, tok, workspace=ws)
        dx, dw = b.grpo_head_logp_bwd(x, w, tok, lse, ent, dlogp, dent, chunk_rows=700, workspace=ws)
        grad = b.grpo_embed_bwd(dx, tok, vocab, workspace=ws)
        _, only = b.grpo_head_logp_bwd(x, w, tok, lse, ent, dlogp, dent, chunk_rows=700, workspace=ws, want_dx=False)
        dx2, _ = b.grpo_head_logp_bwd(x, w, tok, lse, ent, dlogp, dent, chunk_rows=400, workspace=ws, want_dw=False)
        return logp, ent, lse, dx, dw, grad, only, dx2
    want = []
    for p in problems:
        want.append([t.clone() for t in step(p, None)])
        torch.cuda.synchronize()
    got = [step(problems[i % 3], ws) for i in range(24)]
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert all(torch.equal(u, v) for u, v in zip(g, want[i % 3])), i
