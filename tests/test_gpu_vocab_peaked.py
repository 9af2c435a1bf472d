"""Gradients of the head's log-probabilities under peaked policies, where the scored token need not carry the row's gradient.

dx by default takes d z rounded to bf16 (half a step, 2^-8 of each entry but the target's); with exact_dx, and for dw always, as
a sum of two bf16 values, 2^-16 of each.  Every bound is of each element: the rounding of d z, the error of d z itself (p times
that of its exponent), the products' truncations, the rounding of the result."""
import numpy as np
import pytest
import torch

from oracle import vocab_oracle as vo
from tests.test_gpu_vocab_head import B, U, gen, host, wide, z_error

pytestmark = pytest.mark.gpu


def policy(n, d, vocab, spread, scored, gap=0, temperature=1.0):
    g = gen(int(n + d + 10 * spread))
    x = wide(torch.randn(n, d, generator=g, device="cuda").bfloat16(), gap)
    w = wide((torch.randn(vocab, d, generator=g, device="cuda") * (spread / d ** 0.5)).bfloat16(), gap)
    z = x.double() @ w.double().t() / temperature
    if scored == "sampled":
        tok = torch.multinomial(torch.softmax(z, -1), 1, generator=g)[:, 0]
    else:
        tok = z.topk(min(2, vocab), -1).indices[:, {"mode": 0, "second": -1}[scored]]
    tok = tok.int()
    if n > 6:
        tok[3] = -1
        x[3] = float("nan")
    return x, w, tok, torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda") * 0.1


def bounds(x, w, tok, lse, entropy, dlogp, dent, temperature):
    """fp64 gradient of the logits, the bound of the kernel's error before any rounding to bf16, operands."""
    xf, wf, t = host(x), host(w), tok.cpu().numpy()
    live = (t >= 0)[:, None]
    xf[~live[:, 0]] = 0.0
    dz = vo.token_logp_bwd(xf @ wf.T, t, host(dlogp), host(dent), temperature)
    ze, rng = z_error(xf, wf, temperature)
    lse_h, ent_h = host(lse)[:, None], host(entropy)[:, None]
    lp = np.where(live, xf @ wf.T / temperature - lse_h, -np.inf)
    p = np.exp(lp)
    inner = np.abs(host(dlogp))[:, None] + np.abs(host(dent))[:, None] * (np.where(live, np.abs(lp), 0.0) + np.abs(ent_h) + 1)
    rel = (2 * ze + 8 * U * (rng + np.abs(lse_h[:, 0]) + 4) + 2.0 ** -20)[:, None]
    at = np.arange(w.shape[0])[None] == t[:, None]
    # the target's entry is a difference, g - g p: its error is that of g p, and the rounding of the larger of both
    edz = rel * p * inner / temperature + 2 * U * (np.abs(dz) + np.where(at, inner / temperature, 0.0))
    return dz, edz, np.where(at, 0.0, np.abs(dz)), xf, wf


CASES = [(701, 256, 1003, 4, "sampled", 0, 1.0), (300, 128, 2003, 8, "second", 0, 1.0), (300, 128, 2003, 8, "mode", 8, 1.0),
         (40, 64, 5003, 8, "sampled", 0, 0.7), (1, 64, 300, 6, "second", 0, 1.0), (7, 1032, 515, 12, "sampled", 8, 1.3),
         (130, 200, 40, 6, "second", 0, 1.0), (129, 64, 1, 2, "mode", 0, 1.0), (64, 520, 4000, 20, "second", 0, 1.0)]


@pytest.mark.parametrize("n,d,vocab,spread,scored,gap,temperature", CASES)
def test_gradients_of_a_peaked_policy(n, d, vocab, spread, scored, gap, temperature):
    b = B()
    x, w, tok, dlogp, dent = policy(n, d, vocab, spread, scored, gap, temperature)
    _, entropy, lse = b.grpo_head_logp(x, w, tok, temperature)
    dz, edz, rest, xf, wf = bounds(x, w, tok, lse, entropy, dlogp, dent, temperature)
    want = dz @ wf
    mass = np.abs(dz) @ np.abs(wf)
    for exact, cut, adds in ((False, 2.0 ** -8, vocab / 16), (True, 2.0 ** -16, vocab / 8)):
        dx, dw = b.grpo_head_logp_bwd(x, w, tok, lse, entropy, dlogp, dent, temperature, exact_dx=exact)
        # the target's part enters as a product and one addition in fp32
        tol = (edz * (1 + cut)) @ np.abs(wf) + cut * (rest @ np.abs(wf)) + ((adds + 8) * 2.0 ** -23 + 2.0 ** -16) * mass
        if not exact:
            tol = tol + 2.0 ** -8 * 2.0 ** -8 * mass
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol) + 2.0 ** -133
        assert np.all(np.abs(host(dx) - want) <= tol), (exact, np.max(np.abs(host(dx) - want) / tol))
        alone, none = b.grpo_head_logp_bwd(x, w, tok, lse, entropy, dlogp, dent, temperature, want_dw=False, exact_dx=exact)
        assert none is None and torch.equal(alone, dx)
        again, _ = b.grpo_head_logp_bwd(x, w, tok, lse, entropy, dlogp, dent, temperature, exact_dx=exact, chunk_rows=max(1, n // 3))
        assert np.all(np.abs(host(again) - want) <= tol)
        if n > 6:
            assert not dx[3].any()
        wtol = edz.T @ np.abs(xf) + (2.0 ** -16 + 34 * 2.0 ** -23 + 2 * (n / 256 + 4) * U) * (np.abs(dz).T @ np.abs(xf)) + (n + 4) * U * ((np.abs(dz) - rest).T @ np.abs(xf))
        assert np.all(np.abs(host(dw) - dz.T @ xf) <= wtol + 1e-37)


def test_exact_dx_carries_no_rounding_but_its_own():
    """Rounded to bf16, the exact gradient is off by its own rounding; exact_dx by that and by what a value within 2^-15 of the
    exact one can move over a rounding border: for errors e and steps s, sqrt(sum e s), at most sqrt(2^-15 2^-7) of the norm and
    typically a tenth.  The default adds half a step of every other entry, at most another 2^-8."""
    b = B()
    x, w, tok, dlogp, dent = policy(700, 512, 3001, 8, "second")
    _, entropy, lse = b.grpo_head_logp(x, w, tok)
    dz, *_, xf, wf = bounds(x, w, tok, lse, entropy, dlogp, dent, 1.0)
    want = dz @ wf
    norm = np.linalg.norm(want)
    own = np.linalg.norm(host(torch.from_numpy(want).float().bfloat16()) - want) / norm
    err = {e: np.linalg.norm(host(b.grpo_head_logp_bwd(x, w, tok, lse, entropy, dlogp, dent, want_dw=False, exact_dx=e)[0]) - want) / norm for e in (False, True)}
    assert err[True] <= own + 2.0 ** -11 * 0.25 and err[False] <= own + 2.0 ** -8


def test_exact_dx_alone_or_accumulating_changes_no_weight_gradient():
    b = B()
    x, w, tok, dlogp, dent = policy(300, 64, 500, 4, "sampled")
    _, entropy, lse = b.grpo_head_logp(x, w, tok)
    _, dw = b.grpo_head_logp_bwd(x, w, tok, lse, entropy, dlogp, dent)
    dx, dw2 = b.grpo_head_logp_bwd(x, w, tok, lse, entropy, dlogp, dent, exact_dx=True, dw=torch.zeros_like(dw), accumulate=True)
    assert torch.equal(dw, dw2)
    none, dw3 = b.grpo_head_logp_bwd(x, w, tok, lse, entropy, dlogp, dent, exact_dx=True, want_dx=False)
    assert none is None and torch.equal(dw, dw3)
