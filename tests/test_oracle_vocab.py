"""Pins of the fp64 vocabulary oracle: closed forms, a library model with autograd, central differences."""
import numpy as np
import pytest
import torch

from oracle import vocab_oracle as vo


def test_uniform_rows_have_closed_forms():
    z = np.full((2, 50), 3.5)
    out = vo.token_logp(z, [7, -1], temperature=0.5, top=3)
    assert out["logp"][0] == pytest.approx(-np.log(50), abs=1e-14) and out["entropy"][0] == pytest.approx(np.log(50), abs=1e-14)
    assert out["lse"][0] == pytest.approx(7.0 + np.log(50), abs=1e-13)
    assert list(out["top_id"][0]) == [0, 1, 2] and list(out["top_id"][1]) == [-1, -1, -1] and out["lse"][1] == 0.0


def test_large_equal_logits_keep_their_entropy():
    out = vo.token_logp(np.full((1, 13), -3.4e38), [4], temperature=0.9, top=1)
    assert out["entropy"][0] == pytest.approx(np.log(13), abs=1e-14) and out["logp"][0] == pytest.approx(-np.log(13), abs=1e-14)


def test_masked_rows():
    z = np.array([[-np.inf, 2.0, -np.inf, 2.0], [-np.inf] * 4])
    out = vo.token_logp(z, [1, 2], top=4)
    assert out["logp"][0] == pytest.approx(-np.log(2)) and out["entropy"][0] == pytest.approx(np.log(2))
    assert list(out["top_id"][0]) == [1, 3, 0, 2] and out["top_logp"][0][2] == -np.inf
    assert out["logp"][1] == -np.inf and out["entropy"][1] == 0.0
    g = vo.token_logp_bwd(z, [1, 2], [1.0, 1.0], [0.3, 0.3])
    assert np.allclose(g[0], [0, 0.5, 0, -0.5]) and not g[1].any()


def test_top_order_of_nan_infinities_and_zeros():
    assert vo.top_ids([0.0, -0.0, np.nan, np.inf, -np.inf, 0.0], 6) == [2, 3, 0, 1, 5, 4]


def test_logp_and_gradient_against_autograd():
    rng = np.random.default_rng(3)
    n, v, d, T = 6, 37, 11, 1.7
    x, w = rng.normal(size=(n, d)), rng.normal(size=(v, d))
    tok = rng.integers(0, v, n)
    g, h = rng.normal(size=n), rng.normal(size=n)
    xt, wt = torch.tensor(x, requires_grad=True), torch.tensor(w, requires_grad=True)
    z = xt @ wt.T
    z.retain_grad()
    lp = torch.log_softmax(z / T, -1)
    logp = lp[torch.arange(n), torch.tensor(tok)]
    ent = -(lp.exp() * lp).sum(-1)
    (logp * torch.tensor(g) + ent * torch.tensor(h)).sum().backward()
    out = vo.head_logp(x, w, tok, T)
    assert np.allclose(out["logp"], logp.detach().numpy(), atol=1e-12) and np.allclose(out["entropy"], ent.detach().numpy(), atol=1e-12)
    assert np.allclose(vo.token_logp_bwd(x @ w.T, tok, g, h, T), z.grad.numpy(), atol=1e-12)
    dx, dw = vo.head_logp_bwd(x, w, tok, g, h, T)
    assert np.allclose(dx, xt.grad.numpy(), atol=1e-12) and np.allclose(dw, wt.grad.numpy(), atol=1e-12)


def test_gradient_against_central_differences():
    rng = np.random.default_rng(4)
    z, tok, g, h, T = rng.normal(size=(3, 9)) * 2, np.array([2, -1, 8]), rng.normal(size=3), rng.normal(size=3), 0.6
    f = lambda q: float((vo.token_logp(q, tok, T)["logp"] * g + vo.token_logp(q, tok, T)["entropy"] * h).sum())
    num = np.zeros_like(z)
    for i in range(3):
        for j in range(9):
            a, b = z.copy(), z.copy()
            a[i, j] += 1e-5
            b[i, j] -= 1e-5
            num[i, j] = (f(a) - f(b)) / 2e-5
    assert np.allclose(num, vo.token_logp_bwd(z, tok, g, h, T), atol=1e-8)


def test_embedding_and_its_gradient_are_adjoint():
    rng = np.random.default_rng(5)
    table, tok, dout = rng.normal(size=(13, 4)), np.array([3, 3, -1, 12, 0, 13, 3]), rng.normal(size=(7, 4))
    out = vo.embed(table, tok, 2.5)
    assert not out[2].any() and not out[5].any() and np.allclose(out[3], 2.5 * table[12])
    assert np.sum(out * dout) == pytest.approx(np.sum(table * vo.embed_bwd(dout, tok, 13, 2.5)), rel=1e-13)
