"""The vocabulary calls at the edges of what they own, on the GPU: workspaces of exactly the size asked for with other data
behind them, and chunks of rows on both sides of the sizes at which the plan of the sums changes."""
import numpy as np
import pytest
import torch

from oracle import vocab_oracle as vo

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
GUARD = 1 << 22


def B():
    from paper_2605_16154_b200 import binding
    return binding


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def host(t):
    return t.detach().double().cpu().numpy()


class Guarded:
    """A workspace of `need` bytes inside a larger buffer whose other bytes have to stay as they are."""

    def __init__(self, need):
        self.all = torch.full((need + 2 * GUARD + 256,), 0xA5, dtype=torch.uint8, device="cuda")
        at = -self.all.data_ptr() % 256 + GUARD
        self.lo, self.hi = at, at + need

    def view(self):
        return self.all[self.lo:self.hi]

    def intact(self):
        return bool((self.all[:self.lo] == 0xA5).all()) and bool((self.all[self.hi:] == 0xA5).all())


def late_tokens(n, vocab, seed):
    """Few tokens, often, at the end of the vocabulary (action tokens of a language policy); some rows are padded."""
    g = gen(seed)
    tok = vocab - 1 - (torch.rand(n, generator=g, device="cuda") ** 3 * min(vocab, 60)).int()
    tok[torch.rand(n, generator=g, device="cuda") < 0.05] = -1
    return tok.clamp_(-1, vocab - 1)


def check_dw(dw, x, w, tok, dlogp):
    """Against fp64, by the norm: remainder of d z at most 2^-16 of it, exponents a few 2^-20, pieces of 34 truncations of 2^-23
    at most, the targets' sums k additions of 2^-24 on average far below their bound."""
    xd, wd, t = x.double(), w.double(), tok.long()
    live = t >= 0
    xd = torch.where(live[:, None], xd, 0.0)
    p = torch.softmax(xd @ wd.t(), -1)
    dz = -p * torch.where(live, dlogp.double(), 0.0)[:, None]
    dz[live.nonzero()[:, 0], t[live]] += dlogp.double()[live]
    want = dz.t() @ xd
    assert float((dw.double() - want).norm()) <= 2e-5 * float(want.norm())


@pytest.mark.parametrize("n,d,vocab,chunk", [(12000, 64, 900, 10000), (18471, 64, 900, 9472), (18000, 128, 2003, 9500), (20000, 64, 700, 9471)])
def test_head_gradient_of_a_shorter_last_chunk(n, d, vocab, chunk):
    b = B()
    g = gen(n + chunk)
    x = torch.randn(n, d, generator=g, device="cuda").bfloat16()
    w = (torch.randn(vocab, d, generator=g, device="cuda") * (2.0 / d ** 0.5)).bfloat16()
    tok, dlogp = late_tokens(n, vocab, n), torch.randn(n, generator=g, device="cuda")
    _, entropy, lse = b.grpo_head_logp(x, w, tok)
    ws = Guarded(b.grpo_head_logp_bwd_workspace_bytes(n, d, vocab, chunk))
    dx, dw = b.grpo_head_logp_bwd(x, w, tok, lse, entropy, dlogp, chunk_rows=chunk, workspace=ws.view())
    torch.cuda.synchronize()
    assert ws.intact()
    check_dw(dw, x, w, tok, dlogp)
    dx1, dw1 = b.grpo_head_logp_bwd(x, w, tok, lse, entropy, dlogp, chunk_rows=n)
    # other pieces of the contraction and of the tokens' sums: fp32 rounding of up to n / 512 pieces; dx may round to the
    # neighbouring bf16 value, 2^-7 of it
    assert float((dw - dw1).norm() / dw1.norm()) < (n / 512) * U + 34 * 2.0 ** -23
    assert float((dx.float() - dx1.float()).norm() / dx1.float().norm()) < 2.0 ** -7


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 5, 2049, 9471, 9472, 9473, 30000, 262144, 262145])
def test_embedding_gradient_stays_in_its_workspace(kind, n):
    b, vocab, d = B(), 3001, 16
    dout, tok = torch.randn(n, d, generator=gen(n), device="cuda").to(kind), late_tokens(n, vocab, n + 1)
    ws = Guarded(b.grpo_embed_workspace_bytes(n, vocab, d))
    grad = b.grpo_embed_bwd(dout, tok, vocab, workspace=ws.view())
    torch.cuda.synchronize()
    assert ws.intact()
    t = tok.cpu().numpy()
    want, mass = vo.embed_bwd(host(dout), t, vocab), vo.embed_bwd(np.abs(host(dout)), t, vocab)
    k = np.bincount(t[t >= 0].astype(np.int64), minlength=vocab)[:, None]
    assert np.all(np.abs(host(grad) - want) <= (k + 2) * U * mass + 2 * U * np.abs(want))
    # the workspace of the longest batch serves this one
    big = Guarded(b.grpo_embed_workspace_bytes(262145, vocab, d))
    assert torch.equal(b.grpo_embed_bwd(dout, tok, vocab, workspace=big.view()), grad)
    torch.cuda.synchronize()
    assert big.intact()


@pytest.mark.parametrize("n,vocab", [(1, 50001), (16, 40000), (128, 3000), (129, 3000), (700, 5003), (1025, 257)])
def test_head_log_probabilities_stay_in_their_workspace(n, vocab):
    b, d = B(), 64
    g = gen(n + vocab)
    x, w = torch.randn(n, d, generator=g, device="cuda").bfloat16(), (torch.randn(vocab, d, generator=g, device="cuda") * 0.2).bfloat16()
    tok = late_tokens(n, vocab, n)
    ws = Guarded(b.grpo_head_logp_workspace_bytes(n, d, vocab))
    got = b.grpo_head_logp(x, w, tok, workspace=ws.view())
    torch.cuda.synchronize()
    assert ws.intact()
    assert all(torch.equal(p, q) for p, q in zip(got, b.grpo_head_logp(x, w, tok)))


@pytest.mark.parametrize("kind,ints", [(torch.float32, torch.int32), (torch.bfloat16, torch.int16)])
@pytest.mark.parametrize("d,gap", [(64, 0), (2056, 8), (37, 0)])
def test_embedding_with_scale_one_copies_bits(kind, ints, d, gap):
    """Every bit pattern of the type arrives as it is: NaNs with their payloads and signs, infinities, -0, subnormals."""
    vocab = 70
    bits = torch.randint(torch.iinfo(ints).min, torch.iinfo(ints).max, (vocab, d + gap), generator=gen(d), device="cuda", dtype=torch.int64).to(ints)
    special = {torch.int32: [0x7F800001, -0x3FFFFF, 0x7FC12345, -0x800000, -(1 << 31), 1], torch.int16: [0x7F81, -0x3F, 0x7FC9, -0x80, -(1 << 15), 1]}[ints]
    bits[:, :6] = torch.tensor(special, dtype=torch.int64, device="cuda").to(ints)
    table = bits.view(kind)[:, :d]
    tok = torch.randint(-1, vocab, (200,), generator=gen(d + 1), device="cuda", dtype=torch.int32)
    out = B().grpo_embed(table, tok).view(ints)
    want = torch.where((tok >= 0)[:, None], bits[:, :d][tok.clamp(min=0).long()], 0)
    assert torch.equal(out, want)


def test_sizes_beyond_32_bits_are_refused():
    """2^32 + k rows or tokens would arrive as k."""
    b, far = B(), (1 << 32) + 3
    few = torch.zeros(4, dtype=torch.int32, device="cuda")
    m = torch.zeros(4, 8, device="cuda")
    x, w, v = m.bfloat16(), torch.zeros(20, 8, device="cuda").bfloat16(), torch.zeros(4, device="cuda")
    long = torch.empty(far, 1, dtype=torch.bfloat16, device="cuda")             # nothing reads or writes these
    many = torch.empty(far, dtype=torch.int32, device="cuda")
    for f in (lambda: b.grpo_embed_bwd(m, few, far), lambda: b.grpo_embed(long, few), lambda: b.grpo_embed(m, many, out=m),
              lambda: b.grpo_token_logp(long, many), lambda: b.grpo_token_logp(long.t(), few[:1]), lambda: b.grpo_token_logp(m, few, top=(1 << 32) + 2),
              lambda: b.grpo_head_logp_bwd(x, w, few, v, v, v, chunk_rows=far)):
        with pytest.raises(b.PcmError) as e:
            f()
        assert e.value.code == -2


# ---- captured calls at sizes beyond the short kernels --------------------------------------------------------------------
def replays_follow(step, refill):
    """Captures step(), then replays it twice on refilled inputs; the results are those of the same calls made directly."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in (1, 2):
        refill(seed)
        graph.replay()
        torch.cuda.synchronize()
        for p, q in zip(held, step()):
            assert torch.equal(p, q)


@pytest.mark.parametrize("n,vocab,d", [(3000, 70001, 40), (9472, 300, 16), (20011, 1000, 136)])
def test_captured_embedding_gradients_of_long_batches(n, vocab, d):
    """The radix sort of two and three passes, tokens over many tiles."""
    b = B()
    dout, tok = torch.randn(n, d, generator=gen(n), device="cuda"), late_tokens(n, vocab, n)
    grad = torch.zeros(vocab, d, device="cuda")

    def step():
        grad.fill_(0.5)
        return b.grpo_embed_bwd(dout, tok, vocab, 0.7), b.grpo_embed_bwd(dout, tok, vocab, grad=grad, accumulate=True).clone()

    def refill(seed):
        dout.copy_(torch.randn(n, d, generator=gen(seed), device="cuda"))
        tok.copy_(torch.randint(-1, vocab, (n,), generator=gen(seed), device="cuda", dtype=torch.int32))
    replays_follow(step, refill)


def test_captured_head_gradients_in_chunks_on_both_sides_of_the_plans():
    b, n, d, vocab = B(), 12000, 64, 700
    x, w = torch.randn(n, d, generator=gen(1), device="cuda").bfloat16(), (torch.randn(vocab, d, generator=gen(2), device="cuda") * 0.2).bfloat16()
    tok, a = late_tokens(n, vocab, 5), torch.randn(n, generator=gen(3), device="cuda")

    def step():
        logp, ent, lse = b.grpo_head_logp(x, w, tok)
        return (logp, ent, lse) + b.grpo_head_logp_bwd(x, w, tok, lse, ent, a, a, chunk_rows=9500) + \
            b.grpo_head_logp_bwd(x, w, tok, lse, ent, a, None, chunk_rows=2500, exact_dx=True)

    def refill(seed):
        x.copy_(torch.randn(n, d, generator=gen(seed), device="cuda"))
        tok.copy_(late_tokens(n, vocab, seed + 40))
    replays_follow(step, refill)


def test_captured_log_probabilities_of_many_and_of_few_rows():
    b = B()
    many, few = torch.randn(1300, 3001, generator=gen(1), device="cuda").bfloat16(), torch.randn(3, 50001, generator=gen(2), device="cuda")
    t1, t2 = late_tokens(1300, 3001, 3), torch.tensor([5, 50000, -1], dtype=torch.int32, device="cuda")

    def step():
        return b.grpo_token_logp(many, t1, 0.8, 5) + b.grpo_token_logp(few, t2, 1.3, 16)

    def refill(seed):
        many.copy_(torch.randn(1300, 3001, generator=gen(seed), device="cuda"))
        few.copy_(torch.randn(3, 50001, generator=gen(seed + 9), device="cuda"))
    replays_follow(step, refill)


# ---- outputs inside larger buffers: what lies around and between their rows stays ----------------------------------------
def inside(shape, dtype, shift, gap=0, fill=55):
    """An output of `shape` (rows `gap` elements apart) starting `shift` elements into a buffer of `fill`, and a check that only
    the output was written."""
    rows, cols = (1, shape[0]) if len(shape) == 1 else shape
    ld = cols + gap
    buf = torch.full((shift + rows * ld + 64,), fill, dtype=dtype, device="cuda")
    view = buf[shift:shift + rows * ld].view(rows, ld)[:, :cols]

    def only():
        left = torch.ones_like(buf, dtype=torch.bool)
        left[shift:shift + rows * ld].view(rows, ld)[:, :cols] = False
        return bool((buf[left] == fill).all())
    return (view[0] if len(shape) == 1 else view), only


@pytest.mark.parametrize("n,vocab,d,shift", [(50, 33, 24, 1), (3000, 300, 40, 3), (700, 9, 129, 2), (12000, 77, 16, 4)])
def test_embedding_gradient_writes_its_table_only(n, vocab, d, shift):
    b = B()
    dout, tok = torch.randn(n, d, generator=gen(n), device="cuda").bfloat16(), late_tokens(n, vocab, n)
    flat, only = inside((vocab * d,), torch.float32, shift)
    b.grpo_embed_bwd(dout, tok, vocab, 0.5, grad=flat.view(vocab, d))
    assert only()
    t = tok.cpu().numpy()
    want, mass = vo.embed_bwd(host(dout), t, vocab, 0.5), vo.embed_bwd(np.abs(host(dout)), t, vocab, 0.5)
    k = np.bincount(t[t >= 0].astype(np.int64), minlength=vocab)[:, None]
    assert np.all(np.abs(host(flat.view(vocab, d)) - want) <= (k + 2) * U * mass + 2 * U * np.abs(want))


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,vocab,gap,shift", [(3, 50, 3, 1), (9, 1500, 1, 2), (1300, 1100, 0, 5), (2, 40003, 5, 7)])
def test_log_probabilities_write_their_outputs_only(kind, n, vocab, gap, shift):
    b, top = B(), 5
    z, tok = torch.randn(n, vocab, generator=gen(n), device="cuda").to(kind), late_tokens(n, vocab, vocab)
    want = b.grpo_token_logp(z, tok, 1.0, top)
    made = {k: inside((n,), torch.float32, shift) for k in ("logp", "entropy", "lse")}
    made["top_id"], made["top_logp"] = inside((n * top,), torch.int32, shift), inside((n * top,), torch.float32, shift)
    b.grpo_token_logp(z, tok, 1.0, top, out={k: v[0] for k, v in made.items()})
    for (t, only), w in zip(made.values(), want):
        assert only() and torch.equal(t, w.reshape(-1))
    a = torch.randn(n, generator=gen(3), device="cuda")
    near = b.grpo_token_logp_bwd(z, tok, want[2], want[1], a, a)
    out, only = inside((n, vocab), kind, shift, gap)
    b.grpo_token_logp_bwd(z, tok, want[2], want[1], a, a, dlogits=out)
    assert only() and torch.equal(out, near)


@pytest.mark.parametrize("n,d,vocab", [(3, 64, 77), (300, 72, 515), (700, 256, 40)])
def test_head_gradients_write_their_outputs_only(n, d, vocab):
    b = B()
    x, w = torch.randn(n, d, generator=gen(n), device="cuda").bfloat16(), (torch.randn(vocab, d, generator=gen(d), device="cuda") * 0.2).bfloat16()
    tok, a = late_tokens(n, vocab, n), torch.randn(n, generator=gen(1), device="cuda")
    got = {k: inside((n,), torch.float32, 3) for k in ("logp", "entropy", "lse")}
    logp, ent, lse = b.grpo_head_logp(x, w, tok, out={k: v[0] for k, v in got.items()})
    assert all(only() for _, only in got.values())
    for exact in (False, True):
        dx, dw = b.grpo_head_logp_bwd(x, w, tok, lse, ent, a, a, exact_dx=exact)
        dx1, only_dx = inside((n, d), torch.bfloat16, 8, 16)
        dw1, only_dw = inside((vocab * d,), torch.float32, 4)
        b.grpo_head_logp_bwd(x, w, tok, lse, ent, a, a, dx=dx1, dw=dw1.view(vocab, d), exact_dx=exact)
        assert only_dx() and only_dw() and torch.equal(dx1, dx) and torch.equal(dw1.view(vocab, d), dw)
