"""Rotary positions, the paged cache and attention over it on the GPU against the fp64 oracle.

Tolerances, derived before the first run.  u = 2^-24 is half an fp32 step, e half a step of the output's type.
  rotary     sine and cosine of an angle that is right to 2^-22 turns carry 2 u each and the angle's rounding to fp32, pi 2^-24
             of it at most, so 8 u in all with their factor; two products and a sum: 3 u; the result is rounded once:
             12 u amplitude (|a| + |b|) + e |out|.
  scores     dim products and sums in fp32 and the factor: (dim + 4) u scale sum |q k| =: d absolute; tensor cores do not round to
             nearest, which doubles it.
  weights    exp(z - m): d for z and for m, the argument's rounding |z - m| u <= 2 reach u, ex2 2^-22: w = 2 (2 d + 2 reach u + 2^-22),
             twice for the quotient.
  out        (w + n u) mass + r mass + e |out|, mass = sum p |v|, n keys; r = 2^-16 where weights are pairs of bf16 values, 2^-8 where they
             are rounded to bf16, 0 in fp32.
  lse        2 d + 2 reach u + 2^-22 + n u + |lse| u."""
import numpy as np
import pytest
import torch

from oracle import rollout_oracle as ro

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def B():
    from paper_2605_16154_b200 import binding
    return binding


def host(t):
    return t.detach().double().cpu().numpy()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def half_step(t):
    return torch.finfo(t).eps / 2


# ---- rotary -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,heads,dim,rot,gap", [(1, 1, 2, 2, 0), (1, 16, 128, 128, 0), (333, 3, 64, 32, 0), (57, 5, 96, 24, 8), (40, 2, 80, 6, 3),
                                                 (9001, 4, 64, 64, 0), (7, 1, 1024, 1024, 0), (5, 2, 64, 0, 0), (2500, 6, 33, 10, 1)])
def test_rotary_turns_each_pair_by_its_angle(kind, interleaved, n, heads, dim, rot, gap):
    t, g = TYPES[kind], gen(n + dim)
    base = torch.randn(n, heads, dim + gap, generator=g, device="cuda").to(t)
    x = base[..., :dim]
    pos = torch.randint(0, 1 << 30, (n,), generator=g, device="cuda", dtype=torch.int32)
    pos[0] = 2 ** 31 - 1
    pos[n // 2] = 0
    pos[-1] = -77
    if rot:
        turns, amplitude = B().grpo_rotary_freqs(rot, scaling=3, factor=8.0, original_len=4096.0)
    else:
        turns, amplitude = torch.empty(0, dtype=torch.float64), 1.0
    theta = host(turns) * 2 * np.pi
    # the angle as the definition has it: of the turns, whole ones left out in exact arithmetic
    part = np.array([[float((int(p) * int(round(float(f) * 2.0 ** 80))) % 2 ** 80) / 2.0 ** 80 for f in turns] for p in pos.tolist()]).reshape(n, -1)
    pair = lambda v: (v[..., 0:rot:2], v[..., 1:rot:2]) if interleaved else (v[..., :rot // 2], v[..., rot // 2:rot])
    for inverse in (False, True):
        out = B().grpo_rotary(x, pos, turns.cuda(), interleaved=interleaved, amplitude=amplitude, inverse=inverse)
        assert out.shape == x.shape and torch.equal(out[..., rot:], x[..., rot:])
        want = host(x).copy()
        a, b = (v.copy() for v in pair(want))
        c, s = np.cos(2 * np.pi * part)[:, None], np.sin(2 * np.pi * part)[:, None] * (-1 if inverse else 1)
        wa, wb = pair(want)
        wa[...], wb[...] = amplitude * (a * c - b * s), amplitude * (b * c + a * s)
        tol = np.zeros_like(want)
        ta, tb = pair(tol)
        ta[...] = tb[...] = 12 * U * amplitude * (np.abs(a) + np.abs(b)) + (2 * np.pi * 2.0 ** -22) * amplitude * (np.abs(a) + np.abs(b)) * (np.abs(host(pos))[:, None, None] > 2 ** 20)
        tol += half_step(t) * np.abs(want)
        assert np.all(np.abs(host(out) - want) <= tol)
        near = np.abs(host(pos)) < 2 ** 20
        if near.any():
            oracle = ro.rotary(host(x)[near], host(pos)[near], theta, interleaved, amplitude, inverse)
            assert np.allclose(oracle, want[near], rtol=0, atol=1e-8)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_in_place_and_back(kind, interleaved):
    t = TYPES[kind]
    x = torch.randn(300, 6, 64, generator=gen(3), device="cuda").to(t)
    buf = torch.full((300, 8, 64), 5.0, dtype=t, device="cuda")
    buf[:, 1:7] = x
    turns, _ = B().grpo_rotary_freqs(48)
    pos = torch.arange(300, device="cuda", dtype=torch.int32) * 1000
    want = B().grpo_rotary(x, pos, turns.cuda(), interleaved=interleaved)
    view = buf[:, 1:7]
    assert B().grpo_rotary(view, pos, turns.cuda(), interleaved=interleaved, out=view) is view
    assert torch.equal(view, want) and bool((buf[:, 0] == 5).all()) and bool((buf[:, 7] == 5).all())
    back = B().grpo_rotary(want, pos, turns.cuda(), interleaved=interleaved, inverse=True)
    # two rotations, each off by 12 u (|a| + |b|) and a rounding
    assert float((back.double() - x.double()).abs().max()) <= (2 * half_step(t) + 24 * U) * 2 * float(x.double().abs().max())


def test_rotary_gradient_against_differences_and_the_formula():
    """d <w, R x> / d x = R^T w: along random directions, and exactly in fp64 through the oracle."""
    g = gen(11)
    x, w, e = (torch.randn(29, 3, 64, generator=g, device="cuda") for _ in range(3))
    pos = torch.randint(0, 5000, (29,), generator=g, device="cuda", dtype=torch.int32)
    turns, amp = B().grpo_rotary_freqs(32, scaling=3, factor=4.0, original_len=512.0)
    f = lambda v: float((B().grpo_rotary(v, pos, turns.cuda(), amplitude=amp).double() * w.double()).sum())
    dx = B().grpo_rotary(w, pos, turns.cuda(), amplitude=amp, inverse=True)
    h = 0.25                                                        # the function is linear: no error of the difference itself
    slope = (f(x + h * e) - f(x - h * e)) / (2 * h)
    assert abs(slope - float((dx.double() * e.double()).sum())) < 1e-3
    theta, a = ro.frequencies(32, scaling=3, factor=4.0, original_len=512.0)
    assert np.abs(host(dx) - ro.rotary(host(w), host(pos), theta, False, a, True)).max() < 40 * U * 8


# ---- a cache with sequences -------------------------------------------------------------------------------------
class Case:
    """Pages in random order, a table with entries that nothing may follow where no token is, stale values in every slot."""

    def __init__(self, seed, kind, dim, kv, group, page, lens, new, heads_first=False, spare_rows=0, gap=0, stale=float("nan")):
        g = gen(seed)
        self.t, self.kv, self.heads, self.dim, self.page = TYPES[kind], kv, kv * group, dim, page
        n_pages = [-(-x // page) for x in lens]
        total, most = sum(n_pages) + 2, max(n_pages + [1]) + 1
        order = torch.randperm(total, generator=g, device="cuda").cpu()
        self.table_host = np.full((len(lens), most), -1234567, dtype=np.int32)
        used = 0
        for s, a in enumerate(n_pages):
            self.table_host[s, :a] = order[used:used + a].numpy()
            used += a
        self.table = torch.from_numpy(self.table_host).cuda()
        shape = (total, kv, page, dim + gap) if heads_first else (total, page, kv, dim + gap)
        pages = [torch.full(shape, stale, dtype=self.t, device="cuda") for _ in range(2)]
        self.k_pages, self.v_pages = ((p.transpose(1, 2) if heads_first else p)[..., :dim] for p in pages)
        for s, length in enumerate(lens):
            j = np.arange(length)
            at = torch.from_numpy(self.table_host[s][j // page].astype(np.int64)).cuda(), torch.from_numpy(j % page).cuda()
            for p in (self.k_pages, self.v_pages):
                p[at] = torch.randn(length, kv, dim, generator=g, device="cuda").to(self.t)
        self.lens, self.new = list(lens), list(new)
        self.n = sum(new) + spare_rows
        self.seq_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.q_off_host = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.q_off = torch.from_numpy(self.q_off_host).cuda()
        self.q = (torch.randn(self.n, self.heads, dim, generator=g, device="cuda") * 2).to(self.t)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def run(self, window=0, sinks=0, scale=None, **more):
        out = torch.full((self.n, self.heads, self.dim), 7.0, dtype=self.t, device="cuda")
        lse = torch.full((self.n, self.heads), 7.0, device="cuda")
        args = dict(window=window, sinks=sinks, scale=scale, max_new=max(self.new), out=out, lse=lse, status=self.status)
        args.update(more)
        return B().grpo_paged_attention(self.q, self.k_pages, self.v_pages, self.table, self.seq_len, self.q_off, **args)

    def check(self, out, lse, window=0, sinks=0, scale=None, rounded=True, status=0):
        scale = self.dim ** -0.5 if scale is None else scale
        want, wlse, mass, reach = ro.attend(host(self.q), host(self.k_pages), host(self.v_pages), self.table_host, self.lens, self.q_off_host,
                                            scale, window, sinks)
        used = int(self.q_off_host[-1])
        assert bool((out[used:] == 7.0).all()) and bool((lse[used:] == 7.0).all())
        want, wlse, mass, reach = want[:used], wlse[:used], mass[:used], reach[:used]
        n = max(self.lens + [1])
        d = 2 * (self.dim + 4) * U * reach
        w = 2 * (2 * d + 2 * reach * U + 2.0 ** -22)
        r = 0.0 if self.t == torch.float32 else 2.0 ** -8 if rounded else 2.0 ** -16
        tol = (w + n * U + r)[..., None] * mass + half_step(self.t) * np.abs(want)
        o, ls = host(out[:used]), host(lse[:used])
        assert np.all(np.isfinite(o)) and np.all(np.abs(o - want) <= tol), float((np.abs(o - want) / np.maximum(tol, 1e-30)).max())
        none = np.isneginf(wlse)
        assert np.array_equal(none, np.isneginf(ls)) and np.all(o[none] == 0)
        tol = 2 * d + 2 * reach * U + 2.0 ** -22 + n * U + np.abs(np.where(none, 0, wlse)) * U
        assert np.all(np.abs(np.where(none, 0, ls) - np.where(none, 0, wlse)) <= tol)
        assert int(self.status) == status


SHAPES = [
    # dim, kv, group, page, lengths, new, heads first, spare rows, gap
    (64, 2, 1, 16, [1], [1], False, 0, 0),
    (64, 4, 4, 16, [312, 1, 17, 0, 64, 65], [1, 1, 1, 1, 1, 1], False, 0, 0),
    (128, 2, 8, 8, [700, 129, 128, 127], [1, 1, 1, 1], True, 3, 0),
    (32, 3, 5, 24, [40, 333, 8], [1, 3, 8], False, 1, 8),
    (128, 1, 1, 48, [1000, 50], [7, 0], False, 0, 0),
    (64, 2, 3, 16, [130, 700, 5, 0, 257], [130, 33, 9, 2, 1], False, 2, 0),
    (128, 2, 2, 32, [513, 256, 90], [300, 256, 1], True, 0, 0),
    (32, 1, 2, 64, [700, 64], [129, 64], False, 0, 0),
    (64, 1, 7, 128, [1500, 40], [90, 40], False, 0, 0),
    (128, 1, 16, 256, [300, 2200], [20, 3], False, 0, 8),
]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (50, 4), (200, 130), (100000, 3)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"d{s[0]}kv{s[1]}g{s[2]}p{s[3]}")
def test_attention_over_the_cache(kind, window, sinks, shape):
    dim, kv, group, page, lens, new, hf, spare, gap = shape
    c = Case(dim + page, kind, dim, kv, group, page, lens, new, hf, spare, gap)
    c.check(*c.run(window, sinks), window, sinks)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_one_new_token_each_without_offsets(kind):
    c = Case(5, kind, 64, 2, 4, 16, [70, 1, 0, 513, 33], [1] * 5)
    out, lse = c.run(max_new=0)
    q_off, c.q_off = c.q_off, None
    again, lse2 = c.run(max_new=0)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    c.q_off = q_off
    c.check(out, lse)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("dim,kv,group,new", [(128, 2, 4, 1), (64, 1, 2, 3), (32, 2, 1, 1), (64, 2, 2, 40), (128, 1, 1, 300)])
def test_long_histories_are_cut_and_joined(kind, dim, kv, group, new):
    c = Case(9, kind, dim, kv, group, 16, [30011, 200, 7001], [new, 1, new])
    c.check(*c.run())


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("new", [3, 200])
def test_values_that_a_row_does_not_see_do_not_reach_it(kind, new):
    """NaN and infinities at the positions of later tokens, and outside a window: earlier rows stay finite; a row that sees
    one takes it over."""
    c = Case(21, kind, 64, 2, 2, 16, [new + 500], [new])
    clean, lse = c.run()
    page, slot = c.table_host[0][(new + 499) // 16], (new + 499) % 16                 # the last token's slot
    c.v_pages[page, slot, :, ::2] = float("nan")
    c.v_pages[page, slot, :, 1::2] = float("inf")
    out, lse2 = c.run()
    tol = 0 if kind == "f32" else 2.0 ** -7
    assert bool(torch.isfinite(out[:-1]).all()) and torch.equal(lse, lse2)
    assert float((out[:-1].double() - clean[:-1].double()).abs().max()) <= tol * float(clean.double().abs().max()) + 1e-5
    assert bool(torch.isnan(out[-1, :, ::2]).all()) and bool(torch.isinf(out[-1, :, 1::2]).all())
    first = c.table_host[0][100 // 16], 100 % 16                                      # outside every row's window
    c.v_pages[page, slot] = 0
    c.k_pages[first] = float("nan")
    c.v_pages[first] = float("inf")
    out, lse = c.run(300 if new == 3 else 250, 2)
    c.check(out, lse, 300 if new == 3 else 250, 2)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("new", [2, 130])
def test_scores_that_are_infinite_or_nan_stay_in_their_rows(kind, new):
    c = Case(23, kind, 64, 1, 2, 16, [new + 100], [new])
    clean, _ = c.run()
    c.q[0, 0, 0] = float("nan")
    out, lse = c.run()
    assert bool(torch.isnan(out[0, 0]).all()) and bool(torch.isnan(lse[0, 0]))
    out[0, 0] = clean[0, 0]
    assert torch.equal(out, clean)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("new", [1, 150])
def test_large_and_small_scores(kind, new):
    c = Case(25, kind, 64, 2, 2, 16, [400], [new])
    for scale in (1e-6, 3.0):
        c.check(*c.run(scale=scale), scale=scale)


@pytest.mark.parametrize("new", [1, 100])
def test_bad_pages_lengths_and_offsets_are_reported_and_harm_no_other(new):
    c = Case(31, "bf16", 64, 2, 2, 16, [300, 400, 200], [new, new, new])
    clean, _ = c.run()
    c.table[1, 3] = 1 << 30
    c.table[1, 4] = -5
    out, _ = c.run()
    assert int(c.status) == 64 and torch.equal(out[:new], clean[:new]) and torch.equal(out[2 * new:], clean[2 * new:])
    c.table[1, 3:5] = torch.from_numpy(c.table_host[1, 3:5]).cuda()
    for bad_len in (-1, 1 << 30):
        c.status.zero_()
        c.seq_len[1] = bad_len
        if bad_len > 0:
            c.table[1] = 0                                         # the clipped length reaches every entry
        out, _ = c.run()
        assert int(c.status) == 128 and torch.equal(out[:new], clean[:new]) and torch.equal(out[2 * new:], clean[2 * new:])
    c.table.copy_(torch.from_numpy(c.table_host).cuda())
    c.seq_len[1] = 400
    for off in ([0, new, -4, 3 * new], [0, new, 1 << 30, 3 * new]):
        c.status.zero_()
        c.q_off.copy_(torch.tensor(off, dtype=torch.int32))
        out, _ = c.run()
        assert int(c.status) == 128 and torch.equal(out[:new], clean[:new])


# ---- new tokens enter the cache ------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", [SHAPES[1], SHAPES[3], SHAPES[5], SHAPES[6]], ids=lambda s: f"d{s[0]}kv{s[1]}g{s[2]}p{s[3]}")
def test_new_tokens_enter_the_cache(kind, interleaved, shape):
    dim, kv, group, page, lens, new, hf, spare, gap = shape
    c = Case(dim, kind, dim, kv, group, page, lens, new, hf, spare, gap, stale=3.0)
    g = gen(77)
    fused = torch.randn(c.n, c.heads + 2 * kv, dim, generator=g, device="cuda").to(c.t)
    q, k, v = fused[:, :c.heads], fused[:, c.heads:c.heads + kv], fused[:, c.heads + kv:]
    turns, amp = B().grpo_rotary_freqs(dim // 2, scaling=1, factor=2.0)
    q_out = torch.full((c.n, c.heads, dim), 7.0, dtype=c.t, device="cuda")
    before_k, before_v = c.k_pages.clone(), c.v_pages.clone()
    B().grpo_rotary_cache(q, k, v, c.k_pages, c.v_pages, c.table, c.seq_len, c.q_off, turns.cuda(), interleaved=interleaved, q_out=q_out,
                          status=c.status)
    used = int(c.q_off_host[-1])
    pos = np.zeros(used)
    for row, first, count in ro.sequences(lens, c.q_off_host, c.n):
        pos[row:row + count] = first + np.arange(count)
    pos_t = torch.from_numpy(pos.astype(np.int32)).cuda()
    turned = B().grpo_rotary(k[:used], pos_t, turns.cuda(), interleaved=interleaved)
    assert torch.equal(q_out[:used], B().grpo_rotary(q[:used], pos_t, turns.cuda(), interleaved=interleaved))
    assert bool((q_out[used:] == 7.0).all())
    wk, wv = ro.append(host(turned), host(v[:used]), host(before_k), host(before_v), c.table_host, lens, c.q_off_host)
    assert np.array_equal(host(c.k_pages), wk) and np.array_equal(host(c.v_pages), wv)
    assert int(c.status) == 0
    # positions of their own, the queries in place, and no queries at all
    c.k_pages.copy_(before_k)
    other = torch.randint(0, 9000, (c.n,), generator=g, device="cuda", dtype=torch.int32)
    want_q = B().grpo_rotary(q[:used], other[:used], turns.cuda(), interleaved=interleaved)
    spare_q = q[used:].clone()
    B().grpo_rotary_cache(q, k, v, c.k_pages, c.v_pages, c.table, c.seq_len, c.q_off, turns.cuda(), interleaved=interleaved, pos=other, q_out=q)
    assert torch.equal(q[:used], want_q) and torch.equal(q[used:], spare_q)
    with_q = c.k_pages.clone()
    c.k_pages.copy_(before_k)
    B().grpo_rotary_cache(None, k, v, c.k_pages, c.v_pages, c.table, c.seq_len, c.q_off, turns.cuda(), interleaved=interleaved, pos=other)
    assert torch.equal(c.k_pages, with_q)


def test_pages_outside_the_cache_are_not_written():
    c = Case(41, "bf16", 64, 2, 1, 16, [40, 60], [10, 10], stale=3.0)
    k = torch.randn(20, 2, 64, device="cuda").bfloat16()
    c.table[0, 2] = c.k_pages.shape[0]
    before = c.k_pages.clone()
    B().grpo_rotary_cache(None, k, k, c.k_pages, c.v_pages, c.table, c.seq_len, c.q_off, None, status=c.status)
    assert int(c.status) == 64
    changed = (c.k_pages != before).flatten(1).any(1).nonzero().flatten().tolist()
    assert set(changed) <= {int(c.table_host[0][1]), int(c.table_host[1][3])}


# ---- as they are used ------------------------------------------------------------------------------------------------
def test_the_same_inputs_give_the_same_bits():
    for new in ([1, 1, 1], [200, 1, 130], [5, 3, 8]):
        c = Case(51, "bf16", 128, 2, 4, 16, [9000, 700, 3111], new)
        out, lse = c.run()
        for _ in range(3):
            again, lse2 = c.run()
            assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_rows_and_heads_apart_and_a_known_scale(kind):
    c = Case(53, kind, 64, 2, 3, 16, [200, 90], [140, 4], gap=8)
    want, lse = c.run(scale=0.2)
    wide = torch.full((c.n, c.heads + 2, 64 + 8), 9.0, dtype=c.t, device="cuda")
    q = wide[:, 1:-1, :64]
    q.copy_(c.q)
    room = torch.full((c.heads, c.n + 3, 64), 5.0, dtype=c.t, device="cuda")
    out = room.transpose(0, 1)[1:-2]                               # heads outside, rows inside
    got, none = B().grpo_paged_attention(q, c.k_pages, c.v_pages, c.table, c.seq_len, c.q_off, scale=0.2, out=out, want_lse=False)
    assert none is None and got is out and torch.equal(out, want[:c.n])
    assert bool((room[:, 0] == 5).all()) and bool((room[:, -2:] == 5).all())


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_rows_ahead_of_the_first_sequence_are_left_alone(kind):
    c = Case(55, kind, 64, 2, 2, 16, [50, 300], [3, 120])
    want, lse = c.run()
    c.q = torch.cat([c.q[:7] * float("nan"), c.q])
    c.n += 7
    c.q_off += 7
    out, ls = c.run()
    assert torch.equal(out[7:], want) and torch.equal(ls[7:], lse) and bool((out[:7] == 7).all()) and bool((ls[:7] == 7).all())
    kv = torch.randn(c.n, 2, 64, device="cuda").to(c.t)
    before = c.k_pages.clone()
    q_out = torch.full_like(c.q, 7.0)
    B().grpo_rotary_cache(c.q, kv, kv, c.k_pages, c.v_pages, c.table, c.seq_len, c.q_off, None, q_out=q_out)
    assert bool((q_out[:7] == 7).all()) and torch.equal(q_out[7:], c.q[7:])
    changed = (c.k_pages != before) & ~(torch.isnan(c.k_pages) & torch.isnan(before))          # slots never written are NaN
    assert int(changed.flatten(2).any(2).sum()) == 123


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("max_new", [0, 1, 2, 40, 10 ** 6])
def test_max_new_is_a_hint(kind, max_new):
    """Any value gives the right answer, one that is too small too: it chooses among kernels."""
    c = Case(57, kind, 64, 1, 4, 16, [400, 3, 90, 33], [40, 1, 2, 33])
    c.check(*c.run(max_new=max_new))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_many_sequences(kind):
    """More than a block's own plan takes: 1300 sequences, a tenth of them without rows, and a few with many."""
    rng = np.random.default_rng(3)
    lens = [int(a) for a in rng.integers(0, 60, 1300)]
    new = [0 if i % 10 == 0 else min(a, 1 + i % 3) for i, a in enumerate(lens)]
    lens[77], new[77] = 500, 150
    c = Case(59, kind, 32 if kind == "f32" else 64, 1, 2, 8, lens, new)
    c.check(*c.run())


def test_many_row_tiles():
    """A chunk whose row tiles pass what a block plans itself (1024): only its last rows are checked."""
    new, length = 66000, 66100
    g = gen(61)
    k, v = (torch.randn(length // 64 + 1, 64, 1, 64, generator=g, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn(new, 4, 64, generator=g, device="cuda").bfloat16()
    table = torch.randperm(length // 64 + 1, generator=g, device="cuda").to(torch.int32)[None]
    out, lse = B().grpo_paged_attention(q, k, v, table, torch.tensor([length], dtype=torch.int32, device="cuda"),
                                        torch.tensor([0, new], dtype=torch.int32, device="cuda"), window=600, sinks=3, max_new=new)
    rows = [0, 1, 12345, 40000, new - 1]
    flat = lambda t: host(t[table[0].long()].flatten(0, 1)[:length])
    kh, vh = flat(k), flat(v)
    for r in rows:
        want, wlse, mass, _ = ro.attend(host(q[r:r + 1]), kh[None], vh[None], np.zeros((1, 1), int), [length - new + r + 1], np.array([0, 1]), 0.125, 600, 3)
        assert np.all(np.abs(host(out[r:r + 1]) - want) <= 2.0 ** -7 * mass + 2.0 ** -8 * np.abs(want))
        assert np.all(np.abs(host(lse[r:r + 1]) - wlse) < 1e-4)


def test_offsets_beyond_31_bits():
    """Pages at both ends of a cache of more than 2^32 elements."""
    n, page, kv, dim = 264000, 16, 8, 128
    k, v = (torch.empty(n, page, kv, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert k.numel() > 2 ** 32
    table = torch.tensor([[n - 1, 0, n // 2, n - 2, 5]], dtype=torch.int32, device="cuda")
    g = gen(63)
    new = torch.randn(70, 16 + 2 * kv, dim, generator=g, device="cuda").bfloat16()
    q, kn, vn = new[:, :16], new[:, 16:24], new[:, 24:]
    seq_len, q_off = torch.tensor([70], dtype=torch.int32, device="cuda"), torch.tensor([0, 70], dtype=torch.int32, device="cuda")
    B().grpo_rotary_cache(q, kn, vn, k, v, table, seq_len, q_off, None)
    assert torch.equal(k[table[0].long()].flatten(0, 1)[:70], kn)
    kh, vh = host(kn)[None], host(vn)[None]
    for rows in (70, 1):
        out, _ = B().grpo_paged_attention(q[70 - rows:], k, v, table, seq_len, torch.tensor([0, rows], dtype=torch.int32, device="cuda"))
        want, _, mass, _ = ro.attend(host(q[70 - rows:]), kh, vh, np.zeros((1, 1), int), [70], np.array([0, rows]), dim ** -0.5)
        assert np.all(np.abs(host(out) - want) <= 2.0 ** -7 * mass + 2.0 ** -8 * np.abs(want))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("new", [1, 130])
def test_scores_that_rise_by_hundreds_from_tile_to_tile(kind, new):
    """Each tile of keys outweighs all before it by more than a weight's exponent holds, and the other way round."""
    for falling in (False, True):
        c = Case(65, kind, 64, 1, 2, 16, [700], [new])
        c.q[:] = 1.0
        steps = torch.arange(700, device="cuda") // 128 * 90.0
        rows = torch.from_numpy(c.table_host[0][np.arange(700) // 16].astype(np.int64)).cuda(), torch.arange(700, device="cuda") % 16
        noise = torch.randn(700, 1, 64, generator=gen(66), device="cuda") * 0.01
        c.k_pages[rows] = ((noise + ((-steps if falling else steps) / 64)[:, None, None]) * 8).to(c.t)      # scores: 64 x 8 / 8 per step
        c.check(*c.run())


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_captured_calls_follow_the_lengths_and_share_a_workspace(kind):
    """A decoding step and a chunk captured into two graphs with one workspace, replayed in turn as the sequences grow."""
    dim, kv, heads, page = 64, 2, 6, 16
    t, g = TYPES[kind], gen(71)
    k, v = (torch.zeros(40, page, kv, dim, dtype=t, device="cuda") for _ in range(2))
    table = torch.arange(40, dtype=torch.int32, device="cuda").view(2, 20)
    turns, _ = B().grpo_rotary_freqs(dim)
    turns = turns.cuda()
    seq_len = torch.zeros(2, dtype=torch.int32, device="cuda")
    need = max(B().grpo_paged_attention_workspace_bytes(k, 2, n, heads, m) for n, m in ((2, 1), (80, 40)))
    workspace = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    calls = {}
    for new in (40, 1):
        fused = torch.zeros(2 * new, heads + 2 * kv, dim, dtype=t, device="cuda")
        q_off = torch.tensor([0, new, 2 * new], dtype=torch.int32, device="cuda")
        out, lse, q = (torch.empty(2 * new, heads, dim, dtype=t, device="cuda"), torch.empty(2 * new, heads, device="cuda"),
                       torch.empty(2 * new, heads, dim, dtype=t, device="cuda"))

        def step(fused=fused, q_off=q_off, out=out, lse=lse, q=q, new=new):
            B().grpo_rotary_cache(fused[:, :heads], fused[:, heads:heads + kv], fused[:, heads + kv:], k, v, table, seq_len, q_off, turns, q_out=q)
            B().grpo_paged_attention(q, k, v, table, seq_len, q_off, max_new=new, out=out, lse=lse, workspace=workspace)
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        calls[new] = graph, fused, q_off, out, lse, q
    history = []
    length = 0
    for new in (40, 1, 1, 40, 1):
        graph, fused, q_off, out, lse, q = calls[new]
        fused.copy_(torch.randn(fused.shape, generator=g, device="cuda"))
        length += new
        seq_len.fill_(length)
        graph.replay()
        history.append((host(k[table.long()].flatten(1, 2)), host(v[table.long()].flatten(1, 2))))
        kh, vh = history[-1]
        want, _, mass, reach = ro.attend(host(q), kh, vh, np.array([[0], [1]]), [length] * 2, q_off.cpu().numpy(), dim ** -0.5)
        d = 2 * (dim + 4) * U * reach
        tol = ((2 * (2 * d + 2 * reach * U + 2.0 ** -22) + 100 * U + (2.0 ** -8 if kind == "bf16" else 0))[..., None]) * mass + half_step(t) * np.abs(want)
        assert np.all(np.abs(host(out) - want) <= tol)


def test_two_streams_at_once():
    cases = [Case(73 + i, "bf16", 64, 2, 2, 16, [3000, 700], [n, n]) for i, n in enumerate((1, 200))]
    want = [c.run() for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(5):
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                got.append(c.run())
    torch.cuda.synchronize()
    for i, (out, lse) in enumerate(got):
        assert torch.equal(out, want[i % 2][0]) and torch.equal(lse, want[i % 2][1])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_a_layer_token_by_token_is_the_layer_over_the_whole_sequence(kind):
    """The actor update's attention over 96 positions of two chunks, and the rollout's over the same: a prefix of 40 tokens at
    once, then eight, then one at a time, through projection, rotation, cache and attention."""
    H, dh, S, n = 4, 64, 96, 2
    d, t, g = H * dh, TYPES[kind], gen(81)
    x = torch.randn(n * S, d, generator=g, device="cuda").to(t)
    w = (torch.randn(3 * d, d, generator=g, device="cuda") * d ** -0.5).to(t)
    turns, _ = B().grpo_rotary_freqs(dh)
    turns = turns.cuda()
    qkv = B().grpo_gemm(x, True, w, True, n * S, 3 * d, d, out_dtype=t)
    pos = torch.arange(S, dtype=torch.int32, device="cuda").repeat(n)
    whole = qkv.clone().view(n * S, 3, H, dh)
    for i in (0, 1):
        B().grpo_rotary(whole[:, i], pos, turns, out=whole[:, i])
    want, want_lse, _ = B().grpo_attention(whole.view(n * S, 3 * d), n, S, H, dh)
    k, v = (torch.zeros(n * 8, 16, H, dh, dtype=t, device="cuda") for _ in range(2))
    table = torch.randperm(n * 8, generator=g, device="cuda").to(torch.int32).view(n, 8)
    qkv = qkv.view(n, S, 3, H, dh)
    out = torch.empty(n, S, H, dh, dtype=t, device="cuda")
    lse = torch.empty(n, S, H, device="cuda")
    at = 0
    for new in [40, 8] + [1] * 48:
        rows = qkv[:, at:at + new].reshape(n * new, 3, H, dh)
        at += new
        seq_len = torch.full((n,), at, dtype=torch.int32, device="cuda")
        q_off = torch.arange(n + 1, dtype=torch.int32, device="cuda") * new
        q = B().grpo_rotary_cache(rows[:, 0], rows[:, 1], rows[:, 2], k, v, table, seq_len, q_off, turns)
        o, ls = B().grpo_paged_attention(q, k, v, table, seq_len, q_off, max_new=new)
        out[:, at - new:at], lse[:, at - new:at] = o.view(n, new, H, dh), ls.view(n, new, H)
    # both are off from the exact attention by a rounding of the weights (2^-8 of sum p |v|) and one of the result
    vv = whole.view(n, S, 3, H, dh)[:, :, 2].double().abs().max()
    tol = 1e-5 if kind == "f32" else 2 * (2.0 ** -8 + 2.0 ** -8) * float(vv)
    assert float((out.view(n * S, d).double() - want.double()).abs().max()) <= tol
    assert float((lse - want_lse.transpose(1, 2)).abs().max()) <= (1e-5 if kind == "f32" else 1e-3)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("new", [1, 300])
def test_more_sinks_than_a_sequence_can_have_are_all_of_it(kind, new):
    c = Case(71, kind, 64, 2, 2, 16, [900], [new])
    full, lse = c.run()
    out, lse2 = c.run(64, 2 ** 31 - 1)
    assert torch.equal(out, full) and torch.equal(lse, lse2)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("new", [1, 300])
def test_scaled_scores_beyond_fp32_choose_the_largest(kind, new):
    """Scores near 1e34 times a scale of 1e6: any difference leaves the lesser score no weight.  Elements are a power of two
    times small integers: every score is exact and the largest ones are the same in both arithmetics."""
    c = Case(73, kind, 64, 1, 2, 16, [700], [new])
    g = gen(74)
    for t in (c.q, c.k_pages):
        t.copy_((torch.randint(-8, 9, t.shape, generator=g, device="cuda") * 2.0 ** 52).to(c.t))
    out, _ = c.run(scale=1e6)
    want = ro.attend(host(c.q), host(c.k_pages), host(c.v_pages), c.table_host, c.lens, c.q_off_host, 1e6)[0]
    assert bool(torch.isfinite(out).all())
    assert float(np.abs(host(out) - want).max()) <= (2.0 ** -22 if kind == "f32" else 2.0 ** -8) * float(np.abs(want).max())


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("new", [2, 130])
def test_a_score_of_minus_infinity_weighs_nothing_beside_values_that_no_row_sees(kind, new):
    c = Case(75, kind, 64, 1, 2, 16, [new + 400], [new])
    c.q[..., 0] = 1.0
    page, slot = c.table_host[0][0], 0
    c.k_pages[page, slot, 0, 0] = float("-inf")
    clean, lse = c.run()
    assert bool(torch.isfinite(clean).all()) and bool(torch.isfinite(lse).all())
    page, slot = c.table_host[0][(new + 399) // 16], (new + 399) % 16                 # the last token's slot
    c.v_pages[page, slot] = float("nan")
    out, lse2 = c.run()
    tol = 0 if kind == "f32" else 2.0 ** -7
    assert bool(torch.isfinite(out[:-1]).all()) and torch.equal(lse, lse2)
    assert float((out[:-1].double() - clean[:-1].double()).abs().max()) <= tol * float(clean.double().abs().max()) + 1e-5


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(64, 1, 71, 136, [300, 33, 1], [1, 2, 1]), (128, 1, 300, 8, [260, 129], [1, 3]), (32, 1, 100, 40, [500, 7], [1, 7]),
                                   (64, 2, 33, 1000, [2100, 900], [5, 1]), (128, 2, 17, 72, [400, 65, 3], [1, 1, 1])],
                         ids=lambda s: f"d{s[0]}kv{s[1]}g{s[2]}p{s[3]}")
def test_many_heads_of_one_key_and_odd_pages(kind, shape):
    dim, kv, group, page, lens, new = shape
    c = Case(dim + group, kind, dim, kv, group, page, lens, new)
    for window, sinks in ((0, 0), (70, 9)):
        c.check(*c.run(window, sinks), window, sinks, rounded=True)
