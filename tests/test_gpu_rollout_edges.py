"""Calls of the rollout side at their edges.  Tolerances are those of the Case class."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from test_gpu_rollout import B, Case, TYPES, gen, host

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("dim", [64, 128])
def test_a_reference_moves_in_a_warp_with_fewer_rows_too(dim):
    """Scores that rise by 40 powers of two a tile: each row's reference follows from the next tile on, wherever the row's warp
    ends.  The rows of a chunk of 246 tokens are those of a chunk of 256 from the same place, bit by bit: its last warp is the
    only difference, and rows formed once more would round otherwise."""
    c = Case(91, "bf16", dim, 1, 1, 16, [1000], [256])
    c.q[:] = 1.0
    at = torch.from_numpy(c.table_host[0][np.arange(1000) // 16].astype(np.int64)).cuda(), torch.arange(1000, device="cuda") % 16
    rise = torch.arange(1000, device="cuda") // 128 * (40.0 * np.log(2.0) * dim ** 0.5 / dim)
    noise = torch.randn(1000, 1, dim, generator=gen(92), device="cuda") * 0.01
    c.k_pages[at] = (rise[:, None, None] + noise).to(c.t)
    out, lse = c.run()
    c.check(out, lse)
    c.seq_len[0] = 990
    c.q_off[1] = 246
    fewer, lse2 = c.run()
    assert torch.equal(fewer[:246], out[:246]) and torch.equal(lse2[:246], lse[:246])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("new,length", [(3, 60), (3, 20000), (130, 230), (130, 20000)])
@pytest.mark.parametrize("key", ["first", "late"])
def test_a_score_of_infinity_makes_the_rows_that_see_it_nan(kind, new, length, key):
    """.. in units of one piece and in units that are cut, as the first key and as one of the chunk's own; other rows and heads keep their bits."""
    c = Case(93, kind, 64, 2, 2, 16, [length, 90], [new, 1])
    c.q[..., 0] = 1.0
    clean, lse = c.run()
    assert bool(torch.isfinite(clean).all())
    j = 0 if key == "first" else length - (new + 1) // 2
    c.k_pages[c.table_host[0][j // 16], j % 16, 0, 0] = float("inf")
    out, lse2 = c.run()
    first = max(0, j - (length - new))                             # rows from here on see it
    assert bool(torch.isnan(out[first:new, :2]).all()) and bool(torch.isnan(lse2[first:new, :2]).all())
    out[first:new, :2], lse2[first:new, :2] = clean[first:new, :2], lse[first:new, :2]
    assert torch.equal(out, clean) and torch.equal(lse2, lse)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("length", [67, 68, 200, 2 ** 31 - 1])
def test_a_length_beyond_the_table_overwrites_no_stored_token(kind, length):
    """64 slots, all of them taken; new tokens whose places lie behind the table are not stored, and nothing else moves."""
    c = Case(95, kind, 64, 2, 2, 16, [64, 60], [5, 4], stale=3.0)
    c.table = c.table[:, :4].contiguous()
    g = gen(96)
    fused = torch.randn(9, 4 + 2 * 2, 64, generator=g, device="cuda").to(c.t)
    q, k, v = fused[:, :4], fused[:, 4:6], fused[:, 6:]
    turns = B().grpo_rotary_freqs(64)[0].cuda()
    c.seq_len[0] = length
    want_k, want_v = c.k_pages.clone(), c.v_pages.clone()
    pos = np.concatenate([np.arange(length - 5, length), np.arange(56, 60)])
    pos_t = torch.from_numpy(pos.astype(np.int32)).cuda()
    turned = B().grpo_rotary(k, pos_t, turns)
    for r, (s, j) in enumerate(zip([0] * 5 + [1] * 4, pos)):
        if j < 64:
            want_k[c.table_host[s][j // 16], j % 16], want_v[c.table_host[s][j // 16], j % 16] = turned[r], v[r]
    out = B().grpo_rotary_cache(q, k, v, c.k_pages, c.v_pages, c.table, c.seq_len, c.q_off, turns, status=c.status)
    assert torch.equal(c.k_pages, want_k) and torch.equal(c.v_pages, want_v)
    assert torch.equal(out, B().grpo_rotary(q, pos_t, turns))
    assert int(c.status) == 128


@pytest.mark.parametrize("seq_len,q_off", [([40, -1], [0, 10, 10]), ([40, 1 << 20], [0, 10, 10]), ([40, 40], [0, 10, 4]), ([40, 40], [0, 4, 11]),
                                           ([40, 40], [-1, 4, 10])])
def test_both_calls_report_lengths_and_offsets_that_do_not_fit(seq_len, q_off):
    """.. of sequences without rows too."""
    c = Case(97, "bf16", 64, 2, 2, 16, [40, 40], [5, 5])
    c.table = torch.arange(6, dtype=torch.int32, device="cuda").view(2, 3)
    c.seq_len.copy_(torch.tensor(seq_len, dtype=torch.int32))
    c.q_off.copy_(torch.tensor(q_off, dtype=torch.int32))
    kv = torch.ones(10, 2, 64, dtype=c.t, device="cuda")
    c.run()
    assert int(c.status) == 128
    c.status.zero_()
    B().grpo_rotary_cache(c.q, kv, kv, c.k_pages, c.v_pages, c.table, c.seq_len, c.q_off, None, status=c.status)
    assert int(c.status) == 128


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n_pages,kv", [(1, 2), (4, 1), (1, 1)])
def test_strides_that_lead_nowhere_may_differ(kind, n_pages, kv):
    """A cache of one page or one head: the strides of k and v in that dimension mean nothing."""
    g, t = gen(98), TYPES[kind]
    k, v = (torch.randn(n_pages, 16, kv, 64, generator=g, device="cuda").to(t) for _ in range(2))
    table = torch.arange(n_pages, dtype=torch.int32, device="cuda")[None]
    seq_len, q = torch.tensor([n_pages * 16], dtype=torch.int32, device="cuda"), torch.randn(1, 4, 64, generator=g, device="cuda").to(t)
    want, lse = B().grpo_paged_attention(q, k, v, table, seq_len)
    strides = list(v.stride())
    for i, n in ((0, n_pages), (2, kv)):
        if n == 1:
            strides[i] = 24
    other = v.as_strided(v.shape, strides)
    got, lse2 = B().grpo_paged_attention(q, k, other, table, seq_len)
    assert torch.equal(got, want) and torch.equal(lse2, lse)
    got, lse2 = B().grpo_paged_attention(q, k.as_strided(k.shape, strides), v, table, seq_len)
    assert torch.equal(got, want) and torch.equal(lse2, lse)
    with pytest.raises(B().PcmError):                              # the slots' strides do lead somewhere
        B().grpo_paged_attention(q, k, torch.zeros(n_pages, 16, kv, 128, dtype=t, device="cuda")[..., :64], table, seq_len)


def test_calls_of_a_new_thread():
    """The first GPU work of a thread is the call itself: nothing else has made a context current there."""
    import threading
    b, g = B(), gen(99)
    c = {new: Case(99, "bf16", 64, 2, 2, 16, [300, 280], [new, new]) for new in (1, 150)}
    x, w = torch.randn(256, 128, generator=g, device="cuda").bfloat16(), torch.randn(512, 128, generator=g, device="cuda").bfloat16()
    qkv = torch.randn(2 * 96, 3 * 128, generator=g, device="cuda").bfloat16()
    tok = torch.randint(0, 512, (256,), generator=g, device="cuda", dtype=torch.int32)
    paged = []
    for new, case in c.items():
        room = torch.empty(b.grpo_paged_attention_workspace_bytes(case.k_pages, 2, case.n, 4, new) + 256, dtype=torch.uint8, device="cuda")
        paged.append(lambda case=case, new=new, room=room, to=(torch.empty_like(case.q), torch.empty(case.n, 4, device="cuda")): b.grpo_paged_attention(
            case.q, case.k_pages, case.v_pages, case.table, case.seq_len, case.q_off, max_new=new, out=to[0], lse=to[1], workspace=room))
    calls = [*paged, lambda: b.grpo_gemm(x, True, w, True, 256, 512, 128), lambda: b.grpo_attention(qkv, 2, 96, 2, 64)[:2],
             lambda: b.grpo_head_logp(x, w, tok)]
    as_list, failed = (lambda r: list(r) if isinstance(r, (tuple, list)) else [r]), []
    for call in calls:
        want, got = [t.clone() for t in as_list(call())], []
        torch.cuda.synchronize()

        def work():
            try:
                got.append(call())
            except Exception as e:
                got.append(e)
        t = threading.Thread(target=work)
        t.start()
        t.join()
        torch.cuda.synchronize()
        if isinstance(got[0], Exception):
            failed.append(got[0])
        else:
            assert all(torch.equal(p, q) for p, q in zip(as_list(got[0]), want))
    assert not failed


def test_an_expired_wait_is_reported_with_and_without_a_status_word():
    """With a word it is that call's alone; without one the next call that polls has it."""
    b = B()
    x, w = torch.zeros(128, 64, device="cuda").bfloat16(), torch.zeros(256, 64, device="cuda").bfloat16()
    assert b.grpo_gemm_wait_status(0) == 0
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    b.grpo_expired_wait(status)
    assert int(status) == 1 and b.grpo_gemm_wait_status(0) == 0
    b.grpo_expired_wait()
    with pytest.raises(b.PcmError) as e:
        b.grpo_gemm(x, True, w, True, 128, 256, 64)
    assert e.value.code == -5
    b.grpo_gemm(x, True, w, True, 128, 256, 64)
    c = Case(101, "bf16", 64, 1, 2, 16, [300], [200])              # calls that wait for nothing in vain report nothing, with a word and without
    for new in (200, 1):
        c.q_off[1] = new
        c.run()
        c.run(status=None)
    assert int(c.status) == 0 and b.grpo_gemm_wait_status(0) == 0


_CAPTURED_FIRST = """
import torch
from paper_2605_16154_b200 import binding as B
g = torch.Generator(device="cuda").manual_seed(1)
k, v = (torch.randn(40, 16, 2, 64, generator=g, device="cuda").bfloat16() for _ in range(2))
table = torch.arange(40, dtype=torch.int32, device="cuda").view(2, 20)
seq_len = torch.tensor([300, 280], dtype=torch.int32, device="cuda")
new = NEW
q = torch.randn(2 * new, 4, 64, generator=g, device="cuda").bfloat16()
q_off = torch.tensor([0, new, 2 * new], dtype=torch.int32, device="cuda")
room = torch.empty(B.grpo_paged_attention_workspace_bytes(k, 2, 2 * new, 4, new) + 256, dtype=torch.uint8, device="cuda")
out, lse = torch.zeros_like(q), torch.zeros(2 * new, 4, device="cuda")
call = lambda: B.grpo_paged_attention(q, k, v, table, seq_len, q_off, max_new=new, out=out, lse=lse, workspace=room)
graph = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    call()
graph.replay()
torch.cuda.synchronize()
got, got_lse = out.clone(), lse.clone()
call()
torch.cuda.synchronize()
assert torch.equal(got, out) and torch.equal(got_lse, lse) and bool((out != 0).any())
print("captured first ok")
"""


@pytest.mark.parametrize("new", [1, 150])
def test_a_process_whose_first_call_is_captured(new):
    res = subprocess.run([sys.executable, "-c", _CAPTURED_FIRST.replace("NEW", str(new))], cwd=ROOT, env=dict(os.environ, PYTHONPATH=ROOT),
                         capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and "captured first ok" in res.stdout, res.stdout[-2000:] + res.stderr[-2000:]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["pages", "heads first", "slots outside", "heads outside", "beside one another", "page by page", "one page", "one head"])
def test_layouts_of_a_cache_that_are_written(kind, layout):
    """The order of pages, slots and heads in memory is free, and keys and values may lie between one another."""
    t, n, page, kv, dim = TYPES[kind], 1 if layout == "one page" else 6, 16, 1 if layout == "one head" else 2, 32
    make = lambda *shape: torch.full(shape, 3.0, dtype=t, device="cuda")
    if layout == "beside one another":
        k, v = make(n, page, kv, 2, dim).unbind(3)
    elif layout == "page by page":
        k, v = make(n, 2, page, kv, dim).unbind(1)
    elif layout == "heads first":
        k, v = (make(n, kv, page, dim).transpose(1, 2) for _ in range(2))
    elif layout == "slots outside":
        k, v = (make(page, n, kv, dim + 8).transpose(0, 1)[..., :dim] for _ in range(2))
    elif layout == "heads outside":
        k, v = (make(kv, n, page, dim).permute(1, 2, 0, 3) for _ in range(2))
    else:
        k, v = (make(n, page, kv, dim) for _ in range(2))
    g = gen(103)
    new = min(40, n * page - 3)
    kn, vn = (torch.randn(new, kv, dim, generator=g, device="cuda").to(t) for _ in range(2))
    table = torch.randperm(n, generator=g, device="cuda").to(torch.int32)[None]
    at = torch.arange(3, new + 3, device="cuda")
    want_k, want_v = k.clone(), v.clone()
    want_k[table[0].long()[at // page], at % page], want_v[table[0].long()[at // page], at % page] = kn, vn
    B().grpo_rotary_cache(None, kn, vn, k, v, table, torch.tensor([new + 3], dtype=torch.int32, device="cuda"),
                          torch.tensor([0, new], dtype=torch.int32, device="cuda"), None)
    assert torch.equal(k, want_k) and torch.equal(v, want_v)


_FIRST_CALLS = """
import threading
import torch
from paper_2605_16154_b200 import binding as B

def family(dtype, dim, new):
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(40, 16, 2, dim, generator=g, device="cuda").to(dtype) for _ in range(2))
    q = torch.randn(2 * new, 4, dim, generator=g, device="cuda").to(dtype)
    table = torch.arange(40, dtype=torch.int32, device="cuda").view(2, 20)
    seq_len = torch.tensor([300, 280], dtype=torch.int32, device="cuda")
    q_off = torch.tensor([0, new, 2 * new], dtype=torch.int32, device="cuda")
    need = B.grpo_paged_attention_workspace_bytes(k, 2, 2 * new, 4, new)
    n = 8
    outs = [(torch.empty_like(q), torch.empty(2 * new, 4, device="cuda"), torch.empty(need + 256, dtype=torch.uint8, device="cuda")) for _ in range(n)]
    streams = [torch.cuda.Stream() for _ in range(n)]
    gate, failed = threading.Barrier(n), []
    torch.cuda.synchronize()
    def call(i):
        out, lse, ws = outs[i]
        with torch.cuda.stream(streams[i]):
            gate.wait()
            try:
                B.grpo_paged_attention(q, k, v, table, seq_len, q_off, max_new=new, out=out, lse=lse, workspace=ws)
            except Exception as e:
                failed.append(repr(e))
    threads = [threading.Thread(target=call, args=(i,)) for i in range(n)]
    for t in threads: t.start()
    for t in threads: t.join()
    torch.cuda.synchronize()
    assert not failed, (dtype, dim, new, failed)
    for out, lse, _ in outs[1:]:
        assert torch.equal(out, outs[0][0]) and torch.equal(lse, outs[0][1])

for dtype, dim, new in ((torch.bfloat16, 64, 150), (torch.bfloat16, 128, 150), (torch.bfloat16, 64, 1), (torch.bfloat16, 128, 1), (torch.bfloat16, 32, 1),
                        (torch.float32, 64, 150), (torch.float32, 128, 150), (torch.float32, 64, 1), (torch.float32, 128, 1)):
    family(dtype, dim, new)
print("first calls ok")
"""


def test_first_calls_of_several_threads():
    """Eight threads make a process's first call of each kernel at the same time."""
    res = subprocess.run([sys.executable, "-c", _FIRST_CALLS], cwd=ROOT, env=dict(os.environ, PYTHONPATH=ROOT), capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and "first calls ok" in res.stdout, res.stdout[-2000:] + res.stderr[-2000:]
