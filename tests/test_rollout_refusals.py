"""Arguments that the rollout calls refuse, through the C ABI and the binding, their sizes and the frequencies of rotary
positions.  Every case is turned down on the host before anything is launched: the addresses are never used."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import rollout_oracle as ro

ARG, SHAPE, WORKSPACE = -1, -2, -3
P = 1 << 20
NAN, INF = float("nan"), float("inf")


def _lib():
    from paper_2605_16154_b200 import binding
    return binding


CACHE = dict(dtype=1, n_pages=10, page_size=16, n_kv_heads=2, head_dim=64, reserved=0, k=P, v=2 * P, ld_page=16 * 128, ld_slot=128, ld_head=64)
BATCH = dict(n_seq=3, max_pages=4, page_table=P, ld_table=4, seq_len=P, q_off=P)
ROTARY = dict(dtype=1, x=P, ld_x=256, ld_x_head=64, n=5, n_heads=4, head_dim=64, rot_dim=32, turns=P, amplitude=1.0, pos=P, flags=0, out=2 * P,
              ld_out=256, ld_out_head=64, stream=None)
APPEND = dict(n_rows=5, q=P, ld_q=256, ld_q_head=64, n_heads=4, k=P, ld_k=128, ld_k_head=64, v=P, ld_v=128, ld_v_head=64, rot_dim=64, turns=P,
              amplitude=1.0, pos=None, flags=0, q_out=2 * P, ld_q_out=256, ld_q_out_head=64, status=None, stream=None)
ATTEND = dict(n_rows=5, q=P, ld_q=256, ld_q_head=64, n_heads=4, scale=0.125, window=0, sinks=0, max_new=0, out=2 * P, ld_out=256, ld_out_head=64,
              lse=P, status=None, workspace=P, workspace_bytes=1 << 40, stream=None)


def _call(name, cache={}, batch={}, **change):
    B = _lib()
    base = {"grpo_rotary": ROTARY, "grpo_rotary_cache": APPEND, "grpo_paged_attention": ATTEND}[name]
    assert set(change) <= set(base) and set(cache) <= set(CACHE) and set(batch) <= set(BATCH)
    args = list(dict(base, **change).values())
    if name != "grpo_rotary":
        args = [B.grpo_kv_cache(*dict(CACHE, **cache).values()), B.grpo_kv_batch(*dict(BATCH, **batch).values())] + args
    return getattr(B._lib, name)(*args)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), ARG), (dict(x=None), ARG), (dict(out=None), ARG), (dict(pos=None), ARG), (dict(turns=None), ARG), (dict(n=-1), ARG),
    (dict(n_heads=0), ARG), (dict(head_dim=0), ARG), (dict(rot_dim=-2), ARG), (dict(amplitude=NAN), ARG), (dict(amplitude=INF), ARG),
    (dict(flags=4), ARG), (dict(x=P + 1), ARG), (dict(dtype=0, out=P + 2), ARG), (dict(ld_x=63), ARG), (dict(ld_x_head=32), ARG),
    (dict(ld_out=10), ARG), (dict(ld_out_head=63), ARG), (dict(out=P, ld_out=512), ARG), (dict(out=P, ld_out_head=68), ARG),
    (dict(rot_dim=31), SHAPE), (dict(rot_dim=66), SHAPE), (dict(head_dim=1026, ld_x_head=1026, ld_out_head=1026), SHAPE),
    (dict(n=(1 << 30) + 1), SHAPE), (dict(n_heads=70000), SHAPE)])
def test_rotary_refuses(change, code):
    assert _call("grpo_rotary", **change) == code


CACHES = [(dict(dtype=5), ARG), (dict(n_pages=0), ARG), (dict(page_size=0), ARG), (dict(n_kv_heads=0), ARG), (dict(k=None), ARG), (dict(v=None), ARG),
          (dict(page_size=12), SHAPE), (dict(k=P + 8), SHAPE), (dict(v=P + 2), SHAPE), (dict(ld_slot=129), SHAPE), (dict(ld_page=2052), SHAPE),
          (dict(ld_head=68), SHAPE), (dict(ld_slot=56), ARG), (dict(ld_head=8), ARG), (dict(ld_page=-2048), ARG), (dict(ld_page=0), ARG)]
BATCHES = [(dict(n_seq=-1), ARG), (dict(max_pages=0), ARG), (dict(page_table=None), ARG), (dict(seq_len=None), ARG), (dict(ld_table=3), ARG),
           (dict(q_off=None), ARG), (dict(n_seq=(1 << 30) + 1), SHAPE)]


@pytest.mark.parametrize("name", ["grpo_rotary_cache", "grpo_paged_attention"])
@pytest.mark.parametrize("change,code", CACHES, ids=lambda v: str(v) if isinstance(v, dict) else "")
def test_caches_that_are_refused(name, change, code):
    assert _call(name, cache=change) == code


@pytest.mark.parametrize("name", ["grpo_rotary_cache", "grpo_paged_attention"])
@pytest.mark.parametrize("change,code", BATCHES, ids=lambda v: str(v) if isinstance(v, dict) else "")
def test_batches_that_are_refused(name, change, code):
    assert _call(name, batch=change) == code


@pytest.mark.parametrize("change,code", [
    (dict(n_rows=-1), ARG), (dict(k=None), ARG), (dict(v=None), ARG), (dict(q=None), ARG), (dict(q_out=None), ARG), (dict(turns=None), ARG),
    (dict(n_heads=-1), ARG), (dict(flags=2), ARG), (dict(amplitude=INF), ARG), (dict(rot_dim=-1), ARG), (dict(k=P + 1), ARG), (dict(ld_k=32), ARG),
    (dict(ld_v_head=8), ARG), (dict(ld_q=3), ARG), (dict(q_out=P, ld_q_out=300), ARG), (dict(rot_dim=63), SHAPE), (dict(rot_dim=128), SHAPE),
    (dict(n_rows=(1 << 30) + 1), SHAPE)])
def test_appending_refuses(change, code):
    assert _call("grpo_rotary_cache", **change) == code


@pytest.mark.parametrize("change,code", [
    (dict(n_rows=-2), ARG), (dict(q=None), ARG), (dict(out=None), ARG), (dict(n_heads=0), ARG), (dict(n_heads=3), ARG), (dict(scale=0.0), ARG),
    (dict(scale=-1.0), ARG), (dict(scale=NAN), ARG), (dict(scale=INF), ARG), (dict(scale=3e38), ARG), (dict(window=-1), ARG), (dict(sinks=-1), ARG),
    (dict(max_new=-1), ARG), (dict(lse=P + 2), ARG), (dict(ld_q_head=32), ARG), (dict(ld_out=100), ARG), (dict(q=P + 8), SHAPE), (dict(out=P + 2), SHAPE),
    (dict(ld_q=260), SHAPE), (dict(ld_out=512, ld_out_head=68), SHAPE), (dict(ld_out_head=72), ARG), (dict(workspace=None), WORKSPACE), (dict(workspace=P + 64), WORKSPACE),
    (dict(workspace_bytes=1000), WORKSPACE), (dict(n_rows=1 << 30), SHAPE)])
def test_attention_refuses(change, code):
    assert _call("grpo_paged_attention", **change) == code


@pytest.mark.parametrize("dim", [16, 48, 96, 256])
def test_head_dims_that_attention_does_not_take(dim):
    strides = dict(head_dim=dim, ld_head=dim, ld_slot=2 * dim, ld_page=32 * dim)
    assert _call("grpo_paged_attention", cache=strides, ld_q=4 * dim, ld_q_head=dim, ld_out=4 * dim, ld_out_head=dim) == SHAPE


@pytest.mark.parametrize("name", ["grpo_rotary_cache", "grpo_paged_attention"])
def test_no_rows_and_no_sequences_are_valid_calls(name):
    assert _call(name, cache=dict(k=None, v=None), batch=dict(page_table=None, seq_len=None), n_rows=0, q=None) == 0
    assert _call(name, cache=dict(k=None, v=None), batch=dict(n_seq=0, page_table=None, seq_len=None), q=None) == 0
    assert _call("grpo_rotary", n=0, x=None, out=None, pos=None) == 0


def _need(n_seq, n_rows, n_heads=4, max_new=0, **cache):
    B = _lib()
    return B._lib.grpo_paged_attention_workspace_bytes(ctypes.byref(B.grpo_kv_cache(*dict(CACHE, **cache).values())), n_seq, n_rows, n_heads, max_new)


@pytest.mark.parametrize("cache", [dict(), dict(head_dim=128), dict(head_dim=32), dict(dtype=0)])
def test_the_workspace_never_falls(cache):
    for heads in (2, 4, 64):
        last = 0
        for new in (1, 2, 3, 8, 9, 16, 17, 33, 100, 5000):
            need = [_need(5, 5 * new, heads, new, **cache), _need(5, 5 * new + 1, heads, new, **cache), _need(6, 5 * new + 1, heads, new, **cache)]
            assert 0 < last <= need[0] <= need[1] <= need[2] or last == 0
            last = need[2]
        for rows in range(5, 300, 7):
            assert _need(5, rows, heads, 0, **cache) >= _need(5, rows - 1, heads, 0, **cache) > 0
    assert _need(5, 5, 3, **cache) == 0 and _need(-1, 5, **cache) == 0 and _need(5, -1, **cache) == 0 and _need(5, 5, 4, -1, **cache) == 0
    assert _need(5, 1 << 30, 64, **cache) == 0 and _need(5, 5, head_dim=96) == 0


@pytest.mark.parametrize("rot", [2, 4, 64, 128, 1024])
@pytest.mark.parametrize("kw", [dict(), dict(base=500000.0), dict(scaling=1, factor=4.0), dict(scaling=2, factor=8.0), dict(scaling=3, factor=16.0, original_len=4096.0),
                                dict(scaling=3, factor=2.0, original_len=512.0, low=0.5, high=4.0)])
def test_frequencies_against_the_oracle(rot, kw):
    B = _lib()
    if kw.get("scaling") == 2 and rot < 4:
        with pytest.raises(B.PcmError):
            B.grpo_rotary_freqs(rot, **kw)
        return
    turns, amplitude = B.grpo_rotary_freqs(rot, **kw)
    theta, want = ro.frequencies(rot, **kw)
    assert turns.dtype == torch.float64 and turns.shape == (rot // 2,)
    assert np.allclose(turns.numpy() * 2 * np.pi, theta, rtol=1e-13, atol=0) and abs(amplitude - want) <= 2.0 ** -23 * want


@pytest.mark.parametrize("kw,code", [(dict(rot_dim=0), SHAPE), (dict(rot_dim=7), SHAPE), (dict(rot_dim=1026), SHAPE), (dict(rot_dim=-2), SHAPE), (dict(base=0.0), ARG),
                                     (dict(base=INF), ARG), (dict(scaling=4), ARG), (dict(scaling=-1), ARG), (dict(scaling=1, factor=0.5), ARG),
                                     (dict(scaling=1, factor=NAN), ARG), (dict(scaling=3, factor=2.0), ARG),
                                     (dict(scaling=3, factor=2.0, original_len=10.0, low=3.0, high=3.0), ARG)])
def test_frequencies_that_are_refused(kw, code):
    B = _lib()
    with pytest.raises(B.PcmError) as e:
        B.grpo_rotary_freqs(**dict(dict(rot_dim=64), **kw))
    assert e.value.code == code


def test_binding_refuses_host_tensors_and_sizes_that_do_not_fit():
    B = _lib()
    x, pos, pages = torch.zeros(3, 2, 64), torch.zeros(3, dtype=torch.int32), torch.zeros(4, 16, 2, 64)
    table = torch.zeros(3, 2, dtype=torch.int32)
    for f in (lambda: B.grpo_rotary(x, pos, torch.zeros(8, dtype=torch.float64)), lambda: B.grpo_rotary_cache(x, x, x, pages, pages, table, pos, None, None),
              lambda: B.grpo_paged_attention(x, pages, pages, table, pos), lambda: B.grpo_paged_attention_workspace_bytes(pages, 1, 1, 2)):
        with pytest.raises(B.PcmError) as e:
            f()
        assert e.value.code == ARG
    for f in (lambda: B.grpo_paged_attention_workspace_bytes(pages, 1 << 32, 1, 2), lambda: B.grpo_rotary_freqs((1 << 32) + 64)):
        with pytest.raises(B.PcmError) as e:
            f()
        assert e.value.code == SHAPE


def test_binding_refuses_what_is_no_tensor():
    B = _lib()
    x, pos, pages = torch.zeros(3, 2, 64), torch.zeros(3, dtype=torch.int32), torch.zeros(4, 16, 2, 64)
    for f in (lambda: B.grpo_rotary(None, pos, None), lambda: B.grpo_rotary_cache(x, x, x, None, pages, pos, pos, None, None),
              lambda: B.grpo_rotary_cache(x, x, x, pages, [1], pos, pos, None, None), lambda: B.grpo_paged_attention(x, None, None, None, None),
              lambda: B.grpo_paged_attention_workspace_bytes(None, 1, 1, 2), lambda: B._sequences("x", None, pos, None, pos.device),
              lambda: B._sequences("x", pos.view(3, 1), None, None, pos.device), lambda: B._turns("x", 0.5, pos.device)):
        with pytest.raises(B.PcmError) as e:
            f()
        assert e.value.code == ARG


def test_structs_have_the_header_s_layout():
    B = _lib()
    assert ctypes.sizeof(B.grpo_rotary_cfg) == 8 + 5 * 8
    assert ctypes.sizeof(B.grpo_kv_cache) == 6 * 4 + 2 * 8 + 3 * 8
    assert ctypes.sizeof(B.grpo_kv_batch) == 8 + 4 * 8


@pytest.mark.parametrize("cache", [dict(ld_slot=64, ld_head=64), dict(ld_head=64, ld_slot=96), dict(ld_page=64), dict(ld_page=16 * 128 - 64), dict(v=P),
                                   dict(ld_head=16 * 64 - 8, ld_slot=64), dict(n_kv_heads=1, ld_page=512, ld_slot=64),
                                   dict(ld_page=1 << 61, ld_slot=1 << 62, ld_head=64)])
def test_a_cache_whose_slots_overlap_is_not_written(cache):
    assert _call("grpo_rotary_cache", cache=cache, **(dict(ld_k=64, ld_v=64) if "n_kv_heads" in cache else {})) == ARG
