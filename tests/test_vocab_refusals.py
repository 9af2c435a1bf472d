"""Arguments that the vocabulary calls refuse, through the C ABI and the binding.  Every case is turned down on the host
before anything is launched, so the addresses below are never used and no GPU is needed."""
import ctypes

import pytest
import torch

ARG, SHAPE, WORKSPACE = -1, -2, -3
P = 1 << 20                                   # an aligned address that nothing reads
NAN, INF = float("nan"), float("inf")


def _call(name, base, **change):
    from paper_2605_16154_b200 import binding as B
    args = dict(base)
    assert set(change) <= set(args)
    args.update(change)
    return getattr(B._lib, name)(*args.values())


EMBED = dict(dtype=1, table=P, ld_table=64, vocab=100, d=64, tok=P, n=5, scale=1.0, out=P, ld_out=64, status=None, stream=None)
EMBED_BWD = dict(dtype=1, dout=P, ld_dout=64, tok=P, n=5, vocab=100, d=64, scale=1.0, flags=0, grad=P, status=None, workspace=P,
                 workspace_bytes=1 << 30, stream=None)
LOGP = dict(dtype=1, logits=P, ld=100, n_rows=5, vocab=100, tok=P, temperature=1.0, top=4, logp=P, entropy=P, lse=P, top_id=P,
            top_logp=P, status=None, stream=None)
LOGP_BWD = dict(dtype=1, logits=P, ld=100, n_rows=5, vocab=100, tok=P, temperature=1.0, lse=P, entropy=P, dlogp=P, dentropy=P,
                dlogits=2 * P, ld_dlogits=100, status=None, stream=None)

HEAD = dict(x=P, ld_x=64, n_rows=5, d=64, w=P, ld_w=64, vocab=100, tok=P, temperature=1.0, logp=P, entropy=P, lse=P, status=None,
            workspace=P, workspace_bytes=1 << 30, stream=None)
HEAD_BWD = dict(x=P, ld_x=64, n_rows=5, d=64, w=P, ld_w=64, vocab=100, tok=P, temperature=1.0, lse=P, entropy=P, dlogp=P, dentropy=P,
                chunk_rows=5, flags=0, dx=P, ld_dx=64, dw=P, status=None, workspace=P, workspace_bytes=1 << 30, stream=None)

CASES = [
    ("grpo_head_logp", HEAD, [
        (dict(x=None), ARG), (dict(w=None), ARG), (dict(tok=None), ARG), (dict(x=P + 8), ARG), (dict(w=P + 2), ARG), (dict(n_rows=-1), ARG),
        (dict(d=0), ARG), (dict(vocab=0), ARG), (dict(ld_x=56), ARG), (dict(ld_w=8), ARG), (dict(temperature=0.0), ARG),
        (dict(temperature=NAN), ARG), (dict(n_rows=1 << 30, vocab=1 << 30), SHAPE), (dict(d=60), SHAPE), (dict(ld_x=68), SHAPE), (dict(ld_w=65), SHAPE), (dict(workspace=None), WORKSPACE),
        (dict(workspace=P + 128), WORKSPACE), (dict(workspace_bytes=64), WORKSPACE)]),
    ("grpo_head_logp_bwd", HEAD_BWD, [
        (dict(x=None), ARG), (dict(w=None), ARG), (dict(tok=None), ARG), (dict(lse=None), ARG), (dict(dlogp=None), ARG),
        (dict(entropy=None), ARG), (dict(dx=None, dw=None), ARG), (dict(dx=P + 8), ARG), (dict(dw=P + 4), ARG), (dict(ld_dx=56), ARG),
        (dict(chunk_rows=0), ARG), (dict(flags=6), ARG), (dict(temperature=-2.0), ARG), (dict(d=12), SHAPE), (dict(ld_dx=70), SHAPE),
        (dict(workspace_bytes=1 << 10), WORKSPACE), (dict(workspace=P + 8), WORKSPACE)]),
    ("grpo_embed", EMBED, [
        (dict(dtype=2), ARG), (dict(dtype=-1), ARG), (dict(table=None), ARG), (dict(tok=None), ARG), (dict(out=None), ARG),
        (dict(n=-1), ARG), (dict(vocab=0), ARG), (dict(d=0), ARG), (dict(ld_table=63), ARG), (dict(ld_out=63), ARG),
        (dict(scale=NAN), ARG), (dict(scale=INF), ARG), (dict(table=P + 1), ARG), (dict(dtype=0, out=P + 2), ARG),
        (dict(n=(1 << 30) + 1), SHAPE), (dict(vocab=(1 << 30) + 1), SHAPE)]),
    ("grpo_embed_bwd", EMBED_BWD, [
        (dict(dtype=7), ARG), (dict(dout=None), ARG), (dict(tok=None), ARG), (dict(grad=None), ARG), (dict(n=-3), ARG),
        (dict(vocab=0), ARG), (dict(d=-1), ARG), (dict(ld_dout=1), ARG), (dict(scale=INF), ARG), (dict(flags=1), ARG),
        (dict(grad=P + 2), ARG), (dict(d=70000, ld_dout=70000), SHAPE), (dict(n=2 ** 31 - 1), SHAPE), (dict(workspace=None), WORKSPACE),
        (dict(workspace=P + 64), WORKSPACE), (dict(workspace_bytes=1000), WORKSPACE)]),
    ("grpo_token_logp", LOGP, [
        (dict(dtype=3), ARG), (dict(logits=None), ARG), (dict(n_rows=-1), ARG), (dict(vocab=0, top=0), ARG), (dict(ld=99), ARG),
        (dict(temperature=0.0), ARG), (dict(temperature=-1.0), ARG), (dict(temperature=NAN), ARG), (dict(temperature=INF), ARG),
        (dict(temperature=1e-42), ARG), (dict(tok=None), ARG), (dict(top=-1), ARG), (dict(top=17), SHAPE),
        (dict(vocab=3, top=4), SHAPE), (dict(vocab=2 ** 31 - 1, ld=2 ** 31), SHAPE), (dict(top_id=None), ARG), (dict(top_logp=None), ARG), (dict(logits=P + 1), ARG),
        (dict(dtype=0, logits=P + 2), ARG)]),
    ("grpo_token_logp_bwd", LOGP_BWD, [
        (dict(dtype=3), ARG), (dict(logits=None), ARG), (dict(tok=None), ARG), (dict(lse=None), ARG), (dict(dlogp=None), ARG),
        (dict(dlogits=None), ARG), (dict(entropy=None), ARG), (dict(ld=99), ARG), (dict(ld_dlogits=50), ARG),
        (dict(temperature=0.0), ARG), (dict(temperature=NAN), ARG), (dict(n_rows=-1), ARG), (dict(vocab=-2), ARG),
        (dict(dlogits=P, ld_dlogits=104), ARG), (dict(n_rows=2 ** 31 - 1), SHAPE), (dict(dlogits=P + 1), ARG)]),
]


@pytest.mark.parametrize("name,base,change,code", [(n, b, c, e) for n, b, cs in CASES for c, e in cs],
                         ids=lambda v: v if isinstance(v, str) else "-".join(v) if isinstance(v, dict) and len(v) < 5 else "")
def test_the_call_refuses(name, base, change, code):
    assert _call(name, base, **change) == code


@pytest.mark.parametrize("name,base,change", [
    ("grpo_embed", EMBED, dict(n=0, table=None, out=None, tok=None)), ("grpo_token_logp", LOGP, dict(n_rows=0, logits=None, tok=None)),
    ("grpo_token_logp_bwd", LOGP_BWD, dict(n_rows=0, logits=None, dlogits=None))])
def test_no_rows_is_a_valid_call(name, base, change):
    assert _call(name, base, **change) == 0


def test_workspace_sizes():
    from paper_2605_16154_b200 import binding as B
    assert B.grpo_embed_workspace_bytes(-1, 10, 8) == 0 and B.grpo_embed_workspace_bytes(5, 0, 8) == 0
    assert B.grpo_embed_workspace_bytes(5, 10, 70000) == 0
    small, large = B.grpo_embed_workspace_bytes(1, 2, 1), B.grpo_embed_workspace_bytes(119808, 32000, 1024)
    assert 0 < small < large
    # two buffers of (token, position) pairs, and two partial rows for every 64 sorted rows
    assert B.grpo_head_logp_workspace_bytes(5, 12, 100) == 0 and B.grpo_head_logp_bwd_workspace_bytes(5, 16, 100, 0) == 0
    assert B.grpo_head_logp_workspace_bytes(1000, 64, 129) >= 2 * 16 * 1000
    assert B.grpo_head_logp_bwd_workspace_bytes(100, 64, 500, 10) < B.grpo_head_logp_bwd_workspace_bytes(100, 64, 500, 100)
    assert B.grpo_head_logp_bwd_workspace_bytes(100, 64, 500, 100) == B.grpo_head_logp_bwd_workspace_bytes(100, 64, 500, 1000)
    assert large >= 2 * 8 * 119808 + 2 * 4 * 1024 * 119808 // 64


def test_binding_refuses_host_tensors():
    from paper_2605_16154_b200 import binding as B
    t, tok = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32)
    for f in (lambda: B.grpo_embed(t, tok), lambda: B.grpo_embed_bwd(t, tok, 10), lambda: B.grpo_token_logp(t, tok),
              lambda: B.grpo_token_logp_bwd(t, tok, t[:, 0], t[:, 0], t[:, 0])):
        with pytest.raises(B.PcmError) as e:
            f()
        assert e.value.code == ARG
