"""Whose expired wait a status word reports: a vocabulary call's own, not what another call left behind on the device."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def B():
    from paper_2605_16154_b200 import binding
    return binding


@pytest.mark.parametrize("n,d,vocab", [(16, 64, 700), (300, 128, 2003), (40, 4096, 300)])
def test_a_report_left_by_another_call_is_not_this_calls(n, d, vocab):
    b = B()
    g = torch.Generator(device="cuda").manual_seed(n)
    x, w = torch.randn(n, d, generator=g, device="cuda").bfloat16(), (torch.randn(vocab, d, generator=g, device="cuda") * 0.1).bfloat16()
    tok = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    a = torch.randn(n, generator=g, device="cuda")
    clean = b.grpo_head_logp(x, w, tok)
    assert b.grpo_gemm_wait_status(1) == 0                       # a wait of some other call expired
    try:
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = b.grpo_head_logp(x, w, tok, status=status)
        assert int(status) == 0
        b.grpo_head_logp_bwd(x, w, tok, got[2], got[1], a, a, status=status)
        assert int(status) == 0
        assert all(torch.equal(p, q) for p, q in zip(got, clean))
        assert b.grpo_gemm_wait_status(1) == 1                   # still there for the one that polls
        with pytest.raises(b.PcmError) as e:
            b.grpo_gemm(x, True, w[:32], True, n, 32, d)
        assert e.value.code == -5
    finally:
        b.grpo_gemm_wait_status(0)
    assert b.grpo_gemm_wait_status(0) == 0
    status.fill_(64)                                             # only OR-ed into
    tok[0] = vocab
    b.grpo_head_logp(x, w, tok, status=status)
    assert int(status) == 64 | 32


def test_a_status_word_costs_no_launch():
    b = B()
    x, w = torch.zeros(200, 64, device="cuda").bfloat16(), torch.zeros(500, 64, device="cuda").bfloat16()
    tok, v = torch.zeros(200, dtype=torch.int32, device="cuda"), torch.zeros(200, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def launches(**kw):
        at = b.pcm_launch_count()
        b.grpo_head_logp(x, w, tok, **kw)
        b.grpo_head_logp_bwd(x, w, tok, v, v, v, **kw)
        return b.pcm_launch_count() - at
    assert launches(status=status) == launches()
