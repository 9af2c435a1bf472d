"""Sizes and factors at the edge of what the vocabulary calls take, on the host: nothing is launched."""
import pytest

from tests.test_vocab_refusals import ARG, EMBED, EMBED_BWD, HEAD, HEAD_BWD, LOGP, LOGP_BWD, SHAPE, _call

WIDE = (1 << 30) + 8


@pytest.mark.parametrize("d", [(1 << 30) + 1, WIDE, 2 ** 31 - 200, 2 ** 31 - 1])
def test_rows_whose_columns_pass_31_bits_are_refused(d):
    """A thread steps through a row's columns in 32 bits: the step behind the last one has to fit too."""
    assert _call("grpo_embed", EMBED, n=1, d=d, ld_table=d, ld_out=d) == SHAPE
    assert _call("grpo_embed", EMBED, n=0, d=1 << 30, ld_table=1 << 30, ld_out=1 << 30) == 0


@pytest.mark.parametrize("d", [WIDE, 2 ** 31 - 8])
def test_hidden_widths_whose_blocks_pass_31_bits_are_refused(d):
    from paper_2605_16154_b200 import binding as B
    for name, base, lead in (("grpo_head_logp", HEAD, {}), ("grpo_head_logp_bwd", HEAD_BWD, dict(ld_dx=d))):
        assert _call(name, base, n_rows=1, d=d, ld_x=d, ld_w=d, vocab=1, **lead) == SHAPE
    assert B.grpo_head_logp_workspace_bytes(1, d, 1) == 0 and B.grpo_head_logp_bwd_workspace_bytes(1, d, 1, 1) == 0


@pytest.mark.parametrize("name,base", [("grpo_token_logp", LOGP), ("grpo_token_logp_bwd", LOGP_BWD), ("grpo_head_logp", HEAD),
                                       ("grpo_head_logp_bwd", HEAD_BWD)])
def test_temperatures_whose_factors_are_infinite_are_refused(name, base):
    """1 / T is finite from 2.94e-39 on, log2(e) / T, which scales the exponents, from 4.24e-39 on."""
    for t in (2.95e-39, 3.5e-39, 4.2e-39, float("inf"), 0.0, -1.0, float("nan")):
        assert _call(name, base, temperature=t, n_rows=0) == ARG
    for t in (4.3e-39, 1e-3, 1.0, 1e30, 3.4028e38):
        assert _call(name, base, temperature=t, n_rows=0, **({"dw": None} if "dw" in base else {})) == 0


def test_flags_of_the_head_gradient():
    from paper_2605_16154_b200 import binding as B
    for flags in (0, B.GRPO_ACCUMULATE, B.GRPO_EXACT_DX, B.GRPO_ACCUMULATE | B.GRPO_EXACT_DX):
        assert _call("grpo_head_logp_bwd", HEAD_BWD, n_rows=0, dw=None, flags=flags) == 0
    for flags in (1, 4, 12, 16, 1 << 31):
        assert _call("grpo_head_logp_bwd", HEAD_BWD, n_rows=0, dw=None, flags=flags) == ARG
    assert _call("grpo_embed_bwd", EMBED_BWD, flags=B.GRPO_EXACT_DX) == ARG


def test_the_binding_refuses_sizes_that_do_not_fit_the_interface():
    """The C interface takes int32: what ctypes would cut to its low half is refused, not computed for another size."""
    from paper_2605_16154_b200 import binding as B
    far = 1 << 32
    for f in (lambda: B.grpo_embed_workspace_bytes(far + 5, 10, 8), lambda: B.grpo_embed_workspace_bytes(5, far + 10, 8),
              lambda: B.grpo_embed_workspace_bytes(5, 10, far + 8), lambda: B.grpo_head_logp_workspace_bytes(far + 5, 64, 100),
              lambda: B.grpo_head_logp_workspace_bytes(5, 64, 100 - far), lambda: B.grpo_head_logp_bwd_workspace_bytes(5, 64, far + 100, 5),
              lambda: B.grpo_head_logp_bwd_workspace_bytes(5, 64, 100, far + 5), lambda: B.grpo_head_logp_bwd_workspace_bytes(5, 64, 100, 1 << 31)):
        with pytest.raises(B.PcmError) as e:
            f()
        assert e.value.code == SHAPE
    assert B.grpo_embed_workspace_bytes(5, 10, 8) > 0 and B.grpo_embed_workspace_bytes(-1, 10, 8) == 0
