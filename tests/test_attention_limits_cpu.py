"""Limits of comet_linear_attention's and comet_linear_attention_step's sizes and strides as the header states them, from both sides: what is
refused for its workspace alone is not refused for its sizes."""
import ctypes

from tests.test_attention_abi_cpu import caller, group_args, prompt_args, step_args
from tests.test_layers_abi_cpu import cb  # noqa: F401

SHAPE, INVALID = -2, -1


def test_sequences_times_heads(cb):  # noqa: F811
    call = caller(cb, lambda c: prompt_args(c, Hq=32, Hk=32), cb.library().comet_linear_attention)
    assert call(sequences=(1 << 19) + 1) == SHAPE
    # at the limit the states, made up for three sequences, would lie on what comes behind them
    assert call(sequences=1 << 19) == INVALID


def test_strides(cb):  # noqa: F811
    prompt = lambda T: caller(cb, lambda c: prompt_args(c, T=T, S=1, chunks=1), cb.library().comet_linear_attention)
    step = lambda B: caller(cb, lambda c: step_args(c, B=B), cb.library().comet_linear_attention_step)
    for name, row in (("q_stride", 24), ("k_stride", 12), ("v_stride", 8)):
        for several, one in ((prompt(4), prompt(1)), (step(4), step(1))):
            for call in (several, one):
                assert call(**{name: -1}) == SHAPE and call(**{name: (1 << 32) + 1}) == SHAPE
            assert several(**{name: row - 1}) == SHAPE and several(**{name: 0}) == SHAPE
        # one token has no next one: its stride may be anything, and the call goes on to the next check
        one = caller(cb, lambda c: prompt_args(c, T=1, S=1, chunks=1), cb.library().comet_linear_attention)
        assert one(**{name: 0, "workspace_bytes": 64}) == SHAPE and one(**{name: 0, "Eq": (0, None)}) == INVALID


def test_workspace_of_the_norm_needs_no_device(cb):  # noqa: F811
    out = ctypes.c_int64(-1)
    call = cb.library().comet_group_norm_workspace
    assert call(1, 1 << 14, 1, 1, ctypes.byref(out)) == 0 and out.value == 0
    assert call(3, 1 << 14, 10, 5, ctypes.byref(out)) == 0 and out.value == 3 * 5 * 32
    assert group_args(cb).workspace % 256 == 0
