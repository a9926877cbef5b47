"""`zero_unwritten` of comet_linear_attention: neither 0 nor 1 is refused."""
from tests.test_attention_abi_cpu import caller, prompt_args
from tests.test_layers_abi_cpu import cb  # noqa: F401


def test_refusals(cb):  # noqa: F811
    call = caller(cb, prompt_args, cb.library().comet_linear_attention)
    for value in (-1, 2, 1 << 16):
        assert call(zero_unwritten=value) == -1
    assert call(zero_unwritten=1, workspace_bytes=64) == -2  # (on to the next check)
