"""Sizes that the workspace of a linear layer is asked for: refused where the layer is, however many bits they take."""
import pytest


@pytest.fixture(scope="module")
def cb():
    from paper_2505_07239_b200.build import build_library

    build_library()
    from paper_2505_07239_b200 import binding

    return binding


@pytest.mark.parametrize("at", [0, 1, 2])
@pytest.mark.parametrize("beyond", [1 << 32, 1 << 31, -(1 << 32), 1 << 64])
def test_sizes_beyond_32_bits(cb, at, beyond):
    sizes = [4, 16, 8]
    sizes[at] += beyond                                    # cut to 32 bits it would be the good one, or a negative one
    with pytest.raises(cb.CometError) as e:
        cb.linear_workspace(*sizes)
    assert e.value.code == -2


@pytest.mark.parametrize("sizes", [(0, 16, 8), (-4, 16, 8), (4, 12, 8), (4, 16, 6), ((1 << 20) + 1, 16, 8)])
def test_sizes_that_a_layer_refuses(cb, sizes):
    with pytest.raises(cb.CometError) as e:
        cb.linear_workspace(*sizes)
    assert e.value.code == -2
