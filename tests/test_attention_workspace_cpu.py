"""What comet_linear_attention_workspace reports: room that goes by the tokens there are, not by whole chunks for each of the chunks."""
import ctypes

import pytest

from tests.test_layers_abi_cpu import cb  # noqa: F401


def workspace(cb, tokens, chunks, Hq, Hk, Dk, Dv, C):
    out = ctypes.c_int64()
    assert cb.library().comet_linear_attention_workspace(tokens, chunks, Hq, Hk, Dk, Dv, C, ctypes.byref(out)) == 0
    return out.value


def words(tokens, chunks, Hq, Hk, Dk, Dv, C):
    """Of the values that are cut into planes and of the sums: q, k, d, v, P and the states."""
    return tokens * (Hq * (Dk + C) + Hk * (2 * Dk + Dv)) + chunks * Hk * Dk * Dv, 2 * chunks * Hk * Dk * Dv


HEADS = [(8, 8, 32, 32), (32, 8, 128, 128), (5, 1, 2, 30)]


@pytest.mark.parametrize("Hq,Hk,Dk,Dv", HEADS)
@pytest.mark.parametrize("C", [32, 64])
def test_whole_chunks_take_their_words(cb, Hq, Hk, Dk, Dv, C):  # noqa: F811
    """Rows are whole sixteens and blocks whole ones, but for head sizes: 24 bytes a word, 8 a sum, 16 a chunk."""
    n = 37
    up = lambda d, to: -(-d // to) * to
    planes, sums = words(n * C, n, Hq, Hk, up(Dk, 32), up(Dv, 16), C)
    d = n * C * Hk * (up(Dk, 32) - up(Dk, 16))               # (of d k_dim is rows, rounded up to 16)
    assert workspace(cb, n * C, n, Hq, Hk, Dk, Dv, C) <= 24 * (planes - d) + 8 * sums + 16 * n + 512


@pytest.mark.parametrize("Hq,Hk,Dk,Dv", HEADS)
@pytest.mark.parametrize("length", [1, 3, 17, 40])
def test_short_sequences(cb, Hq, Hk, Dk, Dv, length):  # noqa: F811
    """A chunk that is not whole takes the rows and blocks of its tokens.  The weights alone have two blocks a row where a whole chunk has."""
    n = 5000
    up = lambda d, to: -(-d // to) * to
    rows, blocks = up(length + 15, 16), up(length + 31, 32)
    planes, sums = words(rows * n, n, Hq, 0, up(Dk, 32), 0, 64)[0] + n * Hk * (rows * up(Dk, 32) + blocks * (up(Dk, 16) + up(Dv, 16)) + up(Dk, 32) * up(Dv, 16)), 2 * n * Hk * Dk * Dv
    assert workspace(cb, n * length, n, Hq, Hk, Dk, Dv, 64) <= 24 * planes + 8 * sums + 16 * n + 512


def test_sizes_that_fit_a_device(cb):  # noqa: F811
    """Prompts of one token each.  65536 of 8 heads of 32 have 48 GB of arguments and results; 4096 of 32 on 8 heads of 128 have 32."""
    assert workspace(cb, 65536, 65536, 8, 8, 32, 32, 64) < 80e9
    assert workspace(cb, 4096, 4096, 32, 8, 128, 128, 64) < 40e9


def test_no_more_than_whole_chunks(cb):  # noqa: F811
    for tokens in (1, 63, 64, 65, 1000, 1 << 20):
        for C in (1, 16, 33, 64):
            assert workspace(cb, tokens, 9, 4, 2, 64, 48, C) <= workspace(cb, 9 * C, 9, 4, 2, 64, 48, C)
    assert workspace(cb, 9, 9, 4, 2, 64, 48, 64) < workspace(cb, 300, 9, 4, 2, 64, 48, 64) < workspace(cb, 576, 9, 4, 2, 64, 48, 64)
