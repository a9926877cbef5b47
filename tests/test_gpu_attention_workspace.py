"""Linear attention of prompts whose chunks are mostly not whole: planes of tokens lie where those of the chunks before end, and nothing is
written behind the bytes that the library asks for."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import attention  # noqa: E402
from tests.test_gpu_linear import cb  # noqa: E402,F401
from tests.test_gpu_linear_attention import ring_prompt, run_raw  # noqa: E402


def same(got, ref, rows=slice(None)):
    for name in got:
        for i in (0, 1):
            a, b = got[name][i], ref[name][i]
            if name not in ("s", "S"):
                a, b = a[rows], b[rows]
            assert np.array_equal(a, b), (name, i, np.argwhere(a != b)[:4])


# every length around the sixteens and blocks once; all of one token; whole chunks but for the last
LENGTHS = [list(range(1, 67)), [1] * 90, [64, 64, 1, 64, 128, 2], [0, 33, 0, 0, 31, 32, 0, 129, 15, 16, 17, 0], [130, 1]]


@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda v: f"{len(v)}-{sum(v)}")
@pytest.mark.parametrize("Hq,Hk,Dk,Dv,C", [(2, 1, 16, 24, 64), (3, 3, 34, 2, 33), (4, 2, 130, 144, 48), (1, 1, 2, 2, 17)])
def test_ragged(cb, lengths, Hq, Hk, Dk, Dv, C):  # noqa: F811
    case = ring_prompt(41 + C, [0, *np.cumsum(lengths).tolist()], Hq, Hk, Dk, Dv, C, 16)
    ref = attention.linear_attention(**case)
    got, flag = run_raw(cb, case)
    assert flag == 0
    same(got, ref)


def test_drawn_lengths(cb):  # noqa: F811
    rng = np.random.default_rng(42)
    for _ in range(12):
        lengths = np.exp(rng.uniform(0, np.log(150), rng.integers(1, 40))).astype(int).tolist()
        Hk, first = int(rng.integers(1, 4)), int(rng.integers(0, 40))
        case = ring_prompt(43, [first, *(first + np.cumsum(lengths)).tolist()], Hk * int(rng.integers(1, 4)), Hk, 2 * int(rng.integers(1, 50)), 2 * int(rng.integers(1, 80)),
                           int(rng.integers(1, 65)), 13)
        got, flag = run_raw(cb, case)
        assert flag == 0
        same(got, attention.linear_attention(**case), slice(first, None))


@pytest.mark.parametrize("times,n", [(3, 100), (3, 120), (2, 100), (1, 40), (40, 1600)])
def test_sequences_that_overlap(cb, times, n):  # noqa: F811
    """Starts that go back: every second sequence counts, over the same forty tokens, in chunks of one.  There is room for what forty tokens can
    be in n chunks, (40 + 15 n) / 16 of sixteen rows and (40 + 31 n) / 32 blocks; the first chunks have it, the others are not worked out."""
    T = 40
    one = ring_prompt(44, [0, T], 2, 1, 8, 6, 1, 16)
    ref = attention.linear_attention(**one)
    room = min(n, (T + 15 * n) // 16, (T + 31 * n) // 32, T * times)
    again = lambda p: [np.concatenate([v] * times + [np.repeat(v[:1], max(0, n - T * times), 0)])[:n] for v in p]
    state = [np.repeat(v, 2 * times - 1, 0) for v in one["state"]]
    case = dict(one, starts=[0, T] * times, state=state, dealer=dict(one["dealer"], s=again(one["dealer"]["s"]), dv=again(one["dealer"]["dv"])))
    got, flag = run_raw(cb, case)
    assert flag == (times > 1)
    part = attention.linear_attention(**dict(one, starts=[0, room % T]))
    for i in (0, 1):
        for j in range(2 * times - 1):
            whole, some = j // 2 < room // T, j // 2 == room // T
            want = state[i][j] if j % 2 or not (whole or some) else ref["S"][i][0] if whole else part["S"][i][0]
            assert np.array_equal(got["S"][i][j], want), j
        assert np.array_equal(got["s"][i][:room], again(ref["s"])[i][:room]) and (got["s"][i][room:] == 77).all()
        for name in "qkvd":
            assert np.array_equal(got[name][i], ref[name][i])


def test_thousands_of_single_tokens(cb):  # noqa: F811
    """Chunks are up to 64 tokens, sequences have one: with room for whole chunks these planes would be 10 GB."""
    n = 6000
    case = ring_prompt(45, list(range(n + 1)), 4, 4, 32, 32, 64, 16)
    ref = attention.linear_attention(**case)
    got, flag = run_raw(cb, case)
    assert flag == 0
    same(got, ref)
