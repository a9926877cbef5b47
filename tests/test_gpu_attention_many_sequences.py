"""Linear attention of very many packed sequences: the chunks are found, and the starts checked, with work in step with their number."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import attention  # noqa: E402
from tests.test_gpu_linear import cb  # noqa: E402,F401
from tests.test_gpu_linear_attention import ring_prompt, run_raw  # noqa: E402


def same(got, ref, first=0):
    for name in got:
        for i in (0, 1):
            at = 0 if name in ("s", "S") else first
            assert np.array_equal(got[name][i][at:], ref[name][i][at:]), (name, i)


def check(cb, lengths, C, first=0, **kw):
    case = ring_prompt(51, [first, *(first + np.cumsum(lengths)).tolist()], 1, 1, 4, 2, C, 16, **kw)
    got, flag = run_raw(cb, case)
    assert flag == 0
    same(got, attention.linear_attention(**case), first)


# on both sides of as many as a CTA has threads, and of a multiple of it
@pytest.mark.parametrize("n", [31, 32, 33, 255, 256, 257, 511, 512, 513, 1500])
def test_numbers(cb, n):  # noqa: F811
    check(cb, [(5 * j) % 4 for j in range(n)], 2, first=n % 3)
    check(cb, [0] * (n - 1) + [9], 4)
    check(cb, [9] + [0] * (n - 1), 4)


def test_long_ones_among_many(cb):  # noqa: F811
    """Sequences of hundreds of chunks, which several CTAs list, before, between and behind short and empty ones."""
    check(cb, [700] + [1, 0, 3] * 100 + [1300] + [0] * 50 + [515], 1)
    check(cb, [0] * 300 + [3000] + [0] * 300 + [2], 3, state=False)


@pytest.mark.parametrize("n", [40, 700])
def test_flags(cb, n):  # noqa: F811
    """Starts out of order and another number of chunks, wherever among the sequences."""
    good = ring_prompt(52, list(range(0, 2 * n + 1, 2)), 1, 1, 2, 2, 2, 16)
    ref = attention.linear_attention(**good)
    got, flag = run_raw(cb, good)
    assert flag == 0
    same(got, ref)
    for j in (0, 1, n // 2, n - 1, n):
        starts = list(good["starts"])
        starts[j] = -1 if j == 0 else 2 * n + 1 if j == n else starts[j - 1] - 1
        got, flag = run_raw(cb, dict(good, starts=starts))
        assert flag == 1, j
        for i in (0, 1):                                     # what comes before is as it was, states of what does not count stay
            assert np.array_equal(got["S"][i][:max(0, j - 1)], ref["S"][i][:max(0, j - 1)])
            if j:
                assert np.array_equal(got["S"][i][j - 1], good["state"][i][j - 1])
    for cut in (1, n - 1, n + 3):
        words = lambda p: [np.concatenate([v, v[:3]])[:cut] for v in p]
        got, flag = run_raw(cb, dict(good, dealer=dict(good["dealer"], s=words(good["dealer"]["s"]), dv=words(good["dealer"]["dv"]))))
        assert flag == 1
        there = min(cut, n)
        for i in (0, 1):
            assert np.array_equal(got["s"][i][:there], ref["s"][i][:there]) and (got["s"][i][there:] == 77).all()
            assert np.array_equal(got["S"][i][:there], ref["S"][i][:there]) and np.array_equal(got["S"][i][there:], good["state"][i][there:])


def test_time_in_step_with_the_number(cb):  # noqa: F811
    """Eight times the sequences take eight times as long at most, give or take a factor of two; where every CTA looks through all of
    them it is sixty-four."""
    def time(n):
        gen = torch.Generator(device="cuda").manual_seed(n)
        pair = lambda *s: [torch.randint(-2**63, 2**63 - 1, s, generator=gen, device="cuda", dtype=torch.int64) for _ in (0, 1)]
        row, state = (lambda: pair(n, 1, 2)), (lambda: pair(n, 1, 2, 2))
        dealer = cb.PromptDealer(q=row(), k=row(), v=row(), d=row(), p=pair(n, 1, 1), s=state(), qk=pair(n, 1, 1), pv=row(), qs=row(), dv=state())
        Q, K, V = row(), row(), row()
        starts, decay = torch.arange(n + 1, device="cuda", dtype=torch.int32), torch.ones((1, 2), device="cuda", dtype=torch.int64)
        best = float("inf")
        for _ in range(4):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            cb.linear_attention(Q, K, V, starts, decay, dealer, 16, stream=torch.cuda.current_stream())
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b))
        return best

    few, many = time(8192), time(65536)
    print(f"8192: {few:.3f} ms, 65536: {many:.3f} ms")
    assert many <= 16 * few
