"""Words of linear_attention's results that belong to no token of a sequence or to no chunk: messages leave for the other party, so
nothing that was in their memory before may be in them."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import attention  # noqa: E402
from tests.test_gpu_linear import cb, host  # noqa: E402,F401
from tests.test_gpu_linear_attention import OnGpu, compare, ring_prompt, run_raw  # noqa: E402


def used_memory(cb, c):
    """The call on memory that its allocator has given away before, full of known words."""
    shapes = [t.shape for p in cb.linear_attention(**c)[0] for t in p] + [p[0].shape for p in cb.linear_attention(**c)[1:]]
    for times in range(3):
        held = [torch.full(tuple(s), 0x5A5A5A5A5A5A5A5A, dtype=torch.int64, device="cuda") for s in shapes for _ in (0, 1)]
        held.append(torch.full((sum(t.numel() for t in held),), 0x5A5A5A5A5A5A5A5A, dtype=torch.int64, device="cuda"))
        held += [torch.full((1 << k,), 0x5A5A5A5A5A5A5A5A, dtype=torch.int64, device="cuda") for k in range(6, 18) for _ in range(4)]
        del held
        yield cb.linear_attention(**c)


# tokens before the first sequence, behind the last, in none at all; more of them than a CTA has threads
@pytest.mark.parametrize("starts,tokens,C", [([3, 20, 21], 30, 16), ([0, 9], 2500, 8), ([1200, 1300], 1300, 64), ([0, 0, 40, 40], 41, 33), ([5, 5, 5], 9, 4),
                                             ([1023, 1025, 2049], 2100, 1)])
@pytest.mark.parametrize("Hq,Hk,Dk,Dv", [(2, 1, 16, 8), (3, 3, 6, 34)])
def test_rows_in_no_sequence_are_zero(cb, starts, tokens, C, Hq, Hk, Dk, Dv):  # noqa: F811
    case = ring_prompt(31, starts, Hq, Hk, Dk, Dv, C, 16, tokens=tokens)
    ref = attention.linear_attention(**case)                 # (words that are not written are zero there)
    for got in used_memory(cb, OnGpu(cb)(case)):
        compare(got, ref)


@pytest.mark.parametrize("n", [1, 3, 5, 200])
def test_another_number_of_chunks(cb, n):  # noqa: F811
    """Four chunks, the call says n: rows of those behind it, and states of those that there are not, are zero."""
    case = ring_prompt(32, [0, 10, 20], 2, 1, 8, 6, 8, 16)
    ref = attention.linear_attention(**case)
    words = lambda p: [np.concatenate([v, np.repeat(v[:1], max(0, n - 4), 0)])[:n] for v in p]
    c = OnGpu(cb)(dict(case, dealer=dict(case["dealer"], s=words(case["dealer"]["s"]), dv=words(case["dealer"]["dv"]))))
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    rows = {1: 8, 3: 18}.get(n, 20)
    for msg, O, S in used_memory(cb, dict(c, bad_starts_flag=flag)):
        assert int(flag) == 1
        for name, p in (*msg._asdict().items(), ("O", O)):
            top = min(n, 4) if name == "s" else rows
            for i in (0, 1):
                a = host(p[i])
                assert np.array_equal(a[:top], ref[name][i][:top]) and not a[top:].any(), name


def test_starts_out_of_order(cb):  # noqa: F811
    """Sequences that count as empty: their rows are zero, the other's are not touched."""
    good = ring_prompt(33, [0, 10, 24], 2, 1, 8, 8, 8, 16)
    ref = attention.linear_attention(**good)
    for starts, rows in (([0, 10, 25], slice(0, 10)), ([-1, 10, 24], slice(10, 24)), ([0, 10, 9], slice(0, 10)), ([24, 10, 24], slice(10, 24))):
        for msg, O, S in used_memory(cb, OnGpu(cb)(dict(good, starts=starts))):
            for name, p in (*msg._asdict().items(), ("O", O)):
                if name == "s":
                    continue
                for i in (0, 1):
                    a, want = host(p[i]), np.zeros_like(ref[name][i])
                    if name in "qkv":                        # (what does not depend on the chunk's number)
                        want[rows] = ref[name][i][rows]
                        assert np.array_equal(a, want), (name, starts)
                    else:
                        assert not np.delete(a, np.arange(24)[rows], 0).any(), (name, starts)


def test_no_chunks(cb):  # noqa: F811
    """No token in any sequence, no chunk: there is no workspace and nothing but the states has a value."""
    case = ring_prompt(34, [4, 4, 4], 2, 1, 8, 8, 16, 16, tokens=6)
    ref = attention.linear_attention(**case)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    for got in used_memory(cb, dict(OnGpu(cb)(case), bad_starts_flag=flag)):
        compare(got, ref)
        assert int(flag) == 0
    for got in used_memory(cb, dict(OnGpu(cb)(dict(case, starts=[0, 1, 6])), bad_starts_flag=flag)):
        assert int(flag) == 1
        assert not any(t.any() for p in (*got[0], got[1]) for t in p)
        compare((got[0], got[1], got[2]), ref)


def test_the_caller_s_own_memory_stays(cb):  # noqa: F811
    """Through the C ABI rows in no sequence are the caller's, unless it asks for zeros."""
    case = ring_prompt(35, [3, 20, 21], 2, 1, 16, 8, 16, 16, tokens=30)
    ref = attention.linear_attention(**case)
    kept, _ = run_raw(cb, case)
    for name in kept:
        for i in (0, 1):
            if name not in ("s", "S"):
                assert (kept[name][i][:3] == 77).all() and (kept[name][i][21:] == 77).all(), name
                assert np.array_equal(kept[name][i][3:21], ref[name][i][3:21]), name
