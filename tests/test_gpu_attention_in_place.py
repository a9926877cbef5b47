"""A prompt's states replaced in place through the C ABI, and what the Python call makes of a flag and of no chunks."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import attention  # noqa: E402
from tests.test_gpu_linear import cb, host  # noqa: E402,F401
from tests.test_gpu_linear_attention import OnGpu, compare, ring_prompt, ring_step  # noqa: E402


def call(cb, c, state_out, stream=None, zero=0):
    """comet_linear_attention into new memory but for the states: (messages and O by name, everything it needs to stay alive)."""
    (T, Hq, Dk), (_, Hk, Dv) = c["Q"][0].shape, c["V"][0].shape
    C, n = c["decay"].shape[1] - 1, c["dealer"].s[0].shape[0]
    a = cb.CometLinearAttentionArgs()
    a.tokens, a.sequences, a.q_heads, a.kv_heads, a.k_dim, a.v_dim, a.chunk, a.chunks, a.frac_bits = T, len(c["starts"]) - 1, Hq, Hk, Dk, Dv, C, n, c["frac_bits"]
    a.q_stride, a.k_stride, a.v_stride, a.zero_unwritten = Hq * Dk, Hk * Dk, Hk * Dv, zero
    m = c["dealer"]
    out = {k: [torch.empty_like(t) for t in p] for k, p in dict(q=m.q, k=m.k, v=m.v, d=m.d, p=m.p, s=m.s, O=m.qs).items()}
    pairs = dict({k: c[k] for k in "QKV"}, **{"m" + k if len(k) == 1 else k: p for k, p in m._asdict().items()},
                 **{"O" if k == "O" else "E" + k: p for k, p in out.items()}, state=c["state"], state_out=state_out)
    for name, p in pairs.items():
        setattr(a, name, (ctypes.c_void_p * 2)(*(t.data_ptr() for t in p)))
    a.starts, a.decay = c["starts"].data_ptr(), c["decay"].data_ptr()
    need = ctypes.c_int64()
    assert cb.library().comet_linear_attention_workspace(T, n, Hq, Hk, Dk, Dv, C, ctypes.byref(need)) == 0
    room = torch.empty(need.value // 8 + 1, dtype=torch.int64, device="cuda")
    a.workspace, a.workspace_bytes = room.data_ptr(), need.value
    stream = stream or torch.cuda.current_stream()
    assert cb.library().comet_linear_attention(ctypes.c_void_p(stream.cuda_stream), ctypes.byref(a)) == 0
    return out, (a, room, pairs)


# sequences of several chunks, of one, of none; sizes that fill no sixteen, no block
@pytest.mark.parametrize("starts,Hq,Hk,Dk,Dv,C", [([0, 100, 100, 107, 240], 2, 1, 34, 30, 32), ([0, 0, 65], 3, 3, 130, 2, 64), ([0, 33, 70, 71], 4, 2, 64, 144, 16), ([0, 9], 1, 1, 2, 2, 1)])
def test_prompt_in_place(cb, starts, Hq, Hk, Dk, Dv, C):  # noqa: F811
    case = ring_prompt(71, starts, Hq, Hk, Dk, Dv, C, 16)
    ref = attention.linear_attention(**case)
    c = OnGpu(cb)(case)
    out, keep = call(cb, c, c["state"])
    torch.cuda.synchronize()
    for i in (0, 1):
        assert np.array_equal(host(c["state"][i]), ref["S"][i])
        for name, p in out.items():
            assert np.array_equal(host(p[i]), ref[name][i]), name


def test_prompt_in_place_again_and_again(cb):  # noqa: F811
    """Captured once, replayed: every replay goes on from the states that the one before left."""
    case = ring_prompt(72, [0, 40, 40, 110], 2, 2, 32, 32, 32, 16)
    c = OnGpu(cb)(case)
    call(cb, dict(c, state=[t.clone() for t in c["state"]]), [torch.empty_like(t) for t in c["state"]])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, keep = call(cb, c, c["state"])
    state = case["state"]
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        ref = attention.linear_attention(**dict(case, state=state))
        state = ref["S"]
        for i in (0, 1):
            assert np.array_equal(host(c["state"][i]), state[i]) and np.array_equal(host(out["O"][i]), ref["O"][i])


def test_one_party_s_state_in_place_is_refused(cb):  # noqa: F811
    c = OnGpu(cb)(ring_prompt(73, [0, 9], 1, 1, 4, 4, 4, 16))
    with pytest.raises(AssertionError):
        call(cb, c, [c["state"][0], torch.empty_like(c["state"][1])])
    with pytest.raises(AssertionError):
        call(cb, c, c["state"][::-1])


@pytest.mark.parametrize("n,flagged", [(3, True), (4, False), (5, True)])
def test_flag_in_python(cb, n, flagged):  # noqa: F811
    case = ring_prompt(74, [0, 10, 20], 2, 1, 8, 6, 8, 16)
    words = lambda p: [np.concatenate([v, v[:1]])[:n] for v in p]
    c = OnGpu(cb)(dict(case, dealer=dict(case["dealer"], s=words(case["dealer"]["s"]), dv=words(case["dealer"]["dv"]))))
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = cb.linear_attention(**c, bad_starts_flag=flag)
    assert int(flag) == flagged
    if n == 4:
        compare(got, attention.linear_attention(**case))
    cb.linear_attention(**OnGpu(cb)(case), bad_starts_flag=flag)
    assert int(flag) == flagged                              # the caller clears it


def test_no_chunks_in_python(cb):  # noqa: F811
    case = ring_prompt(75, [4, 4, 4], 2, 1, 8, 8, 16, 16, tokens=6)
    compare(cb.linear_attention(**OnGpu(cb)(case)), attention.linear_attention(**case))
    compare(cb.linear_attention(**OnGpu(cb)(dict(case, state=None))), attention.linear_attention(**dict(case, state=None)))


def test_a_prompt_s_states_go_on_token_by_token_and_back(cb):  # noqa: F811
    """Prompt, token, prompt on the same states, each replaced in place."""
    first, last = ring_prompt(76, [0, 70, 75], 2, 2, 16, 24, 64, 16), ring_prompt(77, [0, 3, 40], 2, 2, 16, 24, 16, 16)
    step = ring_step(78, 2, 2, 2, 16, 24, 16)
    c = OnGpu(cb)(first)
    held = [call(cb, c, c["state"])]
    msg, O, S = cb.linear_attention_step(**dict(OnGpu(cb)(step), state=c["state"]))
    d = dict(OnGpu(cb)(last), state=S)
    held.append(call(cb, d, S))
    torch.cuda.synchronize()
    one = attention.linear_attention(**first)
    two = attention.linear_attention_step(**dict(step, state=one["S"]))
    three = attention.linear_attention(**dict(last, state=two["S"]))
    for i in (0, 1):
        assert np.array_equal(host(O[i]), two["O"][i]) and np.array_equal(host(S[i]), three["S"][i])
        assert np.array_equal(host(held[1][0]["O"][i]), three["O"][i])
