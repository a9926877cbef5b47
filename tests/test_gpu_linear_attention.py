"""GPU parity of linear attention on shares (comet_linear_attention, comet_linear_attention_step) with the CPU oracle, word for word."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import attention  # noqa: E402
from tests.test_gpu_linear import cb, dev, host, words  # noqa: E402,F401
from tests.test_oracle_attention import prompt_case, step_case  # noqa: E402

PROMPT_SHAPES = dict(q="Q", k="K", v="V", d="K")


def pair(seed, name, *shape):
    return [words(seed, f"{name}{i}", *shape) for i in (0, 1)]


def ring_prompt(seed, starts, Hq, Hk, Dk, Dv, C, f, state=True, tokens=None):
    """Uniform words everywhere: what the words of a result are does not depend on the dealer's products being products."""
    T = starts[-1] if tokens is None else tokens
    n = sum(max(0, b - a + C - 1) // C for a, b in zip(starts, starts[1:]))
    q, k, v, p, o, s = (T, Hq, Dk), (T, Hk, Dk), (T, Hk, Dv), (T, Hq, C), (T, Hq, Dv), (n, Hk, Dk, Dv)
    dealer = {name: pair(seed, "m" + name, *shape) for name, shape in zip(("q", "k", "v", "d", "p", "s", "qk", "pv", "qs", "dv"), (q, k, v, k, p, s, p, o, o, s))}
    return dict(Q=pair(seed, "Q", *q), K=pair(seed, "K", *k), V=pair(seed, "V", *v), starts=list(starts), decay=words(seed, "w", Hk, C + 1),
                dealer=dealer, frac_bits=f, state=pair(seed, "S", len(starts) - 1, Hk, Dk, Dv) if state else None)


def ring_step(seed, B, Hq, Hk, Dk, Dv, f, state=True):
    q, k, v, o, s = (B, Hq, Dk), (B, Hk, Dk), (B, Hk, Dv), (B, Hq, Dv), (B, Hk, Dk, Dv)
    dealer = {name: pair(seed, "m" + name, *shape) for name, shape in zip(("q", "k", "v", "s", "kv", "qs"), (q, k, v, s, s, o))}
    return dict(Q=pair(seed, "Q", *q), K=pair(seed, "K", *k), V=pair(seed, "V", *v), decay=words(seed, "w", Hk), dealer=dealer, frac_bits=f,
                state=pair(seed, "S", *s) if state else None)


class OnGpu:
    """Moves a case to the GPU: Q, K, V as views whose rows lie `pad` words further apart, every tensor `shift` words into its memory."""

    def __init__(self, cb, pad=0, shift=0):
        self.cb, self.pad, self.shift = cb, pad, shift

    def up(self, a):
        if a.size == 0:
            return dev(a)
        t = torch.zeros(a.size + self.shift, dtype=torch.int64, device="cuda")[self.shift:].view(a.shape)
        t.copy_(dev(a))
        return t

    def rows(self, a):
        T, H, D = a.shape
        room = torch.zeros(T * (H * D + self.pad) + self.shift, dtype=torch.int64, device="cuda")
        view = torch.as_strided(room, (T, H, D), (H * D + self.pad, D, 1), self.shift)
        view.copy_(dev(a))
        return view

    def __call__(self, case):
        pairs = lambda p: None if p is None else [self.up(v) for v in p]
        out = {k: [self.rows(v) for v in case[k]] for k in "QKV"}
        kind = self.cb.PromptDealer if "starts" in case else self.cb.StepDealer
        out.update(decay=self.up(case["decay"]), dealer=kind(**{k: pairs(v) for k, v in case["dealer"].items()}), frac_bits=case["frac_bits"],
                   state=pairs(case["state"]))
        if "starts" in case:
            out["starts"] = torch.tensor(case["starts"], dtype=torch.int32, device="cuda")
        return out


def compare(got, ref, rows=None):
    """rows: the tokens that are in a sequence."""
    msg, O, S = got
    for name, p in (*msg._asdict().items(), ("O", O), ("S", S)):
        for i in (0, 1):
            a, b = host(p[i]), ref[name][i]
            if rows is not None and name not in ("s", "S"):
                a, b = a[rows], b[rows]
            assert np.array_equal(a, b), (name, i, np.argwhere(a != b)[:4])


def check_prompt(cb, case, **kw):
    compare(cb.linear_attention(**OnGpu(cb, **kw)(case)), attention.linear_attention(**case))


def check_step(cb, case, **kw):
    compare(cb.linear_attention_step(**OnGpu(cb, **kw)(case)), attention.linear_attention_step(**case))


# lengths of one token, of a chunk, around its tiles, of several chunks, none at all, packed
STARTS = [[0, 1], [0, 16], [0, 31], [0, 32], [0, 33], [0, 63], [0, 64], [0, 65], [0, 129], [0, 0, 5], [0, 7, 7, 7, 40], [0, 1, 2, 3, 4, 5, 6, 7, 8, 9],
          [0, 64, 65, 129, 192], [0, 100, 101]]


@pytest.mark.parametrize("starts", STARTS, ids=str)
@pytest.mark.parametrize("C", [64, 33])
def test_lengths(cb, starts, C):  # noqa: F811
    check_prompt(cb, ring_prompt(1, starts, 2, 2, 16, 24, C, 16))


@pytest.mark.parametrize("C", [1, 2, 3, 8, 15, 16, 17, 31, 32, 40, 47, 48, 63, 64])
def test_chunks(cb, C):  # noqa: F811
    check_prompt(cb, ring_prompt(C, [0, 50, 53], 2, 1, 12, 8, C, 13))


@pytest.mark.parametrize("Dk,Dv", [(2, 2), (2, 128), (64, 64), (80, 96), (96, 80), (128, 128), (126, 130), (130, 30), (256, 256), (62, 254), (254, 34), (34, 66)])
def test_dims(cb, Dk, Dv):  # noqa: F811
    check_prompt(cb, ring_prompt(Dk + Dv, [0, 70, 75], 2, 1, Dk, Dv, 64, 16))


@pytest.mark.parametrize("Hq,Hk", [(1, 1), (5, 5), (8, 2), (7, 1), (12, 12), (33, 3)])
@pytest.mark.parametrize("state", [True, False])
def test_heads(cb, Hq, Hk, state):  # noqa: F811
    check_prompt(cb, ring_prompt(Hq, [0, 9, 42], Hq, Hk, 32, 16, 32, 12, state))


@pytest.mark.parametrize("f", [1, 12, 31])
@pytest.mark.parametrize("pad,shift", [(0, 0), (2, 0), (3, 0), (64, 2), (0, 1), (5, 3)])
def test_fixed_point_strides_and_alignment(cb, f, pad, shift):  # noqa: F811
    check_prompt(cb, ring_prompt(f, [0, 37, 90], 4, 2, 34, 40, 48, f), pad=pad, shift=shift)
    check_step(cb, ring_step(f, 3, 4, 2, 34, 40, f), pad=pad, shift=shift)


def test_many_sequences(cb):  # noqa: F811
    """More sequences than a CTA has threads, most of them short, some without tokens."""
    lengths = [(7 * j) % 5 for j in range(700)]
    check_prompt(cb, ring_prompt(3, [0, *np.cumsum(lengths).tolist()], 1, 1, 4, 4, 3, 16))


def test_more_chunks_than_the_device_holds_at_once(cb):  # noqa: F811
    check_prompt(cb, ring_prompt(4, [0, 900, 1300], 16, 16, 16, 16, 16, 16))


EXTREMES = [0, 1, (1 << 64) - 1, 1 << 63, 0xFF00FF00FF00FF00, 0x00FF00FF00FF00FF]


@pytest.mark.parametrize("value", EXTREMES, ids=hex)
def test_extreme_words(cb, value):  # noqa: F811
    """All words the same: every sum of byte products at its largest where the bytes are 0xFF."""
    case = ring_prompt(5, [0, 64, 100], 2, 1, 128, 128, 64, 16)
    one = np.uint64(value)
    fill = lambda p: [np.full_like(v, one) for v in p]
    case.update(Q=fill(case["Q"]), K=fill(case["K"]), V=fill(case["V"]), state=fill(case["state"]), decay=np.full_like(case["decay"], one))
    zeros = {k: [np.zeros_like(v) for v in p] for k, p in case["dealer"].items()}
    for dealer in (case["dealer"], zeros, {k: fill(p) for k, p in case["dealer"].items()}):
        check_prompt(cb, dict(case, dealer=dealer))
    step = ring_step(5, 2, 4, 2, 64, 64, 16)
    check_step(cb, dict(step, Q=fill(step["Q"]), K=fill(step["K"]), state=fill(step["state"])))


@pytest.mark.parametrize("B,Hq,Hk,Dk,Dv", [(1, 1, 1, 2, 2), (1, 12, 12, 64, 64), (7, 10, 2, 80, 96), (3, 3, 3, 256, 256), (2, 16, 1, 34, 130), (5, 8, 8, 128, 128),
                                           (2, 33, 1, 16, 6), (1, 5, 1, 250, 2), (40, 6, 3, 2, 254), (300, 2, 2, 16, 16), (9, 4, 4, 62, 66), (1, 9, 3, 128, 128)])
@pytest.mark.parametrize("state", [True, False])
def test_steps(cb, B, Hq, Hk, Dk, Dv, state):  # noqa: F811
    check_step(cb, ring_step(B, B, Hq, Hk, Dk, Dv, 16, state))


def test_real_values(cb):  # noqa: F811
    """The dealer's products are products, the values real numbers."""
    check_prompt(cb, prompt_case(7, [0, 60, 61, 130], 4, 2, 32, 48, 64, 16))
    check_step(cb, step_case(7, 5, 4, 2, 32, 48, 16))


def run_raw(cb, case, fill=None):
    """Through the C ABI into memory that holds known words: (results by name, flag)."""
    c = OnGpu(cb)(case)
    T, Hq, Dk = case["Q"][0].shape
    Hk, Dv, C, n = case["K"][0].shape[1], case["V"][0].shape[2], case["decay"].shape[1] - 1, case["dealer"]["s"][0].shape[0]
    a = cb.CometLinearAttentionArgs()
    a.tokens, a.sequences, a.q_heads, a.kv_heads, a.k_dim, a.v_dim, a.chunk, a.chunks, a.frac_bits = T, len(case["starts"]) - 1, Hq, Hk, Dk, Dv, C, n, case["frac_bits"]
    a.q_stride, a.k_stride, a.v_stride = Hq * Dk, Hk * Dk, Hk * Dv
    keep = []

    def give(name, tensors):
        keep.append(tensors)
        setattr(a, name, (ctypes.c_void_p * 2)(*(t.data_ptr() for t in tensors)))

    for name in "QKV":
        give(name, c[name])
    for name, p in c["dealer"]._asdict().items():
        give("m" + name if len(name) == 1 else name, p)
    if c["state"] is not None:
        give("state", c["state"])
    new = lambda *shape: [torch.full(shape, 77 if fill is None else fill, dtype=torch.int64, device="cuda") for _ in (0, 1)]
    out = dict(q=new(T, Hq, Dk), k=new(T, Hk, Dk), v=new(T, Hk, Dv), d=new(T, Hk, Dk), p=new(T, Hq, C), s=new(n, Hk, Dk, Dv), O=new(T, Hq, Dv),
               S=new(a.sequences, Hk, Dk, Dv))
    for name, p in out.items():
        give({"O": "O", "S": "state_out"}.get(name, "E" + name), p)
    a.starts, a.decay = c["starts"].data_ptr(), c["decay"].data_ptr()
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    a.bad_starts_flag = flag.data_ptr()
    need = ctypes.c_int64()
    assert cb.library().comet_linear_attention_workspace(T, n, Hq, Hk, Dk, Dv, C, ctypes.byref(need)) == 0
    room = torch.zeros(need.value // 8 + 32, dtype=torch.int64, device="cuda")
    a.workspace, a.workspace_bytes = room.data_ptr(), need.value
    stream = torch.cuda.current_stream().cuda_stream
    assert cb.library().comet_linear_attention(ctypes.c_void_p(stream), ctypes.byref(a)) == 0
    torch.cuda.synchronize()
    assert int(cb.static_status()) == 0
    assert not room[need.value // 8:].any()
    return {k: [host(t) for t in p] for k, p in out.items()}, int(flag)


def test_rows_in_no_sequence_stay(cb):  # noqa: F811
    case = ring_prompt(8, [3, 20, 21], 2, 1, 16, 8, 16, 16, tokens=30)
    ref = attention.linear_attention(**case)
    got, flag = run_raw(cb, case)
    assert flag == 0
    for name in got:
        for i in (0, 1):
            if name in ("s", "S"):
                assert np.array_equal(got[name][i], ref[name][i])
            else:
                assert np.array_equal(got[name][i][3:21], ref[name][i][3:21]), name
                assert (got[name][i][:3] == 77).all() and (got[name][i][21:] == 77).all(), name


def test_no_tokens_in_any_sequence(cb):  # noqa: F811
    case = ring_prompt(9, [4, 4, 4], 2, 1, 8, 8, 16, 16, tokens=6)
    got, flag = run_raw(cb, case)
    assert flag == 0
    for i in (0, 1):
        assert np.array_equal(got["S"][i], case["state"][i])
        assert all((got[k][i] == 77).all() for k in ("q", "k", "v", "d", "p", "O"))


def test_starts_out_of_order(cb):  # noqa: F811
    """A sequence whose starts descend or leave the tokens counts as empty; the others are what they are without it."""
    good = ring_prompt(10, [0, 10, 10, 24], 2, 1, 8, 8, 8, 16)
    ref = attention.linear_attention(**good)
    for starts in ([0, 10, 10, 25], [-1, 10, 10, 24], [0, 10, 9, 9]):
        got, flag = run_raw(cb, dict(good, starts=starts))
        assert flag == 1
    # sequences 0 (two chunks) and, of the surplus ones, none
    got, flag = run_raw(cb, dict(good, starts=[0, 10, 10, 25]))
    for i in (0, 1):
        assert np.array_equal(got["O"][i][:10], ref["O"][i][:10]) and (got["O"][i][10:] == 77).all()
        assert np.array_equal(got["S"][i][:2], ref["S"][i][:2]) and np.array_equal(got["S"][i][2], good["state"][i][2])
        assert (got["s"][i][2:] == 77).all()


@pytest.mark.parametrize("n", [1, 3, 4])
def test_another_number_of_chunks(cb, n):  # noqa: F811
    """Two chunks a sequence, four in all; the call says n."""
    case = ring_prompt(11, [0, 10, 20], 1, 1, 8, 8, 8, 16)
    ref = attention.linear_attention(**case)
    cut = dict(case, dealer=dict(case["dealer"], s=[v[:n] for v in case["dealer"]["s"]], dv=[v[:n] for v in case["dealer"]["dv"]]))
    got, flag = run_raw(cb, cut)
    assert flag == (n != 4)
    rows = {1: 8, 3: 18, 4: 20}[n]
    for i in (0, 1):
        assert np.array_equal(got["O"][i][:rows], ref["O"][i][:rows]) and (got["O"][i][rows:] == 77).all()
        assert np.array_equal(got["s"][i], ref["s"][i][:n])


def test_starts_with_more_chunks_than_an_int_counts(cb):  # noqa: F811
    """Starts that go back and forth over 2^20 tokens, chunks of one: 2^31 of them and more, of which four are asked for."""
    T, n, times = 1 << 20, 4, 2100
    case = ring_prompt(9, [0, n], 1, 1, 2, 2, 1, 16, tokens=T)
    ref = attention.linear_attention(**case)
    many = pair(9, "more", 2 * times - 1, 1, 2, 2)
    for i in (0, 1):
        many[i][0] = case["state"][i][0]
    got, flag = run_raw(cb, dict(case, starts=[0, T] * times, state=many))
    assert flag == 1
    for i in (0, 1):
        assert np.array_equal(got["O"][i][:n], ref["O"][i][:n]) and (got["O"][i][n:] == 77).all()
        assert np.array_equal(got["s"][i], ref["s"][i])
        assert np.array_equal(got["S"][i][0], ref["S"][i][0]) and np.array_equal(got["S"][i][1:], many[i][1:])


def test_state_in_place(cb):  # noqa: F811
    case = ring_step(12, 4, 4, 2, 64, 48, 16)
    ref = attention.linear_attention_step(**case)
    c = OnGpu(cb)(case)
    a = cb.CometLinearAttentionStepArgs()
    a.batch, a.q_heads, a.kv_heads, a.k_dim, a.v_dim, a.frac_bits = 4, 4, 2, 64, 48, 16
    a.q_stride, a.k_stride, a.v_stride = 256, 128, 96
    out = {k: [torch.empty_like(t) for t in p] for k, p in dict(Eq=c["Q"], Ek=c["K"], Ev=c["V"], Es=c["state"], O=c["dealer"].qs).items()}
    m = c["dealer"]
    for name, p in dict(out, Q=c["Q"], K=c["K"], V=c["V"], mq=m.q, mk=m.k, mv=m.v, ms=m.s, kv=m.kv, qs=m.qs, state=c["state"], state_out=c["state"]).items():
        setattr(a, name, (ctypes.c_void_p * 2)(*(t.data_ptr() for t in p)))
    a.decay = c["decay"].data_ptr()
    assert cb.library().comet_linear_attention_step(ctypes.c_void_p(torch.cuda.current_stream().cuda_stream), ctypes.byref(a)) == 0
    for i in (0, 1):
        assert np.array_equal(host(c["state"][i]), ref["S"][i]) and np.array_equal(host(out["O"][i]), ref["O"][i])
        assert np.array_equal(host(out["Es"][i]), ref["s"][i])


def test_prompt_then_tokens_in_a_graph(cb):  # noqa: F811
    """A prompt and a token behind it, captured, replayed on other words; eager calls on another stream in between."""
    first, second = (ring_prompt(s, [0, 70, 75], 4, 2, 32, 32, 64, 16) for s in (13, 14))
    steps = [ring_step(s, 2, 4, 2, 32, 32, 16) for s in (15, 16)]
    c, s = OnGpu(cb)(first), OnGpu(cb)(steps[0])
    del s["state"]

    def both(stream):
        one = cb.linear_attention(**c, stream=stream)
        return one, cb.linear_attention_step(**s, state=one[2], stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one, two = both(torch.cuda.current_stream())
    for case, step in ((first, steps[0]), (second, steps[1])):
        with torch.no_grad():
            for name in "QKV":
                for i in (0, 1):
                    c[name][i].copy_(dev(case[name][i]))
                    s[name][i].copy_(dev(step[name][i]))
        eager = both(side)
        graph.replay()
        torch.cuda.synchronize()
        ref = attention.linear_attention(**dict(first, Q=case["Q"], K=case["K"], V=case["V"]))
        after = attention.linear_attention_step(**dict(steps[0], Q=step["Q"], K=step["K"], V=step["V"], state=ref["S"]))
        for o, t in ((one, two), eager):
            compare(o, ref)
            compare(t, after)


def test_two_calls_at_once(cb):  # noqa: F811
    cases = [ring_prompt(20 + j, [0, 150 + j], 8, 4, 64, 64, 64, 16) for j in (0, 1)]
    on = [OnGpu(cb)(c) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = [[cb.linear_attention(**c, stream=s) for _ in range(4)] for c, s in zip(on, streams)]
    torch.cuda.synchronize()
    for case, results in zip(cases, got):
        ref = attention.linear_attention(**case)
        for r in results:
            compare(r, ref)


@pytest.mark.parametrize("starts,Dk,Dv", [([0, 70, 75], 2, 128), ([0, 16], 16, 24), ([0, 1], 2, 2), ([0, 3, 40], 64, 4)])
def test_short_work_again_and_again(cb, starts, Dk, Dv):  # noqa: F811
    """CTAs that are over as soon as their last sums are: what they left to the tensor core has to be over before them."""
    case = ring_prompt(30, starts, 4, 2, Dk, Dv, 64, 16)
    c, ref = OnGpu(cb)(case), attention.linear_attention(**case)
    got = [cb.linear_attention(**c) for _ in range(200)]
    torch.cuda.synchronize()
    for g in got[::20]:
        compare(g, ref)
    assert cb.static_status() == 0


def test_refusals_in_python(cb):  # noqa: F811
    case = OnGpu(cb)(ring_prompt(1, [0, 9], 2, 1, 8, 6, 4, 16))
    with pytest.raises(AssertionError):
        cb.linear_attention(**dict(case, starts=case["starts"].long()))
    with pytest.raises(AssertionError):
        cb.linear_attention(**dict(case, decay=case["decay"][:, 1:]))
    with pytest.raises(AssertionError):
        cb.linear_attention(**dict(case, Q=[v[:, :, ::2] for v in case["Q"]]))
    with pytest.raises(AssertionError):
        cb.linear_attention(**dict(case, state=[v[:, :, 1:] for v in case["state"]]))
    with pytest.raises(cb.CometError):
        cb.linear_attention(**dict(case, frac_bits=32))
    odd = OnGpu(cb)(ring_prompt(1, [0, 9], 2, 1, 7, 6, 4, 16))
    with pytest.raises(cb.CometError):
        cb.linear_attention(**odd)
    step = OnGpu(cb)(ring_step(1, 2, 2, 1, 8, 6, 16))
    with pytest.raises(cb.CometError):
        cb.linear_attention_step(**dict(step, frac_bits=0))
    with pytest.raises(AssertionError):
        cb.linear_attention_step(**dict(step, K=[v[:1] for v in step["K"]]))
