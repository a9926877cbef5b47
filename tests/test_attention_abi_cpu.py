"""Refusals of comet_linear_attention, comet_linear_attention_step and comet_group_norm, which come before any CUDA call: addresses here are
made up and never read."""
import ctypes

import pytest

from tests.test_layers_abi_cpu import Places, cb  # noqa: F401


def prompt_args(cb, T=9, S=3, Hq=4, Hk=2, Dk=6, Dv=4, C=4, chunks=5):
    at = Places()
    a = cb.CometLinearAttentionArgs()
    a.tokens, a.sequences, a.q_heads, a.kv_heads, a.k_dim, a.v_dim, a.chunk, a.chunks, a.frac_bits = T, S, Hq, Hk, Dk, Dv, C, chunks, 16
    a.q_stride, a.k_stride, a.v_stride = Hq * Dk, Hk * Dk, Hk * Dv
    sizes = dict(Q=T * Hq * Dk, K=T * Hk * Dk, V=T * Hk * Dv, mp=T * Hq * C, pv=T * Hq * Dv, ms=chunks * Hk * Dk * Dv, state=S * Hk * Dk * Dv)
    like = dict(mq="Q", mk="K", mv="V", md="K", qk="mp", qs="pv", dv="ms", Eq="Q", Ek="K", Ev="V", Ed="K", Ep="mp", Es="ms", O="pv", state_out="state")
    for name in (*sizes, *like):
        setattr(a, name, at.pair(sizes[like.get(name, name)]))
    a.starts, a.bad_starts_flag = at.pair(S + 1)
    a.decay, _ = at.pair(Hk * (C + 1))
    need = ctypes.c_int64()
    assert cb.library().comet_linear_attention_workspace(T, chunks, Hq, Hk, Dk, Dv, C, ctypes.byref(need)) == 0
    a.workspace, _ = at.pair(need.value // 8)
    a.workspace_bytes = need.value
    return a


def step_args(cb, B=3, Hq=4, Hk=2, Dk=6, Dv=4):
    at = Places()
    a = cb.CometLinearAttentionStepArgs()
    a.batch, a.q_heads, a.kv_heads, a.k_dim, a.v_dim, a.frac_bits = B, Hq, Hk, Dk, Dv, 16
    a.q_stride, a.k_stride, a.v_stride = Hq * Dk, Hk * Dk, Hk * Dv
    sizes = dict(Q=B * Hq * Dk, K=B * Hk * Dk, V=B * Hk * Dv, ms=B * Hk * Dk * Dv, qs=B * Hq * Dv)
    like = dict(mq="Q", mk="K", mv="V", kv="ms", state="ms", Eq="Q", Ek="K", Ev="V", Es="ms", O="qs", state_out="ms")
    for name in (*sizes, *like):
        setattr(a, name, at.pair(sizes[like.get(name, name)]))
    a.decay, _ = at.pair(Hk)
    return a


def group_args(cb, S=2, P=3, C=8, G=2, steps=5):
    at = Places()
    a = cb.CometGroupNormArgs()
    a.samples, a.positions, a.channels, a.groups, a.x_stride, a.frac_bits, a.steps, a.guess, a.eps, a.quadratic = S, P, C, G, C, 16, steps, 1 << 15, 1, 1
    n = S * P * C
    for name, words in (*((k, n) for k in ("X", "U", "UT", "R", "Q", "M", "N", "Z")), ("words", S * G * (6 * steps - 3)), ("S", S * G * (3 * steps - 1)),
                        *((k, C) for k in ("gain", "gain_mask", "bias", "G")), *((k, S * C) for k in ("T", "VW", "D"))):
        setattr(a, name, at.pair(words))
    need = ctypes.c_int64(1 << 20)
    a.workspace, _ = at.pair(need.value // 8)
    a.workspace_bytes = need.value
    return a


def caller(cb, make, call):
    def run(**kw):
        a = make(cb)
        for name, v in kw.items():
            if isinstance(v, tuple):                        # (party, address)
                getattr(a, name)[v[0]] = v[1]
            else:
                setattr(a, name, v)
        return call(None, ctypes.byref(a))
    return run


PROMPT_IN = ("Q", "K", "V", "mq", "mk", "mv", "md", "mp", "ms", "qk", "pv", "qs", "dv")
PROMPT_OUT = ("Eq", "Ek", "Ev", "Ed", "Ep", "Es", "O", "state_out")


def test_prompt_refusals(cb):  # noqa: F811
    lib = cb.library()
    call, good = caller(cb, prompt_args, lib.comet_linear_attention), prompt_args(cb)
    assert lib.comet_linear_attention(None, None) == -1
    for name in PROMPT_IN + PROMPT_OUT:
        for p in (0, 1):
            assert call(**{name: (p, None)}) == -1, name
            assert call(**{name: (p, getattr(good, name)[p] + 4)}) == -1, name
    assert call(state=(0, None)) == -1                       # half a state
    for name in ("starts", "decay", "workspace"):
        assert call(**{name: None}) == -1, name
    assert call(starts=good.starts + 2) == -1 and call(decay=good.decay + 4) == -1 and call(bad_starts_flag=good.bad_starts_flag + 1) == -1
    assert call(workspace=good.workspace + 64) == -1
    for name in PROMPT_OUT:
        for other in PROMPT_IN + PROMPT_OUT + ("state",):
            if other != name:
                assert call(**{name: (0, getattr(good, other)[1])}) == -1, (name, other)
        assert call(**{name: (1, good.workspace)}) == -1 and call(**{name: (1, good.decay)}) == -1 and call(**{name: (0, good.starts)}) == -1
    assert call(state_out=(0, good.state[0])) == -1          # in place for one party alone
    assert call(state_out=(0, good.state[0] + 8)) == -1
    for kw in (dict(tokens=0), dict(sequences=0), dict(chunks=-1), dict(q_heads=0), dict(q_heads=4098), dict(kv_heads=0), dict(kv_heads=3), dict(k_dim=5), dict(k_dim=0),
               dict(k_dim=258), dict(v_dim=3), dict(v_dim=258), dict(chunk=0), dict(chunk=65), dict(q_stride=23), dict(k_stride=11), dict(v_stride=-8),
               dict(q_stride=(1 << 32) + 1), dict(frac_bits=0), dict(frac_bits=32), dict(tokens=(1 << 20) + 1), dict(sequences=(1 << 20) + 1),
               dict(chunks=(1 << 20) + 1), dict(tokens=1 << 20, q_heads=18), dict(chunks=1 << 20, q_heads=18), dict(workspace_bytes=64)):
        assert call(**kw) == -2, kw
    assert lib.comet_linear_attention_workspace(9, 4, 4, 2, 6, 4, 8, None) == -1
    out = ctypes.c_int64()
    assert lib.comet_linear_attention_workspace(9, 4, 4, 2, 7, 4, 8, ctypes.byref(out)) == -2
    assert lib.comet_linear_attention_workspace(9, 4, 4, 2, 6, 4, 65, ctypes.byref(out)) == -2
    assert lib.comet_linear_attention_workspace(9, 0, 4, 2, 6, 4, 8, ctypes.byref(out)) == 0 and out.value == 0


STEP_IN = ("Q", "K", "V", "mq", "mk", "mv", "ms", "kv", "qs")
STEP_OUT = ("Eq", "Ek", "Ev", "Es", "O", "state_out")


def test_step_refusals(cb):  # noqa: F811
    lib = cb.library()
    call, good = caller(cb, step_args, lib.comet_linear_attention_step), step_args(cb)
    assert lib.comet_linear_attention_step(None, None) == -1
    for name in STEP_IN + STEP_OUT:
        for p in (0, 1):
            assert call(**{name: (p, None)}) == -1, name
            assert call(**{name: (p, getattr(good, name)[p] + 4)}) == -1, name
    assert call(state=(1, None)) == -1 and call(decay=None) == -1 and call(decay=good.decay + 4) == -1
    for name in STEP_OUT:
        for other in STEP_IN + STEP_OUT + ("state",):
            if other != name:
                assert call(**{name: (0, getattr(good, other)[1])}) == -1, (name, other)
        assert call(**{name: (1, good.decay)}) == -1
    assert call(state_out=(1, good.state[1])) == -1
    for kw in (dict(batch=0), dict(q_heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(k_dim=5), dict(k_dim=258), dict(v_dim=0), dict(v_dim=258),
               dict(q_stride=23), dict(k_stride=-1), dict(v_stride=(1 << 32) + 1), dict(frac_bits=0), dict(frac_bits=32), dict(batch=(1 << 20) + 1),
               dict(batch=1 << 20, q_heads=18)):
        assert call(**kw) == -2, kw


GROUP_IN = ("X", "U", "UT", "words", "gain", "gain_mask", "bias", "T", "VW", "R", "Q")
GROUP_OUT = ("M", "S", "D", "G", "N", "Z")


def test_group_refusals(cb):  # noqa: F811
    lib = cb.library()
    call, good = caller(cb, group_args, lib.comet_group_norm), group_args(cb)
    assert lib.comet_group_norm(None, None) == -1
    for name in GROUP_IN + GROUP_OUT:
        for p in (0, 1):
            assert call(**{name: (p, None)}) == -1, name
            assert call(**{name: (p, getattr(good, name)[p] + 4)}) == -1, name
    for name in GROUP_OUT:
        for other in GROUP_IN + GROUP_OUT:
            if other != name:
                assert call(**{name: (0, getattr(good, other)[1])}) == -1, (name, other)
        assert call(**{name: (1, good.workspace)}) == -1
    assert call(quadratic=2) == -1 and call(workspace=good.workspace + 8) == -1 and call(workspace_bytes=-8) == -1
    for kw in (dict(samples=0), dict(positions=0), dict(channels=0), dict(groups=0), dict(groups=3), dict(x_stride=7), dict(x_stride=(1 << 32) + 1),
               dict(steps=1), dict(steps=25), dict(guess=0), dict(guess=1 << 32), dict(frac_bits=0), dict(frac_bits=32),
               dict(positions=1 << 23), dict(samples=1 << 24), dict(channels=(1 << 20) + 2)):
        assert call(**kw) == -2, kw
    assert lib.comet_group_norm_workspace(2, 3, 8, 2, None) == -1
    out = ctypes.c_int64()
    assert lib.comet_group_norm_workspace(2, 3, 8, 3, ctypes.byref(out)) == -2


def test_python_refusals(cb):  # noqa: F811
    import torch

    def words(*shape):
        return [torch.zeros(shape, dtype=torch.int64) for _ in (0, 1)]

    with pytest.raises(AssertionError):                      # not on a GPU
        cb.linear_attention(words(3, 2, 4), words(3, 2, 4), words(3, 2, 4), torch.zeros(2, dtype=torch.int32), torch.zeros((2, 5), dtype=torch.int64),
                            cb.PromptDealer(*[words(3, 2, 4)] * 10), 16)
    with pytest.raises(AssertionError):
        cb.linear_attention_step(words(3, 2, 4), words(3, 2, 4), words(3, 2, 4), torch.zeros(2, dtype=torch.int64), None,
                                 cb.StepDealer(*[words(3, 2, 4)] * 6), 16)
    with pytest.raises(AssertionError):
        cb.group_norm(words(3, 2, 4), 2, 16, cb.GroupNorm(words(3, 2, 4), words(3, 2, 9), words(3, 2, 4), 2, 1))
