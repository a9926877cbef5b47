"""Refusals of comet_linear and comet_norm_rotate, which come before any CUDA call: addresses here are made up and never read."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def cb():
    from paper_2505_07239_b200.build import build_library

    build_library()
    from paper_2505_07239_b200 import binding

    return binding


class Places:
    """Disjoint made-up addresses, 16-byte aligned."""

    def __init__(self):
        self.next = 1 << 40

    def pair(self, words):
        out = []
        for _ in (0, 1):
            out.append(self.next)
            self.next += (words * 8 + 4095) // 4096 * 4096 + 4096
        return (ctypes.c_void_p * 2)(*out)


def linear_args(cb, T=4, K=16, N=8, quadratic=1, f=16):
    at = Places()
    a = cb.CometLinearArgs()
    a.tokens, a.inner, a.cols, a.frac_bits, a.quadratic = T, K, N, f, quadratic
    for name, words in (("X", T * K), ("A", T * K), ("E", T * K), ("W", N * K), ("B", N * K), ("F", N * K), ("C", T * N), ("Y", T * N),
                        ("R", T * N), ("Q", T * N), ("M", T * N), ("residual", T * N), ("bias", N)):
        setattr(a, name, at.pair(words))
    return a


def test_linear_refusals(cb):
    lib = cb.library()

    def call(**kw):
        a = linear_args(cb)
        for name, v in kw.items():
            if isinstance(v, tuple):                        # (party, address)
                getattr(a, name)[v[0]] = v[1]
            else:
                setattr(a, name, v)
        return lib.comet_linear(None, ctypes.byref(a))

    good = linear_args(cb)
    assert lib.comet_linear(None, None) == -1
    for name in ("X", "A", "W", "B", "C", "E", "F", "Y", "R", "Q", "M", "bias", "residual"):
        for p in (0, 1):
            assert call(**{name: (p, None)}) == -1, name
            assert call(**{name: (p, getattr(good, name)[p] + 8)}) == -1, name              # 16-byte accesses
    for name in ("E", "F", "M", "Y"):                        # results on the memory of another argument
        for other in ("X", "A", "W", "B", "C", "R", "Q", "bias", "residual", "E", "F", "M", "Y"):
            if other != name:
                assert call(**{name: (1, getattr(good, other)[0])}) == -1, (name, other)
    assert call(quadratic=2) == -1
    assert call(workspace=ctypes.c_void_p((1 << 50) + 64)) == -1
    assert call(workspace=ctypes.c_void_p(good.X[0]), workspace_bytes=256) == -1
    assert call(workspace=ctypes.c_void_p(1 << 50), workspace_bytes=-8) == -1
    for kw in (dict(tokens=0), dict(tokens=-3), dict(inner=12), dict(inner=0), dict(cols=6), dict(cols=2), dict(frac_bits=0),
               dict(frac_bits=32), dict(tokens=(1 << 20) + 1), dict(inner=(1 << 20) + 8), dict(cols=(1 << 20) + 4),
               dict(tokens=1 << 20, inner=1 << 20, cols=1 << 20)):
        assert call(**kw) == -2, kw
    assert lib.comet_linear_workspace(4, 16, 8, None) == -1
    out = ctypes.c_int64()
    assert lib.comet_linear_workspace(4, 12, 8, ctypes.byref(out)) == -2


def norm_args(cb, T=3, H=4, D=8, steps=5, rot=8):
    at = Places()
    a = cb.CometNormRotateArgs()
    a.tokens, a.heads, a.q_heads, a.dim, a.x_stride, a.frac_bits, a.steps = T, H, 2, D, H * D, 16, steps
    a.guess, a.eps, a.rot_dim, a.interleaved, a.table_rows = 1 << 15, 1, rot, 0, 16
    n = T * H * D
    for name, words in (("X", n), ("U", n), ("UV", n), ("A", n), ("C", n), ("M", n), ("D", n), ("Z", n),
                        ("row_words", T * H * (6 * steps - 3)), ("S", T * H * (3 * steps - 1)), ("gain", 2 * D),
                        ("gain_mask", 2 * D), ("G", 2 * D)):
        setattr(a, name, at.pair(words))
    a.cos, a.sin = at.pair(16 * rot // 2)
    a.positions, a.bad_index_flag = at.pair(T)
    return a


def test_norm_rotate_refusals(cb):
    lib = cb.library()

    def call(**kw):
        a = norm_args(cb)
        for name, v in kw.items():
            if isinstance(v, tuple):
                getattr(a, name)[v[0]] = v[1]
            else:
                setattr(a, name, v)
        return lib.comet_norm_rotate(None, ctypes.byref(a))

    good = norm_args(cb)
    assert lib.comet_norm_rotate(None, None) == -1
    pairs = ("X", "U", "UV", "A", "C", "M", "D", "Z", "row_words", "S", "gain", "gain_mask", "G")
    for name in pairs:
        for p in (0, 1):
            assert call(**{name: (p, None)}) == -1, name
            assert call(**{name: (p, getattr(good, name)[p] + 4)}) == -1, name              # not even a word
    for name in ("cos", "sin", "positions"):
        assert call(**{name: None}) == -1, name
        assert call(**{name: getattr(good, name) + 2}) == -1, name
    for name in ("M", "D", "Z", "S", "G"):
        for other in pairs:
            if other != name:
                assert call(**{name: (0, getattr(good, other)[1])}) == -1, (name, other)
        assert call(**{name: (0, good.positions)}) == -1 and call(**{name: (0, good.cos)}) == -1
    assert call(bad_index_flag=good.Z[0]) == -1
    assert call(steps=0, rot_dim=0) == -1                                                   # nothing to do
    assert call(steps=0) == -1                                                              # a gain without a norm
    assert call(interleaved=2) == -1
    for kw in (dict(tokens=0), dict(heads=0), dict(dim=7), dict(dim=0), dict(dim=8194), dict(x_stride=31), dict(x_stride=-32),
               dict(x_stride=(1 << 32) + 1), dict(q_heads=5), dict(q_heads=-1), dict(rot_dim=3), dict(rot_dim=10), dict(rot_dim=-2),
               dict(table_rows=0), dict(steps=1), dict(steps=25), dict(steps=-4), dict(guess=0), dict(guess=1 << 32),
               dict(frac_bits=0), dict(frac_bits=32), dict(tokens=1 << 26, heads=4)):
        assert call(**kw) == -2, kw


def test_python_refusals(cb):
    import torch

    def words(*shape):
        return [torch.zeros(shape, dtype=torch.int64) for _ in (0, 1)]

    with pytest.raises(AssertionError):                      # not on a GPU
        cb.linear(words(2, 8), words(2, 8), words(4, 8), words(4, 8), words(2, 4), 16)
    with pytest.raises(AssertionError):
        cb.norm_rotate(words(2, 3, 8), 16, rotation=cb.Rotation(*words(4, 4), torch.zeros(2, dtype=torch.int32)))
