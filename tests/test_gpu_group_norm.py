"""GPU parity of the norm of channel groups (comet_group_norm) with the CPU oracle, word for word."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import attention  # noqa: E402
from tests.test_gpu_linear import cb, dev, host, words  # noqa: E402,F401
from tests.test_gpu_linear_attention import pair  # noqa: E402
from tests.test_oracle_attention import group_case  # noqa: E402


def ring_group(seed, S, P, C, G, f, steps=3, gained=True, act=True):
    n = (S, P, C)
    case = dict(X=pair(seed, "X", *n), groups=G, frac_bits=f, gain=None, act=None,
                norm=dict(U=pair(seed, "U", *n), words=pair(seed, "w", S, G, 6 * steps - 3), UT=pair(seed, "UT", *n), steps=steps, guess=max(1, int(0.55 * (1 << f))), eps=3))
    if gained:
        case["gain"] = dict(weight=pair(seed, "g", C), mask=pair(seed, "gm", C), T=pair(seed, "T", S, C), VW=pair(seed, "VW", S, C), bias=pair(seed, "b", C))
    if act:
        case["act"] = ((1 << (f - 1), -(1 << f >> 2), 1 << f >> 3), pair(seed, "R", *n), pair(seed, "Q", *n))
    return case


def on_gpu(case, cb, pad=0, shift=0):
    def up(a):
        t = torch.zeros(a.size + shift, dtype=torch.int64, device="cuda")[shift:].view(a.shape)
        t.copy_(dev(a))
        return t

    def rows(a):
        S, P, C = a.shape
        room = torch.zeros(S * P * (C + pad) + shift, dtype=torch.int64, device="cuda")
        view = torch.as_strided(room, (S, P, C), (P * (C + pad), C + pad, 1), shift)
        view.copy_(dev(a))
        return view

    ups = lambda p: [up(v) for v in p]
    n, g = case["norm"], case["gain"]
    return dict(X=[rows(v) for v in case["X"]], groups=case["groups"], frac_bits=case["frac_bits"],
                norm=cb.GroupNorm(ups(n["U"]), ups(n["words"]), ups(n["UT"]), n["steps"], n["guess"], n["eps"]),
                gain=None if g is None else cb.GroupGain(**{k: ups(v) for k, v in g.items()}),
                act=None if case["act"] is None else (case["act"][0], ups(case["act"][1]), ups(case["act"][2])))


def compare(got, ref):
    msg, Z = got
    for name, p in (("Z", Z), *msg._asdict().items()):
        assert (p is None) == (name not in ref), name
        for i in (0, 1):
            if p is not None:
                a = host(p[i])
                assert np.array_equal(a, ref[name][i]), (name, i, np.argwhere(a != ref[name][i])[:4])


def check(cb, case, **kw):
    compare(cb.group_norm(**on_gpu(case, cb, **kw)), attention.group_norm(**case))


# groups of one word to more than a CTA's, of neighbours that fill no access, one position and many
@pytest.mark.parametrize("S,P,C,G", [(1, 1, 1, 1), (1, 1, 2, 1), (3, 1, 5, 5), (1, 1, 768, 12), (7, 1, 96, 3), (2, 1, 1300, 1), (1, 1, 4100, 1), (1, 1, 9001, 1),
                                     (65, 1, 64, 4), (2, 3, 6, 3), (3, 77, 90, 5), (1, 1000, 8, 4), (2, 64, 320, 32), (1, 257, 33, 1), (5, 2, 7, 7), (1, 4096, 4, 1),
                                     (1, 5000, 1, 1), (2, 16, 1024, 2), (1, 3, 20000, 4), (1, 130, 640, 32), (600, 1, 12, 4), (1, 30000, 2, 1), (1, 20000, 6, 2)])
def test_shapes(cb, S, P, C, G):  # noqa: F811
    check(cb, ring_group(S + P, S, P, C, G, 16))


@pytest.mark.parametrize("gained", [True, False])
@pytest.mark.parametrize("act", [True, False])
@pytest.mark.parametrize("pad,shift", [(0, 0), (2, 0), (3, 0), (64, 2), (0, 1), (5, 3)])
@pytest.mark.parametrize("S,P,C,G", [(9, 1, 48, 4), (2, 40, 24, 4), (2, 33, 30, 2), (1, 700, 40, 2)])
def test_parts_strides_and_alignment(cb, gained, act, pad, shift, S, P, C, G):  # noqa: F811
    check(cb, ring_group(C, S, P, C, G, 16, 4, gained, act), pad=pad, shift=shift)


@pytest.mark.parametrize("steps", [2, 3, 12, 24])
@pytest.mark.parametrize("f", [1, 12, 31])
def test_steps_and_fixed_point(cb, steps, f):  # noqa: F811
    for S, P, C, G in ((5, 1, 64, 2), (2, 50, 24, 3), (1, 3000, 8, 2)):
        check(cb, ring_group(steps, S, P, C, G, f, steps))


def test_real_values(cb):  # noqa: F811
    check(cb, group_case(3, 40, 1, 256, 4, 16, 12))
    check(cb, group_case(4, 2, 100, 60, 3, 13, 12))


def test_any_words(cb):  # noqa: F811
    for value in (0, (1 << 64) - 1, 1 << 63):
        case = ring_group(5, 2, 30, 12, 3, 16)
        case["X"] = [np.full_like(v, np.uint64(value)) for v in case["X"]]
        check(cb, case)
        case["norm"]["U"] = [np.full_like(v, np.uint64(value)) for v in case["norm"]["U"]]
        check(cb, case)


@pytest.mark.parametrize("S,P,C,G", [(30, 1, 128, 4), (2, 60, 24, 4), (1, 6000, 16, 2)])
def test_captured_and_on_two_streams(cb, S, P, C, G):  # noqa: F811
    first, second = ring_group(21, S, P, C, G, 16), ring_group(22, S, P, C, G, 16)
    c = on_gpu(first, cb)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    cb.group_norm(**c, stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = cb.group_norm(**c, stream=torch.cuda.current_stream())
    for case in (first, second):
        for i in (0, 1):
            c["X"][i].copy_(dev(case["X"][i]))
        torch.cuda.synchronize()
        other = cb.group_norm(**c, stream=side)
        graph.replay()
        torch.cuda.synchronize()
        ref = attention.group_norm(**dict(first, X=case["X"]))
        compare(kept, ref)
        compare(other, ref)


def test_refusals_in_python(cb):  # noqa: F811
    c = on_gpu(ring_group(1, 2, 3, 8, 2, 16), cb)
    with pytest.raises(AssertionError):
        cb.group_norm(**dict(c, X=[v.transpose(1, 2) for v in c["X"]]))
    with pytest.raises(AssertionError):
        cb.group_norm(**dict(c, X=[v[:, ::2] for v in c["X"]]))
    with pytest.raises(AssertionError):
        cb.group_norm(**dict(c, groups=4))                   # the words of two groups
    with pytest.raises(cb.CometError):
        cb.group_norm(**dict(c, groups=0))
    with pytest.raises(cb.CometError):
        cb.group_norm(**dict(c, frac_bits=0))
    with pytest.raises(cb.CometError):
        cb.group_norm(**dict(c, norm=c["norm"]._replace(guess=0)))
