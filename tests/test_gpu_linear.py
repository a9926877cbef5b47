"""GPU parity of the shared linear layer (comet_linear) with the CPU oracle, word for word."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import layers  # noqa: E402
from paper_2505_07239_b200 import workloads as wl  # noqa: E402


@pytest.fixture(scope="module")
def cb():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2505_07239_b200 import binding

    return binding


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int64)).cuda()


def host(t):
    return t.cpu().numpy().view(np.uint64)


def words(seed, name, *shape):
    return wl.random_u64(seed, name, int(np.prod(shape))).reshape(shape)


def ring_case(seed, T, K, N, f, bias, act, residual):
    """Uniform words everywhere: an additive share is one whatever it stands for, and the words of the result do not depend
    on the triple being one."""
    pair = lambda name, *shape: [words(seed, f"{name}{i}", *shape) for i in (0, 1)]
    k = tuple(int(v) - (1 << 62) for v in words(seed, "k", 3) >> np.uint64(1)) if act == "wild" else (1 << (f - 1), -(1 << f >> 2), 1 << f >> 3)
    return dict(X=pair("X", T, K), A=pair("A", T, K), W=pair("W", N, K), B=pair("B", N, K), C=pair("C", T, N), frac_bits=f,
                bias=pair("b", N) if bias else None, act=(k, pair("R", T, N), pair("Q", T, N)) if act else None,
                residual=pair("r", T, N) if residual else None)


def on_gpu(case):
    up = lambda p: None if p is None else [dev(v) for v in p]
    out = {k: up(case[k]) for k in ("X", "A", "W", "B", "C", "bias", "residual")}
    out["act"] = None if case["act"] is None else (case["act"][0], up(case["act"][1]), up(case["act"][2]))
    return dict(out, frac_bits=case["frac_bits"])


def compare(got, ref):
    E, F, M, Y = got
    assert (M is None) == ("M" not in ref)
    for name, pair in (("E", E), ("F", F), ("M", M), ("Y", Y)):
        for i in (0, 1):
            if pair is not None:
                assert np.array_equal(host(pair[i]), ref[name][i]), (name, i)


_product = {}


def oracle_linear(case, key):
    """The oracle's product is the slow part and the same for every combination of a shape's parts."""
    if key not in _product:
        t = lambda p: [np.ascontiguousarray(v.T) for v in p]
        _product[key] = layers.pi_matmul(case["X"], t(case["W"]), case["A"], t(case["B"]), case["C"])
    keep, layers.pi_matmul = layers.pi_matmul, lambda *_: _product[key]
    try:
        return layers.linear(**case)
    finally:
        layers.pi_matmul = keep


# one row to a few (the streaming kernel, tiles of 32 and of 128 features), up to 64 on either side of its line, planes of limbs,
# planes of residues from either side (more rows, more features); depths and widths that no tile divides
SHAPES = [(1, 8, 4), (1, 768, 768), (7, 40, 132), (16, 256, 96), (17, 520, 36), (32, 1024, 4), (32, 2048, 1300),
          (33, 64, 68), (48, 1024, 772), (64, 56, 132), (64, 1032, 764), (65, 8, 4), (65, 1000, 132), (128, 264, 2052),
          (129, 776, 324), (203, 1000, 364), (512, 1024, 1024), (300, 1992, 1388), (257, 2048, 2052), (1100, 1024, 516)]


@pytest.mark.parametrize("T,K,N", SHAPES)
def test_shapes_match_the_oracle(cb, T, K, N):
    f = (12, 13, 16)[(T + N) % 3]
    case = ring_case(T * 7 + N, T, K, N, f, bias=True, act=True, residual=True)
    compare(cb.linear(**on_gpu(case)), layers.linear(**case))
    assert cb.static_status() == 0


# one to four rows, in one launch or not: blocks of one feature and of several, a second round of blocks, a ragged last one; a
# contraction index of one pair and more, slices with and without words, one chunk and more, lanes and chunks not filled
FEW = [(1, 8, 8192), (1, 8, 8196), (1, 40, 4), (1, 64, 4800), (1, 72, 9600), (1, 96, 148), (1, 136, 152), (1, 200, 596), (1, 392, 36),
       (1, 768, 1188), (1, 1000, 68), (1, 1792, 20), (1, 1800, 148), (1, 3592, 12), (1, 4096, 300), (1, 4104, 8), (2, 8, 12), (2, 96, 8200),
       (2, 192, 296), (2, 904, 44), (2, 1024, 1024), (2, 1024, 1028), (2, 1032, 8), (3, 8, 4), (3, 64, 2048), (3, 392, 180), (3, 512, 256),
       (3, 520, 8), (4, 16, 8), (4, 200, 640), (4, 384, 340), (4, 512, 100), (4, 256, 516)]


@pytest.mark.parametrize("T,K,N", FEW)
def test_few_rows(cb, T, K, N):
    case = ring_case(T * 5 + N, T, K, N, (12, 13, 16)[N % 3], bias=True, act=True, residual=True)
    compare(cb.linear(**on_gpu(case)), layers.linear(**case))
    bare = dict(case, bias=None, act=None, residual=None)
    compare(cb.linear(**on_gpu(bare)), layers.linear(**bare))


def test_few_rows_behind_one_another_and_replayed(cb):
    """The product of each call reads what the call before wrote."""
    f, seed = 16, 8
    sizes = [(2, 264, 520), (2, 520, 520), (2, 520, 100)]
    cases = [ring_case(seed + k, *s, f, True, "tame", False) for k, s in enumerate(sizes)]
    gpu = [on_gpu(c) for c in cases]

    def chain(stream):
        x, out = gpu[0]["X"], []
        for g in gpu:
            out.append(cb.linear(**dict(g, X=x), stream=stream))
            x = out[-1][3]
        return out

    graph = torch.cuda.CUDAGraph()
    chain(None)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        captured = chain(torch.cuda.current_stream())
    eager = chain(None)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for k, c in enumerate(cases):
        ref = layers.linear(**c)
        compare(eager[k], ref)
        compare(captured[k], ref)
        if k + 1 < len(cases):
            cases[k + 1]["X"] = ref["Y"]


@pytest.mark.parametrize("T,K,N", [(1, 264, 36), (2, 64, 36), (4, 128, 36), (5, 64, 36), (64, 72, 68), (90, 264, 132), (512, 1024, 1028)])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("act", [None, "tame", "wild"])
@pytest.mark.parametrize("residual", [False, True])
def test_every_combination_of_parts(cb, T, K, N, bias, act, residual):
    case = ring_case(31, T, K, N, 16, bias, act, residual)
    compare(cb.linear(**on_gpu(case)), oracle_linear(case, (T, K, N)))


@pytest.mark.parametrize("f", [1, 31])
def test_smallest_and_largest_fixed_point(cb, f):
    for T, K, N in ((3, 16, 8), (70, 40, 20)):
        case = ring_case(f, T, K, N, f, True, "wild", True)
        compare(cb.linear(**on_gpu(case)), layers.linear(**case))


def test_extreme_words(cb):
    """All-ones words, the sign bit and zeros: what the kernels accumulate is largest there.  A product of constant matrices is
    one number."""
    for T, K, N in ((20, 512, 132), (70, 512, 132), (512, 1024, 1024)):
        case = ring_case(2, T, K, N, 16, True, "tame", True)
        for value in (0xFFFFFFFFFFFFFFFF, 1 << 63, 0):
            for name in ("X", "W", "A", "B"):
                case[name] = [np.full_like(case[name][i], value if name in "XW" or i else 0) for i in (0, 1)]
            one = {name: [v[0, 0] for v in case[name]] for name in ("X", "W", "A", "B")}
            with np.errstate(over="ignore"):
                E = [one["X"][i] - one["A"][i] for i in (0, 1)]
                F = [one["W"][i] - one["B"][i] for i in (0, 1)]
                e, f = E[0] + E[1], F[0] + F[1]
                Z = [case["C"][i] + np.uint64(K) * (e * one["B"][i] + one["A"][i] * f + (e * f if i else np.uint64(0))) for i in (0, 1)]
            known = {"Z": Z, "E": [np.full((T, K), v) for v in E], "F": [np.full((K, N), v) for v in F]}
            keep, layers.pi_matmul = layers.pi_matmul, lambda *_: known
            try:
                ref = layers.linear(**case)
            finally:
                layers.pi_matmul = keep
            compare(cb.linear(**on_gpu(case)), ref)


def test_depth_beyond_the_residues(cb):
    """Deeper than the residues' number system holds: the product goes through limbs, in several segments."""
    case = ring_case(4, 70, 17000, 40, 16, True, None, True)
    compare(cb.linear(**on_gpu(case)), layers.linear(**case))


def cut(pair, dim, at):
    index = torch.as_tensor(at, device="cuda")
    return [np.ascontiguousarray(host(v.index_select(dim, index))) for v in pair]


@pytest.mark.parametrize("T,K,N", [(512, 2048, 60000), (60000, 2048, 512)])
def test_bands_of_residues(cb, T, K, N):
    """A product that leaves more than the room for residues (1 GiB) behind goes in bands, of features or of rows."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    draw = lambda *s: [torch.randint(-2**63, 2**63 - 1, s, generator=gen, device="cuda", dtype=torch.int64) for _ in (0, 1)]
    X, A, W, B, C, bias, R, Q, res = (draw(T, K), draw(T, K), draw(N, K), draw(N, K), draw(T, N), draw(N), draw(T, N), draw(T, N), draw(T, N))
    k = (3, 5 << 12, 7 << 12)
    E, F, M, Y = cb.linear(X, A, W, B, C, 16, bias=bias, act=(k, R, Q), residual=res)
    assert cb.linear_workspace(T, K, N) > 51 * (N + T) * K            # through residues
    rows = sorted({0, 1, 31, 255, 256, 257, T // 3, T // 2, 8191 % T, 30001 % T, T - 257, T - 256, T - 1})
    cols = sorted({0, 1, 31, 255, 256, 257, N // 3, N // 2, 8191 % N, 30001 % N, N - 257, N - 256, N - 1})
    of = lambda p: cut([torch.as_tensor(v, device="cuda") for v in (x.index_select(0, torch.as_tensor(rows, device="cuda")) for x in p)], 1, cols)
    ref = layers.linear(cut(X, 0, rows), cut(A, 0, rows), cut(W, 0, cols), cut(B, 0, cols), of(C), 16, bias=cut(bias, 0, cols),
                        act=(k, of(R), of(Q)), residual=of(res))
    for i in (0, 1):
        assert np.array_equal(of(Y)[i], ref["Y"][i]) and np.array_equal(of(M)[i], ref["M"][i])
        assert np.array_equal(cut(F, 0, cols)[i], ref["F"][i]) and np.array_equal(cut(E, 0, rows)[i], ref["E"][i])


def test_another_stream_and_calls_behind_one_another(cb):
    """Calls of all three kernels on a stream of the caller's, nothing waited for in between, workspaces handed on."""
    cases = [ring_case(50 + k, *s, 16, True, "tame", True) for k, s in enumerate(((9, 64, 36), (90, 264, 132), (512, 1024, 1024), (80, 128, 68)))]
    gpu = [on_gpu(c) for c in cases]
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    got = [[cb.linear(**g, stream=stream) for g in gpu] for _ in range(3)]
    stream.synchronize()
    refs = [layers.linear(**c) for c in cases]
    for results in got:
        for result, ref in zip(results, refs):
            compare(result, ref)
    assert cb.static_status(stream) == 0


def test_calls_on_two_streams_at_once(cb):
    """No memory is shared between calls: two streams at once, each with its own workspaces, give the same words."""
    cases = [ring_case(60 + k, *s, 16, True, "tame", True) for k, s in enumerate(((9, 64, 36), (90, 264, 132), (512, 1024, 1024)))]
    gpu, refs = [on_gpu(c) for c in cases], [layers.linear(**c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[cb.linear(**g, stream=streams[(k + j) % 2]) for j, g in enumerate(gpu)] for k in range(4)]
    torch.cuda.synchronize()
    for results in got:
        for result, ref in zip(results, refs):
            compare(result, ref)


@pytest.mark.parametrize("T,K", [(1, 264), (9, 64), (90, 264), (512, 1024)])
def test_one_tensor_in_several_places(cb, T, K):
    """What is only read may be given twice: the input as the residual, the product's share as the square's mask, one tensor as both
    parties' bias, the weights as their own masks (the messages are zero then)."""
    case = ring_case(70, T, K, K, 16, True, "tame", True)
    k, _, Q = case["act"]
    case.update(residual=case["X"], B=case["W"], bias=[case["bias"][0]] * 2, act=(k, case["C"], Q))
    gpu = on_gpu(case)
    gpu.update(residual=gpu["X"], B=gpu["W"], bias=[gpu["bias"][0]] * 2, act=(k, gpu["C"], gpu["act"][2]))
    got = cb.linear(**gpu)
    compare(got, layers.linear(**case))
    assert not any(v.any() for v in got[1])


@pytest.mark.parametrize("T,K,N", [(1, 768, 300), (9, 64, 36), (90, 264, 132), (512, 1024, 1024)])
def test_captured_and_replayed(cb, T, K, N):
    case, other = ring_case(3, T, K, N, 13, True, "tame", True), ring_case(4, T, K, N, 13, True, "tame", True)
    g, g_other = on_gpu(case), on_gpu(other)
    ref_of = {id(c): layers.linear(**c) for c in (case, other)}
    cb.linear(**g)
    torch.cuda.synchronize()
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = cb.linear(**g, stream=torch.cuda.current_stream())
    with torch.cuda.graph(second):                         # a second capture, alive at the same time
        got2 = cb.linear(**g, stream=torch.cuda.current_stream())
    for source in (case, other, case):
        fresh = on_gpu(source)
        for name in ("X", "A", "W", "B", "C", "bias", "residual"):
            for i in (0, 1):
                g[name][i].copy_(fresh[name][i])
        for j in (1, 2):
            for i in (0, 1):
                g["act"][j][i].copy_(fresh["act"][j][i])
        graph.replay()
        second.replay()
        eager = cb.linear(**g_other)                        # an eager call between replays
        graph.replay()
        torch.cuda.synchronize()
        compare(got, ref_of[id(source)])
        compare(got2, ref_of[id(source)])
        compare(eager, ref_of[id(other)])


def test_agrees_with_the_calls_that_it_replaces(cb):
    """The product through a context with every neuron active, the bias at scale 2f, the truncation."""
    T, d, D, f = 100, 128, 192, 16
    case = ring_case(77, T, d, D, f, True, None, False)
    ctx = cb.Comet(T, d, D, 16, f)
    try:
        ctx.set_mask(np.ones(D // 16, np.uint8))
        g = on_gpu(case)
        for p in (0, 1):
            for tid, name in ((cb.X, "X"), (cb.W1, "W"), (cb.A_UP, "A"), (cb.B_UP, "B"), (cb.C_UP, "C")):
                ctx.load_shares(p, tid, g[name][p])
        ctx.ffn_up(T)
        view = [ctx.result_view(p, cb.Z_UP, (T, D)) for p in (0, 1)]
        ctx.synchronize()
        cb.add_bias(view, [b << f for b in g["bias"]])
        torch.cuda.synchronize()
        ctx.truncate(cb.Z_UP)
        E, F, M, Y = cb.linear(**g)
        for p in (0, 1):
            assert np.array_equal(ctx.get(p, cb.Z_UP, (T, D)), host(Y[p]))
            assert np.array_equal(ctx.get(p, cb.E_UP, (T, d)), host(E[p]))
            assert np.array_equal(ctx.get(p, cb.F_UP, (D, d)), host(F[p]))
    finally:
        ctx.close()


@pytest.mark.parametrize("T", [1, 8])
def test_words_beyond_32_bits(cb, T):
    """More than 2^31 weights.  Both parties' shares and masks of W are the same words of one buffer, 16 words apart."""
    K, N = 4096, 528000
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB of device memory")
    gen = torch.Generator(device="cuda").manual_seed(3)
    draw = lambda *s: torch.randint(-2**63, 2**63 - 1, s, generator=gen, device="cuda", dtype=torch.int64)
    room = draw(N * K + 48)
    W0, W1, B0, B1 = (room[k:k + N * K].view(N, K) for k in (0, 16, 32, 48))
    X, A, C = ([draw(T, K), draw(T, K)], [draw(T, K), draw(T, K)], [draw(T, N), draw(T, N)])
    E, F, M, Y = cb.linear(X, A, [W0, W1], [B0, B1], C, 16)
    cols = [0, 1, 127, N // 2, (1 << 31) // K - 1, (1 << 31) // K, (1 << 31) // K + 1, N - 2, N - 1]
    ref = layers.linear([host(v) for v in X], [host(v) for v in A], cut([W0, W1], 0, cols), cut([B0, B1], 0, cols), cut(C, 1, cols), 16)
    for i in (0, 1):
        assert np.array_equal(cut(Y, 1, cols)[i], ref["Y"][i])
        assert np.array_equal(cut(F, 0, cols)[i], ref["F"][i])


def test_refusals_on_a_device(cb):
    lib = cb.library()
    t = lambda *s: [torch.zeros(s, dtype=torch.int64, device="cuda") for _ in (0, 1)]
    good = [t(8, 16), t(8, 16), t(12, 16), t(12, 16), t(8, 12)]
    with pytest.raises(AssertionError):
        cb.linear(*good[:4], t(8, 8), 16)
    with pytest.raises(AssertionError):
        cb.linear(*good, 16, bias=t(8))
    with pytest.raises(AssertionError):
        cb.linear([v.t() for v in t(16, 8)], *good[1:], 16)                  # strides that are not the documented ones
    with pytest.raises(AssertionError):
        cb.linear([v.double() for v in good[0]], *good[1:], 16)
    with pytest.raises(TypeError):
        cb.linear(*good, 16, act=(t(8, 12), t(8, 12)))
    for bad in (lambda: cb.linear(*good, 0), lambda: cb.linear(*good, 32), lambda: cb.linear(t(8, 12), t(8, 12), t(12, 12), t(12, 12), good[4], 16),
                lambda: cb.linear(t(0, 16), t(0, 16), *good[2:4], t(0, 12), 16)):
        with pytest.raises(cb.CometError) as e:
            bad()
        assert e.value.code == -2
    # a workspace that is too small, or none
    T, K, N = 512, 1024, 1024
    need = cb.linear_workspace(T, K, N)
    a = cb.CometLinearArgs()
    a.tokens, a.inner, a.cols, a.frac_bits = T, K, N, 16
    keep = []
    for name, shape in (("X", (T, K)), ("A", (T, K)), ("E", (T, K)), ("W", (N, K)), ("B", (N, K)), ("F", (N, K)), ("C", (T, N)), ("Y", (T, N))):
        pair = t(*shape)
        keep.append(pair)
        setattr(a, name, (ctypes.c_void_p * 2)(pair[0].data_ptr(), pair[1].data_ptr()))
    torch.cuda.synchronize()
    assert lib.comet_linear(None, ctypes.byref(a)) == -1
    room = torch.empty(need, dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = room.data_ptr(), need - 1
    assert lib.comet_linear(None, ctypes.byref(a)) == -2
    a.workspace_bytes = need
    assert lib.comet_linear(None, ctypes.byref(a)) == 0
    torch.cuda.synchronize()
    assert cb.linear_workspace(1, K, N) == 0 and cb.static_status() == 0


def test_a_wait_that_ran_out_is_reported(cb):
    """The word that a kernel of comet_linear sets is the one that static_status reads."""
    torch.cuda.synchronize()
    assert cb.static_status() == 0
    assert cb.library().comet_static_inject_timeout(None) == 0
    assert cb.static_status() == cb.ERR_TIMEOUT and cb.static_status() == 0
