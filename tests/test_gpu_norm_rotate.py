"""GPU parity of the norm, gain and rotation of shared heads (comet_norm_rotate) with the CPU oracle, word for word."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import layers  # noqa: E402
from paper_2505_07239_b200 import workloads as wl  # noqa: E402
from tests.test_gpu_linear import cb, dev, host, words  # noqa: E402,F401
from tests.test_oracle_layers import float_norm_rotate, norm_case  # noqa: E402


def on_gpu(case, cb, pad=0, shift=0):
    """The case on the GPU: X as a view whose tokens lie `pad` words further apart, every tensor `shift` words into its memory."""
    def up(a):
        room = torch.zeros(a.size + shift, dtype=torch.int64, device="cuda")
        t = room[shift:].view(a.shape)
        t.copy_(dev(a))
        return t

    def rows(a):
        T, H, D = a.shape
        room = torch.zeros(T * (H * D + pad) + shift, dtype=torch.int64, device="cuda")
        view = torch.as_strided(room, (T, H, D), (H * D + pad, D, 1), shift)
        view.copy_(dev(a))
        return view

    out = dict(X=[rows(v) for v in case["X"]], frac_bits=case["frac_bits"], q_heads=case["q_heads"])
    if case["norm"]:
        n = case["norm"]
        out["norm"] = cb.Norm(*([up(v) for v in n[k]] for k in ("U", "words", "UV")), n["steps"], n["guess"], n["eps"])
    if case["gain"]:
        out["gain"] = cb.Gain(*([up(v) for v in case["gain"][k]] for k in ("weight", "mask", "A", "C")))
    if case["rotation"]:
        r = case["rotation"]
        out["rotation"] = cb.Rotation(up(r["cos"]), up(r["sin"]), torch.from_numpy(r["positions"]).cuda(), r["interleaved"])
    return out


def compare(got, ref):
    msg, Z = got
    for name, pair in (("Z", Z), ("M", msg.M), ("S", msg.S), ("D", msg.D), ("G", msg.G)):
        assert (pair is None) == (name not in ref), name
        for i in (0, 1):
            if pair is not None:
                assert np.array_equal(host(pair[i]), ref[name][i]), (name, i)


# tiles of sixteen rows to one, one to eight CTAs a row, lengths that fill neither threads nor pairs of pairs
DIMS = [2, 4, 6, 30, 32, 34, 62, 64, 66, 80, 126, 128, 130, 132, 256, 1022, 1024, 1026, 1030, 2048, 2050, 3466, 4096, 4098, 8190, 8192]


@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("rot", ["none", "all", "part"])
def test_row_lengths(cb, D, rot):
    rot = {"none": 0, "all": D, "part": 2 * max(1, D // 8)}[rot]
    T, H = (5, 3) if D <= 256 else (3, 1)
    case, _, _ = norm_case(D + rot, T, H, D, 16, 4, rot, interleaved=D % 3 == 0, q_heads=2 if H > 1 else None)
    compare(cb.norm_rotate(**on_gpu(case, cb)), layers.norm_rotate(**case))


@pytest.mark.parametrize("T,H,q", [(1, 1, 1), (1, 2, 1), (1, 24, 12), (7, 5, 4), (33, 3, 0), (13, 4, 4), (512, 2, 1), (2, 300, 299)])
@pytest.mark.parametrize("D,rot,interleaved", [(16, 16, False), (40, 40, True), (64, 64, False), (128, 32, True), (160, 160, False)])
def test_rows_and_heads(cb, T, H, q, D, rot, interleaved):
    case, _, _ = norm_case(T + H, T, H, D, 13, 6, rot, interleaved=interleaved, q_heads=q)
    compare(cb.norm_rotate(**on_gpu(case, cb)), layers.norm_rotate(**case))


@pytest.mark.parametrize("normed,gained,rot", [(True, True, 0), (True, False, 0), (True, False, 24), (False, False, 24), (True, True, 24)])
@pytest.mark.parametrize("D", [24, 48, 96, 264])
@pytest.mark.parametrize("pad,shift", [(0, 0), (2, 0), (3, 0), (96, 2), (0, 1)])
def test_parts_strides_and_alignment(cb, normed, gained, rot, D, pad, shift):
    case, _, _ = norm_case(D, 6, 3, D, 16, 3, rot, interleaved=D == 48, q_heads=1, gained=gained, normed=normed)
    compare(cb.norm_rotate(**on_gpu(case, cb, pad, shift)), layers.norm_rotate(**case))


@pytest.mark.parametrize("steps", [2, 3, 12, 24])
@pytest.mark.parametrize("f", [1, 12, 31])
def test_steps_and_fixed_point(cb, steps, f):
    for D in (32, 128, 520):
        case, _, _ = norm_case(steps, 3, 2, D, f, steps, D, table=8)
        case["norm"]["guess"] = max(1, case["norm"]["guess"])
        compare(cb.norm_rotate(**on_gpu(case, cb)), layers.norm_rotate(**case))


@pytest.mark.parametrize("D", [8, 12, 20, 28, 36, 44, 60, 82, 100, 122, 170, 172, 254, 258, 300, 340, 342, 384, 510, 512, 514, 516])
@pytest.mark.parametrize("rot,interleaved", [("all", False), ("all", True), ("odd", False), ("odd", True), ("even", False)])
def test_tiles(cb, D, rot, interleaved):
    """Tiles of whole rows: as many as 128 threads of four words cover, sixteen at most, the last one not full; pairs of one
    thread's, and pairs through shared memory."""
    rot = {"all": D, "odd": 2 * (2 * (D // 8) + 1), "even": 4 * max(1, D // 10)}[rot]
    tile = min(16, 128 // ((D + 3) // 4)) if D <= 512 else 1
    for T, H, q in ((1, 1, 1), (1, tile + 1, tile), (5, 7, 3)):
        case, _, _ = norm_case(D + rot, T, H, D, 16, 3, min(rot, D), interleaved=interleaved, q_heads=q)
        compare(cb.norm_rotate(**on_gpu(case, cb)), layers.norm_rotate(**case))


# more rows than the CTAs that run at once and what they ask for ahead, the last tile ragged, tokens apart, an odd number of a row's words
@pytest.mark.parametrize("T,H,D,rot,pad", [(447, 1, 512, 512, 0), (67, 31, 128, 64, 2), (91, 41, 64, 64, 0), (601, 13, 16, 16, 6), (203, 1, 1030, 0, 4),
                                           (41, 4, 4096, 1024, 0), (331, 11, 66, 32, 0)])
def test_many_rows(cb, T, H, D, rot, pad):
    case = norm_case(12, T, H, D, 16, 3, rot, q_heads=H // 2)[0]
    for shift in (0, 1):
        compare(cb.norm_rotate(**on_gpu(case, cb, pad, shift)), layers.norm_rotate(**case))


def test_any_words(cb):
    """Uniform words everywhere, triples that are none, the largest guess and eps: the words are still the formulas'."""
    for D, T, H in ((20, 9, 5), (128, 4, 2), (2052, 2, 1)):
        case, _, _ = norm_case(1, T, H, D, 16, 7, D, q_heads=1 if H > 1 else None)
        for k, v in list(case["norm"].items()):
            if isinstance(v, list):
                case["norm"][k] = [words(i, k, *a.shape) for i, a in enumerate(v)]
        case["norm"].update(guess=(1 << 32) - 1, eps=(1 << 64) - 1)
        for k, v in case["gain"].items():
            case["gain"][k] = [words(i, "g" + k, *a.shape) for i, a in enumerate(v)]
        case["X"] = [words(i, "x", *a.shape) for i, a in enumerate(case["X"])]
        case["rotation"]["cos"] = words(0, "cos", *case["rotation"]["cos"].shape)
        case["rotation"]["sin"] = words(0, "sin", *case["rotation"]["sin"].shape)
        compare(cb.norm_rotate(**on_gpu(case, cb)), layers.norm_rotate(**case))


@pytest.mark.parametrize("normed", [True, False])
@pytest.mark.parametrize("D", [32, 130, 256])
def test_positions_outside_the_tables(cb, normed, D):
    case, _, _ = norm_case(5, 6, 2, D, 16, 3, D, normed=normed, table=9)
    case["rotation"]["positions"] = np.array([0, 8, 9, -1, 2**31 - 1, -2**31], np.int32)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    compare(cb.norm_rotate(**on_gpu(case, cb), bad_index_flag=flag), layers.norm_rotate(**case))
    assert flag.item() == 1
    compare(cb.norm_rotate(**on_gpu(case, cb)), layers.norm_rotate(**case))
    case["rotation"]["positions"] = np.array([0, 8, 0, 1, 2, 8], np.int32)
    flag.zero_()
    compare(cb.norm_rotate(**on_gpu(case, cb), bad_index_flag=flag), layers.norm_rotate(**case))
    assert flag.item() == 0


def test_reconstructs_the_float_result(cb):
    """The shares' sum against float64, within the truncations' errors (float_norm_rotate derives them)."""
    for kw in (dict(T=64, H=8, D=128, f=16, steps=12, rot=128, q_heads=5), dict(T=9, H=1, D=4096, f=16, steps=12, rot=0)):
        case, x, weight = norm_case(77, **kw)
        _, Z = cb.norm_rotate(**on_gpu(case, cb))
        want, bound = float_norm_rotate(case, x, weight)
        off = np.abs(wl.decode(host(Z[0]) + host(Z[1]), kw["f"]) - want)
        assert (off <= bound).all(), (off / bound).max()


def test_memory_around_the_results_stays(cb):
    """Nothing before or past a result's words is written: results in the middle of a filled buffer, through the C interface."""
    for D, T, H in ((20, 5, 3), (128, 3, 1), (1030, 2, 1)):
        case, _, _ = norm_case(9, T, H, D, 16, 5, D, q_heads=1 if H > 1 else None)
        g = on_gpu(case, cb)
        ref = layers.norm_rotate(**case)
        gains = case["gain"]["weight"][0].shape[0]
        a = cb.CometNormRotateArgs()
        a.tokens, a.heads, a.q_heads, a.dim, a.x_stride, a.frac_bits, a.steps = T, H, case["q_heads"], D, H * D, 16, 5
        a.guess, a.eps, a.rot_dim, a.table_rows = case["norm"]["guess"], case["norm"]["eps"], D, case["rotation"]["cos"].shape[0]
        put = lambda name, pair: setattr(a, name, (ctypes.c_void_p * 2)(pair[0].data_ptr(), pair[1].data_ptr()))
        for name, pair in (("X", g["X"]), ("U", g["norm"].U), ("row_words", g["norm"].words), ("UV", g["norm"].UV), ("gain", g["gain"].weight),
                           ("gain_mask", g["gain"].mask), ("A", g["gain"].A), ("C", g["gain"].C)):
            put(name, pair)
        a.cos, a.sin, a.positions = g["rotation"].cos.data_ptr(), g["rotation"].sin.data_ptr(), g["rotation"].positions.data_ptr()
        a.interleaved = int(g["rotation"].interleaved)
        rooms = {}
        for name, shape in (("Z", (T, H, D)), ("M", (T, H, D)), ("D", (T, H, D)), ("S", (T, H, 14)), ("G", (gains, D))):
            rooms[name] = [torch.full((int(np.prod(shape)) + 64,), 12345, dtype=torch.int64, device="cuda") for _ in (0, 1)]
            put(name, [r[32:] for r in rooms[name]])
        torch.cuda.synchronize()
        assert cb.library().comet_norm_rotate(None, ctypes.byref(a)) == 0
        torch.cuda.synchronize()
        for name, pair in rooms.items():
            for i in (0, 1):
                got = host(pair[i])
                assert (got[:32] == 12345).all() and (got[-32:] == 12345).all(), name
                assert np.array_equal(got[32:-32].reshape(ref[name][i].shape), ref[name][i]), name


def test_tokens_far_apart(cb):
    """Tokens more than 2^31 words apart in X."""
    T, H, D, far = 3, 2, 64, (1 << 30) + 6                # 2 far words: the last token
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    case, _, _ = norm_case(4, T, H, D, 16, 3, D, q_heads=1)
    g = on_gpu(case, cb)
    room = torch.zeros(2 * far + 4 * H * D, dtype=torch.int64, device="cuda")
    g["X"] = [torch.as_strided(room, (T, H, D), (far, D, 1), i * 2 * H * D) for i in (0, 1)]
    for i in (0, 1):
        g["X"][i].copy_(dev(case["X"][i]))
    compare(cb.norm_rotate(**g), layers.norm_rotate(**case))
    bare = dict(g, norm=None, gain=None)
    compare(cb.norm_rotate(**bare), layers.norm_rotate(**dict(case, norm=None, gain=None)))


@pytest.mark.parametrize("D,rot", [(64, 64), (66, 30), (1024, 0)])
def test_one_tensor_in_several_places(cb, D, rot):
    """What is only read may be given twice: the rows as their own masks, both parties' material alike, the tables each other's."""
    case = norm_case(45, 3, 4, D, 16, 4, rot)[0]
    X = case["X"]
    n, g = case["norm"], case["gain"]
    case = dict(case, norm=dict(n, U=X, UV=[n["UV"][0]] * 2), gain=dict(g, mask=g["weight"], A=X, C=X))
    if rot:
        case["rotation"] = dict(case["rotation"], sin=case["rotation"]["cos"])
    gpu = on_gpu(case, cb)
    x, n, g = gpu["X"], gpu["norm"], gpu["gain"]
    gpu.update(norm=n._replace(U=x, UV=[n.UV[0]] * 2), gain=g._replace(mask=g.weight, A=x, C=x))
    if rot:
        gpu["rotation"] = gpu["rotation"]._replace(sin=gpu["rotation"].cos)
    got = cb.norm_rotate(**gpu)
    compare(got, layers.norm_rotate(**case))
    assert not any(v.any() for v in got[0].M) and not any(v.any() for v in got[0].G)


@pytest.mark.parametrize("normed", [True, False])
def test_calls_on_two_streams_at_once(cb, normed):
    """Calls share no memory: two streams at once, rows of tiles and of clusters, give the words of calls one by one."""
    cases = [norm_case(50 + k, *s)[0] for k, s in enumerate(((70, 6, 128, 13, 5, 128), (9, 3, 66, 16, 6, 30), (40, 1, 2048, 16, 6, 512)))]
    if not normed:
        cases = [dict(c, norm=None, gain=None) for c in cases]
    gpu, refs = [on_gpu(c, cb) for c in cases], [layers.norm_rotate(**c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[cb.norm_rotate(**g, stream=streams[(k + j) % 2]) for j, g in enumerate(gpu)] for k in range(4)]
    torch.cuda.synchronize()
    for results in got:
        for result, ref in zip(results, refs):
            compare(result, ref)


def test_streams_and_replays(cb):
    cases = [norm_case(40 + k, *s)[0] for k, s in enumerate(((5, 4, 64, 16, 6, 64), (3, 1, 2048, 16, 6, 0), (70, 6, 128, 13, 5, 128)))]
    gpu = [on_gpu(c, cb) for c in cases]
    refs = [layers.norm_rotate(**c) for c in cases]
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    got = [[cb.norm_rotate(**g, stream=stream) for g in gpu] for _ in range(3)]
    stream.synchronize()
    for results in got:
        for result, ref in zip(results, refs):
            compare(result, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = [cb.norm_rotate(**g, stream=torch.cuda.current_stream()) for g in gpu]
    for k in range(3):
        for g, c in zip(gpu, cases):                       # other rows, the material kept
            for i in (0, 1):
                c["X"][i] = words(k, f"other{i}", *c["X"][i].shape)
                g["X"][i].copy_(dev(c["X"][i]))
        graph.replay()
        torch.cuda.synchronize()
        for result, c in zip(captured, cases):
            compare(result, layers.norm_rotate(**c))


def test_refusals_on_a_device(cb):
    case, _, _ = norm_case(2, 3, 4, 8, 16, 4, 8, q_heads=2)
    g = on_gpu(case, cb)
    cut = lambda pair: [v[:2].contiguous() for v in pair]
    for bad in (dict(X=[v.transpose(0, 1) for v in g["X"]]), dict(norm=g["norm"]._replace(U=cut(g["norm"].U))),
                dict(norm=g["norm"]._replace(steps=5)), dict(gain=g["gain"]._replace(weight=[v[:1].contiguous() for v in g["gain"].weight])),
                dict(q_heads=4), dict(rotation=g["rotation"]._replace(positions=g["rotation"].positions[:2])),
                dict(rotation=g["rotation"]._replace(positions=g["rotation"].positions.long())),
                dict(X=[g["X"][0], g["X"][1].clone()[:, :2]]), dict(bad_index_flag=torch.zeros(1, device="cuda"))):
        with pytest.raises(AssertionError):
            cb.norm_rotate(**dict(g, **bad))
    for bad, code in ((dict(norm=None, gain=None, rotation=None), -1), (dict(norm=None), -1), (dict(frac_bits=0), -2),
                      (dict(norm=g["norm"]._replace(guess=0)), -2), (dict(q_heads=-1, gain=None), -2), (dict(q_heads=5, gain=None), -2),
                      (dict(norm=g["norm"]._replace(steps=1)), -2)):
        with pytest.raises(cb.CometError) as e:
            cb.norm_rotate(**dict(g, **bad))
        assert e.value.code == code, bad
    # one token may lie anywhere
    one = norm_case(2, 1, 4, 8, 16, 4, 8, q_heads=2)[0]
    compare(cb.norm_rotate(**on_gpu(one, cb, pad=5)), layers.norm_rotate(**one))
