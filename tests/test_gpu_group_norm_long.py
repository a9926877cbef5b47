"""Norms of channel groups that no cluster holds (more than 16384 words), in three passes over slabs of positions: tiles of groups, groups in parts,
one position, every part of the norm there or not, rows that lie apart and off 16 bytes."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.test_gpu_group_norm import check, compare, dev, on_gpu, ring_group  # noqa: E402
from tests.test_gpu_linear import cb  # noqa: E402,F401
from tests.test_oracle_attention import group_case  # noqa: E402

# several samples, tiles of several groups (the last one not full), tiles of one group, groups in parts of pairs and of single channels, one position
SHAPES = [(3, 1000, 640, 32), (2, 820, 630, 30), (2, 20, 1800, 2), (1, 19, 2703, 3), (2, 1, 40000, 2), (1, 1, 16386, 1), (2, 33, 512, 1), (2, 65, 514, 2), (40, 4200, 4, 1),
          (1, 16385, 1, 1), (2, 5500, 21, 7), (1, 70, 257, 1)]


@pytest.mark.parametrize("S,P,C,G", SHAPES)
@pytest.mark.parametrize("gained,act", [(True, True), (True, False), (False, True), (False, False)])
def test_parts(cb, S, P, C, G, gained, act):  # noqa: F811
    check(cb, ring_group(61 + C, S, P, C, G, 16, 4, gained, act))


@pytest.mark.parametrize("pad,shift", [(2, 0), (3, 0), (64, 2), (0, 1), (5, 3)])
@pytest.mark.parametrize("S,P,C,G", [(2, 1000, 640, 32), (2, 20, 1800, 2), (2, 1, 33000, 2), (2, 5500, 21, 7)])
def test_strides_and_alignment(cb, pad, shift, S, P, C, G):  # noqa: F811
    check(cb, ring_group(62, S, P, C, G, 16, 3), pad=pad, shift=shift)


@pytest.mark.parametrize("steps", [2, 24])
@pytest.mark.parametrize("f", [1, 31])
def test_steps_and_fixed_point(cb, steps, f):  # noqa: F811
    for S, P, C, G in ((2, 900, 80, 4), (1, 20, 1700, 2)):
        check(cb, ring_group(steps, S, P, C, G, f, steps))


def test_on_both_sides_of_what_is_held(cb):  # noqa: F811
    for P in (16383, 16384, 16385):
        check(cb, ring_group(63, 2, P, 3, 3, 16))


def test_real_values(cb):  # noqa: F811
    check(cb, group_case(64, 2, 700, 96, 4, 16, 12))


def test_captured_with_several_samples(cb):  # noqa: F811
    """The sums begin at zero in every replay; an eager call on another stream in between has its own."""
    first, second = ring_group(65, 3, 900, 80, 4, 16), ring_group(66, 3, 900, 80, 4, 16)
    c, side = on_gpu(first, cb), torch.cuda.Stream()
    from oracle import attention
    torch.cuda.synchronize()
    cb.group_norm(**c, stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = cb.group_norm(**c, stream=torch.cuda.current_stream())
    for case in (first, second, first):
        for i in (0, 1):
            c["X"][i].copy_(dev(case["X"][i]))
        torch.cuda.synchronize()
        other = cb.group_norm(**c, stream=side)
        graph.replay()
        torch.cuda.synchronize()
        ref = attention.group_norm(**dict(first, X=case["X"]))
        compare(kept, ref)
        compare(other, ref)
