"""What the results of comet_linear and comet_norm_rotate lie in: a party's share in memory of its own, so that what is saved, sent or
grown with it is that share and nothing else; a party's messages in none of the other party's memory."""
import io

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import layers  # noqa: E402
from tests import test_gpu_norm_rotate as norms  # noqa: E402
from tests.test_gpu_linear import cb, compare, host, on_gpu, ring_case  # noqa: E402,F401
from tests.test_oracle_layers import norm_case  # noqa: E402


def saved(t):
    file = io.BytesIO()
    torch.save(t, file)
    return file.getvalue()


def check(results, messages):
    """`results`: pairs; `messages`: pairs that may lie together, each party's."""
    memory = lambda t: t.untyped_storage().data_ptr()
    everything = [memory(t) for p in [*results, *messages] for t in p]
    for pair in results:
        for i in (0, 1):
            assert everything.count(memory(pair[i])) == 1
            assert pair[i].storage_offset() == 0 and pair[i].untyped_storage().nbytes() == pair[i].numel() * 8
            if pair[i].numel() < 1 << 20:
                data = saved(pair[i])
                assert host(pair[i]).tobytes() in data and host(pair[1 - i]).tobytes() not in data
    for a in messages:
        for b in messages:
            assert memory(a[0]) != memory(b[1])
    for i in (0, 1):                                       # words of this party's messages and no others, not even between them
        pieces = {memory(p[i]): p[i].untyped_storage().nbytes() for p in messages}
        assert sum(pieces.values()) == sum(p[i].numel() * 8 for p in messages)
        spans = sorted((p[i].data_ptr(), p[i].data_ptr() + p[i].numel() * 8) for p in messages)
        assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:]))
    # grown, a result takes nothing of another's
    for pair in results:
        before = [t.clone() for p in [*results, *messages] for t in p if t is not pair[0]]
        pair[0].resize_(2 * pair[0].numel()).zero_()
        after = [t for p in [*results, *messages] for t in p if t is not pair[0]]
        assert all(torch.equal(a, b) for a, b in zip(before, after))


@pytest.mark.parametrize("T,K,N", [(1, 264, 36), (9, 64, 36), (90, 264, 132), (512, 1024, 1024)])
@pytest.mark.parametrize("act", [None, "tame"])
def test_linear(cb, T, K, N, act):
    case = ring_case(90 + T, T, K, N, 16, True, act, True)
    E, F, M, Y = got = cb.linear(**on_gpu(case))
    compare(got, layers.linear(**case))
    check([Y], [p for p in (E, F, M) if p is not None])


@pytest.mark.parametrize("T,K,N", [(1, 1024, 6000), (1100, 64, 6000)])
def test_linear_of_many_words(cb, T, K, N):
    """Messages, and a result, of more than 32 MiB."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    draw = lambda *s: [torch.randint(-2**63, 2**63 - 1, s, generator=gen, device="cuda", dtype=torch.int64) for _ in (0, 1)]
    E, F, M, Y = cb.linear(draw(T, K), draw(T, K), draw(N, K), draw(N, K), draw(T, N), 16)
    check([Y], [E, F])


@pytest.mark.parametrize("D,T,H,rot", [(64, 3, 5, 64), (66, 7, 3, 30), (2050, 2, 1, 4)])
@pytest.mark.parametrize("normed,gained", [(True, True), (True, False), (False, False)])
def test_norm_rotate(cb, D, T, H, rot, normed, gained):
    case = norm_case(91, T, H, D, 16, 4, rot, q_heads=1 if H > 1 else None, gained=gained, normed=normed)[0]
    got = cb.norm_rotate(**norms.on_gpu(case, cb))
    norms.compare(got, layers.norm_rotate(**case))
    msg, Z = got
    check([Z], [p for p in msg if p is not None])
    for pair in (msg.M, msg.D, msg.G):                     # 16-byte accesses go to these
        assert pair is None or all(t.data_ptr() % 16 == 0 for t in pair)
