"""A block of linear attention as it is used: a stacked projection, the norm and gain of query and key heads, linear attention over packed prompts and then
token by token, the norm of every head, the output projection; word for word against the same chain of the CPU oracle."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import attention, layers  # noqa: E402
from tests.test_gpu_group_norm import on_gpu as group_on_gpu, ring_group  # noqa: E402
from tests.test_gpu_linear import cb, dev, host, on_gpu as linear_on_gpu, ring_case, words  # noqa: E402,F401
from tests.test_gpu_linear_attention import OnGpu, compare, pair, ring_prompt, ring_step  # noqa: E402
from tests.test_gpu_norm_rotate import on_gpu as norm_on_gpu  # noqa: E402

F = 16


def norm_case(seed, T, H, q_heads, D, steps=3):
    return dict(X=None, frac_bits=F, q_heads=q_heads, rotation=None,
                norm=dict(U=pair(seed, "U", T, H, D), words=pair(seed, "w", T, H, 6 * steps - 3), UV=pair(seed, "UV", T, H, D), steps=steps, guess=1 << (F - 1), eps=5),
                gain=dict(weight=pair(seed, "g", 2, D), mask=pair(seed, "gm", 2, D), A=pair(seed, "gA", T, H, D), C=pair(seed, "gC", T, H, D)))


class Block:
    """A block's material for T rows; `on` runs it on the GPU, `by` the oracle's."""

    def __init__(self, seed, T, K, Hq, Hk, D, prompt=None):
        self.Hq, self.Hk, self.D = Hq, Hk, D
        self.inward = ring_case(seed, T, K, (Hq + 2 * Hk) * D, F, True, None, False)
        self.norm = norm_case(seed + 1, T, Hq + Hk, Hq, D)
        self.attend = ring_prompt(seed + 2, prompt, Hq, Hk, D, D, 64, F) if prompt else ring_step(seed + 2, T, Hq, Hk, D, D, F)
        self.heads = ring_group(seed + 3, T, 1, Hq * D, Hq, F)
        self.outward = ring_case(seed + 4, T, Hq * D, K, F, True, None, True)

    def on(self, cb, stream, state=None):
        T, Hq, Hk, D = self.inward["X"][0].shape[0], self.Hq, self.Hk, self.D
        y = cb.linear(**linear_on_gpu(self.inward), stream=stream)[-1]
        y = [t.view(T, Hq + 2 * Hk, D) for t in y]
        n = norm_on_gpu(dict(self.norm, X=[np.zeros((T, Hq + Hk, D), np.uint64)] * 2), cb)
        n["X"] = [t[:, :Hq + Hk] for t in y]                                     # views of the stacked result
        z = cb.norm_rotate(**n, stream=stream)[1]
        a = OnGpu(cb)(self.attend)
        a.update(Q=[t[:, :Hq] for t in z], K=[t[:, Hq:] for t in z], V=[t[:, Hq + Hk:] for t in y])
        if state is not None:
            a["state"] = state
        got = (cb.linear_attention if "starts" in self.attend else cb.linear_attention_step)(**a, stream=stream)
        g = group_on_gpu(self.heads, cb)
        g["X"] = [t.view(T, 1, Hq * D) for t in got[1]]
        h = cb.group_norm(**g, stream=stream)[1]
        o = linear_on_gpu(self.outward)
        o["X"] = [t.view(T, Hq * D) for t in h]
        return got, cb.linear(**o, stream=stream)[-1]

    def by(self, state=None):
        T, Hq, Hk, D = self.inward["X"][0].shape[0], self.Hq, self.Hk, self.D
        y = [t.reshape(T, Hq + 2 * Hk, D) for t in layers.linear(**self.inward)["Y"]]
        z = layers.norm_rotate(**dict(self.norm, X=[t[:, :Hq + Hk] for t in y]))["Z"]
        case = dict(self.attend, Q=[t[:, :Hq] for t in z], K=[t[:, Hq:] for t in z], V=[t[:, Hq + Hk:] for t in y])
        if state is not None:
            case["state"] = state
        ref = (attention.linear_attention if "starts" in case else attention.linear_attention_step)(**case)
        h = attention.group_norm(**dict(self.heads, X=[t.reshape(T, 1, Hq * D) for t in ref["O"]]))["Z"]
        return ref, layers.linear(**dict(self.outward, X=[t.reshape(T, Hq * D) for t in h]))["Y"]


@pytest.mark.parametrize("Hq,Hk,D,starts", [(4, 2, 32, [0, 70, 75, 139]), (3, 3, 64, [0, 1, 40])])
@pytest.mark.parametrize("other_stream", [False, True])
def test_block_over_prompts_and_tokens(cb, Hq, Hk, D, starts, other_stream):  # noqa: F811
    K, B = 64, len(starts) - 1
    prompt = Block(1, starts[-1], K, Hq, Hk, D, starts)
    tokens = [Block(10 * j, B, K, Hq, Hk, D) for j in (1, 2)]
    stream = torch.cuda.Stream() if other_stream else torch.cuda.current_stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        done = [prompt.on(cb, stream)]
        for t in tokens:
            done.append(t.on(cb, stream, done[-1][0][2]))
    torch.cuda.synchronize()
    refs = [prompt.by()]
    for t in tokens:
        refs.append(t.by(refs[-1][0]["S"]))
    for (got, y), (ref, want) in zip(done, refs):
        compare(got, ref)
        for i in (0, 1):
            assert np.array_equal(host(y[i]), want[i])
    assert cb.static_status() == 0
