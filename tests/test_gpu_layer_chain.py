"""The projections of an attention layer as they are used one behind the other: row norm, stacked q, k, v projection with bias,
norm and rotation of the q and k heads read out of its result, output projection added to the residual stream."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import layers  # noqa: E402
from paper_2505_07239_b200 import workloads as wl  # noqa: E402
from tests.test_gpu_linear import cb, dev, host  # noqa: E402,F401


@pytest.mark.parametrize("T", [1, 32, 150])
def test_projections_of_an_attention_layer(cb, T):
    heads, dim, f, steps, seed = 4, 64, 16, 12, 11
    d = heads * dim
    share = lambda v, name: list(wl.split_shares(v, seed, name))
    draw = lambda name, sigma, *shape: wl.encode(wl.random_normal(seed, name, int(np.prod(shape)), sigma).reshape(shape), f)
    x = draw("x", 1.0, T, d)
    w_qkv, b_qkv, w_out = draw("wqkv", d ** -0.5, 3 * d, d), draw("bqkv", 0.1, 3 * d), draw("wout", d ** -0.5, d, d)
    gains = [draw(f"g{k}", 0.1, *s) + np.uint64(1 << f) for k, s in enumerate(((1, d), (2, dim)))]
    cos, sin = wl.rotation_tables(256, dim, f)
    positions = (wl.random_u64(seed, "pos", T) % np.uint64(256)).astype(np.int32)

    def material(name, rows, D, g, q):
        n = wl.dealer_norm(seed, name, T, rows, D, steps)
        t = wl.dealer_gain(seed, name, T, rows, D, g.shape[0], q)
        return (dict(U=list(n["U"][1:]), words=list(n["words"][1:]), UV=list(n["UV"][1:]), steps=steps, guess=int(0.55 * (1 << f)), eps=1),
                dict(weight=share(g, name + "w"), mask=list(t["mask"][1:]), A=list(t["A"][1:]), C=list(t["C"][1:])))

    def triple(name, K, N):
        t = wl.dealer_triple(seed, name, T, K, N)
        return list(t["A"][1:]), [wl.lib_layout(v) for v in t["B"][1:]], list(t["C"][1:])

    X, W1, B1, W2 = share(x, "xs"), share(w_qkv, "ws"), share(b_qkv, "bs"), share(w_out, "os")
    row_norm, row_gain = material("row", 1, d, gains[0], 1)
    head_norm, head_gain = material("head", 2 * heads, dim, gains[1], heads)
    t1, t2 = triple("t1", d, 3 * d), triple("t2", d, d)
    rotation = dict(cos=cos, sin=sin, positions=positions, interleaved=False)

    # the oracle
    r1 = layers.norm_rotate([v.reshape(T, 1, d) for v in X], f, norm=row_norm, gain=row_gain)
    r2 = layers.linear([v.reshape(T, d) for v in r1["Z"]], t1[0], W1, t1[1], t1[2], f, bias=B1)
    qk = [np.ascontiguousarray(v[:, :2 * d]).reshape(T, 2 * heads, dim) for v in r2["Y"]]
    r3 = layers.norm_rotate(qk, f, norm=head_norm, gain=head_gain, rotation=rotation, q_heads=heads)
    r4 = layers.linear([np.ascontiguousarray(v[:, 2 * d:]) for v in r2["Y"]], t2[0], W2, t2[1], t2[2], f, residual=X)

    # the library, nothing waited for in between
    up = lambda p: [dev(v) for v in p]
    norm = lambda m: cb.Norm(up(m["U"]), up(m["words"]), up(m["UV"]), m["steps"], m["guess"], m["eps"])
    gain = lambda m: cb.Gain(*(up(m[k]) for k in ("weight", "mask", "A", "C")))
    Xd, rn, rg, hn, hg = up(X), norm(row_norm), gain(row_gain), norm(head_norm), gain(head_gain)
    W1d, B1d, W2d = up(W1), up(B1), up(W2)
    A1, M1, C1, A2, M2, C2 = (up(v) for v in (*t1, *t2))
    rot = cb.Rotation(dev(cos), dev(sin), torch.from_numpy(positions).cuda())
    m1, z1 = cb.norm_rotate([v.view(T, 1, d) for v in Xd], f, norm=rn, gain=rg)
    _, _, _, y = cb.linear([v.view(T, d) for v in z1], A1, W1d, M1, C1, f, bias=B1d)
    m3, z3 = cb.norm_rotate([v[:, :2 * d].view(T, 2 * heads, dim) for v in y], f, norm=hn, gain=hg, rotation=rot, q_heads=heads)
    _, _, _, out = cb.linear([v[:, 2 * d:].contiguous() for v in y], A2, W2d, M2, C2, f, residual=Xd)
    for i in (0, 1):
        assert np.array_equal(host(z1[i]), r1["Z"][i]) and np.array_equal(host(m1.S[i]), r1["S"][i])
        assert np.array_equal(host(y[i]), r2["Y"][i])
        assert np.array_equal(host(z3[i]), r3["Z"][i]) and np.array_equal(host(m3.D[i]), r3["D"][i])
        assert np.array_equal(host(out[i]), r4["Y"][i])
    assert cb.static_status() == 0

    # what it stands for, in float64, within the truncations: with |x| < 5, a root of about 1 and gains below 2 the normed row is
    # off by less than 40 ulps, a product by its input's error times the weights' absolute row sums and one ulp
    real = lambda v: wl.decode(v, f)
    n = real(x) / np.sqrt((real(x) ** 2).mean(-1, keepdims=True) + 2.0 ** -f) * real(gains[0])
    v = n @ real(w_qkv).T + real(b_qkv)
    want = v[:, 2 * d:] @ real(w_out).T + real(x)
    bound = 2.0 ** -f * ((40 * np.abs(real(w_qkv)).sum(1).max() + 1) * np.abs(real(w_out)).sum(1).max() + 1)
    assert np.abs(real(host(out[0]) + host(out[1])) - want).max() <= bound
