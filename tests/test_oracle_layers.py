"""Pins of oracle/layers.py: the linear layer and the norm / gain / rotation of shared heads."""
import numpy as np
import pytest

from oracle import layers
from paper_2505_07239_b200 import workloads as wl

U64 = np.uint64


def _signed(a):
    return np.ascontiguousarray(a).view(np.int64)


def _linear_case(seed, T, K, N, f):
    x = wl.encode(wl.random_normal(seed, "x", T * K, 1.0).reshape(T, K), f)
    w = wl.encode(wl.random_normal(seed, "w", N * K, K ** -0.5).reshape(N, K), f)
    t = wl.dealer_triple(seed, "t", T, K, N)
    pair = wl.dealer_square_pair(seed, "p", (T, N))
    b = wl.encode(wl.random_normal(seed, "b", N, 0.5), f)
    r = wl.encode(wl.random_normal(seed, "r", T * N, 1.0).reshape(T, N), f)
    k = tuple(int(v * (1 << f)) for v in (0.5, 0.25, 0.125))
    share = lambda v, n: list(wl.split_shares(v, seed, n))
    args = dict(X=share(x, "x"), A=list(t["A"][1:]), W=share(w, "w"), B=[wl.lib_layout(v) for v in t["B"][1:]], C=list(t["C"][1:]),
                frac_bits=f, bias=share(b, "b"), act=(k, list(pair["R"][1:]), list(pair["Q"][1:])), residual=share(r, "r"))
    return args, (x, w, b, r, k)


def test_linear_against_python_integers():
    """Every truncation is the floor or one more, so the sum of the shares is bracketed by integer arithmetic on the plaintexts."""
    f = 13
    args, (x, w, b, r, k) = _linear_case(5, 6, 24, 12, f)
    got = layers.linear(**args)
    total = _signed(got["Y"][0] + got["Y"][1])
    for t in range(6):
        for n in range(12):
            z = sum(int(_signed(x)[t, j]) * int(_signed(w)[n, j]) for j in range(24)) + (int(_signed(b)[n]) << f)
            allowed = set()
            for y in (z >> f, (z >> f) + 1):
                for s in (y * y >> f, (y * y >> f) + 1):
                    u = k[2] * s + k[1] * y >> f
                    allowed |= {u + k[0] + int(_signed(r)[t, n]), u + 1 + k[0] + int(_signed(r)[t, n])}
            assert int(total[t, n]) in allowed


def test_linear_parts_one_by_one():
    f = 12
    full, (x, w, b, r, k) = _linear_case(7, 3, 8, 4, f)
    bare = layers.linear(**dict(full, bias=None, act=None, residual=None))
    z = _signed(x) @ _signed(w).T
    assert set(np.unique(_signed(bare["Y"][0] + bare["Y"][1]) - (z >> f))) <= {0, 1}
    assert "M" not in bare
    with_residual = layers.linear(**dict(full, bias=None, act=None))
    assert all(np.array_equal(with_residual["Y"][i] - full["residual"][i], bare["Y"][i]) for i in (0, 1))
    # messages: E_0 + E_1 = X - A, F_0 + F_1 = W - B
    assert np.array_equal(bare["E"][0] + bare["E"][1], x - (full["A"][0] + full["A"][1]))
    assert np.array_equal(bare["F"][0] + bare["F"][1], w - (full["B"][0] + full["B"][1]))


def test_quadratic_with_zero_mask_and_identity_coefficients():
    """Shares of R and Q that are zero make the message the whole value; k = (0, 1, 0) at scale f gives y back within a
    truncation."""
    f = 12
    args, _ = _linear_case(9, 2, 8, 4, f)
    zero = [np.zeros((2, 4), U64)] * 2
    plain = layers.linear(**dict(args, act=None, residual=None))
    got = layers.linear(**dict(args, act=((0, 1 << f, 0), zero, zero), residual=None))
    assert all(np.array_equal(got["M"][i], plain["Y"][i]) for i in (0, 1))
    assert np.abs(_signed(got["Y"][0] + got["Y"][1]) - _signed(plain["Y"][0] + plain["Y"][1])).max() <= 1


def norm_case(seed, T, H, D, f, steps, rot, interleaved=False, q_heads=None, gained=True, normed=True, table=64):
    q = H if q_heads is None else q_heads
    gains = 2 if 0 < q < H else 1
    x = wl.encode(wl.random_normal(seed, "x", T * H * D, 1.0).reshape(T, H, D) *
                  np.exp2(2 * wl.random_unit(seed, "size", T * H).reshape(T, H, 1) - 1), f)
    n = wl.dealer_norm(seed, "n", T, H, D, steps)
    g = wl.dealer_gain(seed, "g", T, H, D, gains, q)
    weight = wl.encode(1 + wl.random_normal(seed, "w", gains * D, 0.2).reshape(gains, D), f)
    case = dict(X=list(wl.split_shares(x, seed, "xs")), frac_bits=f, q_heads=q, norm=None, gain=None, rotation=None)
    if normed:
        case["norm"] = dict(U=list(n["U"][1:]), words=list(n["words"][1:]), UV=list(n["UV"][1:]), steps=steps,
                            guess=int(0.55 * (1 << f)), eps=max(1, (1 << f) // 100000))
    if normed and gained:
        case["gain"] = dict(weight=list(wl.split_shares(weight, seed, "ws")), mask=list(g["mask"][1:]), A=list(g["A"][1:]),
                            C=list(g["C"][1:]))
    if rot:
        cos, sin = wl.rotation_tables(table, rot, f)
        at = (wl.random_u64(seed, "pos", T) % U64(table)).astype(np.int32)
        case["rotation"] = dict(cos=cos, sin=sin, positions=at, interleaved=interleaved)
    return case, x, weight


def float_norm_rotate(case, x, weight):
    """The same in float64 on the decoded inputs, and a bound of the fixed-point result's distance from it.

    ulp = 2^-f; a local truncation is off by at most 1 ulp.  s by 1 ulp.  A Newton step at the fixed point adds
    y (s + 1) / 2 + 1 ulp to y (p off by 1, w by s + 1, y by its own truncation), errors of earlier steps enter squared; the
    root of a mean square that is off by d is off by d r^3 / 2.  One ulp more for the squares.  Then a product off by
    |x| dy + |y| dx + 1, and so on."""
    f = case["frac_bits"]
    ulp = 2.0 ** -f
    v, err = wl.decode(x, f), np.zeros(x.shape)
    if case["norm"] is not None:
        s = (v * v).mean(-1, keepdims=True) + case["norm"]["eps"] * ulp
        assert s.min() > 0.12 and s.max() < 8
        r = 1 / np.sqrt(s)
        dr = r ** 3 / 2 + r * (s + 1) / 2 + 2
        err = np.abs(v) * dr + 1
        v = v * r
    if case["gain"] is not None:
        row = np.where(np.arange(x.shape[1]) < case["q_heads"], 0, weight.shape[0] - 1)
        g = wl.decode(weight, f)[row][None]
        err = np.abs(g) * err + 1
        v = v * g
    if case["rotation"] is not None:
        rot = case["rotation"]
        c, t = (wl.decode(rot[k][rot["positions"]], f)[:, None, :] for k in ("cos", "sin"))
        j = np.arange(c.shape[-1])
        one, two = (2 * j, 2 * j + 1) if rot["interleaved"] else (j, j + c.shape[-1])
        a, b, da, db = v[..., one], v[..., two], err[..., one], err[..., two]
        v, err = v.copy(), err.copy()
        v[..., one], v[..., two] = a * c - b * t, b * c + a * t
        err[..., one] = np.abs(c) * da + np.abs(t) * db + 1
        err[..., two] = np.abs(c) * db + np.abs(t) * da + 1
    return v, err * ulp


@pytest.mark.parametrize("kw", [
    dict(T=3, H=2, D=64, f=16, steps=12, rot=64), dict(T=5, H=3, D=10, f=13, steps=11, rot=6, interleaved=True, q_heads=1),
    dict(T=2, H=1, D=512, f=16, steps=12, rot=0), dict(T=4, H=2, D=34, f=12, steps=12, rot=34, gained=False),
    dict(T=9, H=4, D=16, f=16, steps=2, rot=16, normed=False), dict(T=3, H=4, D=20, f=16, steps=12, rot=0, q_heads=3)])
def test_norm_rotate_against_float64(kw):
    case, x, weight = norm_case(31, **kw)
    got = layers.norm_rotate(**case)
    want, bound = float_norm_rotate(case, x, weight)
    off = np.abs(wl.decode(got["Z"][0] + got["Z"][1], case["frac_bits"]) - want)
    assert (off <= bound).all(), (off / bound).max()


def test_norm_of_a_constant_row_and_of_zeros():
    """x = c everywhere has root 1 / c; a row of zeros stays within a truncation of zero."""
    f, D = 16, 32
    case, _, _ = norm_case(3, 2, 1, D, f, 12, 0, gained=False)
    x = np.stack([np.full((1, D), 2 << f, U64), np.zeros((1, D), U64)])
    got = layers.norm_rotate(**dict(case, X=list(wl.split_shares(x, 4, "c"))))
    z = wl.decode(got["Z"][0] + got["Z"][1], f)
    assert np.abs(z[0] - 1).max() < 16 * 2.0 ** -f and np.abs(z[1]).max() <= 2.0 ** -f


def test_rotation_closed_forms():
    """Position 0 leaves every word within a truncation, a quarter turn swaps the pair's members; a position outside the
    table gives zeros; words behind the rotated ones keep their bits."""
    f = 14
    case, x, _ = norm_case(8, 4, 2, 8, f, 2, 4, normed=False)
    case["rotation"]["cos"] = np.array([[1 << f] * 2, [0] * 2], U64)
    case["rotation"]["sin"] = np.array([[0] * 2, [1 << f] * 2], U64)
    case["rotation"]["positions"] = np.array([0, 1, -1, 2], np.int32)
    got = layers.norm_rotate(**case)["Z"]
    z, v = _signed(got[0] + got[1]), _signed(x)
    assert np.isin(z[0, :, :4] - v[0, :, :4], (0, 1)).all()
    assert np.isin(z[1, :, :2] + v[1, :, 2:4], (0, 1)).all() and np.isin(z[1, :, 2:4] - v[1, :, :2], (0, 1)).all()
    assert not got[0][2:, :, :4].any() and not got[1][2:, :, :4].any()
    assert all(np.array_equal(got[i][..., 4:], case["X"][i][..., 4:]) for i in (0, 1))


@pytest.mark.parametrize("plant", ["square", "mask", "gain row", "party"])
def test_planted_mistakes_show(plant, monkeypatch):
    case, x, weight = norm_case(12, 3, 4, 16, 16, 12, 16, q_heads=2)
    if plant == "square":
        # the square of the last step's mask (Newton's iteration forgets what is wrong in an early step)
        case["norm"]["words"][0] = case["norm"]["words"][0].copy()
        case["norm"]["words"][0][..., 2 + 6 * 10 + 1] += U64(1 << 28)
    elif plant == "mask":
        case["norm"]["UV"][1] = case["norm"]["UV"][0]
    elif plant == "gain row":
        case["q_heads"] = 3
    else:                                      # the public term is the other party's: the sums stay, the shares do not
        monkeypatch.setattr(layers, "_eq1", lambda c, a, b, d, e: [c[0] + d * b[0] + e * a[0] + d * e, c[1] + d * b[1] + e * a[1]])
        wrong = layers.norm_rotate(**case)
        monkeypatch.undo()
        assert not np.array_equal(wrong["Z"][0], layers.norm_rotate(**case)["Z"][0])
        return
    got = layers.norm_rotate(**case)
    case["q_heads"] = 2
    want, bound = float_norm_rotate(case, x, weight)
    assert (np.abs(wl.decode(got["Z"][0] + got["Z"][1], 16) - want) > bound).any()
