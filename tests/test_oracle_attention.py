"""Pins of oracle/attention.py: linear attention of prompts and single tokens, norms of channel groups."""
import numpy as np
import pytest

from oracle import attention
from paper_2505_07239_b200 import workloads as wl

U64 = np.uint64


def signed(a):
    return np.ascontiguousarray(a).view(np.int64)


def big(a):
    """Signed values as Python integers, whose sums and products wrap nowhere."""
    return signed(a).astype(object)


def total(pair):
    with np.errstate(over="ignore"):
        return pair[0] + pair[1]


def near_floor(got, number, bits):
    """Whether every local truncation of `number` by `bits` is the floor or one more."""
    off = got - (number >> bits)
    return bool(((off == 0) | (off == 1)).all())


def shares(seed, name, value):
    return list(wl.split_shares(value, seed, name))


def prompt_case(seed, starts, Hq, Hk, Dk, Dv, C, f, state=True, tokens=None):
    T = starts[-1] if tokens is None else tokens
    draw = lambda name, sigma, *shape: shares(seed, name, wl.encode(wl.random_normal(seed, name, int(np.prod(shape)), sigma).reshape(shape), f))
    dealer = wl.dealer_prompt(seed, "t", starts, Hq, Hk, Dk, Dv, C, T)
    return dict(Q=draw("q", Dk ** -0.5, T, Hq, Dk), K=draw("k", Dk ** -0.25, T, Hk, Dk), V=draw("v", 1.0, T, Hk, Dv), starts=list(starts),
                decay=wl.decay_powers(Hk, C, f), dealer={k: list(v[1:]) for k, v in dealer.items()}, frac_bits=f,
                state=draw("s", 0.5, len(starts) - 1, Hk, Dk, Dv) if state else None)


def step_case(seed, B, Hq, Hk, Dk, Dv, f, state=True):
    draw = lambda name, sigma, *shape: shares(seed, name, wl.encode(wl.random_normal(seed, name, int(np.prod(shape)), sigma).reshape(shape), f))
    dealer = wl.dealer_step(seed, "t", B, Hq, Hk, Dk, Dv)
    return dict(Q=draw("q", Dk ** -0.5, B, Hq, Dk), K=draw("k", Dk ** -0.25, B, Hk, Dk), V=draw("v", 1.0, B, Hk, Dv),
                decay=np.ascontiguousarray(wl.decay_powers(Hk, 1, f)[:, 1]), dealer={k: list(v[1:]) for k, v in dealer.items()}, frac_bits=f,
                state=draw("s", 0.5, B, Hk, Dk, Dv) if state else None)


def group_case(seed, S, P, C, G, f, steps, gained=True, act=True):
    size = np.exp2(2 * wl.random_unit(seed, "size", S * G).reshape(S, 1, G, 1) - 1)
    x = size * wl.random_normal(seed, "x", S * P * C, 1.0).reshape(S, P, G, C // G) + wl.random_normal(seed, "mean", S * G, 0.5).reshape(S, 1, G, 1)
    m = {k: list(v[1:]) for k, v in wl.dealer_group(seed, "t", S, P, C, G, steps, gained).items()}
    draw = lambda name, centre, sigma, *shape: shares(seed, name, wl.encode(centre + wl.random_normal(seed, name, int(np.prod(shape)), sigma).reshape(shape), f))
    case = dict(X=shares(seed, "xs", wl.encode(x.reshape(S, P, C), f)), groups=G, frac_bits=f, gain=None, act=None,
                norm=dict(U=m["U"], words=m["words"], UT=m["UT"], steps=steps, guess=max(1, int(0.55 * (1 << f))), eps=max(1, (1 << f) // 100000)))
    if gained:
        case["gain"] = dict(weight=draw("w", 1.0, 0.2, C), mask=m["mask"], T=m["T"], VW=m["VW"], bias=draw("b", 0.0, 0.3, C))
    if act:
        pair = wl.dealer_square_pair(seed, "p", (S, P, C))
        case["act"] = (tuple(int(v * (1 << f)) for v in (0.5, 0.25, 0.125)), list(pair["R"][1:]), list(pair["Q"][1:]))
    return case


PROMPTS = [([0, 7], 1, 1, 4, 6, 3), ([0, 1, 1, 6, 14], 4, 2, 6, 4, 4), ([0, 5, 13], 3, 3, 8, 2, 8)]


@pytest.mark.parametrize("starts,Hq,Hk,Dk,Dv,C", PROMPTS)
def test_prompt_against_python_integers(starts, Hq, Hk, Dk, Dv, C):
    """Every truncation is the floor or one more, so every value that is opened, put together again with its mask, is bracketed by
    integer arithmetic on those before it."""
    f = 13
    case = prompt_case(3, starts, Hq, Hk, Dk, Dv, C, f)
    got, m = attention.linear_attention(**case), case["dealer"]
    q, k, v = (big(total(case[n])) for n in "QKV")
    value = lambda name: total(got[name]) + total(m[name])
    for name, x in (("q", q), ("k", k), ("v", v)):
        assert (big(value(name)) == x).all()
    w, P, D, start = big(case["decay"]), big(value("p")), big(value("d")), big(value("s"))
    S, O = big(total(case["state"])), big(total(got["O"]))
    number = 0
    for j in range(len(starts) - 1):
        for first in range(starts[j], starts[j + 1], C):
            L = min(C, starts[j + 1] - first)
            for h in range(Hk):
                assert (start[number, h] == S[j, h]).all()
                for hq in range(h * Hq // Hk, (h + 1) * Hq // Hk):
                    for r in range(L):
                        t = first + r
                        for s in range(r + 1):
                            score = sum(q[t, hq] * k[first + s, h])
                            assert P[t, hq, s] in {(w[h, r - s] * (z + e) >> f) + g for z in [score >> f] for e in (0, 1) for g in (0, 1)}
                        near = sum(P[t, hq, s] * v[first + s, h] for s in range(r + 1))
                        far = q[t, hq] @ S[j, h] >> f
                        ok = [(near + w[h, r + 1] * (far + e) >> f) + g == O[t, hq] for e in (0, 1) for g in (0, 1)]
                        assert np.any(ok, 0).all()
                for s in range(L):
                    assert near_floor(D[first + s, h], w[h, L - 1 - s] * k[first + s, h], f)
                z = w[h, L] * S[j, h] + sum(np.multiply.outer(D[first + s, h], v[first + s, h]) for s in range(L))
                S[j, h] = z >> f
                # (the next chunk's opening, or the result, tells which of the two it was)
                later = start[number + 1, h] if first + C < starts[j + 1] else big(total(got["S"]))[j, h]
                assert near_floor(later, z, f)
                S[j, h] = later
            number += 1
    assert (big(total(got["S"])) == S).all()
    # off the triangle nothing is sent
    at = np.concatenate([(np.arange(a, b) - a) % C for a, b in zip(starts, starts[1:])])
    for i in (0, 1):
        assert not got["p"][i][np.broadcast_to(np.arange(C)[None, None] > at[:, None, None], got["p"][i].shape)].any()


def test_step_against_python_integers():
    f = 16
    case = step_case(5, 3, 4, 2, 6, 4, f)
    got, m = attention.linear_attention_step(**case), case["dealer"]
    q, k, v, S0 = (big(total(case[n])) for n in ("Q", "K", "V", "state"))
    S, O, w = big(total(got["S"])), big(total(got["O"])), big(case["decay"])
    assert (big(total(got["s"]) + total(m["s"])) == S).all()
    for b in range(3):
        for h in range(2):
            assert near_floor(S[b, h], w[h] * S0[b, h] + np.multiply.outer(k[b, h], v[b, h]), f)
            for hq in (2 * h, 2 * h + 1):
                assert near_floor(O[b, hq], q[b, hq] @ S[b, h], f)


@pytest.mark.parametrize("C", [1, 4, 32])
def test_prompt_against_float64(C):
    """The recurrence in float64.  In units of 2^-f: a chunk's scores are off by 1, weighted by at most 1 and 1 again, so sum |v| 2 of the
    near part; far part and result 1 each and |q|_1 times the state's error; the state takes 1 a chunk and 1 |v| a token for the decayed key
    and |d v| times half a unit for every power."""
    f, T, H, D = 16, 37, 2, 8
    case = prompt_case(9, [0, T], H, H, D, D, C, f)
    got = attention.linear_attention(**case)
    q, k, v = (wl.decode(total(case[n]), f) for n in "QKV")
    S, w = wl.decode(total(case["state"]), f)[0], 1.0 - 2.0 ** (-3.0 - 5.0 * np.arange(H) / H)
    ulp, state_off = 2.0 ** -f, np.zeros(H)
    top = lambda x: np.abs(x).max()
    grown = top(S)
    for t in range(T):
        S = w[:, None, None] * S + k[t][:, :, None] * v[t][:, None, :]
        grown = max(grown, top(S))
        state_off += 2 + top(v) + 0.5 * (grown + top(k) * top(v))
        want = np.einsum("hk,hkv->hv", q[t], S)
        length = np.abs(q[t]).sum(-1)
        bound = ulp * (length * state_off + 4 + min(T, C) * top(v) * (2 + 0.5 * np.abs(q[t]).sum(-1).max() * top(k)) + 0.5 * length * grown)
        off = np.abs(wl.decode(total([o[t] for o in got["O"]]), f) - want)
        assert (off <= bound[:, None]).all()
    assert np.abs(wl.decode(total(got["S"]), f)[0] - S).max() <= ulp * state_off.max()


def test_prompt_token_by_token():
    """Chunks of one token and single tokens differ by their truncations alone: decayed keys and weights are multiplied by w[0] = 1 and
    truncated once more, which is exact or one unit up, the far part is decayed behind its truncation."""
    f, T, H, D = 13, 9, 2, 6
    case = prompt_case(4, [0, T], H, H, D, D, 1, f)
    got = attention.linear_attention(**case)
    state = case["state"]
    for t in range(T):
        one = step_case(50 + t, 1, H, H, D, D, f)
        one.update(Q=[x[t:t + 1] for x in case["Q"]], K=[x[t:t + 1] for x in case["K"]], V=[x[t:t + 1] for x in case["V"]], state=state)
        out = attention.linear_attention_step(**one)
        state = out["S"]
        v, q = (np.abs(big(total(one[n]))).max() for n in "VQ")
        # per token the state moves apart by one truncation each and a unit of the key times the largest |v| (at scale f)
        apart = (t + 1) * (3 + (int(v) >> f))
        off = np.abs(big(total([o[t:t + 1] for o in got["O"]])) - big(total(out["O"]))).max()
        assert off <= (D * int(q) * apart >> f) + D * apart + 6 + 3 * (int(v) >> f)
    assert np.abs(big(total(got["S"])) - big(total(state))).max() <= T * (3 + (int(v) >> f))


def test_state_none_is_zero():
    case = prompt_case(6, [0, 3, 3, 8], 2, 1, 4, 4, 4, 12, state=False)
    zero = dict(case, state=[np.zeros((3, 1, 4, 4), U64)] * 2)
    a, b = attention.linear_attention(**case), attention.linear_attention(**zero)
    assert all(np.array_equal(a[k][i], b[k][i]) for k in a for i in (0, 1))
    assert not total(a["S"])[1].any()                        # the sequence without tokens keeps it


@pytest.mark.parametrize("S,P,C,G,f,steps", [(2, 1, 24, 3, 16, 12), (2, 5, 12, 2, 16, 12), (1, 7, 15, 5, 13, 12), (3, 4, 6, 1, 16, 12)])
def test_group_against_python_integers(S, P, C, G, f, steps):
    case = group_case(8, S, P, C, G, f, steps)
    got, per = attention.group_norm(**case), C // G
    n = P * per
    x, U = big(total(case["X"])).reshape(S, P, G, per), total(case["norm"]["U"])
    d = big(total(got["M"]) + U).reshape(S, P, G, per)
    words = total(case["norm"]["words"])
    root = big(total([t[..., -1] for t in got["S"]]) + words[..., -1])
    second = big(total([t[..., 0] for t in got["S"]]) + words[..., 1]) - case["norm"]["eps"]
    gain, bias = big(total(case["gain"]["weight"])).reshape(G, per), big(total(case["gain"]["bias"])).reshape(G, per)
    t = big(total(got["D"]) + total(case["gain"]["T"])).reshape(S, G, per)
    R = total(case["act"][1])
    z = big(total(got["N"]) + R).reshape(S, P, G, per)
    Z = big(total(got["Z"])).reshape(S, P, G, per)
    k0, k1, k2 = case["act"][0]
    for s in range(S):
        for g in range(G):
            mean = x[s, :, g] - d[s, :, g]
            assert len(set(mean.ravel())) == 1 and mean.ravel()[0] - x[s, :, g].sum() // n in (0, 1)
            assert second[s, g] - (d[s, :, g] ** 2).sum() // (n << f) in (0, 1)
            # Newton at the fixed point: y (s + 1) / 2 + 1 units, twice that for the steps before
            real, y = (float(second[s, g]) + case["norm"]["eps"]) / (1 << f), float(root[s, g]) / (1 << f)
            assert 0.12 < real < 8 and abs(y - real ** -0.5) <= 2.0 ** -f * (y * (real + 1) + 2)
            assert near_floor(t[s, g], root[s, g] * gain[g], f)
            assert near_floor(z[s, :, g], t[s, g] * d[s, :, g] + (bias[g] << f), f)
            ok = [(k2 * ((z[s, :, g] ** 2 >> f) + e) + k1 * z[s, :, g] >> f) + c + k0 == Z[s, :, g] for e in (0, 1) for c in (0, 1)]
            assert np.any(ok, 0).all()


def test_group_of_a_constant_and_of_one_word():
    """A group without variance is its bias: d is zero or one unit, however large the root."""
    f = 16
    for P, C, G in ((4, 6, 2), (1, 5, 5)):
        case = group_case(2, 2, P, C, G, f, 8, act=False)
        case["X"] = shares(3, "c", np.full((2, P, C), 5 << (f - 1), U64))
        got = attention.group_norm(**case)
        d = signed(total(got["M"]) + total(case["norm"]["U"]))
        assert set(np.unique(d)) <= {-1, 0}
        t = big(total(got["D"]) + total(case["gain"]["T"]))[:, None]
        assert (np.abs(big(total(got["Z"])) - big(total(case["gain"]["bias"]))) <= (np.abs(t) >> f) + 2).all()


def test_group_parts():
    f = 12
    full = group_case(11, 2, 3, 8, 2, f, 5)
    bare = dict(group_case(11, 2, 3, 8, 2, f, 5, gained=False), act=None)
    got = attention.group_norm(**bare)
    assert set(got) == {"M", "S", "Z"}
    d, root = big(total(got["M"]) + total(bare["norm"]["U"])), big(total([t[..., -1] for t in got["S"]]) + total(bare["norm"]["words"])[..., -1])
    assert near_floor(big(total(got["Z"])), d * np.repeat(root, 4, 1)[:, None], f)
    assert set(attention.group_norm(**dict(full, act=None))) == {"M", "S", "Z", "D", "G"}


def test_planted_mistakes_are_found():
    """What the pins would miss, they would miss here."""
    case = prompt_case(3, [0, 7], 1, 1, 4, 6, 3, 13)
    good = attention.linear_attention(**case)
    wrong = [dict(case, decay=np.roll(case["decay"], 1, 1)), dict(case, starts=[0, 6]), dict(case, state=None)]
    for bad in wrong:
        got = attention.linear_attention(**bad)
        assert any(not np.array_equal(total(got[k]), total(good[k])) for k in ("O", "S"))
