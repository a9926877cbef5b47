"""TEST INFRASTRUCTURE -- plain statements of linear attention on shares, for prompts and for single tokens, and of the norm of channel
groups with gain, bias and activation.

Composed like oracle/layers.py: every product goes through Eq. 1 with a dealer's triple, every rescaling through the two parties'
local division.  numpy uint64 words; a pair is (party 0, party 1).

Pins (tests/test_oracle_attention.py): Python integers and float64 on the reconstructed values, tokens one by one against a prompt in chunks,
closed forms.
"""
from __future__ import annotations

import numpy as np

from .layers import U64, _divide, _eq1, _open, _public, _trunc


def product(c, a, b, d, e):
    """Matrix form of Eq. 1: [c]_i + d [b]_i + [a]_i e + i d e (numpy multiplies uint64 matrices mod 2^64)."""
    z = [c[i] + d @ b[i] + a[i] @ e for i in (0, 1)]
    z[1] = z[1] + d @ e
    return z


def _times(pair, word):
    return [v * word for v in pair]


def linear_attention(Q, K, V, starts, decay, dealer, frac_bits, state=None):
    """Q [T, Hq, Dk], K [T, Hk, Dk], V [T, Hk, Dv]; starts ascending; decay [Hk, C + 1]; dealer: dict of pairs q, k, v, d, p, s, qk, pv, qs, dv.
    Returns dict of pairs: the messages q, k, v, d, p, s, the result O and the states S.  Words that are not written are zero."""
    f, C, m = frac_bits, decay.shape[1] - 1, dealer
    (T, Hq, Dk), (_, Hk, Dv) = Q[0].shape, V[0].shape
    n_seq, group = len(starts) - 1, Hq // Hk
    out = {k: [np.zeros_like(v) for v in m[k]] for k in ("q", "k", "v", "d", "p", "s")}
    out["O"] = [np.zeros((T, Hq, Dv), U64) for _ in (0, 1)]
    out["S"] = [np.zeros((n_seq, Hk, Dk, Dv), U64) for _ in (0, 1)] if state is None else [v.copy() for v in state]
    with np.errstate(over="ignore"):
        number = 0
        for j in range(n_seq):
            for first in range(starts[j], starts[j + 1], C):
                L = min(C, starts[j + 1] - first)
                rows = slice(first, first + L)
                at = np.arange(L)
                below = at[:, None] >= at[None]
                for h in range(Hk):
                    w = decay[h]
                    part = lambda pair, head: [np.ascontiguousarray(v[rows, head]) for v in pair]

                    def opened(name, value, head):
                        msg, e = _open(value, part(m[name], head))
                        for i in (0, 1):
                            out[name][i][rows, head] = msg[i]
                        return e

                    k, v = part(K, h), part(V, h)
                    ke, ve = opened("k", k, h), opened("v", v, h)
                    km, vm = part(m["k"], h), part(m["v"], h)
                    S, sm = [out["S"][i][j, h] for i in (0, 1)], [m["s"][i][number, h] for i in (0, 1)]
                    msg, se = _open(S, sm)
                    for i in (0, 1):
                        out["s"][i][number, h] = msg[i]
                    for hq in range(h * group, (h + 1) * group):
                        qe, qm = opened("q", part(Q, hq), hq), part(m["q"], hq)
                        scores = product([t[:, :L] for t in part(m["qk"], hq)], qm, [t.T for t in km], qe, ke.T)
                        P = _trunc(_times(_trunc(scores, f), w[np.where(below, at[:, None] - at[None], 0)]), f)
                        P, pm = ([np.where(below, t[:, :L], U64(0)) for t in pair] for pair in (P, part(m["p"], hq)))
                        msg, pe = _open(P, pm)
                        near = product(part(m["pv"], hq), pm, vm, pe, ve)
                        far = _trunc(product(part(m["qs"], hq), qm, sm, qe, se), f)
                        o = _trunc([near[i] + w[1:L + 1, None] * far[i] for i in (0, 1)], f)
                        for i in (0, 1):
                            out["p"][i][rows, hq, :L] = msg[i]
                            out["O"][i][rows, hq] = o[i]
                    de = opened("d", _trunc(_times(k, w[L - 1 - at][:, None]), f), h)
                    add = product([t[number, h] for t in m["dv"]], [t.T for t in part(m["d"], h)], vm, de.T, ve)
                    S = _trunc([w[L] * S[i] + add[i] for i in (0, 1)], f)
                    for i in (0, 1):
                        out["S"][i][j, h] = S[i]
                number += 1
    return out


def linear_attention_step(Q, K, V, decay, dealer, frac_bits, state=None):
    """Q [B, Hq, Dk], K [B, Hk, Dk], V [B, Hk, Dv]; decay [Hk]; dealer: dict of pairs q, k, v, s, kv, qs."""
    f, m = frac_bits, dealer
    (B, Hq, _), Hk = Q[0].shape, K[0].shape[1]
    state = [np.zeros_like(v) for v in m["s"]] if state is None else state
    out = {}
    with np.errstate(over="ignore"):
        out["q"], qe = _open(Q, m["q"])
        out["k"], ke = _open(K, m["k"])
        out["v"], ve = _open(V, m["v"])
        col, row = (lambda t: t[..., :, None]), (lambda t: t[..., None, :])
        add = _eq1(m["kv"], [col(t) for t in m["k"]], [row(t) for t in m["v"]], col(ke), row(ve))
        out["S"] = _trunc([decay[:, None, None] * state[i] + add[i] for i in (0, 1)], f)
        out["s"], se = _open(out["S"], m["s"])
        out["O"] = [np.zeros_like(t) for t in m["qs"]]
        for b in range(B):
            for h in range(Hq):
                s = h // (Hq // Hk)
                o = _trunc(product([t[b, h][None] for t in m["qs"]], [t[b, h][None] for t in m["q"]], [t[b, s] for t in m["s"]], qe[b, h][None], se[b, s]), f)
                for i in (0, 1):
                    out["O"][i][b, h] = o[i][0]
    return out


def group_norm(X, groups, frac_bits, norm, gain=None, act=None):
    """X [S, P, C].  norm = dict(U, words, UT, steps, guess, eps); gain = dict(weight, mask, T, VW, bias); act = ((k0, k1, k2), R, Q).
    Returns dict of pairs Z, M, S and, as the parts are there, D, G, N."""
    f, out, sent = frac_bits, {}, []
    S, P, C = X[0].shape
    per = C // groups
    total = lambda t: t.reshape(S, P, groups, per).sum((1, 3), dtype=U64)
    wide = lambda pair: [np.repeat(t, per, 1) for t in pair]                       # [S, groups] to [S, C]

    def reveal(v, mask):
        msg, value = _open(v, mask)
        sent.append(msg)
        return value

    with np.errstate(over="ignore"):
        words = [[norm["words"][i][..., j] for i in (0, 1)] for j in range(norm["words"][0].shape[-1])]
        mean = wide([_divide(total(X[i]), i, P * per) for i in (0, 1)])
        out["M"], m = _open([X[i] - mean[i][:, None] for i in (0, 1)], norm["U"])
        squares = _eq1([np.zeros_like(m)] * 2, norm["U"], norm["U"], m, m)
        s = [_divide(words[0][i] + total(squares[i]), i, P * per << f) for i in (0, 1)]
        s[1] = s[1] + U64(norm["eps"])
        three = _public(3 << f, (S, groups))
        w = _trunc(_times(s, U64(norm["guess"] * norm["guess"] >> f)), f)
        y = _trunc([U64(norm["guess"]) * (three[i] - w[i]) for i in (0, 1)], f + 1)
        ds = reveal(s, words[1])
        for k in range(norm["steps"] - 1):
            ym, yy, pm, ap, wm, yw = words[2 + 6 * k:8 + 6 * k]
            dy = reveal(y, ym)
            p = _trunc(_eq1(yy, ym, ym, dy, dy), f)
            sp = _trunc(_eq1(ap, words[1], pm, ds, reveal(p, pm)), f)
            w = [three[i] - sp[i] for i in (0, 1)]
            y = _trunc(_eq1(yw, ym, wm, dy, reveal(w, wm)), f + 1)
        root, mask = reveal(y, words[-1]), words[-1]
        out["S"] = [np.stack([msg[i] for msg in sent], -1) for i in (0, 1)]
        t, mask = wide([root, root])[0], wide(mask)
        bias = _public(0)
        if gain is not None:
            out["G"], e = _open(gain["weight"], gain["mask"])
            scaled = _trunc(_eq1(gain["VW"], mask, gain["mask"], t, e), f)
            mask = gain["T"]
            out["D"], t = _open(scaled, mask)
            bias = _times(gain["bias"], U64(1 << f))
        z = _eq1(norm["UT"], norm["U"], [v[:, None] for v in mask], m, t[:, None])
        z = _trunc([z[i] + bias[i] for i in (0, 1)], f)
        if act is not None:
            (k0, k1, k2), R, Q = act
            word = lambda k: U64(k & ((1 << 64) - 1))
            out["N"], b = _open(z, R)
            square = _trunc(_eq1(Q, R, R, b, b), f)
            z = _trunc([word(k2) * square[i] + word(k1) * z[i] for i in (0, 1)], f)
            z[1] = z[1] + word(k0)
        out["Z"] = z
    return out
