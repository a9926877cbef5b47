"""TEST INFRASTRUCTURE -- plain statements of the shared linear layer's epilogue and of the norm and rotation of shared heads.

Both are composed of Section 2.1's Multiplication (Eq. 1 with a dealer's triple) and Addition and of the two parties' local
truncation, so they are written here from those: every product goes through `_eq1`, every rescaling through `_divide`.  numpy
uint64 words; a pair is (party 0, party 1); party 1 carries the public terms.

Pins (tests/test_oracle_layers.py): the sums of the shares against Python integers and against float64 within the truncations'
errors, closed forms (zero masks, position 0, a quarter turn, a constant row) and planted mistakes.
"""
from __future__ import annotations

import numpy as np

from . import pi_matmul

U64 = np.uint64


def _divide(share, party: int, divisor: int):
    """The party's half of a division of a shared number by a public one."""
    d = U64(divisor)
    return share // d if party == 0 else U64(0) - (U64(0) - share) // d


def _trunc(pair, bits: int):
    return [_divide(pair[i], i, 1 << bits) for i in (0, 1)]


def _open(x, mask):
    """Messages x_i - mask_i and the opened value."""
    msg = [x[i] - mask[i] for i in (0, 1)]
    return msg, msg[0] + msg[1]


def _eq1(c, a, b, d, e):
    """[c]_i + d [b]_i + e [a]_i + i d e."""
    z = [c[i] + d * b[i] + e * a[i] for i in (0, 1)]
    z[1] = z[1] + d * e
    return z


def _public(value: int, shape=()):
    return [np.zeros(shape, U64), np.full(shape, value & ((1 << 64) - 1), U64)]


def linear(X, A, W, B, C, frac_bits, bias=None, act=None, residual=None):
    """X, A [T, K]; W, B [N, K]; C [T, N]; act = ((k0, k1, k2), R, Q).  Returns dict of pairs E, F [N, K], Y and, with an
    activation, M."""
    with np.errstate(over="ignore"):
        t = lambda p: [np.ascontiguousarray(v.T) for v in p]                 # the oracle's right operands are [K, N]
        product = pi_matmul(X, t(W), A, t(B), C)
        z = [product["Z"][i] for i in (0, 1)]
        if bias is not None:
            z = [z[i] + bias[i] * U64(1 << frac_bits) for i in (0, 1)]
        y = _trunc(z, frac_bits)
        out = {"E": list(product["E"]), "F": t(product["F"])}
        if act is not None:
            (k0, k1, k2), R, Q = act
            out["M"], m = _open(y, R)
            square = _trunc(_eq1(Q, R, R, m, m), frac_bits)
            mixed = [U64(k2 & ((1 << 64) - 1)) * square[i] + U64(k1 & ((1 << 64) - 1)) * y[i] for i in (0, 1)]
            y = _trunc(mixed, frac_bits)
            y[1] = y[1] + U64(k0 & ((1 << 64) - 1))
        if residual is not None:
            y = [y[i] + residual[i] for i in (0, 1)]
        out["Y"] = y
        return out


def norm_rotate(X, frac_bits, norm=None, gain=None, rotation=None, q_heads=None):
    """X [T, H, D].  norm = dict(U, words, UV, steps, guess, eps); gain = dict(weight, mask, A, C); rotation = dict(cos, sin,
    positions, interleaved).  Returns dict of pairs Z and M, S, D, G as the parts are there."""
    f, out = frac_bits, {}
    x = [np.ascontiguousarray(v) for v in X]
    T, H, dim = x[0].shape
    with np.errstate(over="ignore"):
        if norm is not None:
            words, sent = norm["words"], []

            def word(j):
                return [words[i][..., j] for i in (0, 1)]

            def reveal(v, mask):
                msg, value = _open(v, mask)
                sent.append(msg)
                return value

            out["M"], m = _open(x, norm["U"])
            squares = _eq1([np.zeros_like(m)] * 2, norm["U"], norm["U"], m, m)
            total = [word(0)[i] + squares[i].sum(-1, dtype=U64) for i in (0, 1)]
            s = [_divide(total[i], i, dim << f) for i in (0, 1)]
            s[1] = s[1] + U64(norm["eps"])
            three = _public(3 << f, (T, H))
            first = U64(norm["guess"] * norm["guess"] >> f)
            w = _trunc([first * s[i] for i in (0, 1)], f)
            y = _trunc([U64(norm["guess"]) * (three[i] - w[i]) for i in (0, 1)], f + 1)
            ds = reveal(s, word(1))
            for k in range(norm["steps"] - 1):
                ym, yy, pm, ap, wm, yw = (word(2 + 6 * k + j) for j in range(6))
                dy = reveal(y, ym)
                p = _trunc(_eq1(yy, ym, ym, dy, dy), f)
                dp = reveal(p, pm)
                sp = _trunc(_eq1(ap, word(1), pm, ds, dp), f)
                w = [three[i] - sp[i] for i in (0, 1)]
                dw = reveal(w, wm)
                y = _trunc(_eq1(yw, ym, wm, dy, dw), f + 1)
            v = word(6 * norm["steps"] - 4)
            root = reveal(y, v)
            x = _trunc(_eq1(norm["UV"], norm["U"], [t[..., None] for t in v], m, root[..., None]), f)
            out["S"] = [np.stack([msg[i] for msg in sent], -1) for i in (0, 1)]
        if gain is not None:
            row = np.where(np.arange(H) < (H if q_heads is None else q_heads), 0, gain["weight"][0].shape[0] - 1)
            out["D"], d = _open(x, gain["A"])
            out["G"], e = _open(gain["weight"], gain["mask"])
            x = _trunc(_eq1(gain["C"], gain["A"], [gain["mask"][i][row][None] for i in (0, 1)], d, e[row][None]), f)
        if rotation is not None:
            cos, sin, at = rotation["cos"], rotation["sin"], rotation["positions"]
            half = cos.shape[1]
            inside = (at >= 0) & (at < cos.shape[0])
            c, t = ((np.where(inside[:, None], tab[np.where(inside, at, 0)], U64(0)))[:, None, :] for tab in (cos, sin))
            j = np.arange(half)
            one, two = (2 * j, 2 * j + 1) if rotation["interleaved"] else (j, j + half)
            a, b = [v[..., one] for v in x], [v[..., two] for v in x]
            x = [v.copy() for v in x]
            turned = _trunc([a[i] * c - b[i] * t for i in (0, 1)], f), _trunc([b[i] * c + a[i] * t for i in (0, 1)], f)
            for i in (0, 1):
                x[i][..., one], x[i][..., two] = turned[0][i], turned[1][i]
    out["Z"] = x
    return out
