"""Two operators on additive shares over Z_{2^64}, as measurable cases: a linear layer whose product is finished in its
epilogue, and the norms of queries and keys with the position rotation behind them.

Both parties are simulated on one GPU.  Every tensor is a pair (party 0, party 1) of 64-bit words, the value is their sum
mod 2^64, a real number v is floor(v 2^f + 1/2), and what a party opens (its share minus a dealer's mask) is an output, the
message that it sends.  Results are whole numbers: there is one right word for every output.

  linear       Y = residual + act(trunc(X W^T + bias)):  Beaver's product with a dealer's triple (A, B, C = A B^T), bias added
               at scale 2^2f, local truncation by f bits, and, where there is an activation, the quadratic
               k2 y^2 + k1 y + k0 on a dealer's square pair (R, Q = R R)
  norm_rotate  for every token and head x -> rotate(gain * x / sqrt(mean(x^2) + eps)), any of the three parts alone where
               that makes sense: the sum of squares from the dealer's sum of squared masks, the inverse root by Newton steps on
               the shares, the gain as a product of its own, the rotation by public angles as a local step

`trunc` by a divisor d is the two parties' local rule: s -> floor(s / d) for party 0, s -> -floor(-s / d) for party 1, s taken
as an unsigned word.

With `own` true `run` calls the public entry points, with `own` false it computes the same words with elementary torch
operations on 64-bit integers (products of matrices through 16-bit pieces in 64-bit floating point, where every sum is exact).
"""
import math

import numpy as np
import torch

own = False

MASK = (1 << 64) - 1


def listed():
    return [
        # one token through a small model's 768 x 768 projection: latency of the call and its launches
        _linear("linear, 1 token, 768 to 768", 1, 768, 768, 13, bias=True),
        # a batch of 32 sequences decodes a token each: the output projection of a 4096-wide model, added to the residual stream
        _linear("linear, 32 tokens, 4096 to 4096", 32, 4096, 4096, 16, bias=True, residual=True),
        # seven sequences on a wide up-projection without bias: nothing but the weights' words counts
        _linear("linear, 7 tokens, 4096 to 11008", 7, 4096, 11008, 16),
        # a prompt through the output projection of a 2048-wide model
        _linear("linear, 512 tokens, 2048 to 2048", 512, 2048, 2048, 16, bias=True, residual=True),
        # the same prompt through the dense first layer of the feed-forward part, with its activation: the heaviest
        _linear("linear, 512 tokens, 2048 to 8192, quadratic", 512, 2048, 8192, 16, bias=True, quadratic=True),
        # a prompt and a layer whose sizes are multiples of nothing, everything switched on
        _linear("linear, 203 tokens, 1000 to 1364, all", 203, 1000, 1364, 12, bias=True, quadratic=True, residual=True),
        # one token's queries and keys, 12 heads of 64 each: latency again
        _norm("heads, 1 token, 12 + 12 of 64", 1, 12, 12, 64, 13, rot=64),
        # a batch of 32 sequences decodes: 32 query and 32 key heads of 128, read out of the stacked q, k, v result
        _norm("heads, 32 tokens, 32 + 32 of 128", 32, 32, 32, 128, 16, rot=128, pad=4096),
        # a prompt of 512 tokens, the same heads: the largest
        _norm("heads, 512 tokens, 32 + 32 of 128", 512, 32, 32, 128, 16, rot=128, pad=4096),
        # a prompt on a model that rotates without a norm
        _norm("rotation alone, 256 tokens, 32 + 32 of 128", 256, 32, 32, 128, 16, norm=False, gain=False, rot=128, pad=4096),
        # whole rows of 4096 instead of heads: the norm before a layer, no rotation
        _norm("rows of 4096, 203 tokens", 203, 1, 0, 4096, 16),
        # few key heads, an odd head size, a part of it rotated, neighbours as pairs
        _norm("heads, 77 tokens, 10 + 2 of 80, 32 rotated", 77, 10, 2, 80, 12, rot=32, pad=160, interleaved=True),
    ]


def _linear(name, tokens, inner, cols, frac, bias=False, residual=False, quadratic=False):
    case = {"kind": "linear", "tokens": tokens, "inner": inner, "cols": cols, "frac": frac, "bias": bias,
            "residual": residual, "quadratic": quadratic}
    return dict(case, name=name) if name else case


def _norm(name, tokens, q_heads, k_heads, dim, frac, norm=True, gain=True, rot=0, pad=0, interleaved=False, steps=10):
    case = {"kind": "norm", "tokens": tokens, "q_heads": q_heads, "k_heads": k_heads, "dim": dim, "frac": frac,
            "norm": norm, "gain": gain, "rot": rot, "pad": pad, "interleaved": interleaved, "steps": steps}
    return dict(case, name=name) if name else case


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    frac = rng.choice((12, 13, 16))
    if rng.random() < 0.5:
        while True:
            tokens, inner, cols = _log_int(rng, 1, 512), 8 * _log_int(rng, 8, 512), 4 * _log_int(rng, 16, 2752)
            if tokens * inner * cols <= 512 * 2048 * 8192 and inner * cols <= 4096 * 11008:
                break
        return _linear(None, tokens, inner, cols, frac, rng.random() < 0.7, rng.random() < 0.5, rng.random() < 0.4)
    kind = rng.choices(("heads", "rows", "rotation"), (6, 2, 2))[0]
    while True:
        tokens = _log_int(rng, 1, 512)
        q_heads = _log_int(rng, 1, 2) if kind == "rows" else _log_int(rng, 1, 32)
        k_heads = 0 if kind == "rows" else max(1, q_heads // rng.choice((1, 1, 2, 4, 8)))
        dim = 2 * (_log_int(rng, 64, 2048) if kind == "rows" else _log_int(rng, 8, 128))
        if tokens * (q_heads + k_heads) * dim <= 512 * 64 * 128:
            break
    rot = 0 if kind == "rows" else rng.choice((dim, dim, 2 * max(1, dim // 8)))
    if kind == "heads" and rng.random() < 0.2:
        rot = 0
    return _norm(None, tokens, q_heads, k_heads, dim, frac, norm=kind != "rotation", gain=kind != "rotation" and rng.random() < 0.8,
                 rot=rot, pad=rng.choice((0, 0, k_heads * dim, 2 * _log_int(rng, 1, 64))), interleaved=rng.random() < 0.4,
                 steps=rng.randint(6, 14))


def work(case):
    """Words that one pass reads and writes once, and its operations."""
    if case["kind"] == "linear":
        T, K, N = case["tokens"], case["inner"], case["cols"]
        # X, A in, E out; W, B in, F out; C in, Y out; R, Q in, M out; residual in; bias in
        words = 3 * T * K + 3 * K * N + 2 * T * N + (3 * T * N if case["quadratic"] else 0)
        words += (T * N if case["residual"] else 0) + (N if case["bias"] else 0)
        # two ring products per party, the fewest known in the fused form of Beaver's product.  A ring multiply-add takes 18
        # multiply-adds of bytes at least, and bytes go through the tensor cores at twice the rate of 16-bit numbers: counted as one
        # operation each
        return {"bytes": 2 * 8 * words, "flops": 2 * 2 * 18 * T * K * N}
    T, H, D = case["tokens"], case["q_heads"] + case["k_heads"], case["dim"]
    words = 2 * T * H * D                                                # X in, Z out
    if case["norm"]:
        words += 3 * T * H * D + T * H * (9 * case["steps"] - 4)         # U, product in, message out; a row's own words
    if case["gain"]:
        words += 3 * T * H * D + 3 * _gains(case) * D                    # A, C in, message out; the gain, its mask, its message
    # the angles are public and serve both parties
    tables = T * case["rot"] if case["rot"] else 0
    # word multiplications of the element-wise steps, both parties
    per = (6 if case["norm"] else 0) + (3 if case["gain"] else 0)
    return {"bytes": 8 * (2 * words + tables), "flops": 2 * 2 * (per * T * H * D + 2 * T * H * case["rot"])}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
class _Draw:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def words(self, *shape):
        return torch.randint(-(1 << 63), (1 << 63) - 1, shape, generator=self.g, device="cuda", dtype=torch.int64)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float64)

    def share(self, value):
        """A uniform share for party 0, the rest for party 1."""
        s = self.words(*value.shape)
        return [s, value - s]


def _encode(v, frac):
    return torch.floor(v * float(1 << frac) + 0.5).to(torch.int64)


def _gains(case):
    return 2 if case["q_heads"] and case["k_heads"] else 1


def _guess(case):
    """Newton's starting value: the inputs' mean squares lie in (1/8, 8), and 0.55 is below sqrt(3 / 8)."""
    return int(0.55 * (1 << case["frac"]))


def prepare(case, seed):
    d = _Draw(seed)
    f = case["frac"]
    if case["kind"] == "linear":
        T, K, N = case["tokens"], case["inner"], case["cols"]
        s = {"case": case,
             "X": d.share(_encode(d.normal(T, K), f)), "W": d.share(_encode(d.normal(N, K) / math.sqrt(K), f)),
             "A": [d.words(T, K), d.words(T, K)], "B": [d.words(N, K), d.words(N, K)], "bias": None, "act": None, "residual": None}
        s["C"] = d.share(_matmul(s["A"][0] + s["A"][1], s["B"][0] + s["B"][1]))
        if case["bias"]:
            s["bias"] = d.share(_encode(0.5 * d.normal(N), f))
        if case["residual"]:
            s["residual"] = d.share(_encode(d.normal(T, N), f))
        if case["quadratic"]:
            R = [d.words(T, N), d.words(T, N)]
            s["act"] = (tuple(int(v * (1 << f)) for v in (0.5, 0.25, 0.125)), R, d.share((R[0] + R[1]) * (R[0] + R[1])))
        return s
    T, H, D, n = case["tokens"], case["q_heads"] + case["k_heads"], case["dim"], case["steps"]
    # heads differ in size by up to a factor of four: mean squares in (1/4, 4), and the rows of a token lie `pad` words apart
    size = torch.exp2(2.0 * torch.rand((1, H, 1), generator=d.g, device="cuda", dtype=torch.float64) - 1.0)
    value = _encode(size * d.normal(T, H, D), f)
    X = []
    for share in d.share(value):
        rows = d.words(T, H * D + case["pad"])
        rows[:, :H * D] = share.view(T, H * D)
        X.append(rows[:, :H * D].view(T, H, D))
    s = {"case": case, "X": X, "norm": None, "gain": None, "rotation": None}
    if case["norm"]:
        U = [d.words(T, H, D), d.words(T, H, D)]
        u = U[0] + U[1]
        # a row's own words: sum of the squared masks, mask a of the mean square, per Newton step behind the first the mask of y,
        # its square, the mask of p, its product with a, the mask of w, its product with that of y; the mask of the root
        own_words = torch.empty((T, H, 6 * n - 3), dtype=torch.int64, device="cuda")
        own_words[..., 0] = (u * u).sum(-1)
        a = own_words[..., 1] = d.words(T, H)
        for k in range(n - 1):
            y, p, w = d.words(T, H), d.words(T, H), d.words(T, H)
            own_words[..., 2 + 6 * k:8 + 6 * k] = torch.stack((y, y * y, p, a * p, w, y * w), -1)
        v = own_words[..., 6 * n - 4] = d.words(T, H)
        s["norm"] = dict(U=U, words=d.share(own_words), UV=d.share(u * v[..., None]), steps=n, guess=_guess(case),
                         eps=max(1, (1 << f) // 100000))
    if case["gain"]:
        weight = d.share(_encode(1.0 + 0.2 * d.normal(_gains(case), D), f))
        mask = [d.words(_gains(case), D), d.words(_gains(case), D)]
        A = [d.words(T, H, D), d.words(T, H, D)]
        b = _per_head(mask[0] + mask[1], case)
        s["gain"] = dict(weight=weight, mask=mask, A=A, C=d.share((A[0] + A[1]) * b))
    if case["rot"]:
        # positions of a batch: anywhere in a context of 4096
        half = case["rot"] // 2
        angle = torch.arange(4096, device="cuda", dtype=torch.float64)[:, None] * \
            torch.pow(10000.0, -torch.arange(half, device="cuda", dtype=torch.float64) / half)
        s["rotation"] = dict(cos=_encode(torch.cos(angle), f), sin=_encode(torch.sin(angle), f),
                             positions=torch.randint(0, 4096, (T,), generator=d.g, device="cuda", dtype=torch.int32),
                             interleaved=case["interleaved"])
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(state):
    if own:
        return _run_own(state)
    return _plain_linear(state) if state["case"]["kind"] == "linear" else _plain_norm(state)


def _run_own(s):
    from paper_2505_07239_b200 import binding as cb

    case = s["case"]
    stream = torch.cuda.current_stream()
    if case["kind"] == "linear":
        E, F, M, Y = cb.linear(s["X"], s["A"], s["W"], s["B"], s["C"], case["frac"], bias=s["bias"], act=s["act"],
                               residual=s["residual"], stream=stream)
        return {"E": E, "F": F, "Y": Y, **({"M": M} if M is not None else {})}
    norm = cb.Norm(**s["norm"]) if s["norm"] else None
    gain = cb.Gain(**s["gain"]) if s["gain"] else None
    rotation = cb.Rotation(**s["rotation"]) if s["rotation"] else None
    msg, Z = cb.norm_rotate(s["X"], case["frac"], norm=norm, gain=gain, rotation=rotation, q_heads=case["q_heads"], stream=stream)
    out = {"Z": Z}
    if norm:
        out.update(M=msg.M, S=msg.S)
    if gain:
        out.update(D=msg.D, G=msg.G)
    return out


# ---------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------
def _matmul(a, b):
    """a b^T mod 2^64.  Words in four pieces of 16 bits; a sum of K products of pieces stays below 2^53 for K up to 2^21."""
    def pieces(x):
        return [((x >> (16 * p)) & 0xFFFF).to(torch.float64) for p in range(4)]

    left, right = pieces(a), pieces(b)
    out = torch.zeros((a.shape[0], b.shape[0]), dtype=torch.int64, device=a.device)
    for p in range(4):
        for q in range(4 - p):
            out += (left[p] @ right[q].t()).to(torch.int64) << (16 * (p + q))
    return out


def _shift(x, bits):
    """Unsigned shift to the right."""
    return (x >> bits) & (MASK >> bits)


def _truncate(x, party, bits):
    return _shift(x, bits) if party == 0 else -_shift(-x, bits)


def _divide(x, party, divisor):
    def unsigned(v):
        q = _shift(v, 1) // divisor * 2
        return q + (v - q * divisor >= divisor).to(torch.int64)

    return unsigned(x) if party == 0 else -unsigned(-x)


def _plain_linear(s):
    f = s["case"]["frac"]
    E = [s["X"][i] - s["A"][i] for i in (0, 1)]
    F = [s["W"][i] - s["B"][i] for i in (0, 1)]
    e, w = E[0] + E[1], F[0] + F[1]
    Y = []
    for i in (0, 1):
        z = s["C"][i] + _matmul(e, s["B"][i] + (w if i else 0)) + _matmul(s["A"][i], w)
        if s["bias"] is not None:
            z = z + (s["bias"][i] << f)
        Y.append(_truncate(z, i, f))
    out = {"E": E, "F": F, "Y": Y}
    if s["act"] is not None:
        (k0, k1, k2), R, Q = s["act"]
        M = [Y[i] - R[i] for i in (0, 1)]
        m = M[0] + M[1]
        for i in (0, 1):
            square = _truncate(Q[i] + 2 * m * R[i] + (m * m if i else 0), i, f)
            Y[i] = _truncate(k2 * square + k1 * Y[i], i, f) + (k0 if i else 0)
        out["M"] = M
    if s["residual"] is not None:
        out["Y"] = [Y[i] + s["residual"][i] for i in (0, 1)]
    return out


def _per_head(t, case):
    """[gains, D] to [H, D]: the first for the query heads, the last for the key heads."""
    return torch.cat((t[:1].expand(case["q_heads"], -1), t[-1:].expand(case["k_heads"], -1)))


def _plain_norm(s):
    case = s["case"]
    f, z, out = case["frac"], s["X"], {}
    if s["norm"]:
        U, words, UV, n = s["norm"]["U"], s["norm"]["words"], s["norm"]["UV"], s["norm"]["steps"]
        guess, eps, three = s["norm"]["guess"], s["norm"]["eps"], 3 << f
        M = [z[i] - U[i] for i in (0, 1)]
        m = M[0] + M[1]
        S = [torch.empty((*m.shape[:2], 3 * n - 1), dtype=torch.int64, device=m.device) for _ in (0, 1)]

        def opened(v, mask, at):
            for i in (0, 1):
                S[i][..., at] = v[i] - words[i][..., mask]
            return S[0][..., at] + S[1][..., at]

        square = [words[i][..., 0] + (2 * m * U[i] + (m * m if i else 0)).sum(-1) for i in (0, 1)]
        ms = [_divide(square[i], i, case["dim"] << f) + (eps if i else 0) for i in (0, 1)]
        first = guess * guess >> f
        y = [_truncate(guess * ((three if i else 0) - _truncate(ms[i] * first, i, f)), i, f + 1) for i in (0, 1)]
        g = opened(ms, 1, 0)
        for k in range(n - 1):
            mat = [[words[i][..., 2 + 6 * k + j] for j in range(6)] for i in (0, 1)]
            d = opened(y, 2 + 6 * k, 1 + 3 * k)
            p = [_truncate(mat[i][1] + 2 * d * mat[i][0] + (d * d if i else 0), i, f) for i in (0, 1)]
            e = opened(p, 4 + 6 * k, 2 + 3 * k)
            w = [(three if i else 0) - _truncate(mat[i][3] + g * mat[i][2] + e * words[i][..., 1] + (g * e if i else 0), i, f)
                 for i in (0, 1)]
            h = opened(w, 6 + 6 * k, 3 + 3 * k)
            y = [_truncate(mat[i][5] + d * mat[i][4] + h * mat[i][0] + (d * h if i else 0), i, f + 1) for i in (0, 1)]
        r = opened(y, 6 * n - 4, 3 * n - 2)[..., None]
        z = [_truncate(UV[i] + m * words[i][..., 6 * n - 4, None] + r * U[i] + (m * r if i else 0), i, f) for i in (0, 1)]
        out.update(M=M, S=S)
    if s["gain"]:
        weight, mask, A, C = (s["gain"][k] for k in ("weight", "mask", "A", "C"))
        G = [weight[i] - mask[i] for i in (0, 1)]
        D = [z[i] - A[i] for i in (0, 1)]
        d, e = D[0] + D[1], _per_head(G[0] + G[1], case)
        z = [_truncate(C[i] + d * _per_head(mask[i], case) + e * A[i] + (d * e if i else 0), i, f) for i in (0, 1)]
        out.update(D=D, G=G)
    if s["rotation"]:
        half = case["rot"] // 2
        at = s["rotation"]["positions"].long()
        c, t = s["rotation"]["cos"][at][:, None], s["rotation"]["sin"][at][:, None]
        turned = []
        for i in (0, 1):
            o = z[i].clone()
            one, two = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if case["interleaved"] else (slice(0, half), slice(half, 2 * half))
            x, y = z[i][..., one], z[i][..., two]
            o[..., one] = _truncate(x * c - y * t, i, f)
            o[..., two] = _truncate(y * c + x * t, i, f)
            turned.append(o)
        z = turned
    out["Z"] = z
    return out


# ---------------------------------------------------------------------------
# the definition, in numpy on the host's 64-bit unsigned words
# ---------------------------------------------------------------------------
def _ring_product(a, b):
    """a b^T mod 2^64 with pieces of 22, 21 and 21 bits and sums of at most 256 products, below 2^52."""
    starts, widths = (0, 22, 43), (22, 21, 21)
    cut = [[((x >> np.uint64(s)) & np.uint64((1 << w) - 1)).astype(np.float64) for s, w in zip(starts, widths)] for x in (a, b)]
    total = np.zeros((a.shape[0], b.shape[0]), np.uint64)
    for k in range(0, a.shape[1], 256):
        for p in range(3):
            for q in range(3):
                if starts[p] + starts[q] < 64:
                    part = cut[0][p][:, k:k + 256] @ cut[1][q][:, k:k + 256].T
                    total += part.astype(np.uint64) << np.uint64(starts[p] + starts[q])
    return total


def _local(share, party, divisor):
    """One party's half of a division by a public number."""
    d = np.uint64(divisor)
    return share // d if party == 0 else np.uint64(0) - (np.uint64(0) - share) // d


def exact(case, seed):
    if case["kind"] == "linear" and case["tokens"] * case["inner"] * case["cols"] > 3 << 30:
        return None
    state = prepare(case, seed)

    def host(v):
        if isinstance(v, torch.Tensor):
            return v.cpu().numpy().view(np.uint64) if v.dtype == torch.int64 else v.cpu().numpy()
        if isinstance(v, dict):
            return {k: host(x) for k, x in v.items() if k != "case"}
        return [host(x) for x in v] if isinstance(v, (list, tuple)) else v

    with np.errstate(over="ignore"):
        result = (_exact_linear if case["kind"] == "linear" else _exact_norm)(case, host(state))
    return {k: [torch.from_numpy(np.ascontiguousarray(x).view(np.int64)) for x in v] for k, v in result.items()}


def _u(v):
    return np.uint64(v & MASK)


def _exact_linear(case, s):
    one = 1 << case["frac"]
    E = [x - a for x, a in zip(s["X"], s["A"])]
    F = [w - b for w, b in zip(s["W"], s["B"])]
    e, f = E[0] + E[1], F[0] + F[1]
    Y = [s["C"][0] + _ring_product(e, s["B"][0]) + _ring_product(s["A"][0], f),
         s["C"][1] + _ring_product(e, s["B"][1]) + _ring_product(s["A"][1] + e, f)]
    if case["bias"]:
        Y = [y + b * _u(one) for y, b in zip(Y, s["bias"])]
    Y = [_local(y, i, one) for i, y in enumerate(Y)]
    out = {"E": E, "F": F}
    if case["quadratic"]:
        (k0, k1, k2), R, Q = s["act"]
        out["M"] = M = [y - r for y, r in zip(Y, R)]
        m = M[0] + M[1]
        squares = [Q[0] + m * R[0] + m * R[0], Q[1] + m * (R[1] + R[1] + m)]
        Y = [_local(_u(k2) * _local(q, i, one) + _u(k1) * y, i, one) for i, (q, y) in enumerate(zip(squares, Y))]
        Y[1] = Y[1] + _u(k0)
    out["Y"] = [y + r for y, r in zip(Y, s["residual"])] if case["residual"] else Y
    return out


def _beaver(c, a, b, d, e):
    """Shares of (a + d)(b + e) from those of a, b and c = a b."""
    return [c[0] + d * b[0] + e * a[0], c[1] + d * b[1] + e * a[1] + d * e]


def _exact_norm(case, s):
    one, z, out = 1 << case["frac"], s["X"], {}
    if case["norm"]:
        m_, n = s["norm"], case["steps"]
        word = [[m_["words"][i][..., j] for i in (0, 1)] for j in range(6 * n - 3)]
        sent = []

        def reveal(v, mask):
            sent.append([v[i] - mask[i] for i in (0, 1)])
            return sent[-1][0] + sent[-1][1]

        M = [z[i] - m_["U"][i] for i in (0, 1)]
        m = M[0] + M[1]
        cross = [(m * m_["U"][i]).sum(-1, dtype=np.uint64) for i in (0, 1)]
        total = [word[0][i] + cross[i] + cross[i] for i in (0, 1)]
        total[1] = total[1] + (m * m).sum(-1, dtype=np.uint64)
        ms = [_local(total[i], i, case["dim"] * one) for i in (0, 1)]
        ms[1] = ms[1] + _u(m_["eps"])
        three = [_u(0), _u(3 * one)]
        guess = m_["guess"]
        y = [_local(_u(guess) * (three[i] - _local(ms[i] * _u(guess * guess // one), i, one)), i, 2 * one) for i in (0, 1)]
        a = word[1]
        da = reveal(ms, a)
        for k in range(n - 1):
            my, myy, mp, map_, mw, myw = word[2 + 6 * k:8 + 6 * k]
            dy = reveal(y, my)
            p = [_local(v, i, one) for i, v in enumerate(_beaver(myy, my, my, dy, dy))]
            dp = reveal(p, mp)
            w = [three[i] - _local(v, i, one) for i, v in enumerate(_beaver(map_, a, mp, da, dp))]
            dw = reveal(w, mw)
            y = [_local(v, i, 2 * one) for i, v in enumerate(_beaver(myw, my, mw, dy, dw))]
        v = word[6 * n - 4]
        root = reveal(y, v)[..., None]
        z = [_local(x, i, one) for i, x in enumerate(_beaver(m_["UV"], m_["U"], [v[i][..., None] for i in (0, 1)], m, root))]
        out["M"] = M
        out["S"] = [np.stack([t[i] for t in sent], -1) for i in (0, 1)]
    if case["gain"]:
        g = s["gain"]
        row = np.array([0] * case["q_heads"] + [_gains(case) - 1] * case["k_heads"])
        out["G"] = G = [g["weight"][i] - g["mask"][i] for i in (0, 1)]
        out["D"] = D = [z[i] - g["A"][i] for i in (0, 1)]
        z = [_local(x, i, one) for i, x in enumerate(
            _beaver(g["C"], g["A"], [g["mask"][i][row] for i in (0, 1)], D[0] + D[1], (G[0] + G[1])[row]))]
    if case["rot"]:
        r, half = s["rotation"], case["rot"] // 2
        c, t = r["cos"][r["positions"]][:, None, :], r["sin"][r["positions"]][:, None, :]
        first = np.arange(half) * (2 if case["interleaved"] else 1)
        second = first + (1 if case["interleaved"] else half)
        z = [v.copy() for v in z]
        for i in (0, 1):
            x, y = z[i][..., first], z[i][..., second]
            z[i][..., first], z[i][..., second] = _local(x * c - y * t, i, one), _local(y * c + x * t, i, one)
    out["Z"] = z
    return out
