"""Attention without a softmax and the norm behind it, on additive shares over Z_{2^64}, as measurable cases: linear attention with
a decay for every head, for prompts in chunks and for single tokens, and the norm of groups of channels with its activation.

Both parties are simulated on one GPU.  Every tensor is a pair (party 0, party 1) of 64-bit words, the value is their sum
mod 2^64, a real number v is floor(v 2^f + 1/2), and what a party opens (its share minus a dealer's mask) is an output, the
message that it sends.  Results are whole numbers: there is one right word for every output.  tr is the parties' local truncation by
f bits, div_d the same by a divisor d (s -> floor(s / d) for party 0, s -> -floor(-s / d) for party 1, s taken as an unsigned word),
w the public powers of a head's decay at scale f, w[n] = decay^n.

  prompt   sequences of any lengths packed behind one another, each in chunks of C tokens, the last one shorter; of a chunk of L
           tokens that finds the state S [k_dim, v_dim]:
             P[r, s] = tr(w[r - s] tr(q_r . k_s)) for s <= r,   O_r = tr(sum_{s <= r} P[r, s] v_s + w[r + 1] tr(q_r S))
             d_s = tr(w[L - 1 - s] k_s),                        S <- tr(w[L] S + sum_s d_s v_s^T)
  step     one token for every sequence of a batch:  S <- tr(w S + k v^T),  o = tr(q S)
  group    x [samples, positions, channels], its channels in groups of neighbours; of every sample and group, n words:
             d = x - div_n(sum x),  s = div_{n 2^f}(sum d^2) + eps,  y ~ 1 / sqrt(s) by Newton steps on the shares
             t_c = tr(y gain_c),  z = tr(t_c d + 2^f bias_c)  (without a gain z = tr(y d)), then k2 z^2 + k1 z + k0 where there is an activation

Every value that enters a product is masked and opened once, and the dealer hands out the products of the masks.

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
        # a first message to a small model of 12 heads: latency of the whole call
        _prompt("prompt, 16 tokens, 12 heads of 64", "16", 12, 12, 64, 64, 64, 13),
        # four users' prompts in one batch, one of them a single token, on a model of few key heads and odd head sizes
        _prompt("prompts of 1+64+77+61, 10 on 2 of 80x96", "1+64+77+61", 10, 2, 80, 96, 48, 12, state=True),
        # a prompt on a model of 32 heads
        _prompt("prompt, 512 tokens, 32 heads of 128", "512", 32, 32, 128, 128, 64, 16),
        # further parts of eight long documents, their states known, grouped heads: the longest
        _prompt("prompts, 8 x 256, 32 on 8 of 128", "+".join(["256"] * 8), 32, 8, 128, 128, 64, 16, state=True),
        # one user's next token on the small model
        _step("step, 1 sequence, 12 heads of 64", 1, 12, 12, 64, 64, 13),
        # a batch of 32 sequences decodes: nothing but the states' words counts
        _step("step, 32 sequences, 32 heads of 128", 32, 32, 32, 128, 128, 16),
        # an odd batch, few key heads, odd head sizes
        _step("step, 7 sequences, 10 on 2 of 80x96", 7, 10, 2, 80, 96, 12),
        # one token's heads behind the attention, no gain, no activation
        _group("heads, 1 token, 12 of 64", 1, 1, 768, 12, 13, gain=False),
        # the same of a prompt, with gain, bias and activation
        _group("heads, 512 tokens, 32 of 128", 512, 1, 4096, 32, 16, quadratic=True),
        # feature maps of an image encoder, channels last: one of 64 x 64, a batch of 32 x 32
        _group("map, 1 x 4096 x 320 in 32", 1, 4096, 320, 32, 16, quadratic=True),
        _group("maps, 8 x 1024 x 640 in 32", 8, 1024, 640, 32, 16, quadratic=True),
        # sizes that are multiples of nothing
        _group("maps, 3 x 77 x 90 in 5", 3, 77, 90, 5, 12, pad=6, quadratic=True),
    ]


def _prompt(name, lengths, q_heads, kv_heads, k_dim, v_dim, chunk, frac, state=False):
    case = {"kind": "prompt", "lengths": lengths, "q_heads": q_heads, "kv_heads": kv_heads, "k_dim": k_dim, "v_dim": v_dim,
            "chunk": chunk, "frac": frac, "state": state}
    return dict(case, name=name) if name else case


def _step(name, batch, q_heads, kv_heads, k_dim, v_dim, frac):
    case = {"kind": "step", "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads, "k_dim": k_dim, "v_dim": v_dim, "frac": frac}
    return dict(case, name=name) if name else case


def _group(name, samples, positions, channels, groups, frac, gain=True, quadratic=False, pad=0, steps=10):
    case = {"kind": "group", "samples": samples, "positions": positions, "channels": channels, "groups": groups, "frac": frac,
            "gain": gain, "quadratic": quadratic, "pad": pad, "steps": steps}
    return dict(case, name=name) if name else case


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _heads(rng):
    kv = _log_int(rng, 1, 32)
    q = kv * rng.choice([g for g in (1, 1, 2, 4, 5, 8) if g * kv <= 32])
    k_dim = 2 * _log_int(rng, 8, 64)
    return q, kv, k_dim, k_dim if rng.random() < 0.6 else 2 * _log_int(rng, 8, 64)


def draw(rng):
    frac = rng.choice((12, 13, 16))
    kind = rng.choices(("prompt", "step", "group"), (4, 3, 3))[0]
    if kind == "prompt":
        while True:
            q, kv, k_dim, v_dim = _heads(rng)
            lengths = [_log_int(rng, 1, 512) for _ in range(_log_int(rng, 1, 8))]
            case = _prompt(None, "+".join(map(str, lengths)), q, kv, k_dim, v_dim, rng.choice((16, 32, 40, 64, 64)), frac, rng.random() < 0.5)
            if work(case)["bytes"] <= work(listed()[3])["bytes"] and work(case)["flops"] <= work(listed()[3])["flops"]:
                return case
    if kind == "step":
        while True:
            case = _step(None, _log_int(rng, 1, 64), *_heads(rng), frac)
            if work(case)["bytes"] <= work(listed()[5])["bytes"]:
                return case
    while True:
        groups, wide = _log_int(rng, 1, 32), rng.random() < 0.5
        channels = groups * (2 * _log_int(rng, 8, 64) if wide else _log_int(rng, 1, 40))
        samples, positions = (_log_int(rng, 1, 512), 1) if wide else (_log_int(rng, 1, 8), _log_int(rng, 2, 4096))
        if channels * positions >= 16 * groups and samples * positions * channels <= 8 * 1024 * 640:
            return _group(None, samples, positions, channels, groups, frac, rng.random() < 0.7, rng.random() < 0.5,
                          rng.choice((0, 0, 2 * _log_int(rng, 1, 64))), rng.randint(6, 14))


def _lengths(case):
    return [int(v) for v in case["lengths"].split("+")]


def _chunks(case):
    """(sequence, first token, tokens) of every chunk."""
    out, at = [], 0
    for j, n in enumerate(_lengths(case)):
        for first in range(0, n, case["chunk"]):
            out.append((j, at + first, min(case["chunk"], n - first)))
        at += n
    return out


def work(case):
    """Words that one pass reads and writes once, and its operations.  A ring multiply-add takes 18 multiply-adds of bytes at
    least, and bytes go through the tensor cores at twice the rate of 16-bit numbers: counted as one operation each."""
    if case["kind"] == "group":
        S, P, C, G, n = (case[k] for k in ("samples", "positions", "channels", "groups", "steps"))
        words = 5 * S * P * C + S * G * (9 * n - 4)                      # x, U, U t in, message and result out; a group's own words
        words += (3 * S * C + 4 * C if case["gain"] else 0)              # mask and product in, message out; gain, mask, message, bias
        words += 3 * S * P * C if case["quadratic"] else 0
        return {"bytes": 2 * 8 * words, "flops": 2 * 2 * (6 + (4 if case["quadratic"] else 0)) * S * P * C}
    Hq, Hk, Dk, Dv = (case[k] for k in ("q_heads", "kv_heads", "k_dim", "v_dim"))
    if case["kind"] == "step":
        B, kv = case["batch"], case["batch"] * case["kv_heads"] * Dk * Dv
        words = 5 * kv                                                   # state, mask, product in, message and state out
        words += B * (3 * Hq * Dk + 3 * Hk * Dk + 3 * Hk * Dv)           # q, k, v, their masks, their messages
        words += 2 * B * Hq * Dv                                         # product in, result out
        return {"bytes": 2 * 8 * words + 8 * Hk, "flops": 2 * 2 * (3 * kv + 2 * B * Hq * Dk * Dv)}
    chunks, lengths = _chunks(case), _lengths(case)
    T, pairs = sum(lengths), sum(n * (n + 1) // 2 for _, _, n in chunks)
    words = T * (3 * Hq * Dk + 5 * Hk * Dk + 3 * Hk * Dv)                # q, k, v with masks and messages; mask and message of d
    words += 3 * T * Hq * Dv + 3 * Hq * pairs                            # products of P v and q S in, result out; product, mask, message of P
    words += 3 * len(chunks) * Hk * Dk * Dv                              # of S: mask and product of d v in, message out
    words += (2 if case["state"] else 1) * len(lengths) * Hk * Dk * Dv
    macs = Hq * pairs * (Dk + Dv) + T * (Hq + Hk) * Dk * Dv
    return {"bytes": 2 * 8 * words + 8 * Hk * (case["chunk"] + 1), "flops": 2 * 2 * 2 * 18 * macs}


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

    def mask(self, *shape):
        return [self.words(*shape), self.words(*shape)]

    def share(self, value):
        """A uniform share for party 0, the rest for party 1."""
        s = self.words(*value.shape)
        return [s, value - s]


def _encode(v, frac):
    return torch.floor(v * float(1 << frac) + 0.5).to(torch.int64)


def _decays(case, powers):
    """decay^n at scale f for n in `powers`; heads forget with half-lives from a few tokens to a few hundred."""
    h = torch.arange(case["kv_heads"], device="cuda", dtype=torch.float64)
    rate = 1.0 - torch.exp2(-3.0 - 5.0 * h / case["kv_heads"])
    return _encode(rate[:, None] ** torch.as_tensor(powers, device="cuda", dtype=torch.float64)[None], case["frac"])


def _projected(d, case, T):
    """q, k, v of T tokens read out of the result of one stacked projection, a token's words behind one another."""
    Hq, Hk, Dk, Dv = (case[k] for k in ("q_heads", "kv_heads", "k_dim", "v_dim"))
    scale = torch.cat((torch.full((Hq * Dk,), Dk ** -0.5, device="cuda", dtype=torch.float64),
                       torch.full((Hk * Dk,), Dk ** -0.25, device="cuda", dtype=torch.float64),
                       torch.ones(Hk * Dv, device="cuda", dtype=torch.float64)))
    rows = d.share(_encode(d.normal(T, scale.numel()) * scale, case["frac"]))
    cut = lambda a, n, D: [r[:, a:a + n * D].unflatten(1, (n, D)) for r in rows]
    return dict(Q=cut(0, Hq, Dk), K=cut(Hq * Dk, Hk, Dk), V=cut((Hq + Hk) * Dk, Hk, Dv))


def _total(pair):
    return pair[0] + pair[1]


def _spread(t, case):
    """[..., kv_heads, D] to the query heads."""
    return t.repeat_interleave(case["q_heads"] // case["kv_heads"], -2)


def prepare(case, seed):
    d = _Draw(seed)
    f = case["frac"]
    if case["kind"] == "group":
        return _prepare_group(case, d)
    Hq, Hk, Dk, Dv = (case[k] for k in ("q_heads", "kv_heads", "k_dim", "v_dim"))
    if case["kind"] == "step":
        B = case["batch"]
        s = dict(case=case, **_projected(d, case, B), decay=_decays(case, [1])[:, 0].contiguous())
        mask = dict(q=d.mask(B, Hq, Dk), k=d.mask(B, Hk, Dk), v=d.mask(B, Hk, Dv), s=d.mask(B, Hk, Dk, Dv))
        kv = d.share(_total(mask["k"])[..., :, None] * _total(mask["v"])[..., None, :])
        sm = _total(mask["s"]).repeat_interleave(Hq // Hk, 1)
        qs = d.share(_matmul(_total(mask["q"])[:, :, None], sm)[:, :, 0])
        s.update(mask=mask, triple=dict(kv=kv, qs=qs), state=d.share(_encode(0.5 * d.normal(B, Hk, Dk, Dv), f)))
        return s
    lengths, chunks, C = _lengths(case), _chunks(case), case["chunk"]
    T = sum(lengths)
    s = dict(case=case, **_projected(d, case, T), decay=_decays(case, range(C + 1)))
    s["starts"] = torch.tensor([0, *np.cumsum(lengths)], device="cuda", dtype=torch.int32)
    mask = dict(q=d.mask(T, Hq, Dk), k=d.mask(T, Hk, Dk), v=d.mask(T, Hk, Dv), d=d.mask(T, Hk, Dk), p=d.mask(T, Hq, C),
                s=d.mask(len(chunks), Hk, Dk, Dv))
    q, k, v, dk, p, st = (_total(mask[x]) for x in ("q", "k", "v", "d", "p", "s"))
    qk, pv = d.words(T, Hq, C), torch.empty((T, Hq, Dv), dtype=torch.int64, device="cuda")
    qs, dv = torch.empty_like(pv), torch.empty_like(st)
    for c, (_, at, n) in enumerate(chunks):
        rows = slice(at, at + n)
        kh, vh = _spread(k[rows], case).transpose(0, 1), _spread(v[rows], case).transpose(0, 1)
        qh, sh = q[rows].transpose(0, 1), st[c].repeat_interleave(Hq // Hk, 0)
        qk[rows, :, :n] = _matmul(qh, kh.transpose(1, 2)).transpose(0, 1)
        low = torch.tril(p[rows, :, :n].transpose(0, 1))
        pv[rows] = _matmul(low, vh).transpose(0, 1)
        qs[rows] = _matmul(qh, sh).transpose(0, 1)
        dv[c] = _matmul(dk[rows].permute(1, 2, 0), v[rows].transpose(0, 1))
    s.update(mask=mask, triple=dict(qk=d.share(qk), pv=d.share(pv), qs=d.share(qs), dv=d.share(dv)))
    s["state"] = d.share(_encode(0.5 * d.normal(len(lengths), Hk, Dk, Dv), f)) if case["state"] else None
    return s


def _prepare_group(case, d):
    S, P, C, G, f, n = (case[k] for k in ("samples", "positions", "channels", "groups", "frac", "steps"))
    # groups differ in mean and by up to a factor of four in size; a position's channels lie `pad` words apart from the next one's
    size = torch.exp2(2.0 * torch.rand((S, 1, G, 1), generator=d.g, device="cuda", dtype=torch.float64) - 1.0)
    value = _encode(size * d.normal(S, P, G, C // G) + 0.5 * d.normal(S, 1, G, 1), f).view(S, P, C)
    X = []
    for share in d.share(value):
        rows = d.words(S, P, C + case["pad"])
        rows[..., :C] = share
        X.append(rows[..., :C])
    U = d.mask(S, P, C)
    u = _total(U)
    own_words = torch.empty((S, G, 6 * n - 3), dtype=torch.int64, device="cuda")
    own_words[..., 0] = (u * u).view(S, P, G, C // G).sum((1, 3))
    a = own_words[..., 1] = d.words(S, G)
    for k in range(n - 1):
        y, p, w = d.words(S, G), d.words(S, G), d.words(S, G)
        own_words[..., 2 + 6 * k:8 + 6 * k] = torch.stack((y, y * y, p, a * p, w, y * w), -1)
    v = own_words[..., 6 * n - 4] = d.words(S, G)
    s = {"case": case, "X": X, "gain": None, "act": None}
    t = v.repeat_interleave(C // G, 1)
    if case["gain"]:
        mask, T = d.mask(C), d.mask(S, C)
        s["gain"] = dict(weight=d.share(_encode(1.0 + 0.2 * d.normal(C), f)), mask=mask, T=T, VW=d.share(t * _total(mask)),
                         bias=d.share(_encode(0.3 * d.normal(C), f)))
        t = _total(T)
    s["norm"] = dict(U=U, words=d.share(own_words), UT=d.share(u * t[:, None]), steps=n, guess=int(0.55 * (1 << f)),
                     eps=max(1, (1 << f) // 100000))
    if case["quadratic"]:
        R = d.mask(S, P, C)
        s["act"] = (tuple(int(x * (1 << f)) for x in (0.5, 0.25, 0.125)), R, d.share(_total(R) * _total(R)))
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(state):
    if own:
        return _run_own(state)
    return {"prompt": _plain_prompt, "step": _plain_step, "group": _plain_group}[state["case"]["kind"]](state)


def _run_own(s):
    from paper_2505_07239_b200 import binding as cb

    case, stream = s["case"], torch.cuda.current_stream()
    if case["kind"] == "group":
        gain = cb.GroupGain(**s["gain"]) if s["gain"] else None
        msg, Z = cb.group_norm(s["X"], case["groups"], case["frac"], cb.GroupNorm(**s["norm"]), gain=gain, act=s["act"], stream=stream)
        out = {"M": msg.M, "S": msg.S, "Z": Z}
        if gain:
            out.update(D=msg.D, G=msg.G)
        if s["act"] is not None:
            out["N"] = msg.N
        return out
    m, t = s["mask"], s["triple"]
    if case["kind"] == "step":
        dealer = cb.StepDealer(q=m["q"], k=m["k"], v=m["v"], s=m["s"], kv=t["kv"], qs=t["qs"])
        msg, O, S = cb.linear_attention_step(s["Q"], s["K"], s["V"], s["decay"], s["state"], dealer, case["frac"], stream=stream)
        return {"q": msg.q, "k": msg.k, "v": msg.v, "s": msg.s, "O": O, "S": S}
    dealer = cb.PromptDealer(q=m["q"], k=m["k"], v=m["v"], d=m["d"], p=m["p"], s=m["s"], qk=t["qk"], pv=t["pv"], qs=t["qs"], dv=t["dv"])
    msg, O, S = cb.linear_attention(s["Q"], s["K"], s["V"], s["starts"], s["decay"], dealer, case["frac"], state=s["state"], stream=stream)
    return {"q": msg.q, "k": msg.k, "v": msg.v, "d": msg.d, "p": msg.p, "s": msg.s, "O": O, "S": S}


# ---------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------
def _matmul(a, b):
    """a b mod 2^64, batched.  Words in four pieces of 16 bits; a sum of K products of pieces stays below 2^53 for K up to 2^21."""
    def pieces(x):
        return [((x >> (16 * p)) & 0xFFFF).to(torch.float64) for p in range(4)]

    left, right = pieces(a), pieces(b)
    out = None
    for p in range(4):
        for q in range(4 - p):
            part = (left[p] @ right[q]).to(torch.int64) << (16 * (p + q))
            out = part if out is None else out + part
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


def _open(x, mask):
    msg = [x[i] - mask[i] for i in (0, 1)]
    return msg, msg[0] + msg[1]


def _plain_prompt(s):
    case, m, t = s["case"], s["mask"], s["triple"]
    f, C, g = case["frac"], case["chunk"], case["q_heads"] // case["kv_heads"]
    mq, q = _open(s["Q"], m["q"])
    mk, k = _open(s["K"], m["k"])
    mv, v = _open(s["V"], m["v"])
    md, mp, ms = ([torch.zeros_like(x) for x in m[y]] for y in ("d", "p", "s"))
    O = [torch.empty_like(x) for x in t["pv"]]
    shape = (len(_lengths(case)), case["kv_heads"], case["k_dim"], case["v_dim"])
    S = [x.clone() for x in s["state"]] if s["state"] is not None else [torch.zeros(shape, dtype=torch.int64, device="cuda") for _ in (0, 1)]
    heads = lambda x: _spread(x, case).transpose(0, 1)                       # [tokens, kv_heads, D] to [q_heads, tokens, D]
    w = s["decay"]
    wq = w.repeat_interleave(g, 0)
    for c, (j, at, n) in enumerate(_chunks(case)):
        rows = slice(at, at + n)
        i_ = torch.arange(n, device="cuda")
        lag = (i_[:, None] - i_[None]).clamp(min=0)
        low = (i_[:, None] >= i_[None])[None]
        # scores, weighted and opened
        P = []
        for i in (0, 1):
            z = t["qk"][i][rows, :, :n].transpose(0, 1) + _matmul(m["q"][i][rows].transpose(0, 1), heads(k[rows]).transpose(1, 2))
            z = z + _matmul(q[rows].transpose(0, 1), heads(m["k"][i][rows] + (k[rows] if i else 0)).transpose(1, 2))
            P.append(torch.where(low, _truncate(_truncate(z, i, f) * wq[:, lag], i, f), 0))
            mp[i][rows, :, :n] = torch.where(low, P[i] - m["p"][i][rows, :, :n].transpose(0, 1), 0).transpose(0, 1)
        p = (mp[0] + mp[1])[rows, :, :n].transpose(0, 1)
        for i in (0, 1):
            ms[i][c] = S[i][j] - m["s"][i][c]
        st = ms[0][c] + ms[1][c]
        for i in (0, 1):
            x = t["qs"][i][rows].transpose(0, 1) + _matmul(m["q"][i][rows].transpose(0, 1), st.repeat_interleave(g, 0))
            x = x + _matmul(q[rows].transpose(0, 1), (m["s"][i][c] + (st if i else 0)).repeat_interleave(g, 0))
            mask = torch.where(low, m["p"][i][rows, :, :n].transpose(0, 1), 0)
            y = t["pv"][i][rows].transpose(0, 1) + _matmul(mask, heads(v[rows])) + _matmul(p, heads(m["v"][i][rows] + (v[rows] if i else 0)))
            O[i][rows] = _truncate(y + wq[:, 1:n + 1, None] * _truncate(x, i, f), i, f).transpose(0, 1)
        # the state behind the chunk
        back = w[:, n - 1 - i_].t()[..., None]
        for i in (0, 1):
            md[i][rows] = _truncate(s["K"][i][rows] * back, i, f) - m["d"][i][rows]
        dk = (md[0] + md[1])[rows].permute(1, 2, 0)
        for i in (0, 1):
            z = t["dv"][i][c] + _matmul(m["d"][i][rows].permute(1, 2, 0), v[rows].transpose(0, 1))
            z = z + _matmul(dk, (m["v"][i][rows] + (v[rows] if i else 0)).transpose(0, 1))
            S[i][j] = _truncate(w[:, n, None, None] * S[i][j] + z, i, f)
    return {"q": mq, "k": mk, "v": mv, "d": md, "p": mp, "s": ms, "O": O, "S": S}


def _plain_step(s):
    case, m, t = s["case"], s["mask"], s["triple"]
    f, g = case["frac"], case["q_heads"] // case["kv_heads"]
    mq, q = _open(s["Q"], m["q"])
    mk, k = _open(s["K"], m["k"])
    mv, v = _open(s["V"], m["v"])
    outer = lambda a, b: a[..., :, None] * b[..., None, :]
    S = []
    for i in (0, 1):
        z = t["kv"][i] + outer(k, m["v"][i] + (v if i else 0)) + outer(m["k"][i], v)
        S.append(_truncate(s["decay"][:, None, None] * s["state"][i] + z, i, f))
    ms, st = _open(S, m["s"])
    O = []
    for i in (0, 1):
        z = _matmul(q[:, :, None], (m["s"][i] + (st if i else 0)).repeat_interleave(g, 1))
        z = z + _matmul(m["q"][i][:, :, None], st.repeat_interleave(g, 1))
        O.append(_truncate(t["qs"][i] + z[:, :, 0], i, f))
    return {"q": mq, "k": mk, "v": mv, "s": ms, "O": O, "S": S}


def _plain_group(s):
    case = s["case"]
    f, n, G, C, P = (case[k] for k in ("frac", "steps", "groups", "channels", "positions"))
    U, words, UT, guess, eps, three = *(s["norm"][k] for k in ("U", "words", "UT", "guess", "eps")), 3 << f
    count, per = P * (C // G), C // G
    sums = lambda x: x.unflatten(2, (G, per)).sum((1, 3))                   # [samples, positions, channels] to [samples, groups]
    wide = lambda x: x.repeat_interleave(per, 1)                             # [samples, groups] to [samples, channels]
    x = [s["X"][i] - wide(_divide(sums(s["X"][i]), i, count))[:, None] for i in (0, 1)]
    M, m = _open(x, U)
    S = [torch.empty((*words[0].shape[:2], 3 * n - 1), dtype=torch.int64, device=m.device) for _ in (0, 1)]

    def opened(v, mask, at):
        for i in (0, 1):
            S[i][..., at] = v[i] - words[i][..., mask]
        return S[0][..., at] + S[1][..., at]

    square = [words[i][..., 0] + sums(2 * m * U[i] + (m * m if i else 0)) for i in (0, 1)]
    var = [_divide(square[i], i, count << f) + (eps if i else 0) for i in (0, 1)]
    first = guess * guess >> f
    y = [_truncate(guess * ((three if i else 0) - _truncate(var[i] * first, i, f)), i, f + 1) for i in (0, 1)]
    a = opened(var, 1, 0)
    for k in range(n - 1):
        mat = [[words[i][..., 2 + 6 * k + j] for j in range(6)] for i in (0, 1)]
        d = opened(y, 2 + 6 * k, 1 + 3 * k)
        p = [_truncate(mat[i][1] + 2 * d * mat[i][0] + (d * d if i else 0), i, f) for i in (0, 1)]
        e = opened(p, 4 + 6 * k, 2 + 3 * k)
        w = [(three if i else 0) - _truncate(mat[i][3] + a * mat[i][2] + e * words[i][..., 1] + (a * e if i else 0), i, f) for i in (0, 1)]
        h = opened(w, 6 + 6 * k, 3 + 3 * k)
        y = [_truncate(mat[i][5] + d * mat[i][4] + h * mat[i][0] + (d * h if i else 0), i, f + 1) for i in (0, 1)]
    r, T = wide(opened(y, 6 * n - 4, 3 * n - 2)), [wide(words[i][..., 6 * n - 4]) for i in (0, 1)]
    out = {"M": M, "S": S}
    if s["gain"]:
        weight, mask, VW, bias = (s["gain"][k] for k in ("weight", "mask", "VW", "bias"))
        out["G"], e = _open(weight, mask)
        t = [_truncate(VW[i] + r * mask[i] + e * T[i] + (r * e if i else 0), i, f) for i in (0, 1)]
        T = s["gain"]["T"]
        out["D"], r = _open(t, T)
    z = [UT[i] + m * T[i][:, None] + r[:, None] * U[i] + (m * r[:, None] if i else 0) for i in (0, 1)]
    if s["gain"]:
        z = [z[i] + (bias[i] << f) for i in (0, 1)]
    z = [_truncate(z[i], i, f) for i in (0, 1)]
    if s["act"] is not None:
        (k0, k1, k2), R, Q = s["act"]
        out["N"], b = _open(z, R)
        for i in (0, 1):
            square = _truncate(Q[i] + 2 * b * R[i] + (b * b if i else 0), i, f)
            z[i] = _truncate(k2 * square + k1 * z[i], i, f) + (k0 if i else 0)
    out["Z"] = z
    return out


# ---------------------------------------------------------------------------
# the definition, in numpy on the host's 64-bit unsigned words
# ---------------------------------------------------------------------------
def _ring_product(a, b):
    """a b mod 2^64 with pieces of 22, 21 and 21 bits and sums of at most 256 products, below 2^52."""
    starts, widths = (0, 22, 43), (22, 21, 21)
    cut = [[((x >> np.uint64(s)) & np.uint64((1 << w) - 1)).astype(np.float64) for s, w in zip(starts, widths)] for x in (a, b)]
    total = np.zeros((a.shape[0], b.shape[1]), np.uint64)
    for k in range(0, a.shape[1], 256):
        for p in range(3):
            for q in range(3):
                if starts[p] + starts[q] < 64:
                    part = cut[0][p][:, k:k + 256] @ cut[1][q][k:k + 256]
                    total += part.astype(np.uint64) << np.uint64(starts[p] + starts[q])
    return total


def _local(share, party, divisor):
    """One party's half of a division by a public number."""
    d = np.uint64(divisor)
    return share // d if party == 0 else np.uint64(0) - (np.uint64(0) - share) // d


def _u(v):
    return np.uint64(v & MASK)


def _beaver(c, a, b, d, e, times=np.multiply):
    """Shares of (a + d)(b + e) from those of a, b and c = a b."""
    return [c[0] + times(d, b[0]) + times(a[0], e), c[1] + times(d, b[1]) + times(a[1], e) + times(d, e)]


def exact(case, seed):
    cost = work(case)
    if cost["bytes"] > 2e8 or cost["flops"] > 2e10:
        return None
    state = prepare(case, seed)

    def host(v):
        if isinstance(v, torch.Tensor):
            return v.cpu().numpy().view(np.uint64) if v.dtype == torch.int64 else v.cpu().numpy()
        if isinstance(v, dict):
            return {k: host(x) for k, x in v.items() if k != "case"}
        return [host(x) for x in v] if isinstance(v, (list, tuple)) else v

    with np.errstate(over="ignore"):
        result = {"prompt": _exact_prompt, "step": _exact_step, "group": _exact_group}[case["kind"]](case, host(state))
    return {k: [torch.from_numpy(np.ascontiguousarray(x).view(np.int64)) for x in v] for k, v in result.items()}


def _reveal(x, mask):
    msg = [a - b for a, b in zip(x, mask)]
    return msg, msg[0] + msg[1]


def _exact_prompt(case, s):
    one, C, group = 1 << case["frac"], case["chunk"], case["q_heads"] // case["kv_heads"]
    m, t, out = s["mask"], s["triple"], {}
    opened = {}
    for name, x in (("q", s["Q"]), ("k", s["K"]), ("v", s["V"])):
        out[name], opened[name] = _reveal(x, m[name])
    out["d"], out["p"], out["s"] = ([np.zeros_like(x) for x in m[y]] for y in ("d", "p", "s"))
    out["O"] = [np.zeros_like(x) for x in t["pv"]]
    ends = s["starts"]
    shape = (len(ends) - 1, case["kv_heads"], case["k_dim"], case["v_dim"])
    out["S"] = [x.copy() for x in s["state"]] if case["state"] else [np.zeros(shape, np.uint64) for _ in (0, 1)]
    c = 0
    for j in range(len(ends) - 1):
        for at in range(ends[j], ends[j + 1], C):
            n = min(C, ends[j + 1] - at)
            for h in range(case["kv_heads"]):
                w = s["decay"][h]
                side = lambda x, head: [np.ascontiguousarray(v[at:at + n, head]) for v in x]
                vm, ve = side(m["v"], h), opened["v"][at:at + n, h]
                km, ke = [x.T for x in side(m["k"], h)], opened["k"][at:at + n, h].T
                S = [out["S"][i][j, h] for i in (0, 1)]
                sent, se = _reveal(S, [m["s"][i][c, h] for i in (0, 1)])
                for i in (0, 1):
                    out["s"][i][c, h] = sent[i]
                for hq in range(h * group, (h + 1) * group):
                    qm, qe = side(m["q"], hq), opened["q"][at:at + n, hq]
                    z = _beaver([x[:, :n] for x in side(t["qk"], hq)], qm, km, qe, ke, _ring_product)
                    z = [_local(x, i, one) for i, x in enumerate(z)]
                    pm = [np.tril(x[:, :n]) for x in side(m["p"], hq)]
                    weight = np.array([[w[max(r - u, 0)] for u in range(n)] for r in range(n)], np.uint64)
                    P = [np.tril(_local(x * weight, i, one)) for i, x in enumerate(z)]
                    sent, pe = _reveal(P, pm)
                    y = _beaver(side(t["pv"], hq), pm, vm, pe, ve, _ring_product)
                    x = _beaver(side(t["qs"], hq), qm, [m["s"][i][c, h] for i in (0, 1)], qe, se, _ring_product)
                    for i in (0, 1):
                        out["p"][i][at:at + n, hq, :n] = sent[i]
                        out["O"][i][at:at + n, hq] = _local(y[i] + w[1:n + 1, None] * _local(x[i], i, one), i, one)
                D = [_local(x * w[n - 1 - np.arange(n)][:, None], i, one) for i, x in enumerate(side(s["K"], h))]
                sent, de = _reveal(D, side(m["d"], h))
                z = _beaver([t["dv"][i][c, h] for i in (0, 1)], [x.T for x in side(m["d"], h)], vm, de.T, ve, _ring_product)
                for i in (0, 1):
                    out["d"][i][at:at + n, h] = sent[i]
                    out["S"][i][j, h] = _local(w[n] * S[i] + z[i], i, one)
            c += 1
    return out


def _exact_step(case, s):
    one, group = 1 << case["frac"], case["q_heads"] // case["kv_heads"]
    m, t, out, opened = s["mask"], s["triple"], {}, {}
    for name, x in (("q", s["Q"]), ("k", s["K"]), ("v", s["V"])):
        out[name], opened[name] = _reveal(x, m[name])
    row, col = (lambda x: x[..., None, :]), (lambda x: x[..., :, None])
    z = _beaver(t["kv"], [col(x) for x in m["k"]], [row(x) for x in m["v"]], col(opened["k"]), row(opened["v"]))
    out["S"] = [_local(s["decay"][:, None, None] * s["state"][i] + z[i], i, one) for i in (0, 1)]
    out["s"], se = _reveal(out["S"], m["s"])
    out["O"] = [np.empty_like(x) for x in t["qs"]]
    for b in range(case["batch"]):
        for h in range(case["q_heads"]):
            o = _beaver([x[b, h][None] for x in t["qs"]], [x[b, h][None] for x in m["q"]], [x[b, h // group] for x in m["s"]],
                        opened["q"][b, h][None], se[b, h // group], _ring_product)
            for i in (0, 1):
                out["O"][i][b, h] = _local(o[i][0], i, one)
    return out


def _exact_group(case, s):
    one, n, G, per = 1 << case["frac"], case["steps"], case["groups"], case["channels"] // case["groups"]
    m_, count = s["norm"], case["positions"] * per
    shape = (case["samples"], case["positions"], G, per)
    cut = lambda pair: [np.ascontiguousarray(x).reshape(shape) for x in pair]
    word = [[m_["words"][i][..., j] for i in (0, 1)] for j in range(6 * n - 3)]
    sent, out = [], {}

    def reveal(v, mask):
        sent.append([v[i] - mask[i] for i in (0, 1)])
        return sent[-1][0] + sent[-1][1]

    x, U = cut(s["X"]), cut(m_["U"])
    mean = [_local(v.sum((1, 3), dtype=np.uint64), i, count) for i, v in enumerate(x)]
    M, m = _reveal([v - mean[i][:, None, :, None] for i, v in enumerate(x)], U)
    cross = [(m * u).sum((1, 3), dtype=np.uint64) for u in U]
    total = [word[0][i] + cross[i] + cross[i] for i in (0, 1)]
    total[1] = total[1] + (m * m).sum((1, 3), dtype=np.uint64)
    var = [_local(total[i], i, count * one) for i in (0, 1)]
    var[1] = var[1] + _u(m_["eps"])
    three, guess = [_u(0), _u(3 * one)], m_["guess"]
    y = [_local(_u(guess) * (three[i] - _local(var[i] * _u(guess * guess // one), i, one)), i, 2 * one) for i in (0, 1)]
    da = reveal(var, word[1])
    for k in range(n - 1):
        my, myy, mp, map_, mw, myw = word[2 + 6 * k:8 + 6 * k]
        dy = reveal(y, my)
        p = [_local(v, i, one) for i, v in enumerate(_beaver(myy, my, my, dy, dy))]
        dp = reveal(p, mp)
        w = [three[i] - _local(v, i, one) for i, v in enumerate(_beaver(map_, word[1], mp, da, dp))]
        dw = reveal(w, mw)
        y = [_local(v, i, 2 * one) for i, v in enumerate(_beaver(myw, my, mw, dy, dw))]
    mask, value = word[6 * n - 4], reveal(y, word[6 * n - 4])
    mask, value = [v[..., None] for v in mask], value[..., None]                # [samples, groups, 1]
    out["S"] = [np.stack([v[i] for v in sent], -1) for i in (0, 1)]
    split = lambda pair: [v.reshape(*v.shape[:-1], G, per) for v in pair]
    if case["gain"]:
        g = s["gain"]
        out["G"], e = _reveal(g["weight"], g["mask"])
        t = _beaver(split(g["VW"]), mask, split(g["mask"]), value, e.reshape(G, per))
        mask = split(g["T"])
        D, value = _reveal([_local(v, i, one) for i, v in enumerate(t)], mask)
        out["D"] = [v.reshape(case["samples"], -1) for v in D]
    z = _beaver(cut(m_["UT"]), U, [v[:, None] for v in mask], m, value[:, None])
    if case["gain"]:
        z = [v + b * _u(one) for v, b in zip(z, split(s["gain"]["bias"]))]
    z = [_local(v, i, one) for i, v in enumerate(z)]
    flat = lambda pair: [v.reshape(case["samples"], case["positions"], -1) for v in pair]
    if case["quadratic"]:
        (k0, k1, k2), R, Q = s["act"]
        N, b = _reveal(z, cut(R))
        q = _beaver(cut(Q), cut(R), cut(R), b, b)
        z = [_local(_u(k2) * _local(v, i, one) + _u(k1) * z[i], i, one) for i, v in enumerate(q)]
        z[1] = z[1] + _u(k0)
        out["N"] = flat(N)
    out["M"], out["Z"] = flat(M), flat(z)
    return out
