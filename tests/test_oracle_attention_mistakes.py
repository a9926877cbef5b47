"""The pins of oracle/attention.py against oracles with a mistake in them: each is planted in the source of the oracle's own function, and the integer
brackets of tests/test_oracle_attention.py, run on what it then returns, have to reject it."""
import inspect

import pytest

from oracle import attention
from tests import test_oracle_attention as pins


def planted(function, old, new):
    source = inspect.getsource(function)
    assert source.count(old) == 1, old
    space = dict(vars(attention))
    exec(source.replace(old, new), space)
    return space[function.__name__]


def accepted(pin, cases):
    try:
        for case in cases:
            pin(*case)
    except AssertionError:
        return False
    return True


PROMPT = [
    ("w[1:L + 1, None]", "w[:L, None]"),                     # the far part's weight of the token itself
    ("P = _trunc(_times(_trunc(scores, f), w[np.where(below, at[:, None] - at[None], 0)]), f)",
     "P = _times(_trunc(scores, f), w[np.where(below, at[:, None] - at[None], 0)])"),          # weights left at scale 2f
    ("_times(_trunc(scores, f), w[np.where(below, at[:, None] - at[None], 0)])", "_times(_trunc(scores, f), w[np.where(below, L - 1 - at[None], 0)])"),
    ("at[:, None] >= at[None]", "at[:, None] > at[None]"),   # the token does not see itself
    ("below = at[:, None] >= at[None]", "below = at[:, None] >= 0"),                           # it sees those behind it
    ("msg, se = _open(S, sm)", "msg, se = _open(_trunc(_times(S, w[L]), f), sm)"),             # the state opened behind its update
    ("w[L - 1 - at][:, None]", "w[L - at][:, None]"),        # keys decayed once too often
    ("w[L] * S[i] + add[i]", "w[C] * S[i] + add[i]"),        # a short chunk's state decayed like a whole one's
    ("range(h * group, (h + 1) * group)", "range(h, Hq, Hk)"),                                 # query heads dealt out in turn
    ("number += 1", "number += 0"),
    ("P, pm = ([np.where(below, t[:, :L], U64(0)) for t in pair]", "P, pm = ([t[:, :L] for t in pair]"),                  # weights off the triangle sent
]
STEP = [
    ("decay[:, None, None] * state[i] + add[i]", "state[i] + add[i]"),
    ("_open(out[\"S\"], m[\"s\"])", "_open(state, m[\"s\"])"),                                 # o from the old state
    ("s = h // (Hq // Hk)", "s = h % Hk"),
]
GROUP = [
    ("_divide(total(X[i]), i, P * per)", "_divide(total(X[i]), i, P * per + 1)"),
    ("_divide(words[0][i] + total(squares[i]), i, P * per << f)", "_divide(words[0][i] + total(squares[i]), i, C << f)"),
    ("_open([X[i] - mean[i][:, None] for i in (0, 1)], norm[\"U\"])", "_open([X[i] for i in (0, 1)], norm[\"U\"])"),        # the mean left in
    ("_times(gain[\"bias\"], U64(1 << f))", "gain[\"bias\"]"),                                 # the bias at the wrong scale
    ("word(k2) * square[i] + word(k1) * z[i]", "word(k1) * square[i] + word(k2) * z[i]"),
    ("z[1] = z[1] + word(k0)", "z[1] = z[1]"),
    ("t, mask = wide([root, root])[0], wide(mask)", "t, mask = wide([root, root])[0][:, ::-1], [v[:, ::-1] for v in wide(mask)]"),                  # another group's root
]
PROMPT_PIN = (pins.test_prompt_against_python_integers, pins.PROMPTS)
STEP_PIN = (pins.test_step_against_python_integers, [()])
GROUP_PIN = (pins.test_group_against_python_integers, [(2, 1, 24, 3, 16, 12), (2, 5, 12, 2, 16, 12)])


@pytest.mark.parametrize("name,mistakes,pin", [("linear_attention", PROMPT, PROMPT_PIN), ("linear_attention_step", STEP, STEP_PIN), ("group_norm", GROUP, GROUP_PIN)])
def test_mistakes_are_rejected(monkeypatch, name, mistakes, pin):
    good = getattr(attention, name)
    same = mistakes[0][0]
    monkeypatch.setattr(attention, name, planted(good, same, same))
    assert accepted(*pin)                                    # the copy itself is no mistake
    for old, new in mistakes:
        monkeypatch.setattr(attention, name, planted(good, old, new))
        assert not accepted(*pin), (old, new)
