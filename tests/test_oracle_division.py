"""How often the local division of a shared number fails, the figure that comet.h gives for the norm of a row: one case in
2^64 / |z| of uniform shares, z the number, and then by 2^64 / divisor."""
import numpy as np
import pytest

from oracle import layers
from paper_2505_07239_b200 import workloads as wl

U64 = np.uint64


@pytest.mark.parametrize("log_z", [58, 59, 60])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("divisor", [1 << 33, 80 << 20])
def test_failures_of_a_local_division(log_z, sign, divisor):
    count = 1 << 16
    z = np.full(count, sign * (1 << log_z), np.int64).view(U64)
    share = wl.split_shares(z, 11, f"division{log_z}{sign}")
    with np.errstate(over="ignore"):
        got = (layers._divide(share[0], 0, divisor) + layers._divide(share[1], 1, divisor)).view(np.int64)
    off = np.abs(got - sign * ((1 << log_z) // divisor))
    failed = off > 1
    # within a unit where it holds, off by 2^64 / divisor within two where it fails
    assert (np.abs(off[failed] - (1 << 64) // divisor) <= 2).all()
    # binomial: probability 2^(log_z - 64), six deviations on either side
    p = 2.0 ** (log_z - 64)
    assert abs(failed.sum() - p * count) <= 6 * (count * p * (1 - p)) ** 0.5


def test_failures_of_a_row():
    """The mean square of a row of D words at scale f: z = D ms 2^2f, and where the division fails it is off by 2^64 / (D 2^f)."""
    T, D, f, ms_log = 4096, 64, 24, 4
    x = np.full((T, 1, D), 1 << (f + ms_log // 2), np.int64).view(U64)
    n = wl.dealer_norm(3, "row", T, 1, D, 2)
    norm = dict(U=list(n["U"][1:]), words=list(n["words"][1:]), UV=list(n["UV"][1:]), steps=2, guess=1 << (f - 2), eps=0)
    out = layers.norm_rotate(list(wl.split_shares(x, 3, "x")), f, norm=norm)
    with np.errstate(over="ignore"):                       # the opening of s is its first word; its mask the second of the row's
        s = (out["S"][0][..., 0] + out["S"][1][..., 0] + n["words"][0][..., 1]).view(np.int64)
    off = np.abs(s - (1 << (f + ms_log)))
    failed = off > 1
    assert (np.abs(off[failed] - (1 << 64) // (D << f)) <= 2).all()
    p = D * 2.0 ** (ms_log + 2 * f - 64)
    assert abs(failed.sum() - p * T) <= 6 * (T * p * (1 - p)) ** 0.5
