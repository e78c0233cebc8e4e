"""How far the table of frequencies is off 60 digits: 4 units of 2^-64 where no frequency passes a radian a token, 3 + 2 max(f) where some do.

The sum with a half and the cut behind it are off by half a unit each, 1 - x of a frequency that turns backwards by another half.  f / 2 pi is a power (one step of 64 bits, 2^-63, and |e ln base| 2^-64
by its exponent e: at most 0.37 2^-64 of the largest f), and at most four quotients and products of 2^-64 each: 6.4 units of f / 2 pi, 1.02 of the largest f.  A line between low and high is off by 6 steps of
length f / 2 pi <= high, over high - low, and two more; times f / 2 pi <= high / length that is at most 1 unit where length >= 8 high^2 / (high - low).  Together 2.5 + 1.02 max(f), and half a unit for the
reference's own rounding: at most 4 whole units up to a radian, and 3 + 1.02 max(f) beyond."""
import random
from decimal import Decimal

import pytest

from paper_2411_17686_amd import ficoco as fc
from tests.test_rotary_abi import turns


def off(**kw):
    got = [int(x) % 2 ** 64 for x in fc.rotary_turns(kw["rot"], **{k: v for k, v in kw.items() if k != "rot"})]
    return max((min((g - w) % 2 ** 64, (w - g) % 2 ** 64) for g, w in zip(got, turns(**kw))), default=0)


@pytest.mark.parametrize("seed", range(6))
def test_below_a_radian_a_token(seed):
    r = random.Random(seed)
    for _ in range(12):
        kw = dict(rot=2 * r.randint(1, 256), base=10 ** r.uniform(0, 8))
        how = r.randrange(4)
        if how == 1:
            kw["factor"] = 2 ** r.uniform(0, 6)
        elif how == 2:
            kw.update(factor=2 ** r.uniform(0, 6), length=2 ** r.uniform(12, 18), low=r.choice([0.5, 1, 2]), high=r.choice([4, 8, 32]))
        elif how == 3:
            kw["divisors"] = [r.choice([-1, 1]) * r.uniform(1, 50) for _ in range(kw["rot"] // 2)]
        assert off(**kw) <= 4, kw


@pytest.mark.parametrize("kw", [dict(rot=64, base=5e5, factor=0.01), dict(rot=128, base=1e6, factor=1e-4), dict(rot=6, base=100.0, divisors=[1.0, -2.5, 0.125]), dict(rot=2, base=10.0, factor=1e-9),
                                dict(rot=48, base=1e4, divisors=[1 / (3.0 + i) for i in range(24)])])
def test_faster_ones_in_proportion(kw):
    divisors = kw.get("divisors") or [1.0] * (kw["rot"] // 2)
    most = max(float((-Decimal(2 * i) / kw["rot"] * Decimal(kw["base"]).ln()).exp()) / abs(x) for i, x in enumerate(divisors)) / kw.get("factor", 1.0)
    assert off(**kw) <= 3 + 2 * most


def test_a_far_position():
    """The turns of position 2^31, against those of 60 digits: within 2^-31 of one."""
    for w, g in zip(turns(128, 1e6), fc.rotary_turns(128, 1e6).tolist()):
        d = ((g - w) * 2 ** 31) % 2 ** 64
        assert min(d, 2 ** 64 - d) <= 2 ** 33
