"""mtp_rotary_turns on the host: the pairs' turns per position against the formulas in 64 bits.  No GPU is needed."""
import math
from decimal import Decimal, localcontext

import numpy as np
import pytest

from test_lib_cpu import libpath  # noqa: F401


def _turns(rot, scaling, **kw):
    from paper_2410_13839_gb300 import mtp
    return mtp.mtp_rotary_turns(rot, scaling, device="cpu", **kw).numpy().view(np.uint64)


def _formula(i, rot, scaling, base, factor, context, low, high):
    if scaling == "BASE":
        base *= factor ** (rot / (rot - 2))
    f = base ** (-2 * i / rot)
    if scaling == "LINEAR":
        f /= factor
    if scaling == "BANDS":
        kept = min(1.0, max(0.0, (context * f / (2 * math.pi) - low) / (high - low)))
        f = kept * f + (1 - kept) * f / factor
    return f / (2 * math.pi)


@pytest.mark.parametrize("scaling", ["PLAIN", "LINEAR", "BASE", "BANDS"])
@pytest.mark.parametrize("rot,base,factor", [(4, 10000.0, 4.0), (64, 10000.0, 8.0), (128, 500000.0, 32.0), (22, 1.5, 1.0)])
def test_turns(libpath, scaling, rot, base, factor):  # noqa: F811
    from paper_2410_13839_gb300 import mtp
    kw = dict(base=base, factor=factor, context=8192.0, low=1.0, high=4.0)
    got = _turns(rot, getattr(mtp, "MTP_ROTARY_" + scaling), **kw)
    assert got.shape == (rot // 2,)
    for i, x in enumerate(got.tolist()):
        want = _formula(i, rot, scaling, **kw)
        # a few roundings to 53 bits, of the power (whose exponent is up to ln(base) large) and the products, and the last place
        assert abs(x / 2.0 ** 64 - want) <= want * (math.log(base * factor ** 2) + 8) * 2.0 ** -52 + 2.0 ** -64


def test_bands_keep_the_fast_pairs_and_slow_the_slow_ones_down(libpath):  # noqa: F811
    from paper_2410_13839_gb300 import mtp
    plain = _turns(64, mtp.MTP_ROTARY_PLAIN)
    bands = _turns(64, mtp.MTP_ROTARY_BANDS, factor=8.0, context=8192.0, low=1.0, high=4.0)
    turns = plain.astype(np.float64) / 2.0 ** 64 * 8192
    assert np.array_equal(bands[turns >= 4.001], plain[turns >= 4.001]) and (turns >= 4.001).any()
    slow = turns <= 0.999
    assert slow.any()
    for b, x in zip(bands[slow].tolist(), plain[slow].tolist()):  # both are whole: eight halves of a place, and one half
        assert abs(8 * b - x) <= 4.5 + x * 2.0 ** -50


@pytest.mark.parametrize("rot,scaling,kw", [
    (0, 0, {}), (3, 0, {}), (258, 0, {}), (64, 4, {}), (64, -1, {}), (64, 0, dict(base=1.0)), (64, 0, dict(base=float("nan"))),
    (64, 0, dict(base=float("inf"))), (64, 1, dict(factor=0.5)), (64, 1, dict(factor=float("nan"))), (2, 2, dict(factor=2.0)),
    (4, 2, dict(factor=1e300)), (64, 3, dict(factor=2.0)), (64, 3, dict(factor=2.0, context=100.0, low=4.0, high=4.0)),
    (64, 3, dict(factor=2.0, context=float("inf")))])
def test_refusals(libpath, rot, scaling, kw):  # noqa: F811
    from paper_2410_13839_gb300 import mtp
    with pytest.raises(mtp.MTPError) as e:
        _turns(rot, scaling, **kw)
    assert e.value.code == -1 and str(e.value)


def _exact(i, rot, scaling, base, factor, context, low, high):
    """A pair's turns per position in units of 2^-64, to 60 digits."""
    with localcontext() as ctx:
        ctx.prec = 60
        base, factor, context, low, high = (Decimal(x) for x in (base, factor, context, low, high))
        turn = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494")
        if scaling == "BASE":
            base *= (factor.ln() * rot / (rot - 2)).exp()
        f = (-2 * i * base.ln() / rot).exp()
        if scaling == "LINEAR":
            f /= factor
        if scaling == "BANDS":
            kept = min(Decimal(1), max(Decimal(0), (context * f / turn - low) / (high - low)))
            f = kept * f + (1 - kept) * f / factor
        return f / turn * 2 ** 64


@pytest.mark.parametrize("scaling", ["PLAIN", "LINEAR", "BASE", "BANDS"])
@pytest.mark.parametrize("rot,base,factor,context", [
    (4, 10000.0, 4.0, 100.0), (64, 10000.0, 8.0, 8192.0), (64, 1.0 + 2.0 ** -40, 1.0, 30.0), (128, 500000.0, 32.0, 8192.0), (22, 1.5, 1.0, 50.0),
    (256, 1e6, 40.0, 131072.0), (96, 1e300, 1.25, 4096.0), (128, 12345.678, 3.3, 5000.0)])
def test_turns_are_the_formulas_to_their_last_place(libpath, scaling, rot, base, factor, context):  # noqa: F811
    """At position 2^31 a turn's 64th place is 2^-33 of a turn: what the sines and cosines are promised at any position rests on it."""
    from paper_2410_13839_gb300 import mtp
    kw = dict(base=base, factor=factor, context=context, low=1.0, high=4.0)
    for i, x in enumerate(_turns(rot, getattr(mtp, "MTP_ROTARY_" + scaling), **kw).tolist()):
        # one rounding to a whole number; about 100 bits before it
        assert abs(Decimal(x) - _exact(i, rot, scaling, **kw)) <= Decimal(0.5 + 2.0 ** -20), i
