"""Group norm's strides of what there is one of (groups, samples, points): any value, also one
whose bytes pass 64 bits, and never part of an address (no GPU: every call is refused)."""

import pytest

from paper_1910_13444_amd import pigan
from test_group_norm_abi import FAKE, _args, needs_lib

ANY = [0, -1, 1, (1 << 62) + 1, (1 << 63) - 1, -(1 << 63)]
FAR = 1 << 24


@needs_lib
@pytest.mark.parametrize("stride", ANY)
@pytest.mark.parametrize("G,s,p", [(1, 1, 1), (1, 1, 5), (1, 3, 1), (2, 1, 1)])
def test_unused_strides(G, s, p, stride):
    L = pigan.lib()
    c = 24
    at = tuple(used if many else stride for many, used in ((p > 1, c), (s > 1, p * c), (G > 1, s * p * c)))
    for dt in (0, 1):
        x, y = (FAKE, *at), (FAR, *at)
        last = FAR + (G * s * p * c - 1) * (4, 2)[dt] // 4 * 4
        assert L.pigan_group_norm_forward(_args(G=G, s=s, p=p, dt=dt, x=x, y=y, mean=last, rstd=0), None, 0, None) == pigan.EINVAL
        assert pigan.lib().pigan_last_error() == b"mean overlaps y"
        bad = _args(G=G, s=s, p=p, dt=dt, x=x, dy=x, add=x, dx=y, dgamma=1 << 30, dbeta=last)
        assert L.pigan_group_norm_backward(bad, 1 << 36, 1 << 30, None) == pigan.EINVAL
        assert pigan.lib().pigan_last_error() == b"dbeta overlaps dx"
