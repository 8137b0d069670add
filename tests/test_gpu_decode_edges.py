"""Decoding over a shared and a bounded cache on the GPU where it can go wrong.

Tolerances as in test_gpu_decode.py, and: fp16's halves of a weight above zero are raised to 2^-24 of 2^15 each, so that a row adds
2^-38 of the base's weight at most (bf16: 2^-125, nothing beside the smallest numbers)."""
import math

import pytest
import torch

from test_gpu_handoff import DEV, TYPES, half_step, ints, mb, tiny  # noqa: F401

pytestmark = pytest.mark.gpu


def sums_error(dh, n, dz):
    """Relative error of an output's sums over n rows whose scores have products that add up to dz (see test_gpu_decode.py)."""
    return 2 * (dh / 16 + 3) * 2.0 ** -23 * dz + 2.0 ** -19 + 2.0 ** -16 + (n / 8 + n / 64 + 64) * 2.0 ** -23


@pytest.mark.parametrize("gap", [64, 200])
@pytest.mark.parametrize("typ", ["f16", "bf16"])
def test_attend_shared_of_a_row_that_takes_all(mb, typ, gap):  # noqa: F811
    """A row of a small value takes all weight in front of 16000 large values of one sign, all of them in one CTA's run (250 tiles by
    304 heads for 304 CTAs).  Weights of 2^-64 are raised to 2^-38 at most, those of 2^-200 are zero in fp32."""
    typ, dh, hk, page, front, own = TYPES[typ], 64, 304, 16, 16000, 4
    whole, n = front // page, front + own
    cache = mb.Cache.empty(1, whole + 2, hk, page, dh, 2, whole + 1, typ)
    cache.table[:, :whole] = torch.arange(whole, dtype=torch.int32, device=DEV)
    cache.table[:, whole] = ints([whole, whole + 1])
    cache.refs[:] = ints([2] * whole + [1, 1])
    cache.length[:] = n
    cache.pool[0, 0], cache.pool[0, 1] = 0.0, 1000.0
    cache.pool[0, 0, 0, :, 5, 3] = gap * 8 * math.log(2)
    cache.pool[0, 1, 0, :, 5] = 0.001
    q = torch.ones(2, hk, dh, dtype=typ, device=DEV)
    dz = float(cache.pool[0, 0, 0, 0, 5, 3]) / 8
    w, v = math.exp(-dz), float(cache.pool[0, 1, 0, 0, 5, 0])
    want = (v + (n - 1) * 1000 * w) / (1 + (n - 1) * w)
    raised = (n - 1) * 1000 * (2.0 ** -38 if typ == torch.float16 else 2.0 ** -125) if gap < 126 else 0.0
    tol = half_step(typ) * (want + raised) + sums_error(dh, n, dz) * (want + raised) + raised + tiny(typ)
    for out in (cache.attend(q, ints([0, 1]), 0), cache.attend_shared(q, ints([0, 1]), 0, ints([0, 2]))):
        off = (out.double() - want).abs().max().item()
        assert off <= tol, (off, tol)
    cache.check()
