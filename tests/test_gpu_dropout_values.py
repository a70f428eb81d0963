"""Dropped elements that are not finite."""
import numpy as np
import pytest
import torch

import paper_2304_04237_amd as sa
from oracle import region_oracle as ro
from tests.region_cases import DTYPES, numpy_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1])
def test_dropped_infinities_contribute_nothing(dtype, shift):
    """Infinities of both signs and NaN wherever the mask drops, in whole pieces and element by element (an address off by one)."""
    n, bad = 4099, [float("inf"), float("-inf"), float("nan")]
    f = ro.drop_factors(np.arange(n), 0.5, 1, 2)
    values = np.ones(n)
    dropped = np.flatnonzero(f == 0)
    values[dropped] = np.resize(bad, len(dropped))
    room = torch.zeros(n + shift, dtype=DTYPES[dtype], device="cuda")
    x = room[shift:]
    x.copy_(torch.tensor(values))
    assert x.isposinf().any() and x.isneginf().any() and x.isnan().any() and (~x.isfinite()).sum() == len(dropped)
    r = torch.tensor(np.arange(n) % 7 - 3.0).to(DTYPES[dtype]).cuda()
    assert (numpy_of(sa.slide_dropout_fwd(x, 0.5, 1, 2)) == f).all()
    assert (numpy_of(sa.slide_dropout_bwd(x, 0.5, 1, 2)) == f).all()
    assert (numpy_of(sa.slide_dropout_fwd(x, 0.5, 1, 2, residual=r)) == f + numpy_of(r)).all()       # (small whole numbers: exact)
