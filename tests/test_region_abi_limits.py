"""Where the C ABI of region selection and region attention ends: the last problem that is taken and the first that is not (on the host:
nothing is launched)."""
import numpy as np
import pytest

from tests.test_region_abi import lib, problem  # noqa: F401  (lib is a fixture)

SELECT, FWD, BWD = 0, 1, 2
LOG2E = np.float32(1.4426950408889634)


def taken(lib, call, **change):  # noqa: F811
    """Whether the backward (whose scratch is never 0 bytes), the selection takes the problem."""
    return lib.slide_region_workspace_bytes(problem(**change), call) > 0


@pytest.mark.parametrize("scale, dropout", [(3e38, 0.0), (2.4e38, 0.0), (1e38, 0.9), (1e34, 0.99998)])
def test_scales_that_overflow_where_they_are_used_are_refused(lib, scale, dropout):  # noqa: F811
    """Logits are multiplied by scale log2 e, sums of the backward by scale / (1 - dropout): an infinity there makes a NaN of every zero."""
    with np.errstate(over="ignore"):
        assert np.isinf(np.float32(scale) * LOG2E) or np.isinf(np.float32(scale) * np.float32(65536 / (65536 - round(dropout * 65536))))
    assert not taken(lib, BWD, scale=scale, dropout=dropout)


def test_a_scale_that_only_the_backward_cannot_use(lib):  # noqa: F811
    """One token over many keys needs scratch in the forward too, which shows that the forward takes it."""
    one = dict(q_h=1, q_w=1, q_region_h=1, q_region_w=1, k_h=1, k_w=5000, k_region_h=1, k_region_w=32, topk=100, B=1, scale=1e38, dropout=0.9)
    assert taken(lib, FWD, **one) and not taken(lib, BWD, **one)


@pytest.mark.parametrize("scale, dropout", [(2.3e38, 0.0), (1e37, 0.9), (1e33, 0.99998), (1e-45, 0.5)])
def test_scales_that_do_not_are_taken(lib, scale, dropout):  # noqa: F811
    assert taken(lib, BWD, scale=scale, dropout=dropout)
