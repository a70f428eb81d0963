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


def small(**change):
    """Maps of two pixels, so that batches and heads of any number stay within the other limits."""
    a = dict(B=1, heads=1, kv_heads=1, head_dim=8, q_h=1, q_w=2, k_h=1, k_w=2, q_region_h=1, q_region_w=2, k_region_h=1, k_region_w=2, topk=1,
             q_pixel=1 << 20, q_image=1 << 21, k_pixel=1 << 20, k_image=1 << 21, v_pixel=1 << 20, v_image=1 << 21)
    a.update(change)
    return a


@pytest.mark.parametrize("call", [SELECT, BWD])
def test_batches_and_heads(lib, call):  # noqa: F811
    """At most 65535 images, heads, and key heads over all images."""
    for most, more in [(dict(B=65535), dict(B=65536)), (dict(heads=65535), dict(heads=65536)),
                       (dict(B=21845, heads=6, kv_heads=3), dict(B=21846, heads=6, kv_heads=3))]:
        assert taken(lib, call, **small(**most)) and not taken(lib, call, **small(**more))


@pytest.mark.parametrize("call", [SELECT, BWD])
def test_rows_and_places(lib, call):  # noqa: F811
    """Fewer than 2^24 times 32 rows over all regions, key heads and images, and as many places; fewer than 2^29 pixels a map."""
    for most, more in [(dict(q_w=(1 << 24) - 1, q_region_w=1), dict(q_w=1 << 24, q_region_w=1)),
                       (dict(q_w=(1 << 21) - 1, q_region_w=1, heads=8, kv_heads=8), dict(q_w=1 << 21, q_region_w=1, heads=8, kv_heads=8))]:
        assert taken(lib, call, **small(**most)) and not taken(lib, call, **small(**more))
    if call == BWD:
        for most, more in [(dict(k_w=(1 << 24) - 1, k_region_w=1), dict(k_w=1 << 24, k_region_w=1)),
                           (dict(q_w=1 << 20, q_region_w=1, topk=1023), dict(q_w=1 << 20, q_region_w=1, topk=1024))]:
            assert taken(lib, call, **small(**most)) and not taken(lib, call, **small(**more))
    assert not taken(lib, call, **small(q_w=1 << 29)) and not taken(lib, call, **small(k_w=1 << 29))


def test_keys_of_a_list_and_strides(lib):  # noqa: F811
    """Places of a region, counted up to a multiple of 4, times topk: fewer than 2^31 - 256; pixels fewer than 2^31 elements apart, images
    fewer than 2^45."""
    wide = dict(k_w=1 << 27, k_region_w=1 << 27)
    assert taken(lib, BWD, **small(**wide, topk=15)) and not taken(lib, BWD, **small(**wide, topk=16))
    for name, most in (("pixel", (1 << 31) - 1), ("image", (1 << 45) - 1)):
        for side in "qkv":
            assert taken(lib, BWD, **small(**{"%s_%s" % (side, name): most}))
            assert not taken(lib, BWD, **small(**{"%s_%s" % (side, name): most + 1}))
