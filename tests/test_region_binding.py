"""The binding of region selection, region attention and dropout on the host: what one call leaves for the next, and sizes that are refused."""
import pytest
import torch

import paper_2304_04237_amd as sa
from paper_2304_04237_amd import region


def plan_of(q, k, topk=2, **how):
    how = {**dict(heads=2, q_region=(4, 4), k_region=(4, 4), kv_heads=None), **how}
    return region._plan(q, (("k", k), ("v", k)), how["heads"], how["q_region"], how["k_region"], how["kv_heads"], topk)


@pytest.mark.gpu
def test_a_refused_call_leaves_the_next_one_its_scratch():
    """How much scratch a call needs is kept for the next of the same sizes: a call that is refused must not enter it."""
    q = torch.randn(1, 13, 17, 64, device="cuda")
    index = torch.zeros(1, 2, 20, 2, dtype=torch.int32, device="cuda")
    how = dict(heads=2, q_region=(4, 4), k_region=(4, 4))
    lse = torch.empty(1, 2, 13, 17, device="cuda")
    for _ in range(2):
        with pytest.raises(sa.SlideAttnError):
            sa.slide_region_attn_fwd(q, q, q, index, dropout=1.0 - 2.0 ** -17 - 1e-12, **how)
        with pytest.raises(sa.SlideAttnError):
            sa.slide_region_attn_bwd(q, q, q, q, index, q, lse, dropout=1.0 - 2.0 ** -17 - 1e-12, **how)
        out = sa.slide_region_attn_fwd(q, q, q, index, lse=lse, **how)
        assert all(x.isfinite().all() for x in sa.slide_region_attn_bwd(q, q, q, q, index, out, lse, **how))


@pytest.mark.parametrize("dropout", [1.0 - 2.0 ** -17 - 1e-12, 1.0 - 2.0 ** -17, 1.0, float("nan"), -1e-50, 10 ** 400])
def test_dropout_is_refused_as_the_float32_that_it_becomes(dropout):
    """1 - 2^-17 - 1e-12 is 1 - 2^-17 in float32, which rounds to 65536 / 65536 (ties to even)."""
    with pytest.raises(sa.SlideAttnError, match="dropout must be"):
        region._random(dropout, 1, 0, torch.device("cpu"))


def test_the_largest_dropout_that_float32_holds():
    """The next float32 below 1 - 2^-17 rounds to 65535 / 65536."""
    rate = 1.0 - 2.0 ** -17 - 2.0 ** -24
    assert region._random(rate, 1, 0, torch.device("cpu"))[0] == rate
    q = torch.zeros(1, 13, 17, 64)
    p = plan_of(q, q).problem(None, None, q.device)
    p.dropout = rate
    assert region._library().slide_region_workspace_bytes(p, region._BWD) > 0


@pytest.mark.parametrize("q_shape, k_shape, heads", [
    ((1, 1, 2 ** 32 + 5, 8), (1, 1, 20, 8), 1), ((1, 2 ** 32 + 5, 1, 8), (1, 1, 20, 8), 1), ((2 ** 32 + 1, 1, 5, 8), (2 ** 32 + 1, 1, 5, 8), 1),
    ((1, 1, 5, 8), (1, 1, 2 ** 32 + 20, 8), 1), ((1, 1, 5, 8), (1, 2 ** 31, 1, 8), 1), ((1, 1, 5, 2 ** 32 + 32), (1, 1, 5, 2 ** 32 + 32), 1),
    ((1, 1, 5, 2 ** 33 + 64), (1, 1, 5, 2 ** 33 + 64), 2)])
def test_sizes_that_an_int_does_not_hold_are_refused(q_shape, k_shape, heads):
    """The library's sizes are ints: 2^32 + 5 must not arrive there as 5."""
    q, k = torch.empty(q_shape, device="meta"), torch.empty(k_shape, device="meta")
    with pytest.raises(sa.SlideAttnError):
        plan_of(q, k, heads=heads)


@pytest.mark.parametrize("change", [dict(heads=2.0), dict(kv_heads=2.0), dict(q_region=(4.0, 4)), dict(k_region=(4, 4.0)), dict(topk=1.0),
                                    dict(topk=True), dict(q_region=(True, 4)), dict(heads=True)])
def test_what_is_no_integer_is_refused_after_an_equal_integer_too(change):
    """2.0 and True equal 2 and 1: a plan that was made for those must not answer for them."""
    x = torch.zeros(1, 12, 12, 64)
    for topk in (1, 2):
        for heads in (1, 2):
            for height in (1, 4):
                plan_of(x, x, topk=topk, heads=heads, q_region=(height, 4))
                plan_of(x, x, topk=topk, heads=heads, kv_heads=heads, q_region=(height, 4))
    with pytest.raises(sa.SlideAttnError, match="must be an integer"):
        plan_of(x, x, **change)
