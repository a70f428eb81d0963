"""Region selection and region attention at the sizes where a launch of one kernel would have 2^32 threads or more."""
import pytest
import torch

import paper_2304_04237_amd as sa

pytestmark = pytest.mark.gpu


def test_selection_for_as_many_lists_as_there_may_be():
    """2^23 lists over 9216 regions, of whose ranks one list's fill half the LDS: 2^23 blocks of 512 threads.  Rows of 1 and -1 pick the
    key that is the highest and the lowest of their head."""
    heads, rows, keys = 8, 1 << 20, 9216
    gen = torch.Generator(device="cuda").manual_seed(1)
    k = torch.rand((1, 1, keys, heads), generator=gen, device="cuda") - 0.5
    head = torch.arange(heads, device="cuda")
    high, low = 1103 * head + 7, keys - 1 - 1009 * head
    k[0, 0, high, head] = 16.0
    k[0, 0, low, head] = -16.0
    q = torch.where(torch.rand((1, 1, rows, heads), generator=gen, device="cuda") < 0.5, -1.0, 1.0)
    index = sa.slide_region_select(q, k, 1, heads=heads, q_region=(1, 1), k_region=(1, 1))
    want = torch.where(q[0, 0] > 0, high, low).T.reshape(index.shape)
    assert torch.equal(index, want.to(torch.int32))
