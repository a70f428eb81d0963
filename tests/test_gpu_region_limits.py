"""Region selection and region attention at the sizes where a launch of one kernel would have 2^32 threads or more."""
import numpy as np
import pytest
import torch

import paper_2304_04237_amd as sa
from oracle import region_oracle as ro
from tests.region_cases import bounds, case, make, numpy_of

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


def test_backward_over_as_many_regions_as_there_may_be():
    """8 times 2^21 - 1 regions of keys: the lists are turned around by 2^22 blocks of 1024 threads."""
    c = case((1, 1024), (1, (1 << 21) - 1), heads=8, d=1, q_region=(1, 1), k_region=(1, 1), topk=2)
    t, index, how = make(c, "f32", seed=30)
    ref = ro.attention(*(numpy_of(t[n]) for n in ("q", "k", "v")), index, how, numpy_of(t["dout"]))
    g = {n: x.cuda() for n, x in t.items()}
    lists = torch.tensor(index, device="cuda")
    lse = torch.empty((1, 8, 1, 1024), device="cuda")
    out = sa.slide_region_attn_fwd(g["q"], g["k"], g["v"], lists, lse=lse, **how)
    grads = sa.slide_region_attn_bwd(g["dout"], g["q"], g["k"], g["v"], lists, out, lse, **how)
    bound = bounds(c, "f32", ref)
    for n, got in zip(("out", "dq", "dk", "dv"), (out, *grads)):
        assert (np.abs(numpy_of(got) - ref[n]) / bound[n]).max() <= 1, n
