"""Refusals of region selection, region attention and dropout: on the host, before any kernel (the pointers are no device memory)."""
import ctypes

import pytest
import torch

import paper_2304_04237_amd as sa
from paper_2304_04237_amd import region

P = ctypes.c_void_p(0x1000)
OK, NULL, SHAPE, DTYPE, WORKSPACE, ALIGN = 0, 1, 2, 3, 4, 6


@pytest.fixture(scope="module")
def lib():
    return region._library()


def problem(**kw):
    a = dict(B=2, heads=4, kv_heads=2, head_dim=32, q_h=14, q_w=14, k_h=14, k_w=14, q_region_h=7, q_region_w=7, k_region_h=7,
             k_region_w=7, topk=2, dtype=0, q_pixel=128, q_image=128 * 196, k_pixel=64, k_image=64 * 196, v_pixel=64,
             v_image=64 * 196, scale=0.0, dropout=0.0, seed=0, offset=0)
    a.update(kw)
    return region._Problem(**a)


def select(lib, p, q=P, k=P, index=P, ws=P, size=1 << 40):
    return lib.slide_region_select(p, q, k, index, ws, size, None)


def fwd(lib, p, q=P, k=P, v=P, index=P, out=P, lse=None, ws=P, size=1 << 40):
    return lib.slide_region_attn_fwd(p, q, k, v, index, out, lse, ws, size, None)


def bwd(lib, p, dout=P, q=P, k=P, v=P, index=P, out=P, lse=P, dq=P, dk=P, dv=P, ws=P, size=1 << 40):
    return lib.slide_region_attn_bwd(p, dout, q, k, v, index, out, lse, dq, dk, dv, ws, size, None)


@pytest.mark.parametrize("change, status", [
    (dict(dtype=2), DTYPE), (dict(B=0), SHAPE), (dict(heads=3), SHAPE), (dict(kv_heads=0), SHAPE), (dict(heads=0), SHAPE),
    (dict(head_dim=0), SHAPE), (dict(head_dim=129, q_pixel=1000, k_pixel=1000, v_pixel=1000), SHAPE), (dict(topk=0), SHAPE),
    (dict(topk=1025), SHAPE), (dict(q_h=0), SHAPE), (dict(k_w=-1), SHAPE), (dict(q_region_h=0), SHAPE), (dict(k_region_w=0), SHAPE),
    (dict(q_pixel=127), SHAPE), (dict(k_pixel=63), SHAPE), (dict(k_image=-1), SHAPE), (dict(q_pixel=1 << 31), SHAPE),
    (dict(k_h=1 << 15, k_w=1 << 14), SHAPE), (dict(q_h=1 << 14, q_w=1 << 15), SHAPE), (dict(B=40000), SHAPE),
    (dict(q_size=0x1002), ALIGN), (dict(k_size=0x1001), ALIGN)])
def test_every_call_refuses_a_bad_problem(lib, change, status):
    p = problem(**change)
    assert select(lib, p) == fwd(lib, p) == bwd(lib, p) == status
    assert all(lib.slide_region_workspace_bytes(p, c) == 0 for c in range(3))


@pytest.mark.parametrize("change, status", [
    (dict(dropout=1.0), SHAPE), (dict(dropout=-0.1), SHAPE), (dict(dropout=float("nan")), SHAPE), (dict(dropout=1 - 2.0 ** -18), SHAPE),
    (dict(scale=-1.0), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE), (dict(v_pixel=63), SHAPE),
    (dict(v_image=-1), SHAPE), (dict(offset_device=0x1004), ALIGN)])
def test_attention_refuses_a_bad_problem(lib, change, status):
    p = problem(**change)
    assert fwd(lib, p) == bwd(lib, p) == status


def test_selection_refuses_more_regions_than_it_ranks(lib):
    p = problem(k_h=1, k_w=16385, k_region_h=1, k_region_w=1)
    assert select(lib, p) == SHAPE
    assert lib.slide_region_workspace_bytes(p, 0) == 0 and lib.slide_region_workspace_bytes(p, 2) > 0


def test_pointers(lib):
    p, odd = problem(), ctypes.c_void_p(0x1002)
    assert select(lib, None) == fwd(lib, None) == bwd(lib, None) == NULL
    for name in ("q", "k", "index"):
        assert select(lib, p, **{name: None}) == NULL and select(lib, p, **{name: odd}) == ALIGN
    for name in ("q", "k", "v", "index", "out"):
        assert fwd(lib, p, **{name: None}) == NULL and fwd(lib, p, **{name: odd}) == ALIGN
    assert fwd(lib, p, lse=odd) == ALIGN
    for name in ("dout", "q", "k", "v", "index", "out", "lse", "dq", "dk", "dv"):
        assert bwd(lib, p, **{name: None}) == NULL and bwd(lib, p, **{name: odd}) == ALIGN
    assert fwd(lib, problem(dtype=1), q=ctypes.c_void_p(0x1001)) == ALIGN


def test_workspaces(lib):
    p = problem()
    for call, make in ((0, select), (1, fwd), (2, bwd)):
        need = lib.slide_region_workspace_bytes(p, call)
        if need:
            assert make(lib, p, ws=None) == WORKSPACE and make(lib, p, size=need - 1) == WORKSPACE
            assert make(lib, p, ws=ctypes.c_void_p(0x1008)) == ALIGN
    assert lib.slide_region_workspace_bytes(p, 0) > 0 and lib.slide_region_workspace_bytes(p, 2) > 0
    assert lib.slide_region_workspace_bytes(p, 3) == 0 == lib.slide_region_workspace_bytes(p, -1)


def test_dropout_refusals(lib):
    def fwd(x=P, residual=None, y=P, n=8, dtype=0, p=0.1, holder=None):
        return lib.slide_dropout_fwd(x, residual, y, n, dtype, p, 0, 0, holder, None)

    odd = ctypes.c_void_p(0x1002)
    assert fwd(dtype=5) == DTYPE
    assert fwd(n=0) == fwd(n=-1) == fwd(n=1 << 34) == fwd(p=1.0) == fwd(p=-1e-3) == fwd(p=float("nan")) == SHAPE
    assert fwd(x=None) == fwd(y=None) == NULL
    assert fwd(x=odd) == fwd(y=odd) == fwd(residual=odd) == fwd(holder=ctypes.c_void_p(0x1004)) == ALIGN
    assert lib.slide_dropout_bwd(None, P, 8, 0, 0.1, 0, 0, None, None) == NULL
    assert lib.slide_dropout_bwd(P, P, 8, 0, 1.5, 0, 0, None, None) == SHAPE


def test_binding_names_what_is_wrong():
    """Tensors on the CPU never reach the library."""
    q, k = torch.zeros(2, 6, 6, 64), torch.zeros(2, 6, 6, 32)
    how = dict(heads=4, kv_heads=2, q_region=(3, 3), k_region=(3, 3))
    with pytest.raises(sa.SlideAttnError, match="q must live on the GPU"):
        sa.slide_region_select(q, k, 2, **how)
    with pytest.raises(sa.SlideAttnError, match="must be .B, H, W, C."):
        sa.slide_region_select(q[0], k, 2, **how)
    with pytest.raises(sa.SlideAttnError, match="float32 or bfloat16"):
        sa.slide_region_select(q.half(), k, 2, **how)
    with pytest.raises(sa.SlideAttnError, match="int32 .B, kv_heads"):
        sa.slide_region_attn_fwd(q, k, k, torch.zeros(2, 2), **how)
    with pytest.raises(sa.SlideAttnError, match="x must live on the GPU"):
        sa.slide_dropout_fwd(q, 0.1, 0)
    with pytest.raises(sa.SlideAttnError, match="dout must live on the GPU"):
        sa.slide_dropout_bwd(q, 0.1, 0)


def test_binding_names_what_no_plan_can_hold():
    x = torch.zeros(1, 4, 4, 8)
    for region in (3, None):
        with pytest.raises(sa.SlideAttnError, match="q_region"):
            sa.slide_region_select(x, x, 1, heads=1, q_region=region, k_region=(2, 2))
    with pytest.raises(sa.SlideAttnError, match="call must be"):
        sa.slide_region_workspace_bytes("forward", x, x, 1, heads=1, q_region=(2, 2), k_region=(2, 2))


def test_strides_of_parts():
    def strides(t, name):
        return region._strides(t.shape, t.stride(), name)

    x = torch.zeros(2, 4, 5, 96)
    assert strides(x, "x") == (96, 96 * 20)
    assert strides(x[..., 32:64], "x") == (96, 96 * 20)                     # a part of the channels
    assert strides(torch.zeros(2, 1, 50, 8)[:, :, :10], "x") == (8, 400)    # the filled part of a cache
    assert strides(x[:1].expand(3, 4, 5, 96), "x") == (96, 0)               # one map for the whole batch
    assert strides(x[:, :, :1], "x") == (96 * 5, 96 * 20)
    assert strides(x[:, :1], "x") == (96, 96 * 20)
    for bad in (x[:, :, :3], x.permute(0, 2, 1, 3), x[..., ::2]):
        with pytest.raises(sa.SlideAttnError, match="evenly spaced"):
            strides(bad, "x")


@pytest.mark.parametrize("scale", [0.0, -1.0, 1e-46, 1e300, float("inf"), float("nan")])
def test_binding_refuses_scales_that_float32_does_not_hold(scale):
    """1e-46 is below half of float32's smallest number, 2^-149 = 1.4e-45."""
    x = torch.zeros(1, 4, 4, 8)
    with pytest.raises(sa.SlideAttnError, match="scale must be positive"):
        sa.slide_region_attn_fwd(x, x, x, torch.zeros(1, 1, 4, 1, dtype=torch.int32), heads=1, q_region=(2, 2), k_region=(2, 2), scale=scale)
