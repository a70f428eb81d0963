"""Dropout on the GPU against the oracle, and an attention block made of all the calls."""
import numpy as np
import pytest
import torch

import paper_2304_04237_amd as sa
from oracle import region_oracle as ro
from tests.region_cases import DTYPES, NORM, case, make, numpy_of, off

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def normal(n, dtype, seed):
    return torch.tensor(np.random.default_rng(seed).standard_normal(n), dtype=torch.float32).to(DTYPES[dtype]).cuda()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 255, 2048, 2049, 100003])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.999])
def test_against_the_oracle(n, p, dtype):
    seed, offset = 0xfedcba9876543210, 12
    x, r, dout = (normal(n, dtype, s) for s in range(3))
    f = ro.drop_factors(np.arange(n), p, seed, offset)
    for residual in (None, r):
        y = sa.slide_dropout_fwd(x, p, seed, offset, residual=residual)
        want = f * numpy_of(x) + (0 if residual is None else numpy_of(r))
        # the factor, the product and the sum round once each in 32 bits, then once to the type
        assert (np.abs(numpy_of(y) - want) <= HALF[dtype] * np.abs(want) + 3 * 2.0 ** -24 * (np.abs(f * numpy_of(x)) + np.abs(want))).all()
    dx = sa.slide_dropout_bwd(dout, p, seed, offset)
    want = f * numpy_of(dout)
    assert (np.abs(numpy_of(dx) - want) <= (HALF[dtype] + 3 * 2.0 ** -24) * np.abs(want)).all()
    assert ((numpy_of(dx) == 0) == (f == 0)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_unaligned_in_place_and_what_lies_around(dtype):
    n = 5003
    whole = normal(n + 40, dtype, 4)
    want = {}
    for shift in (0, 1, 3, 8):
        x, r = whole[shift:shift + n].clone(), whole[20:20 + n].clone()
        want[shift] = sa.slide_dropout_fwd(x, 0.3, 5, 6, residual=r)
        room = torch.full((n + 40,), 99.0, dtype=DTYPES[dtype], device="cuda")
        y = room[shift:shift + n]
        sa.slide_dropout_fwd(whole[shift:shift + n], 0.3, 5, 6, residual=whole[20:20 + n], out=y)
        assert torch.equal(y, want[shift]) and (room[:shift] == 99).all() and (room[shift + n:] == 99).all()
        same = x.clone()
        assert torch.equal(sa.slide_dropout_fwd(same, 0.3, 5, 6, residual=r, out=same), want[shift])
        same = x.clone()
        sa.slide_dropout_bwd(same, 0.3, 5, 6, dx=same)
        assert torch.equal(same, sa.slide_dropout_bwd(x, 0.3, 5, 6))
        sa.slide_dropout_fwd(whole[shift:shift + n].clone(), 0.3, 5, 6, residual=r, out=r)
        assert torch.equal(r, want[shift])


def test_dropped_elements_contribute_nothing():
    n = 4096
    f = ro.drop_factors(np.arange(n), 0.5, 1, 2)
    x = torch.where(torch.tensor(f == 0), float("nan"), 1.0).cuda()
    x[f == 0][::2] = float("inf")
    y = sa.slide_dropout_fwd(x, 0.5, 1, 2)
    assert (numpy_of(y) == f).all()


def test_more_than_32_bits_of_elements():
    n = (1 << 32) + 1001
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    y = sa.slide_dropout_fwd(x, 0.5, 3, 4)
    for at in (0, (1 << 31) - 500, (1 << 32) - 500, n - 1001):
        i = np.arange(at, at + 1001)
        assert (numpy_of(y[at:at + 1001]) == ro.drop_factors(i, 0.5, 3, 4)).all(), at


def test_offset_in_device_memory_and_in_a_graph():
    x, r = normal(10000, "f32", 6), normal(10000, "f32", 7)
    number = torch.zeros(1, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    sa.slide_dropout_fwd(x, 0.2, 9, number, residual=r)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        y = sa.slide_dropout_fwd(x, 0.2, 9, number, residual=r)
        dx = sa.slide_dropout_bwd(x, 0.2, 9, number)
    for call in (3, 0, 3, 2 ** 32 - 1):
        number.fill_(call)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, sa.slide_dropout_fwd(x, 0.2, 9, call, residual=r)) and torch.equal(dx, sa.slide_dropout_bwd(x, 0.2, 9, call))


def test_refusals():
    x = torch.zeros(4, 6, device="cuda")
    for change, message in [(dict(x=x.half()), "float32 or bfloat16"), (dict(x=x.t()), "contiguous"), (dict(p=1.0), "dropout"),
                            (dict(p=-0.1), "dropout"), (dict(seed=1 << 64), "seed"), (dict(offset=-1), "offset"),
                            (dict(residual=x[:3]), "residual"), (dict(residual=x.bfloat16()), "residual"), (dict(out=x.t()), "result"),
                            (dict(residual=x.cpu()), "GPU")]:
        with pytest.raises(sa.SlideAttnError, match=message):
            sa.slide_dropout_fwd(**{**dict(x=x, p=0.1, seed=1, offset=0), **change})
    assert sa.slide_dropout_fwd(x[:0], 0.1, 1).shape == (0, 6)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_block_of_window_and_region_attention(dtype):
    """Local attention on the map, then region attention on its result with dropout of the weights, dropout and a residual:
    forward and backward of the second half against the oracle."""
    c = case((16, 24), B=2, heads=2, d=32, q_region=(8, 8), topk=3, dropout=0.25)
    t, _, how = make(c, dtype, seed=12)
    g = {n: x.cuda() for n, x in t.items()}
    C = 64
    zeros = torch.zeros((C, 9, 3, 3), device="cuda")
    w = sa.slide_reparam(zeros)
    local = sa.slide_attn_fwd_nhwc(g["q"], g["k"], g["v"], w, w, None, 2, 3)
    maps = dict(heads=2, q_region=(8, 8), k_region=(8, 8))
    index = sa.slide_region_select(local, g["k"], 3, **maps)
    drop = dict(dropout=0.25, seed=how["seed"], offset=1)
    lse = torch.empty((2, 2, 16, 24), device="cuda")
    out = sa.slide_region_attn_fwd(local, g["k"], g["v"], index, lse=lse, **maps, **drop)
    y = sa.slide_dropout_fwd(out, 0.1, how["seed"], 2, residual=local)
    dx = sa.slide_dropout_bwd(g["dout"], 0.1, how["seed"], 2)
    dq, dk, dv = sa.slide_region_attn_bwd(dx, local, g["k"], g["v"], index, out, lse, **maps, **drop)

    assert (index.cpu().numpy() == ro.select(numpy_of(local), numpy_of(g["k"]), 3, maps)).all()
    f = ro.drop_factors(np.arange(out.numel()), 0.1, how["seed"], 2).reshape(out.shape)
    ref = ro.attention(numpy_of(local), numpy_of(g["k"]), numpy_of(g["v"]), index.cpu().numpy(), dict(maps, **drop), numpy_of(dx))
    assert off(y, numpy_of(local) + f * ref["out"]) <= 2 * NORM[dtype]          # (out is rounded, then y)
    assert off(dx, f * numpy_of(g["dout"])) <= NORM[dtype]
    for n, got in (("dq", dq), ("dk", dk), ("dv", dv)):
        assert off(got, ref[n]) <= NORM[dtype], n
