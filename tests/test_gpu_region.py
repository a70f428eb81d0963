"""Region selection and region attention on the GPU against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2304_04237_amd as sa
from oracle import region_oracle as ro
from tests.region_cases import DTYPES, NORM, bounds, case, make, numpy_of, off

pytestmark = pytest.mark.gpu

CASES = {
    "regions_7x7": case((14, 14), q_region=(7, 7), topk=2),
    "stage_like": case((24, 32), B=2, q_region=(8, 8), topk=4),
    "ragged_24_channels": case((13, 19), B=2, heads=3, d=24, q_region=(4, 5), sized=True),
    "unlike_regions": case((9, 17), (11, 6), B=3, heads=2, d=16, q_region=(3, 4), k_region=(5, 2), topk=5, sized=True),
    "grouped_sequence": case((1, 100), B=2, heads=8, kv_heads=2, d=64, q_region=(1, 16), k_region=(1, 20), topk=4, sized=True),
    "own_list_for_each_token": case((1, 37), heads=8, kv_heads=2, d=64, q_region=(1, 1), k_region=(1, 8), topk=3),
    "one_token": case((1, 1), (1, 300), B=3, heads=8, kv_heads=2, d=128, q_region=(1, 1), k_region=(1, 64), topk=3, sized=True),
    "one_token_alone": case((1, 1), (1, 70), heads=1, d=64, q_region=(1, 1), k_region=(1, 16), topk=4),
    "one_token_many_keys": case((1, 1), (1, 5000), B=2, heads=16, kv_heads=2, d=64, q_region=(1, 1), k_region=(1, 32), topk=100),
    "two_tokens_128_rows": case((1, 2), (1, 900), heads=64, kv_heads=1, d=32, q_region=(1, 2), k_region=(1, 33), topk=20),
    "one_pixel": case((1, 1), d=8, q_region=(1, 1), topk=1, lists="all"),
    "one_channel": case((5, 5), heads=1, d=1, q_region=(2, 2), topk=4),
    "odd_channels": case((6, 7), heads=3, d=33, q_region=(3, 3), topk=3),
    "100_channels": case((1, 90), heads=2, d=100, q_region=(1, 24), k_region=(1, 40), topk=3),
    "128_channels": case((1, 130), heads=4, kv_heads=1, d=128, q_region=(1, 32), k_region=(1, 32), topk=3, sized=True),
    "region_larger_than_map": case((5, 6), (7, 4), q_region=(50, 50), k_region=(9, 9), topk=1, lists="all"),
    "regions_of_196": case((28, 15), heads=1, d=32, q_region=(14, 14), topk=2),
    "512_rows_a_group": case((1, 64), (1, 256), heads=8, kv_heads=1, d=16, q_region=(1, 64), k_region=(1, 128), topk=2),
    "many_small_regions": case((1, 200), heads=2, d=32, q_region=(1, 10), k_region=(1, 3), topk=64),
    "everyone_lists_the_same": case((20, 20), B=2, heads=2, d=32, q_region=(2, 2), k_region=(5, 5), topk=2, lists="all"),
    "600_lists": case((1, 600), heads=4, kv_heads=2, d=32, q_region=(1, 1), k_region=(1, 8), topk=4),
    "600_lists_64_channels": case((1, 600), B=2, heads=4, kv_heads=1, d=64, q_region=(1, 1), k_region=(1, 40), topk=4, sized=True),
    "600_lists_128_channels": case((1, 600), heads=2, kv_heads=1, d=128, q_region=(1, 1), k_region=(1, 100), topk=4),
    "600_lists_of_few": case((1, 600), (1, 50), heads=40, kv_heads=1, d=20, q_region=(1, 1), k_region=(1, 10), topk=4),
    "600_lists_odd": case((1, 600), heads=2, d=35, q_region=(1, 1), k_region=(1, 8), topk=4),
    "large_groups_of_few": case((32, 40), (8, 8), heads=1, d=48, q_region=(16, 20), k_region=(4, 4), topk=3),
    "64_channels": case((24, 24), B=2, heads=2, d=64, q_region=(8, 8), topk=3, sized=True),
    "96_channels": case((16, 16), heads=2, d=96, q_region=(8, 8), topk=3),
    "1024_entries": case((1, 70), (1, 300), heads=2, d=32, q_region=(1, 35), k_region=(1, 2), topk=1024),
    "list_ends_early": case((20, 20), B=2, heads=2, d=32, q_region=(5, 5), topk=70, lists="early"),
    "one_token_128_channels_many_keys": case((1, 1), (1, 9000), B=2, heads=8, kv_heads=2, d=128, q_region=(1, 1), k_region=(1, 64), topk=60, sized=True),
    "1088_groups": case((64, 68), heads=4, d=32, q_region=(4, 4), topk=10, sized=True),
    "624_groups_128_channels": case((48, 50), heads=4, d=128, q_region=(4, 4), topk=9),
    "dropped_1088_groups": case((64, 68), heads=4, d=24, q_region=(4, 4), topk=10, dropout=0.2),
    "dropped_two_of_many_regions": case((12, 12), heads=2, d=64, q_region=(6, 6), k_region=(5, 5), topk=9, dropout=0.4, sized=True),
    "dropped_2600_entries": case((1, 650), (1, 2054), heads=1, d=16, q_region=(1, 1), k_region=(1, 1), topk=4, dropout=0.1),
    "dropped_2400_entries_sized": case((1, 300), (1, 1027), B=2, heads=2, d=16, q_region=(1, 2), k_region=(1, 1), topk=16, sized=True, dropout=0.1),
    "map_as_one_region": case((30, 31), heads=1, d=32, q_region=(99, 99), k_region=(99, 99), topk=1, lists="all"),
    "odd_channels_few_keys_attended": case((6, 7), (40, 50), heads=2, d=33, q_region=(6, 7), k_region=(5, 5), topk=2),
    "60_channels": case((18, 15), B=2, heads=3, d=60, q_region=(6, 3), topk=9, sized=True),
    "scale": case((8, 8), d=32, q_region=(4, 4), topk=2, scale=0.7),
    "steep": case((8, 8), d=32, q_region=(4, 4), topk=2, scale=3.0),
    "dropped_ragged": case((13, 19), B=2, heads=3, d=24, q_region=(4, 5), sized=True, dropout=0.3),
    "dropped_odd": case((9, 9), heads=6, kv_heads=2, d=32, q_region=(3, 3), k_region=(3, 5), topk=4, dropout=0.5),
    "dropped_stage_like": case((24, 32), q_region=(8, 8), topk=4, dropout=0.1),
    "dropped_sequence": case((1, 100), heads=8, kv_heads=2, d=64, q_region=(1, 16), k_region=(1, 20), topk=4, dropout=0.2),
    "dropped_600_lists": case((1, 600), heads=4, kv_heads=2, d=32, q_region=(1, 1), k_region=(1, 9), topk=4, dropout=0.2),
    "dropped_64_channels": case((24, 24), heads=2, d=64, q_region=(8, 8), topk=3, dropout=0.3),
    "dropped_128_channels": case((1, 130), heads=4, kv_heads=1, d=128, q_region=(1, 32), k_region=(1, 32), topk=3, dropout=0.3),
    "dropped_one_token_many_keys": case((1, 1), (1, 5000), B=2, heads=16, kv_heads=2, d=64, q_region=(1, 1), k_region=(1, 33), topk=90, dropout=0.3),
    "dropped_one_token": case((1, 1), (1, 300), B=2, heads=8, kv_heads=2, d=128, q_region=(1, 1), k_region=(1, 63), topk=3, dropout=0.2),
}


def on_gpu(t, index, how):
    how = dict(how)
    for n in ("q_size", "k_size"):
        if n in how:
            how[n] = torch.tensor(how[n], device="cuda")
    return {n: x.cuda() for n, x in t.items()}, torch.tensor(index, device="cuda"), how


def clean(t):
    """The oracle's inputs: what no result may depend on (NaN in the padding) as zeros."""
    return {n: np.nan_to_num(numpy_of(x)) for n, x in t.items()}


def forward(g, index, how, **kw):
    B, H, W = g["q"].shape[:3]
    lse = torch.full((B, how["heads"], H, W), 7.0, device="cuda")
    out = sa.slide_region_attn_fwd(g["q"], g["k"], g["v"], index, lse=lse, **how, **kw)
    return out, lse


def backward(g, index, how, out, lse, **kw):
    return sa.slide_region_attn_bwd(g["dout"], g["q"], g["k"], g["v"], index, out, lse, **how, **kw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", CASES)
def test_forward_and_backward(name, dtype):
    c = CASES[name]
    t, index, how = make(c, dtype, seed=3)
    print(name, dtype, flush=True)
    x = clean(t)
    ref = ro.attention(x["q"], x["k"], x["v"], index, how, x["dout"])
    g, idx, gh = on_gpu(t, index, how)
    out, lse = forward(g, idx, gh)
    grads = backward(g, idx, gh, out, lse)
    bound = bounds(c, dtype, ref)
    want_lse = ref["lse"]
    assert (np.isneginf(numpy_of(lse)) == np.isneginf(want_lse)).all()
    finite = np.isfinite(want_lse)
    # a logit's chain of roundings, the maximum's and the logarithm's
    assert np.abs(numpy_of(lse)[finite] - want_lse[finite]).max(initial=0) <= 2.0 ** -24 * ((c["d"] + 4) * ref["score_mag"] + 64)
    for n, got in zip(("out", "dq", "dk", "dv"), (out, *grads)):
        worst = (np.abs(numpy_of(got) - ref[n]) / bound[n]).max()
        print("%-4s error / bound %.3f, 2-norm %.3g" % (n, worst, off(got, ref[n])), flush=True)
        assert worst <= 1, n
        if ref[n].size >= 1000 and c["scale"] is None:
            assert off(got, ref[n]) <= NORM[dtype], n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", [n for n in CASES if not n.startswith("dropped")])
def test_selection(name, dtype):
    c = CASES[name]
    t, _, how = make(c, dtype, seed=4)
    x = clean(t)
    g, _, gh = on_gpu(t, np.zeros(1, np.int32), how)
    for topk in sorted({1, c["topk"], min(c["topk"] + 3, 1024)}):
        print(name, dtype, topk, flush=True)
        got = sa.slide_region_select(g["q"], g["k"], topk, **{n: v for n, v in gh.items() if n != "scale"})
        assert (got.cpu().numpy() == ro.select(x["q"], x["k"], topk, how)).all()


def test_selection_among_equal_and_odd_scores():
    """Ties, infinities and NaN: equal scores go to the lowest region, NaN ranks lowest but is chosen before nothing."""
    inf, nan = float("inf"), float("nan")
    q = torch.ones(1, 1, 3, 1, device="cuda")
    for values in ([1, 1, 1, 1, 1], [0, -0.0, 0, 1, 1], [nan, 2, nan, -inf, 3], [inf, inf, -inf, nan, 0], [-inf] * 5, [nan] * 5):
        k = torch.tensor(values, dtype=torch.float32, device="cuda").reshape(1, 1, 5, 1)
        for topk in (1, 2, 3, 4, 5, 6):
            got = sa.slide_region_select(q, k, topk, heads=1, q_region=(1, 1), k_region=(1, 1))
            order = sorted(range(5), key=lambda j: (-(values[j] if values[j] == values[j] else -inf), j))
            want = sorted(order[:topk]) + [-1] * (topk - 5)
            assert (got.cpu().numpy() == np.array(want)).all(), (values, topk)


def test_selection_among_many_regions():
    rng = np.random.default_rng(11)
    # 16384 regions, the most there may be; values of few levels, so that many scores are equal
    k = torch.tensor(rng.integers(-8, 9, (1, 1, 16384, 2)), dtype=torch.float32, device="cuda")
    q = torch.tensor(rng.integers(-3, 4, (1, 1, 5, 2)), dtype=torch.float32, device="cuda")
    for topk in (1, 64, 65, 1000, 1024):
        got = sa.slide_region_select(q, k, topk, heads=1, q_region=(1, 2), k_region=(1, 1)).cpu().numpy()
        want = ro.select(q.cpu().numpy(), k.cpu().numpy(), topk, dict(heads=1, q_region=(1, 2), k_region=(1, 1)))
        assert (got == want).all(), topk


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parts_of_wider_tensors(dtype):
    """q, k and v as parts of one projection; k and v as the filled part of a cache; one map for the whole batch; unaligned."""
    c = case((6, 10), B=2, heads=2, d=24, q_region=(3, 5), topk=2)
    t, index, how = make(c, dtype, seed=5)
    g, idx, gh = on_gpu(t, index, how)
    want = forward(g, idx, gh)
    want += tuple(backward(g, idx, gh, *want))
    for pad in (0, 1, 8):
        wide = torch.full((2, 6, 10, 3 * 48 + pad), float("nan"), dtype=DTYPES[dtype], device="cuda")
        parts = dict(g)
        for n, name in enumerate(("q", "k", "v")):
            parts[name] = wide[..., 48 * n + pad:48 * n + pad + 48]
            parts[name].copy_(g[name])
        got = forward(parts, idx, gh)
        got += tuple(backward(parts, idx, gh, *got))
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        assert (sa.slide_region_select(parts["q"], parts["k"], 2, **gh) == sa.slide_region_select(g["q"], g["k"], 2, **gh)).all()

    c = case((1, 4), (1, 30), B=2, heads=2, d=32, q_region=(1, 4), k_region=(1, 8), topk=3)
    t, index, how = make(c, dtype, seed=6)
    g, idx, gh = on_gpu(t, index, how)
    want = forward(g, idx, gh)
    cache = {n: torch.full((2, 1, 100, 64), float("nan"), dtype=DTYPES[dtype], device="cuda") for n in ("k", "v")}
    for n in cache:
        cache[n][:, :, :30] = g[n]
    got = forward(dict(g, **{n: x[:, :, :30] for n, x in cache.items()}), idx, gh)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])

    one = dict(g, k=g["k"][:1].expand_as(g["k"]), v=g["v"][:1].expand_as(g["v"]))
    same = dict(g, k=one["k"].contiguous(), v=one["v"].contiguous())
    a, b = forward(one, idx, gh), forward(same, idx, gh)
    assert torch.equal(a[0], b[0])
    for u, w in zip(backward(one, idx, gh, *a), backward(same, idx, gh, *b)):
        assert torch.equal(u, w)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["regions_7x7", "100_channels", "many_small_regions", "64_channels", "1088_groups", "dropped_stage_like",
                                  "dropped_two_of_many_regions", "dropped_128_channels", "dropped_sequence"])
def test_tensors_that_begin_anywhere(name, dtype):
    """Whole strides behind an address that is no multiple of 16 bytes, for inputs and for the gradients' own memory."""
    c = CASES[name]
    t, index, how = make(c, dtype, seed=12)
    print(name, dtype, flush=True)
    x = clean(t)
    ref = ro.attention(x["q"], x["k"], x["v"], index, how, x["dout"])
    g, idx, gh = on_gpu(t, index, how)

    def moved(x):
        room = torch.full((x.numel() + 1,), float("nan"), dtype=x.dtype, device="cuda")
        room[1:].copy_(x.reshape(-1))
        return room[1:].view(x.shape)

    g = {n: moved(x) for n, x in g.items()}
    out, lse = forward(g, idx, gh)
    grads = backward(g, idx, gh, moved(out), lse)
    bound = bounds(c, dtype, ref)
    for n, got in zip(("out", "dq", "dk", "dv"), (out, *grads)):
        assert (np.abs(numpy_of(got) - ref[n]) / bound[n]).max() <= 1, n


@pytest.mark.parametrize("name", ["ragged_24_channels", "one_token_many_keys", "everyone_lists_the_same", "600_lists_64_channels", "dropped_sequence"])
def test_the_same_twice_and_on_another_stream(name):
    t, index, how = make(CASES[name], "bf16", seed=7)
    g, idx, gh = on_gpu(t, index, how)
    out, lse = forward(g, idx, gh)
    first = (out, lse, *backward(g, idx, gh, out, lse))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out, lse = forward(g, idx, gh)
        second = (out, lse, *backward(g, idx, gh, out, lse))
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(first, second):
        assert torch.equal(a.nan_to_num(), b.nan_to_num())


@pytest.mark.parametrize("name", ["dropped_ragged", "odd_channels", "one_token_many_keys"])
def test_outputs_and_workspaces_of_the_caller(name):
    """Given outputs are written whole, and nothing behind a workspace of exactly the size asked for."""
    c = CASES[name]
    t, index, how = make(c, "bf16", seed=8)
    g, idx, gh = on_gpu(t, index, how)
    sizes = {n: gh.pop(n) for n in ("q_size", "k_size") if n in gh}
    drop = {n: gh.pop(n) for n in ("dropout", "seed", "offset") if n in gh}
    out, lse = forward(g, idx, dict(gh, **sizes, **drop))
    want = backward(g, idx, dict(gh, **sizes, **drop), out, lse)

    def room(call):
        need = sa.slide_region_workspace_bytes(call, g["q"], g["k"], c["topk"], **gh)
        whole = torch.full((need + 256,), 165, dtype=torch.uint8, device="cuda")
        return whole, whole[:need]

    whole, ws = room("fwd")
    mine = torch.full_like(out, float("nan"))
    forward(g, idx, dict(gh, **sizes, **drop), out=mine, workspace=ws if ws.numel() else None)
    assert torch.equal(mine, out) and (whole[ws.numel():] == 165).all()
    whole, ws = room("bwd")
    mine = [torch.full_like(x, float("nan")) for x in want]
    backward(g, idx, dict(gh, **sizes, **drop), out, lse, outputs=mine, workspace=ws)
    assert all(torch.equal(a, b) for a, b in zip(mine, want)) and (whole[ws.numel():] == 165).all()
    whole, ws = room("select")
    lists = torch.full_like(idx, 99)
    sa.slide_region_select(g["q"], g["k"], c["topk"], index=lists, workspace=ws, **gh, **sizes)
    assert torch.equal(lists, sa.slide_region_select(g["q"], g["k"], c["topk"], **gh, **sizes)) and (whole[ws.numel():] == 165).all()


def test_binding_refuses_on_the_gpu():
    q = torch.zeros(2, 6, 6, 64, device="cuda")
    idx = torch.zeros(2, 2, 4, 1, dtype=torch.int32, device="cuda")
    how = dict(heads=2, q_region=(3, 3), k_region=(3, 3))
    lse = torch.zeros(2, 2, 6, 6, device="cuda")
    for change, message in [(dict(index=idx.long()), "index"), (dict(index=idx[:, :, :3]), "index"), (dict(index=idx.cpu()), "index"),
                            (dict(k=q[..., :32]), "k must"), (dict(v=q[:, :5]), "v must"), (dict(k=q.bfloat16()), "k must"),
                            (dict(heads=3), "multiple"), (dict(kv_heads=4), "multiple"), (dict(q_region=(0, 3)), "q_region"),
                            (dict(k_region=(3, 3, 3)), "k_region"), (dict(q_size=torch.zeros(2, 2, device="cuda")), "q_size"),
                            (dict(k_size=torch.zeros(1, 2, dtype=torch.int32, device="cuda")), "k_size"), (dict(dropout=1.0), "dropout"),
                            (dict(seed=-1), "seed"), (dict(offset=1 << 32), "offset"), (dict(scale=0.0), "scale"),
                            (dict(offset=torch.zeros(1, device="cuda")), "offset"), (dict(lse=lse[0]), "lse"),
                            (dict(out=q[..., :32]), "out"), (dict(workspace=torch.zeros(8)), "workspace"),
                            (dict(q=q.transpose(1, 2)), "evenly spaced"), (dict(q=q[:0]), "k must")]:
        with pytest.raises(sa.SlideAttnError, match=message):
            sa.slide_region_attn_fwd(**{**dict(q=q, k=q, v=q, index=idx, **how), **change})
    with pytest.raises(sa.SlideAttnError, match="lse"):
        sa.slide_region_attn_bwd(q, q, q, q, idx, q, lse[:, :1], **how)
    with pytest.raises(sa.SlideAttnError, match="dk"):
        sa.slide_region_attn_bwd(q, q, q, q, idx, q, lse, outputs=(q, q[:1], q), **how)
    with pytest.raises(sa.SlideAttnError, match="WORKSPACE"):
        sa.slide_region_attn_bwd(q, q, q, q, idx, q, lse, workspace=torch.zeros(4, dtype=torch.uint8, device="cuda"), **how)


def test_values_that_are_not_finite():
    """An infinite or NaN value reaches the rows that attend it and no others; a logit of -infinity is a weight of zero."""
    for dtype in ("f32", "bf16"):
        c = case((1, 64), heads=1, d=32, q_region=(1, 16), k_region=(1, 16), topk=1)
        t, _, how = make(c, dtype, seed=9)
        index = np.arange(4).reshape(1, 1, 4, 1).astype(np.int32)       # each its own
        t["v"][0, 0, 5, 3] = float("inf")
        t["v"][0, 0, 20, 7] = float("nan")
        t["k"][0, 0, 40, 0] = float("nan")
        g, idx, gh = on_gpu(t, index, how)
        out, lse = forward(g, idx, gh)
        o = out[0, 0]
        assert (o[:16, 3] == float("inf")).all() and o[16:32, 7].isnan().all() and o[32:48].isnan().all()
        whole = torch.ones_like(o, dtype=torch.bool)
        whole[:16, 3] = whole[16:32, 7] = whole[32:48] = False
        assert o[whole].isfinite().all() and lse[0, 0, 0, 32:48].isnan().all() and lse[0, 0, 0, :32].isfinite().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("dropout", [0.0, 0.2])
def test_queries_outside_pass_nothing_whatever_the_keys_hold(dtype, value, dropout):
    """Keys that only rows outside the image list, in regions wholly and partly outside."""
    c = case((16, 16), B=2, heads=2, d=32, q_region=(8, 8), k_region=(4, 4), topk=3, dropout=dropout)
    t, _, how = make(c, dtype, seed=13)
    how["q_size"] = np.array([[5, 16], [16, 8]], dtype=np.int32)
    index = np.zeros((2, 2, 4, 3), dtype=np.int32)
    index[:, :] = [[0, 1, -1], [2, 3, 3], [4, 5, 1], [6, 7, 15]]
    g, idx, gh = on_gpu(t, index, how)
    want = forward(g, idx, gh)
    want += tuple(backward(g, idx, gh, *want))
    for b, inside in ((0, (0, 1)), (1, (0, 2))):        # regions of queries that have rows inside
        listed = {j for i in inside for j in index[0, 0, i]}
        for j in set(range(16)) - listed:
            for n in ("k", "v"):
                g[n][b, 4 * (j // 4), 4 * (j % 4) + 1] = value
    got = forward(g, idx, gh)
    got += tuple(backward(g, idx, gh, *got))
    for a, w in zip(got, want):
        assert torch.equal(a, w)


def test_two_calls_at_once():
    """Two streams, two problems, in turns; each has its own workspace."""
    work, want = [], []
    for name, seed in (("one_token_many_keys", 20), ("600_lists", 21)):
        t, index, how = make(CASES[name], "bf16", seed)
        g, idx, gh = on_gpu(t, index, how)
        out, lse = forward(g, idx, gh)
        work.append((g, idx, gh))
        want.append((out, lse, *backward(g, idx, gh, out, lse)))
    streams = [torch.cuda.Stream() for _ in work]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for n, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                out, lse = forward(*work[n])
                got[n].append((out, lse, *backward(*work[n], out, lse)))
    torch.cuda.synchronize()
    for n in range(2):
        assert all(torch.equal(a, b) for one in got[n] for a, b in zip(one, want[n]))


def test_a_cache_of_more_than_32_bits():
    """Keys and values behind 2^32 elements, queries of one token."""
    across, d = 1 << 16, 128                    # nine rows of 2^22 pixels
    k = torch.empty((1, 9, 64 * across, d), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    lists = [0, 4 * across + 5, 9 * across - 2, 9 * across - 1]
    gen = torch.Generator(device="cuda").manual_seed(1)

    def part(x, j):
        return x[:, j // across:j // across + 1, 64 * (j % across):64 * (j % across) + 64]

    for j in lists:
        for x in (k, v):
            part(x, j).copy_(torch.randn((1, 1, 64, d), generator=gen, device="cuda"))
    q = torch.randn((1, 1, 1, 8 * d), generator=gen, device="cuda").bfloat16()
    index = torch.tensor(lists, dtype=torch.int32, device="cuda").reshape(1, 1, 1, 4)
    out = sa.slide_region_attn_fwd(q, k, v, index, heads=8, kv_heads=1, q_region=(1, 1), k_region=(1, 64))
    near = {m: torch.cat([part(x, j) for j in lists], 2) for m, x in (("k", k), ("v", v))}
    ref = ro.attention(numpy_of(q), numpy_of(near["k"]), numpy_of(near["v"]), np.arange(4).reshape(1, 1, 1, 4),
                       dict(heads=8, kv_heads=1, q_region=(1, 1), k_region=(1, 64)))
    assert off(out, ref["out"]) <= NORM["bf16"]


def test_a_captured_step_draws_new_masks():
    """Forward and backward with dropout in a graph; the number of the call is in device memory and moves on between replays."""
    c = CASES["dropped_stage_like"]
    t, index, how = make(c, "bf16", seed=10)
    g, idx, gh = on_gpu(t, index, how)
    gh["offset"] = torch.zeros(1, dtype=torch.int64, device="cuda")

    def step():
        lists = sa.slide_region_select(g["q"], g["k"], c["topk"], heads=gh["heads"], q_region=gh["q_region"], k_region=gh["k_region"])
        out, lse = forward(g, idx, gh)
        return (lists, out, lse, *backward(g, idx, gh, out, lse))

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    seen = []
    for call in (0, 1, 5, 1, 4294967301):
        gh["offset"].fill_(call)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in held]
        want = step()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), call
        seen.append(got[1])
    assert not torch.equal(seen[0], seen[1]) and torch.equal(seen[1], seen[3]) and torch.equal(seen[2], seen[4])
