"""Inputs and bounds of the GPU tests of region attention."""
import numpy as np
import torch

from oracle import region_oracle as ro

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def case(q_map, k_map=None, B=1, heads=2, kv_heads=None, d=32, q_region=(4, 4), k_region=None, topk=3, sized=False, dropout=0.0,
         scale=None, lists="some"):
    return dict(B=B, q_map=q_map, k_map=k_map or q_map, heads=heads, kv_heads=kv_heads or heads, d=d, q_region=q_region,
                k_region=k_region or q_region, topk=topk, sized=sized, dropout=dropout, scale=scale, lists=lists)


def make(c, dtype, seed, padding=True):
    """numpy inputs (already rounded to dtype), lists and sizes; what lies outside the sizes is NaN."""
    rng = np.random.default_rng(seed)
    heads, kv, d, B = c["heads"], c["kv_heads"], c["d"], c["B"]

    def normal(m, n):
        return torch.tensor(rng.standard_normal((B, *m, n)), dtype=torch.float32).to(DTYPES[dtype])

    t = dict(q=normal(c["q_map"], heads * d), k=normal(c["k_map"], kv * d), v=normal(c["k_map"], kv * d), dout=normal(c["q_map"], heads * d))
    how = dict(heads=heads, kv_heads=kv, q_region=c["q_region"], k_region=c["k_region"])
    if c["sized"]:
        sizes = {}
        for side in ("q", "k"):
            H, W = c[side + "_map"]
            size = np.stack([rng.integers(0 if H > 1 else 1, H + 2, B), rng.integers(1, W + 2, B)], 1)      # (some past the map)
            size[-1] = (max(1, H - 1), max(1, W - 3))
            sizes[side] = size.astype(np.int32)
            if padding:
                for b in range(B):
                    for name in (("q", "dout") if side == "q" else ("k", "v")):
                        t[name][b, size[b, 0]:] = float("nan")
                        t[name][b, :, size[b, 1]:] = float("nan")
        how.update(q_size=sizes["q"], k_size=sizes["k"])
    if c["scale"]:
        how["scale"] = c["scale"]
    if c["dropout"]:
        how.update(dropout=c["dropout"], seed=0x1234567890abcdef + seed, offset=0xfffffffe)
    G, J = len(ro.regions(*c["q_map"], c["q_region"])), len(ro.regions(*c["k_map"], c["k_region"]))
    if c["lists"] == "some":            # anything that a list may hold: outside, missing, twice
        index = rng.integers(0, J, (B, kv, G, c["topk"]))
        index = np.where(rng.random(index.shape) < 0.15, rng.choice([-1, J, J + 7, -2 ** 31, 2 ** 31 - 1], index.shape), index)
        index[-1, -1, -1] = -1          # a group without any
    elif c["lists"] == "early":         # one to three regions, then nothing, in every second group nothing at all
        index = np.full((B, kv, G, c["topk"]), -1)
        index[:, :, ::2, :3] = rng.integers(0, J, index[:, :, ::2, :3].shape)
        index[:, :, ::4, 2] = -1
    else:                               # every group lists the same few regions
        index = np.broadcast_to(np.arange(c["topk"]) % J, (B, kv, G, c["topk"]))
    return t, np.ascontiguousarray(index, dtype=np.int32), how


def numpy_of(t):
    return t.double().cpu().numpy()


def bounds(c, dtype, ref):
    """Largest error of every single value, from the sums of absolute values that the oracle gives.

    Of each attention weight: its logit is a chain of d products (d + 2 roundings of 2^-24 of score_mag), the exponential and the
    statistics add 16 roundings, the sum over the keys one for each of the topk * places.  bf16: the weight and the logit's
    gradient are rounded to bf16 before the products (2^-8 each), D is formed from the rounded out (2^-8 of sum |dout out|, which
    dq_mag and dk_mag hold twice), and the result is rounded once (2^-8)."""
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    places = min(c["k_region"][0], c["k_map"][0]) * min(c["k_region"][1], c["k_map"][1])
    rows = min(c["q_region"][0], c["q_map"][0]) * min(c["q_region"][1], c["q_map"][1]) * c["heads"] // c["kv_heads"]
    chain = (c["d"] + 2) * ref["score_mag"] + 16 + 2 * c["d"]
    weight = (2.0 ** -8 if dtype == "bf16" else 0.0) + 2.0 ** -24 * (chain + c["topk"] * places)
    per_key = weight + 2.0 ** -24 * rows * c["topk"] * len(ro.regions(*c["q_map"], c["q_region"]))
    return {n: (per_key if n in ("dk", "dv") else weight) * ref[n + "_mag"] + half * np.abs(ref[n]) + 1e-30
            for n in ("out", "dq", "dk", "dv") if n in ref}


def off(got, want):
    """2-norm of the difference over the 2-norm of the result."""
    size = np.linalg.norm(want)
    return np.linalg.norm(numpy_of(got) - want) / size if size else np.linalg.norm(numpy_of(got))


# roundings of independent sign: a weight's and the result's, of at most 2^-8, with root mean square 0.58 of that: 0.82 * 2^-8 in all;
# float32: 32 of 2^-24, from logits of a few units and chains of up to 128 products
NORM = {"bf16": 2.0 ** -8, "f32": 32 * 2.0 ** -24}
