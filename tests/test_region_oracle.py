"""Pins of the oracle of region attention and dropout, on the CPU: the generator's published answers, closed forms, differences."""
import numpy as np
import pytest

from oracle import region_oracle as ro


def test_generator_gives_the_published_answers():
    # (known answers that the generator's authors distribute, for all-zero counter and key and 7 and 10 rounds)
    assert [int(x) for x in ro.philox(0, 0, 0, 0, 0, 7)] == [0x5f6fb709, 0x0d893f64, 0x4f121f81, 0x4f730a48]
    assert [int(x) for x in ro.philox(0, 0, 0, 0, 0, 10)] == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]


def test_dropout_keeps_the_share_and_the_mean():
    n = 1 << 16
    for p in (0.0, 0.1, 0.5, 0.9):
        f = ro.drop_factors(np.arange(n), p, 1234567890123, 2)
        dropped = (f == 0).mean()
        assert abs(dropped - p) <= 5 * np.sqrt(p * (1 - p) / n)         # five standard deviations of a share of n draws
        assert len(np.unique(f)) <= 2
    a, b = ro.drop_factors(np.arange(n), 0.5, 1, 0), ro.drop_factors(np.arange(n), 0.5, 1, 1)
    assert abs((a == b).mean() - 0.5) <= 5 * 0.5 / np.sqrt(n)


def _random(rng, B, q_map, k_map, heads, kv, d):
    return [rng.standard_normal(s) for s in ((B, *q_map, heads * d), (B, *k_map, kv * d), (B, *k_map, kv * d), (B, *q_map, heads * d))]


def test_every_region_listed_is_full_attention():
    rng = np.random.default_rng(0)
    q, k, v, _ = _random(rng, 2, (5, 7), (5, 7), 4, 2, 6)
    problem = dict(heads=4, kv_heads=2, q_region=(2, 3), k_region=(3, 2))
    J = len(ro.regions(5, 7, (3, 2)))
    index = ro.select(q, k, J, problem)
    assert (index == np.arange(J)).all()
    got = ro.attention(q, k, v, index, problem)
    Q = q.reshape(2, 35, 2, 2, 6)
    K, V = k.reshape(2, 35, 2, 6), v.reshape(2, 35, 2, 6)
    S = np.einsum("bimgd,bjmd->bmgij", Q, K) / np.sqrt(6)
    P = np.exp(S)
    P /= P.sum(-1, keepdims=True)
    O = np.einsum("bmgij,bjmd->bimgd", P, V).reshape(q.shape)
    assert np.abs(got["out"] - O).max() < 1e-13
    assert np.abs(got["lse"].reshape(2, 2, 2, 35) - np.log(np.exp(S).sum(-1))).max() < 1e-13


def test_selection_takes_the_highest_pooled_score_and_the_lowest_of_equal_ones():
    q = np.ones((1, 1, 4, 1))
    k = np.array([1, 3, 2, 2, 5, -9, 2, 2, 1.0]).reshape(1, 1, 9, 1)    # regions of 2: means 2, 2, -2, 2, 1
    problem = dict(heads=1, q_region=(1, 2), k_region=(1, 2))
    assert ro.select(q, k, 2, problem)[0, 0].tolist() == [[0, 1], [0, 1]]
    assert ro.select(q, k, 4, problem)[0, 0].tolist() == [[0, 1, 3, 4]] * 2
    assert ro.select(-q, k, 1, problem)[0, 0].tolist() == [[2]] * 2
    sized = dict(problem, k_size=np.array([[1, 3]]), q_size=np.array([[1, 2]]))
    assert ro.select(q, k, 3, sized)[0, 0].tolist() == [[0, 1, -1], [-1, -1, -1]]


@pytest.mark.parametrize("dropout", [0.0, 0.4])
def test_gradients_against_differences(dropout):
    rng = np.random.default_rng(1)
    q, k, v, dout = _random(rng, 2, (3, 5), (4, 5), 4, 2, 3)
    problem = dict(heads=4, kv_heads=2, q_region=(2, 2), k_region=(2, 3), dropout=dropout, seed=77, offset=5,
                   k_size=np.array([[4, 5], [3, 4]]), q_size=np.array([[3, 5], [2, 5]]))
    index = rng.integers(-1, 5, (2, 2, 6, 3))                           # (four regions: 4 is outside, and some are listed twice)
    found = ro.attention(q, k, v, index, problem, dout)
    h = 1e-5
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        way = rng.standard_normal(x.shape)
        values = []
        for sign in (1, -1):
            args = dict(q=q, k=k, v=v)
            args[name[1]] = x + sign * h * way
            values.append((ro.attention(args["q"], args["k"], args["v"], index, problem)["out"] * dout).sum())
        # a centred difference is off by h^2 / 6 of the third derivative (here of order 100) and by rounding of 1e-16 * 100 / h
        assert abs((values[0] - values[1]) / (2 * h) - (found[name] * way).sum()) < 1e-7


def test_rows_without_keys_are_zeros():
    rng = np.random.default_rng(2)
    q, k, v, dout = _random(rng, 1, (1, 4), (1, 4), 1, 1, 2)
    problem = dict(heads=1, q_region=(1, 2), k_region=(1, 2))
    found = ro.attention(q, k, v, np.array([[[[-1], [1]]]]), problem, dout)
    assert (found["out"][0, 0, :2] == 0).all() and np.isneginf(found["lse"][0, 0, 0, :2]).all()
    assert (found["dk"][0, 0, :2] == 0).all() and (found["dk"][0, 0, 2:] != 0).any()
