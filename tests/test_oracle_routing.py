"""Pins for the oracle's expert routing."""
import math

import numpy as np
import pytest
import torch

from oracle.routing import route, route_row


@pytest.mark.parametrize("E,k", [(8, 2), (60, 4), (128, 8), (5, 5)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_matches_torch_topk(E, k, score):
    l = np.random.default_rng(E).normal(0, 2, (64, E))
    s = torch.softmax(torch.from_numpy(l), 1) if score == "softmax" else torch.sigmoid(torch.from_numpy(l))
    v, i = torch.topk(s, k, dim=1)
    ids, w = route(l, k, score=score, renorm=False)
    assert (ids == i.numpy()).all()
    assert np.allclose(w, v.numpy(), rtol=1e-14, atol=0)
    ids, w = route(l, k, score=score, factor=2.5)
    assert np.allclose(w, 2.5 * (v / v.sum(1, keepdim=True)).numpy(), rtol=1e-14, atol=0)


def test_bias_selects_but_does_not_weigh():
    l = [math.log(4.0), math.log(2.0), 0.0, 0.0]            # softmax 1/2, 1/4, 1/8, 1/8
    ids, w = route_row(l, 2, bias=[0.0, 0.0, 0.5, 0.0], renorm=False)
    assert ids == [2, 0] and w == pytest.approx([0.125, 0.5])
    ids, w = route_row(l, 2, bias=[0.0, 0.0, 0.5, 0.0])
    assert w == pytest.approx([0.2, 0.8])


def test_groups_by_their_best_one_or_two():
    s = [0.9, 0.1, 0.6, 0.5, 0.7, 0.2]
    l = [math.log(v / (1 - v)) for v in s]
    kw = dict(score="sigmoid", n_groups=3, renorm=False)
    assert route_row(l, 2, top_groups=1, group_best=1, **kw)[0] == [0, 1]     # 0.9 is the best one
    assert route_row(l, 2, top_groups=1, group_best=2, **kw)[0] == [2, 3]     # 0.6 + 0.5 is the best pair
    assert route_row(l, 2, top_groups=2, group_best=1, **kw)[0] == [0, 4]
    assert route_row(l, 4, top_groups=3, group_best=2, **kw)[0] == [0, 4, 2, 3]


def test_ties_go_to_the_lower_id_and_group():
    assert route_row([1.0] * 6, 3)[0] == [0, 1, 2]
    assert route_row([0.0, 1.0, 1.0, 0.0], 3)[0] == [1, 2, 0]
    assert route_row([1.0] * 6, 2, n_groups=3, top_groups=2, group_best=2)[0] == [0, 1]


def test_masked_and_poisoned_rows():
    inf, nan = math.inf, math.nan
    assert route_row([-inf, 2.0, -inf, 1.0], 3)[0] == [1, 3, -1]
    ids, w = route_row([-inf] * 4, 2)
    assert ids == [-1, -1] and w == [0.0, 0.0]
    assert route_row([0.0, 1.0], 1, bias=[0.0, -inf])[0] == [0]
    for bad in ([nan, 0.0], [inf, 0.0]):
        ids, w = route_row(bad, 1)
        assert ids == [-1] and math.isnan(w[0])
    assert math.isnan(route_row([0.0, 0.0], 1, bias=[nan, 0.0])[1][0])
    # a masked expert does not count in its group's value
    assert route_row([3.0, -inf, 1.0, 1.0], 1, score="sigmoid", n_groups=2, group_best=2)[0] == [2]


def test_softmax_shift_and_saturation():
    l = np.random.default_rng(3).normal(0, 1, (8, 16))
    a, b = route(l, 4), route(l + 100.0, 4)
    assert (a[0] == b[0]).all() and np.allclose(a[1], b[1], rtol=1e-12)
    ids, w = route_row([-1000.0, -2000.0], 2, score="sigmoid")
    assert ids == [0, 1] and w == [0.0, 0.0]                   # both scores 0: no weight, not NaN
    assert route_row([0.0, -2000.0], 2)[1] == [1.0, 0.0]
