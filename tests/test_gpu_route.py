"""The router (darts_moe_route) against the float64 oracle: ids equal, weights
within one float32 rounding.  Sizes of one expert to 1024, groups, biases, masks,
rows that are masked out or hold NaN, strided rows, ties; other streams and graph
replays."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"

from oracle.routing import route


def _b():
    from paper_2605_30859_amd import binding
    binding.load_library()
    return binding


def _call(logits, k, score="softmax", bias=None, n_groups=1, top_groups=1, group_best=1, renorm=True, factor=1.0,
          stream=None):
    B = _b()
    ids = torch.full((logits.shape[0] + 1, k), 77, dtype=torch.int32, device=DEV)
    w = torch.full((logits.shape[0] + 1, k), 77.0, device=DEV)
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())       # for what was just filled
    B.darts_moe_route(logits, B.DARTS_BF16 if logits.dtype == torch.bfloat16 else B.DARTS_F32, ids[:-1], w[:-1],
                      score=B.SCORE_SIGMOID if score == "sigmoid" else B.SCORE_SOFTMAX, bias=bias, n_groups=n_groups,
                      top_groups=top_groups, group_best=group_best, renorm=renorm, factor=factor, stream=stream)
    torch.cuda.synchronize()
    assert bool((ids[-1] == 77).all()) and bool((w[-1] == 77.0).all())       # the row behind the last one
    return ids[:-1].cpu().numpy(), w[:-1].cpu().numpy()


def _check(logits, k, **kw):
    """Weights: one rounding to float32, half a step (2^-24), and the last digits of 64-bit arithmetic."""
    ids, w = _call(logits, k, **kw)
    b = kw.pop("bias", None)
    eid, ew = route(logits.float().cpu().numpy(), k, bias=None if b is None else b.cpu().numpy(), **kw)
    assert (ids == eid).all(), np.argwhere(ids != eid)[:5]
    assert (np.isnan(w) == np.isnan(ew)).all()
    assert (np.nan_to_num(np.abs(w - ew)) <= np.nan_to_num(np.abs(ew)) * (2.0 ** -24 * (1 + 1e-6)) + 2.0 ** -149).all()


def _logits(rows, E, dtype=torch.float32, std=1.5):
    g = torch.Generator(device=DEV).manual_seed(rows * 1000 + E)
    return torch.empty(rows, E, device=DEV).normal_(0.0, std, generator=g).to(dtype)


@pytest.mark.parametrize("rows,E,k", [(1, 1, 1), (3, 2, 2), (1, 128, 8), (5, 60, 4), (67, 63, 7), (64, 64, 6), (9, 65, 8),
                                      (33, 160, 6), (130, 256, 8), (17, 257, 10), (6, 1000, 64), (5, 1024, 64)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_sizes(rows, E, k, score):
    print(f"route {rows} {E} {k} {score}", flush=True)
    _check(_logits(rows, E), k, score=score)
    _check(_logits(rows, E, torch.bfloat16), k, score=score, renorm=False, factor=2.5)


@pytest.mark.parametrize("E,k,groups,top,best", [(256, 8, 8, 4, 2), (160, 6, 8, 3, 1), (64, 4, 64, 5, 2), (96, 8, 4, 1, 2),
                                                 (1024, 16, 64, 7, 2), (12, 6, 6, 3, 2), (128, 8, 2, 2, 1), (6, 3, 3, 1, 2)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_groups_and_bias(E, k, groups, top, best, dtype):
    g = torch.Generator(device=DEV).manual_seed(E)
    bias = torch.empty(E, device=DEV).normal_(0.0, 0.1, generator=g)
    for score in ("softmax", "sigmoid"):
        for b in (None, bias):
            _check(_logits(41, E, dtype), k, score=score, bias=b, n_groups=groups, top_groups=top, group_best=best)


def test_masks_and_poisoned_rows():
    inf, nan = float("inf"), float("nan")
    l = _logits(12, 32)
    l[0] = -inf                       # a padding row
    l[1, 3:] = -inf                   # fewer experts than places
    l[2, 5] = nan
    l[3, 31] = inf
    l[4, ::2] = -inf
    l[5, 8:16] = -inf                 # a group with nothing left
    l[6] = torch.finfo(torch.float32).min      # a mask by the type's lowest value
    l[7, 0] = torch.finfo(torch.float32).max
    l[8, :] = -300.0
    l[9, :] = nan
    l[10, :31] = -inf
    bias = torch.linspace(-0.2, 0.2, 32, device=DEV)
    bias2 = bias.clone()
    bias2[4:12] = -inf                # experts taken out
    for score in ("softmax", "sigmoid"):
        for b in (None, bias, bias2):
            _check(l, 6, score=score, bias=b)
            _check(l, 6, score=score, bias=b, n_groups=4, top_groups=2, group_best=2)
            _check(l, 6, score=score, bias=b, n_groups=4, top_groups=2, group_best=1, renorm=False)
    bias2[0] = nan
    ids, w = _call(l, 6, bias=bias2)
    assert (ids == -1).all() and np.isnan(w).all()


def test_saturated_scores():
    l = torch.tensor([[-1000.0, -2000.0, -1500.0, -3e38], [800.0, 900.0, 40.0, -900.0]], device=DEV)
    for score in ("softmax", "sigmoid"):
        _check(l, 3, score=score)


def test_ties_go_to_the_lower_id():
    for E in (8, 128, 300):
        l = torch.zeros(3, E, device=DEV)
        l[1, E // 2:] = 1.0
        l[2, ::3] = 0.5
        for kw in (dict(), dict(n_groups=4, top_groups=2, group_best=2)):
            _check(l, 5, **kw)
            _check(l, 5, score="sigmoid", **kw)


@pytest.mark.parametrize("E,k", [(64, 8), (128, 8), (256, 8), (500, 20), (1024, 40)])
def test_nearly_equal_scores(E, k):
    """Neighbours a few last digits apart, in the logits and after the bias, beside
    equal ones: the 64-bit order decides."""
    g = torch.Generator(device=DEV).manual_seed(E)
    base = torch.randint(0, 6, (40, E), device=DEV, generator=g).float() * 0.25
    step = torch.randint(0, 3, (40, E), device=DEV, generator=g).float()
    l = base + step * torch.tensor([2.0 ** -23, 2.0 ** -20, 2.0 ** -17, 2.0 ** -15], device=DEV).repeat(10)[:, None]
    l[::2] -= 0.75
    bias = torch.randint(0, 4, (E,), device=DEV, generator=g).float() * 0.125
    for score in ("softmax", "sigmoid"):
        for b in (None, bias, bias + step[0] * 2.0 ** -22):
            _check(l, k, score=score, bias=b)
            _check(l, k, score=score, bias=b, n_groups=4, top_groups=2, group_best=2)
            _check(l.bfloat16(), k, score=score, bias=b)
        _check(l + 20.0, k, score=score)
        _check(l * 8.0 - 690.0, k, score=score)


@pytest.mark.parametrize("bias", [-1000.0, 3e4])
def test_large_bias(bias):
    l = _logits(30, 128)
    b = torch.full((128,), bias, device=DEV) + torch.arange(128, device=DEV) % 5
    for score in ("softmax", "sigmoid"):
        _check(l, 8, score=score, bias=b)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("large", [10.0, 1000.0])
def test_groups_of_large_biases_of_either_sign(score, large):
    """Groups whose two best add up to little: float32 keeps few digits of either."""
    bias = torch.full((32,), -3.0 * large, device=DEV)
    bias[0::4], bias[1::4] = large, -large
    # taken: the large ones of three groups
    _check(_logits(20000, 32), 3, score=score, bias=bias, n_groups=8, top_groups=3, group_best=2)


def test_strided_rows():
    wide = _logits(50, 384)
    wide[:, 60:] = float("nan")       # columns beside the logits are not read
    _check(wide[:, :60], 4)
    _check(wide.bfloat16()[:, :60], 4)
    _check(wide[:, 1:61].nan_to_num(0.5), 4)
    flat = _logits(1, 4000).flatten()                     # rows that begin at any address
    _check(torch.as_strided(flat, (30, 64), (67, 1), 1), 6)
    _check(torch.as_strided(flat.bfloat16(), (30, 64), (66, 1), 3), 6)


def test_many_rows():
    """32768 rows: ids against torch's topk of float64 scores (no ties among float32 draws of 128)."""
    l = _logits(32768, 128)
    ids, w = _call(l, 8)
    v, i = torch.topk(torch.softmax(l.double(), 1), 8, dim=1)
    assert (ids == i.int().cpu().numpy()).all()
    ew = (v / v.sum(1, keepdim=True)).cpu().numpy()
    assert (np.abs(w - ew) <= ew * (2.0 ** -24 * (1 + 1e-6))).all()


@pytest.mark.parametrize("E,k", [(4, 2), (4, 4)])
def test_more_rows_than_one_launch_has(E, k):
    """2^24 + 5 rows, copies of 64: all as the first."""
    l = _logits(64, E)
    l = l.repeat((1 << 18) + 1, 1)[:(1 << 24) + 5].contiguous()
    ids, w = _call(l, k)
    eid, ew = _call(l[:64].contiguous(), k)
    n = len(ids)
    assert (ids == np.tile(eid, (n // 64 + 1, 1))[:n]).all() and (w == np.tile(ew, (n // 64 + 1, 1))[:n]).all()


def test_other_stream_and_graph_replays():
    B = _b()
    l = _logits(300, 256)
    exp = _call(l, 8, score="sigmoid", n_groups=8, top_groups=4, group_best=2)
    st = torch.cuda.Stream()
    got = _call(l, 8, score="sigmoid", n_groups=8, top_groups=4, group_best=2, stream=st)
    assert (got[0] == exp[0]).all() and (got[1] == exp[1]).all()
    ids = torch.zeros(300, 8, dtype=torch.int32, device=DEV)
    w = torch.zeros(300, 8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.darts_moe_route(l, B.DARTS_F32, ids, w, score=B.SCORE_SIGMOID, n_groups=8, top_groups=4, group_best=2)
    for i in range(3):
        ids.zero_()
        l.copy_(_logits(300, 256) + i * torch.arange(256, device=DEV) * 0.01)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        exp = _call(l, 8, score="sigmoid", n_groups=8, top_groups=4, group_best=2)
        assert (ids.cpu().numpy() == exp[0]).all() and (w.cpu().numpy() == exp[1]).all()
