"""The router (darts_moe_route) where finite biases are as large as float32 holds, and at
sizes that reach each of its kernels: ids equal to the float64 oracle's, weights within
one float32 rounding."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"

from oracle.routing import route

INF, LOWEST = float("inf"), torch.finfo(torch.float32).min


def _check(logits, k, score, bias, **kw):
    """Weights: half a step of float32 (2^-24), and the last digits of 64-bit arithmetic."""
    from paper_2605_30859_amd import binding as B
    ids = torch.full((logits.shape[0], k), 77, dtype=torch.int32, device=DEV)
    w = torch.full((logits.shape[0], k), 77.0, device=DEV)
    B.darts_moe_route(logits, B.DARTS_F32, ids, w, score=B.SCORE_SIGMOID if score == "sigmoid" else B.SCORE_SOFTMAX,
                      bias=bias, **kw)
    ids, w = ids.cpu().numpy(), w.cpu().numpy()
    eid, ew = route(logits.cpu().numpy(), k, score=score, bias=None if bias is None else bias.cpu().numpy(), **kw)
    assert (ids == eid).all(), np.argwhere(ids != eid)[:5]
    assert (np.abs(w - ew) <= np.abs(ew) * (2.0 ** -24 * (1 + 1e-6)) + 2.0 ** -149).all()


def _logits(rows, E):
    g = torch.Generator(device=DEV).manual_seed(rows * 1000 + E)
    return torch.empty(rows, E, device=DEV).normal_(0.0, 1.5, generator=g)


# the bias of each of 8 groups: of all its experts, or of its two first and of the others
GROUP_BIASES = {
    "a soft mask beside a hard one": [-INF] + [LOWEST] * 6 + [0.0],
    "soft masks alone": [LOWEST] * 5 + [0.0, LOWEST, 0.0],
    "large sums": [0.0, 2e38, 0.0, 3e38, 0.0, 2.5e38, 0.0, 0.0],
    "large negative sums": [-INF, -3e38, -3.2e38, -2e38, -2.5e38, -INF, LOWEST, -2.2e38],
    "one expert of a pair": [(0.0, LOWEST), (0.25, LOWEST), -INF, (3e38, LOWEST), (LOWEST, LOWEST), (0.5, -INF),
                             (2e38, -2e38), (LOWEST, -INF)],
    "sums of opposite signs": [(3e38, -3e38), (-1.0, -1.0), (2e38, -2e38), (0.5, -1.0), (-3e38, 3e38), (0.0, 0.0),
                               (-0.25, -0.5), (3e38, -3.2e38)],
}


@pytest.mark.parametrize("name", sorted(GROUP_BIASES))
@pytest.mark.parametrize("E,k", [(64, 10), (128, 12), (256, 20), (512, 30)])
@pytest.mark.parametrize("best", [1, 2])
def test_groups_of_biases_near_the_ends_of_float32(name, E, k, best):
    print(f"groups {name}, {E} experts, the best {best}", flush=True)
    per = E // 8
    bias = torch.empty(E, device=DEV)
    for g, b in enumerate(GROUP_BIASES[name]):
        pair = b if isinstance(b, tuple) else (b, b)
        bias[g * per:(g + 1) * per] = pair[1] if isinstance(b, tuple) and pair[1] < pair[0] else LOWEST if isinstance(b, tuple) else b
        bias[g * per] = pair[0]
        bias[g * per + 1] = pair[1]
    for score in ("softmax", "sigmoid"):
        for top in (1, 2, 3, 5):
            _check(_logits(37, E), k, score, bias, n_groups=8, top_groups=top, group_best=best)


# experts, experts of a row, groups: 16, 32 and 64 lanes a row with 4, 8 and 16 experts
# each, in the order of logits or scores and by groups; groups of other sizes and 64
# experts a row, which go by the definition alone
SIZES = [(60, 5, 1), (64, 15, 8), (37, 9, 1), (128, 15, 8), (100, 7, 1), (120, 15, 1), (64, 20, 4), (256, 31, 8), (200, 9, 1),
         (129, 16, 3), (512, 40, 8), (300, 33, 1), (128, 63, 16), (1024, 63, 8), (1000, 10, 1), (1024, 63, 64), (777, 31, 7),
         (48, 6, 4), (96, 8, 4), (160, 6, 8), (320, 12, 10), (600, 8, 6), (64, 64, 1), (200, 64, 1), (512, 64, 8), (1000, 64, 5)]


@pytest.mark.parametrize("E,k,groups", SIZES)
@pytest.mark.parametrize("first", [0, 1])
def test_every_kernel(E, k, groups, first):
    """Rows that begin at addresses for wide loads, and rows that do not."""
    print(f"route {E} {k} {groups} from element {first}", flush=True)
    rows = 43
    g = torch.Generator(device=DEV).manual_seed(E + k)
    ld = E + (-E) % 8 + first
    flat = torch.empty(rows * ld + 8, device=DEV).normal_(0.0, 1.5, generator=g)
    bias = torch.empty(E, device=DEV).normal_(0.0, 0.1, generator=g)
    l = torch.as_strided(flat, (rows, E), (ld, 1), first)
    l[3], l[4, : E // 2], l[5, 1:] = -INF, -INF, -INF
    for score in ("softmax", "sigmoid"):
        for b in (bias, torch.zeros_like(bias)):
            for best in (1, 2) if groups > 1 else (1,):
                kw = dict(n_groups=groups, top_groups=(groups + 1) // 2, group_best=best)
                _check(l, k, score, b, **kw)
        _check(l, k, score, None)
