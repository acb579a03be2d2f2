"""The routed experts on 8-bit codes at the ends of their ranges: weights that are
infinite or NaN where no expert is."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"


def _layer(E, d, F):
    g = torch.Generator(device=DEV).manual_seed(E * 7 + d)
    gu = torch.randint(-127, 128, (E, 2 * F, d), dtype=torch.int8, device=DEV, generator=g)
    dn = torch.randint(-127, 128, (E, d, F), dtype=torch.int8, device=DEV, generator=g)
    return gu, torch.full((E, 2 * F), 1e-3, device=DEV), dn, torch.full((E, d), 1e-3, device=DEV)


def _ffn(x, ids, w, layer, epi):
    from paper_2605_30859_amd import binding as B
    (R, d), (E, F2, _) = x.shape, layer[0].shape
    out = torch.full((R, d), 2.0, dtype=torch.bfloat16 if epi == 1 else torch.float32, device=DEV)
    ws = torch.full((B.darts_moe_ffn_i8_workspace_bytes(R, d, E, ids.shape[1], F2 // 2),), 0xff, dtype=torch.uint8, device=DEV)
    B.darts_moe_ffn_i8(x, ids, w, E, F2 // 2, *layer, out, epi, ws)
    return out


@pytest.mark.parametrize("R", [3, 300, 5000])
@pytest.mark.parametrize("epi", [1, 2])
def test_weights_of_places_without_an_expert(R, epi):
    """Infinite weights add nothing there; NaN makes the row NaN.  Everything else is
    the same bits as with weights of 0."""
    print(f"empty places, {R} rows, epilogue {epi}", flush=True)
    E, k, d, F = 16, 4, 256, 128
    g = torch.Generator(device=DEV).manual_seed(R)
    x = torch.empty(R, d, device=DEV).normal_(generator=g).bfloat16()
    ids = torch.randint(0, E, (R, k), dtype=torch.int32, device=DEV, generator=g)
    w = torch.rand(R, k, device=DEV, generator=g)
    ids[:, 1], ids[0], ids[1, 3] = -1, E, 1 << 30
    w[:, 1] = 0.0
    w[0] = 0.0
    w[1, 3] = 0.0
    layer = _layer(E, d, F)
    clean = _ffn(x, ids, w, layer, epi)
    w[:, 1] = float("inf")
    w[0] = -float("inf")
    w[1, 3] = float("inf")
    w[2, 1] = float("nan")
    got = _ffn(x, ids, w, layer, epi)
    assert bool(got[2].isnan().all())
    keep = torch.arange(R, device=DEV) != 2
    assert torch.equal(got[keep], clean[keep]) and bool(clean.isfinite().all())
