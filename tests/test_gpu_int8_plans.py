"""Every kernel of the 8-bit products and expert layers (int8_cases.py; that the sizes
reach all of them is tested on the host), and sizes past 32-bit offsets.

Tolerances.  Products: the roundings counted in test_gpu_int8.py.  Expert layers
against their parts: as there.  Expert layers against 64 bits: h is rounded to bf16,
and where its 64-bit value and the error of SwiGLU, (|g| + 12) 2^-23, leave two
possible bf16 numbers, their codes differ by a known number of steps; y has the
bound that follows, three float32 roundings and half a step of bf16; the sum k + 1
roundings of float32, the residual's one more, and a bf16 result half a step."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"

import int8_cases as S
from oracle import int8 as O
from test_gpu_int8 import (_gen, _i64, _layer, _operands, _rows, _swiglu64, by_parts, check_ffn, check_product, ffn,
                           quantize, same_codes)


def _b():
    from paper_2605_30859_amd import binding
    binding.load_library()
    return binding


@pytest.mark.parametrize("epi", [0, 1, 2, 3])
@pytest.mark.parametrize("M,N,K", S.PRODUCTS)
def test_products(M, N, K, epi):
    print(f"product {M} {N} {K} epi={epi} plan {_b().darts_debug_gemm_i8_plan(M, N, K, epi)}", flush=True)
    check_product(*_operands(M, N, K), epi)


def _ids(R, E, k, extra, seed=0):
    """Uniform ids, and `extra` pairs beside them of expert 1."""
    g = _gen(R, E, k, extra, seed)
    ids = torch.randint(0, E, (R, k), dtype=torch.int32, device=DEV, generator=g)
    ids[:, 0][torch.randperm(R, device=DEV, generator=g)[:extra]] = min(1, E - 1)
    return ids


@pytest.mark.parametrize("epi", [1, 2])
@pytest.mark.parametrize("R,E,k,d,F,extra", S.EXPERTS)
def test_experts_against_their_parts(R, E, k, d, F, extra, epi):
    print(f"experts {R} {E} {k} {d} {F} epi={epi} plan {_b().darts_debug_moe_ffn_i8_plan(R, d, E, k, F)}", flush=True)
    check_ffn(R, E, k, d, F, ids=_ids(R, E, k, extra), epi=epi)


def _codes64(x):
    """Codes and scales of float32 rows by the oracle, as 64-bit numbers."""
    q, s = O.quantize_rows(x.float().cpu().numpy())
    return torch.from_numpy(q).to(DEV).double(), torch.from_numpy(s).to(DEV).double()[:, None]


@pytest.mark.parametrize("epi", [1, 2])
@pytest.mark.parametrize("R,E,k,d,F", [(1, 128, 8, 2048, 768), (61, 128, 8, 2048, 768), (976, 128, 8, 2048, 768),
                                       (2000, 128, 8, 2048, 768), (300, 64, 6, 1024, 1408), (500, 60, 4, 1456, 720)])
def test_full_width_experts_against_64_bits(R, E, k, d, F, epi):
    print(f"experts {R} {E} {k} {d} {F} epi={epi}", flush=True)
    x, layer, ids = _rows(R, d), _layer(E, d, F), _ids(R, E, k, R // 10)
    w = torch.rand(R, k, device=DEV, generator=_gen(R, k))
    got = ffn(x, ids, w, layer, epi).double()
    gu, s_gu, dn, s_dn = layer
    ref = torch.zeros(R, d, dtype=torch.float64, device=DEV)
    off, mag = torch.zeros_like(ref), torch.zeros_like(ref)
    fits = torch.ones(R, dtype=torch.bool, device=DEV)
    xq, xs = _codes64(x)
    for e in range(E):
        row, slot = torch.nonzero(ids == e, as_tuple=True)
        if not row.numel():
            continue
        g, _, h = _swiglu64(xq[row] @ gu[e].double().t() * (xs[row] * s_gu[e].double()))
        err = (g.abs() + 12) * 2.0 ** -23 * h
        a, b = (h - err).float().bfloat16(), (h + err).float().bfloat16()      # the smaller and the larger in magnitude
        # the scale is sure where the row's largest element is: other rows are left out
        sure = a.abs().float().amax(1) == b.abs().float().amax(1)
        fits[row] &= sure
        (qa, s), (qb, _) = _codes64(a), _codes64(b)
        scale = s * s_dn[e].double()
        y = qa @ dn[e].double().t() * scale
        dy = (qa - qb).abs() @ dn[e].double().abs().t() * scale + 3 * 2.0 ** -24 * y.abs()
        dy += 2.0 ** -8 * (y.abs() + dy)
        wt = w[row, slot].double()[:, None]
        ref.index_add_(0, row, wt * y)
        off.index_add_(0, row, wt * dy)
        mag.index_add_(0, row, wt * (y.abs() + dy))
    tol = off + (k + 1) * 2.0 ** -24 * mag
    if epi == 1:
        tol += 2.0 ** -8 * (ref.abs() + tol)
    else:
        ref += 2.0
        tol += 2.0 ** -24 * (ref.abs() + tol)
    assert int(fits.sum()) >= 0.8 * R
    bad = ((got - ref).abs() > tol) & fits[:, None]
    assert not bool(bad.any()), (torch.nonzero(bad)[:4].tolist(), float(((got - ref).abs() - tol)[fits].max()))


# ------------------------------------------------------- rows to codes, by rows
@pytest.mark.parametrize("rows,cols", [(2050, 768), (4099, 72), (2049, 2048), (2100, 1000), (2050, 7)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_codes_of_many_rows(rows, cols, dtype):
    """A wavefront per row, on aligned rows, on strided ones and at any address."""
    print(f"codes {rows} {cols} {dtype}", flush=True)
    x = torch.empty(rows, cols, device=DEV).normal_(0, 2, generator=_gen(rows, cols)).to(dtype)
    x[1, cols - 1], x[2, 0], x[3] = float("nan"), float("inf"), 0.0
    same_codes(x)
    for before, after in ((3, 2), (8, 8)):
        wide = torch.full((rows, before + cols + after), float("nan"), dtype=dtype, device=DEV)
        wide[:, before:before + cols] = x
        same_codes(wide[:, before:before + cols])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [16, 15])
def test_codes_of_more_rows_than_one_launch_has(cols, dtype):
    """2^21 + 5 rows, copies of 64: all as the first."""
    x = torch.empty(64, cols, device=DEV).normal_(generator=_gen(cols)).to(dtype)
    q, s = quantize(x.repeat((1 << 15) + 1, 1)[:(1 << 21) + 5].contiguous())
    same_codes(x)
    eq, es = quantize(x)
    n = len(q)
    assert torch.equal(q, eq.repeat(n // 64 + 1, 1)[:n]) and torch.equal(s, es.repeat(n // 64 + 1)[:n])


# ------------------------------------------------------ past 32-bit offsets
@pytest.mark.parametrize("M,N,K", [(17000, 32, 131072), (17000, 272, 131072), (64, 16992, 131072), (300, 17024, 131072),
                                   (1100000, 512, 2048), (1100000, 80, 2048), (1000, 1100000, 2048), (20, 1100000, 2048)])
def test_operands_beyond_32_bit_offsets(M, N, K):
    """More than 2^31 bytes of codes in rows of either operand."""
    print(f"product {M} {N} {K} plan {_b().darts_debug_gemm_i8_plan(M, N, K, 0)}", flush=True)
    B = _b()
    a, sa, w, sw = _operands(M, N, K)
    assert max(a.numel(), w.numel()) > 1 << 31
    out = torch.full((M, N), 3.0, device=DEV)
    ws = torch.empty(B.darts_gemm_i8_workspace_bytes(M, N, K), dtype=torch.uint8, device=DEV)
    B.darts_gemm_i8(a, sa, w, sw, out, M, N, K, 0, ws)
    rows = torch.unique(torch.tensor([0, M // 2, M - 256, M - 129, M - 1], device=DEV).clamp_min(0))
    cols = torch.unique(torch.cat([torch.arange(max(N - 300, 0), N, device=DEV), torch.arange(0, N, max(N // 500, 1), device=DEV)]))
    ref = _i64(a[rows], w[cols]) * sa[rows].double()[:, None] * sw[cols].double()
    assert bool(((out[rows][:, cols].double() - ref).abs() <= 3.01 * 2.0 ** -24 * ref.abs()).all())


def test_gathered_rows_beyond_32_bit_offsets():
    """270000 rows of d_model 8192: codes of 2.2 GB, from which the routed rows are
    gathered.  The rows past 2^31 bytes are as in a call of their own."""
    R, E, d, F = 270000, 3, 8192, 32
    x = torch.empty(R, d, dtype=torch.bfloat16, device=DEV)
    for at in range(0, R, 30000):
        x[at:at + 30000] = torch.empty(min(30000, R - at), d, device=DEV).normal_(generator=_gen(at, d))
    ids, w, layer = _ids(R, E, 1, 0), torch.rand(R, 1, device=DEV, generator=_gen(R)), _layer(E, d, F)
    B = _b()

    def run(at, end):
        n = end - at
        out = torch.full((n, d), 2.0, dtype=torch.bfloat16, device=DEV)
        ws = torch.empty(B.darts_moe_ffn_i8_workspace_bytes(n, d, E, 1, F), dtype=torch.uint8, device=DEV)
        B.darts_moe_ffn_i8(x[at:end], ids[at:end], w[at:end], E, F, *layer, out, 1, ws)
        return out

    out = run(0, R)
    first = (1 << 31) // d
    assert torch.equal(out[first - 1000:], run(first - 1000, R)) and torch.equal(out[:1000], run(0, 1000))
    ref, mag = by_parts(x[-2000:], ids[-2000:], w[-2000:], layer)
    assert bool(((out[-2000:].double() - ref).abs() <= 2 * 2.0 ** -24 * mag + 2.0 ** -8 * ref.abs() + 1e-37).all())


def test_router_beyond_32_bit_offsets():
    """2^21 + 3 rows of 1024 experts, copies of 64: all as the first."""
    B, E, k = _b(), 1024, 8
    n = (1 << 21) + 3
    few = torch.empty(64, E, device=DEV).normal_(generator=_gen(E)).bfloat16()
    rows = few.repeat(n // 64 + 1, 1)[:n].contiguous()
    assert rows.numel() > 1 << 31
    ids, w = torch.empty(n, k, dtype=torch.int32, device=DEV), torch.empty(n, k, device=DEV)
    B.darts_moe_route(rows, B.DARTS_BF16, ids, w)
    eid, ew = torch.empty(64, k, dtype=torch.int32, device=DEV), torch.empty(64, k, device=DEV)
    B.darts_moe_route(few, B.DARTS_BF16, eid, ew)
    assert torch.equal(ids, eid.repeat(n // 64 + 1, 1)[:n]) and torch.equal(w, ew.repeat(n // 64 + 1, 1)[:n])
    from oracle.routing import route
    oid, ow = route(few.float().cpu().numpy(), k)
    assert (eid.cpu().numpy() == oid).all() and np.allclose(ew.cpu().numpy(), ow, rtol=2.0 ** -23, atol=0)
