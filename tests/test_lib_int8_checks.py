"""Host-side argument checks of the router and of the 8-bit entries (no GPU
needed: every call here returns before any device work)."""
import ctypes as C

import pytest

from paper_2605_30859_amd import binding as B

OK, EINVAL = B.DARTS_OK, B.DARTS_EINVAL
N = None
D = C.c_void_p(4096)          # never dereferenced: the call fails its argument check first
ODD = C.c_void_p(4100)


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def test_zero_rows_are_noops(lib):
    assert lib.darts_moe_route(N, 128, 0, 128, B.DARTS_F32, 0, N, 1, 1, 1, 8, 1, 1.0, N, N, N) == OK
    assert lib.darts_quantize_rows(N, 64, 0, 64, B.DARTS_BF16, N, N, N) == OK
    assert lib.darts_gemm_i8(N, N, N, N, N, 0, 64, 64, 0, N, 0, N) == OK
    assert lib.darts_moe_ffn_i8(N, N, N, 0, 64, 8, 2, 32, N, N, N, N, N, 1, N, 0, N) == OK
    assert lib.darts_moe_ffn_i8_workspace_bytes(0, 64, 8, 2, 32) == 0


def test_router_refusals(lib):
    def call(ld=128, rows=4, E=128, dtype=B.DARTS_F32, score=0, groups=1, top=1, best=1, k=8, factor=1.0, l=D, ids=D, w=D):
        return lib.darts_moe_route(l, ld, rows, E, dtype, score, N, groups, top, best, k, 1, factor, ids, w, N)
    for kw in (dict(ld=127), dict(rows=-1), dict(E=0, ld=8), dict(E=1025, ld=2048), dict(dtype=2), dict(score=2),
               dict(score=-1), dict(groups=0), dict(groups=3), dict(groups=128), dict(groups=4, top=5),
               dict(groups=4, top=0), dict(best=0), dict(best=3), dict(k=0), dict(k=65), dict(E=4, k=5),
               dict(factor=float("nan")), dict(factor=float("inf")), dict(l=N), dict(ids=N), dict(w=N)):
        assert call(**kw) == EINVAL, kw


def test_quantizer_refusals(lib):
    def call(ldx=64, rows=4, cols=64, dtype=B.DARTS_BF16, x=D, q=D, s=D):
        return lib.darts_quantize_rows(x, ldx, rows, cols, dtype, q, s, N)
    for kw in (dict(rows=-1), dict(cols=0), dict(ldx=63), dict(dtype=3), dict(x=N), dict(q=N), dict(s=N)):
        assert call(**kw) == EINVAL, kw


def test_product_refusals(lib):
    def call(M=4, n=64, K=64, epi=0, a=D, sa=D, w=D, sw=D, c=D):
        return lib.darts_gemm_i8(a, sa, w, sw, c, M, n, K, epi, N, 0, N)
    for kw in (dict(M=-1), dict(n=0), dict(n=40), dict(K=0), dict(K=72), dict(K=131072 + 16), dict(epi=4), dict(epi=-1),
               dict(n=48, epi=3), dict(M=1 << 30, n=1 << 16), dict(a=N), dict(sa=N), dict(w=N), dict(sw=N), dict(c=N), dict(a=ODD), dict(w=ODD)):
        assert call(**kw) == EINVAL, kw
    # a plan that needs a workspace, without one and with one too small
    for M, n, K in ((1, 4096, 12288), (45, 4096, 12288), (200, 2048, 4096), (16, 1024, 4096)):
        need = lib.darts_gemm_i8_workspace_bytes(M, n, K)
        if need:
            assert lib.darts_gemm_i8(D, D, D, D, D, M, n, K, 0, N, need, N) == EINVAL
            assert lib.darts_gemm_i8(D, D, D, D, D, M, n, K, 0, D, need - 1, N) == EINVAL
            assert lib.darts_gemm_i8(D, D, D, D, D, M, n, K, 0, ODD, need, N) == EINVAL
    assert lib.darts_gemm_i8_workspace_bytes(0, 64, 64) == 0


def test_expert_refusals(lib):
    need = lib.darts_moe_ffn_i8_workspace_bytes(4, 64, 8, 2, 32)
    assert need > 0

    def call(x=D, ids=D, w=D, rows=4, d=64, E=8, k=2, F=32, gu=D, sgu=D, dn=D, sdn=D, out=D, epi=1, ws=D, nb=need):
        return lib.darts_moe_ffn_i8(x, ids, w, rows, d, E, k, F, gu, sgu, dn, sdn, out, epi, ws, nb, N)
    for kw in (dict(rows=-1), dict(d=0), dict(d=72), dict(d=131088), dict(F=8), dict(F=40), dict(E=0), dict(E=1025),
               dict(k=0), dict(k=65), dict(rows=4194240 // 2 + 1), dict(epi=0), dict(epi=3), dict(x=N), dict(ids=N),
               dict(w=N), dict(gu=N), dict(sgu=N), dict(dn=N), dict(sdn=N), dict(out=N), dict(ws=N), dict(nb=need - 1),
               dict(x=ODD), dict(gu=ODD), dict(dn=ODD), dict(out=ODD), dict(ws=C.c_void_p(4096 + 128))):
        assert call(**kw) == EINVAL, kw
    assert lib.darts_moe_ffn_i8_workspace_bytes(4, 72, 8, 2, 32) == 0


def test_binding_wants_adjacent_elements():
    torch = pytest.importorskip("torch")
    x = torch.zeros(8, 4).t()
    with pytest.raises(ValueError):
        B.darts_quantize_rows(x, B.DARTS_F32, None, None)
    with pytest.raises(ValueError):
        B.darts_moe_route(x, B.DARTS_F32, x, x)


def test_refusals_of_sizes_past_the_kernels_offsets(lib):
    # a row of codes longer than 2^30; results that are not 16-byte aligned; gathered
    # rows beyond 32-bit offsets
    assert lib.darts_quantize_rows(D, 1 << 31, 1, (1 << 30) + 1, B.DARTS_F32, D, D, N) == EINVAL
    assert lib.darts_gemm_i8(D, D, D, D, ODD, 4, 64, 64, 0, D, 1 << 40, N) == EINVAL
    for rows, d in ((1 << 19, 8192), ((1 << 24) // 16, 4096), (32768, 131072), (4194240, 1040)):
        assert lib.darts_moe_ffn_i8_workspace_bytes(rows, d, 8, 1, 32) == 0, (rows, d)
        assert lib.darts_moe_ffn_i8(D, D, D, rows, d, 8, 1, 32, D, D, D, D, D, 1, D, 1 << 50, N) == EINVAL, (rows, d)
    assert lib.darts_moe_ffn_i8_workspace_bytes((1 << 19) - 1, 8192, 8, 1, 32) > 0
