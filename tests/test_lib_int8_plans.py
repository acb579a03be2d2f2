"""The sizes of int8_cases.py reach every kernel that the 8-bit calls can run, as the
library's plans say (no GPU needed)."""
import ctypes as C
import math
import random

import pytest

import int8_cases as S
from paper_2605_30859_amd import binding as B

FEW, RING, ALTERNATING = 0, 1, 2


@pytest.fixture(scope="module", autouse=True)
def _lib():
    B.load_library()


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def _product_kernel(M, N, K):
    """What names the kernel: tiles, splits or not, padded rows and where their K ends."""
    kernel, rows, cols, splits, padded = B.darts_debug_gemm_i8_plan(M, N, K, 0)
    assert splits == 1 or not padded
    return kernel, rows, cols, splits if kernel == FEW else splits > 1, (1 if K % 128 else 2) if padded else 0


def test_products_reach_every_kernel():
    rng = random.Random(5)
    possible = set()
    for _ in range(120000):
        K = _log(rng, 1, 1024) * 16
        K = max(256, K // 256 * 256) if rng.random() < 0.5 else max(128, K // 256 * 256 + 128) if rng.random() < 0.3 else K
        possible.add(_product_kernel(_log(rng, 1, 40000), _log(rng, 1, 2000) * 16, K))
    run = {_product_kernel(*c) for c in S.PRODUCTS}
    assert possible <= run, sorted(possible - run)
    assert {k[1:3] for k in run if k[0] == ALTERNATING} == {(128, 128), (128, 256), (256, 128), (256, 192), (256, 256)}


@pytest.mark.parametrize("cases", ["WHOLE", "PADDED", "PADDED_HALF"])
def test_products_with_more_tiles_than_blocks_and_with_fewer(cases):
    """Both with tiles that rows and channels do not fill."""
    seen = {}
    for M, N, K in getattr(S, cases):
        kernel, rows, cols, _, padded = B.darts_debug_gemm_i8_plan(M, N, K, 0)
        if kernel != ALTERNATING:
            continue
        assert M % rows and N % cols and padded == (cases != "WHOLE")
        blocks = 512 if (rows, cols) == (128, 128) else 256
        seen.setdefault((rows, cols), set()).add(-(-M // rows) * -(-N // cols) > blocks)
    assert len(seen) == 5 and all(True in v for v in seen.values())
    assert sum(False in v for v in seen.values()) >= 4


def test_expert_layers_reach_every_kernel():
    rng = random.Random(6)
    possible = set()
    for _ in range(60000):
        E, k = rng.choice([1, 2, 3, 8, 16, 60, 64, 128, 160, 256, 1024]), min(64, _log(rng, 1, 64))
        d, F = (_log(rng, 1, 512) * 16 for _ in range(2))
        d, F = (max(256, n // 256 * 256) if rng.random() < 0.5 else n for n in (d, F))
        lists, rows, gu, dn, short_gu, short_dn = B.darts_debug_moe_ffn_i8_plan(_log(rng, 1, 30000), d, E, k, F)
        possible |= {("lists", lists, rows)} | ({("gate/up", rows, gu, short_gu), ("down", rows, dn, short_dn)} if lists else set())
    run = set()
    for R, E, k, d, F, _ in S.EXPERTS:
        lists, rows, gu, dn, short_gu, short_dn = B.darts_debug_moe_ffn_i8_plan(R, d, E, k, F)
        run |= {("lists", lists, rows)} | ({("gate/up", rows, gu, short_gu), ("down", rows, dn, short_dn)} if lists else set())
    assert possible <= run, sorted(possible - run)


def test_plans_refuse_what_the_calls_refuse():
    lib, out = B.load_library(), (C.c_int32 * 6)()
    for M, N, K, epi in ((0, 64, 64, 0), (4, 40, 64, 0), (4, 64, 72, 0), (4, 64, 131088, 0), (4, 48, 64, 3), (4, 64, 64, 4),
                         (1 << 30, 1 << 16, 64, 0)):
        assert lib.darts_debug_gemm_i8_plan(M, N, K, epi, out) == B.DARTS_EINVAL
    for R, d, E, k, F in ((0, 64, 8, 2, 32), (4, 72, 8, 2, 32), (4, 64, 1025, 2, 32), (4, 64, 8, 65, 32), (4, 64, 8, 2, 8),
                          (1 << 19, 8192, 8, 1, 32)):
        assert lib.darts_debug_moe_ffn_i8_plan(R, d, E, k, F, out) == B.DARTS_EINVAL
    assert lib.darts_debug_gemm_i8_plan(4, 64, 64, 0, None) == B.DARTS_EINVAL
    assert lib.darts_debug_moe_ffn_i8_plan(4, 64, 8, 2, 32, None) == B.DARTS_EINVAL


@pytest.mark.parametrize("N,K,wavefronts", [(2048, 4096, 8), (4096, 4096, 8), (4096, 512, 8), (4112, 4096, 4), (5120, 2048, 4),
                                            (5120, 8192, 4), (6144, 4096, 4), (8192, 4096, 4), (8208, 4096, 8),
                                            (12288, 4096, 8), (24576, 4096, 8), (12288, 512, 4), (24576, 512, 4)])
def test_wavefronts_of_a_strip_go_by_rounds_of_blocks(N, K, wavefronts):
    """Four where two strips a block make one round over the CUs of two, or K is short."""
    assert B.darts_debug_gemm_i8_plan(1, N, K, 0)[3] == wavefronts
