"""Pins for the roundings of the oracle's 8-bit experts."""
import numpy as np

from oracle.int8 import expert, moe_ffn, product, quantize_rows, round_bf16, swiglu


def _layer():
    rng = np.random.default_rng(7)
    E, d, F, R = 3, 48, 32, 9
    x = round_bf16(rng.normal(0, 1, (R, d)))
    w_gu, w_dn = (rng.integers(-127, 128, s).astype(np.int8) for s in ((E, 2 * F, d), (E, d, F)))
    s_gu, s_dn = (rng.random((E, n)).astype(np.float32) * 1e-3 for n in (2 * F, d))
    return x, w_gu, s_gu, w_dn, s_dn


def test_an_experts_result_is_rounded_to_bf16_before_the_sum():
    x, w_gu, s_gu, w_dn, s_dn = _layer()
    h = round_bf16(swiglu(product(*quantize_rows(x), w_gu[1], s_gu[1])))
    y = product(*quantize_rows(h), w_dn[1], s_dn[1])
    got = expert(x, w_gu[1], s_gu[1], w_dn[1], s_dn[1])
    assert (got == round_bf16(got)).all() and (got == round_bf16(y)).all() and (got != y).any()
    assert (np.abs(got - y) <= 2.0 ** -8 * np.abs(y)).all()          # half a step


def test_the_sum_and_its_weights_are_not_rounded():
    x, *layer = _layer()
    ids = np.array([[0, 1, 2]] * len(x), dtype=np.int32)
    w = np.random.default_rng(8).random(ids.shape).astype(np.float32)
    y = [expert(x, *(t[e] for t in layer)) for e in range(3)]
    ref = sum(w[:, e, None].astype(np.float64) * y[e] for e in range(3))
    assert np.allclose(moe_ffn(x, ids, w, *layer), ref, rtol=1e-13, atol=1e-15)
