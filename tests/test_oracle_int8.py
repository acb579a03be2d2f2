"""Pins for the oracle's 8-bit codes, products and expert layer."""
import numpy as np
import pytest

from oracle.int8 import expert, moe_ffn, product, quantize_rows, round_bf16, silu, swiglu


def test_codes_by_hand():
    q, s = quantize_rows([[127.0, -127.0, 0.5, 1.5, 2.5, -0.5, 0.49, 63.0]])
    assert q.tolist() == [[127, -127, 0, 2, 2, 0, 0, 63]] and s.tolist() == [1.0]     # halves to even
    q, s = quantize_rows([[0.0, 0.0], [2.0 ** -120, 0.0], [np.inf, 1.0], [np.nan, 1.0], [2.0 ** -119, 0.0]])
    assert q[:4].any() == 0 and s[0] == 0 and s[1] == 0 and np.isnan(s[2]) and np.isnan(s[3])
    assert q[4].tolist() == [127, 0] and s[4] == np.float32(2.0 ** -119) / np.float32(127)


def test_a_code_is_within_half_a_step():
    x = np.random.default_rng(0).normal(0, 3, (50, 333)).astype(np.float32)
    q, s = quantize_rows(x)
    assert np.abs(q).max() == 127
    err = np.abs(q.astype(np.float64) * s.astype(np.float64)[:, None] - x)
    # half a step, and the roundings of 127 / a, of the product and of the scale
    assert (err <= s.astype(np.float64)[:, None] * (0.5 + 127 * 3 * 2.0 ** -24)).all()


def test_codes_do_not_depend_on_a_power_of_two():
    x = np.random.default_rng(1).normal(0, 1, (4, 64)).astype(np.float32)
    q, s = quantize_rows(x)
    for p in (2.0 ** -60, 2.0 ** 80):
        q2, s2 = quantize_rows(x * np.float32(p))
        assert (q2 == q).all() and (s2 == s * np.float32(p)).all()


def test_product_in_python_integers():
    rng = np.random.default_rng(2)
    a, w = rng.integers(-127, 128, (3, 48)).astype(np.int8), rng.integers(-127, 128, (5, 48)).astype(np.int8)
    sa, sw = rng.random(3).astype(np.float32), rng.random(5).astype(np.float32)
    c = product(a, sa, w, sw)
    for m in range(3):
        for n in range(5):
            acc = sum(int(x) * int(y) for x, y in zip(a[m], w[n]))
            assert c[m, n] == pytest.approx(acc * float(sa[m]) * float(sw[n]), rel=1e-15)
    big = np.full((1, 131072), 127, dtype=np.int8)
    assert product(big, np.ones(1, np.float32), -big, np.ones(1, np.float32))[0, 0] == -127 * 127 * 131072


def test_swiglu_columns():
    c = np.arange(64, dtype=np.float64)[None, :] / 10
    h = swiglu(c)
    for f in range(32):
        g, u = c[0, f // 16 * 32 + f % 16], c[0, f // 16 * 32 + 16 + f % 16]
        assert h[0, f] == pytest.approx(silu(g) * u)
    assert silu(np.float64(-1e6)) == 0


def test_experts_against_one_dense_layer_each():
    rng = np.random.default_rng(4)
    E, d, F, R = 3, 32, 16, 7
    x = round_bf16(rng.normal(0, 1, (R, d)))
    w_gu = rng.integers(-127, 128, (E, 2 * F, d)).astype(np.int8)
    w_dn = rng.integers(-127, 128, (E, d, F)).astype(np.int8)
    s_gu, s_dn = (rng.random((E, n)).astype(np.float32) * 1e-3 for n in (2 * F, d))
    ids = np.array([[0, 1], [2, 2], [1, -1], [-1, -1], [5, 0], [0, 2], [1, 0]], dtype=np.int32)
    w = rng.random(ids.shape).astype(np.float32)
    dense = [expert(x, w_gu[e], s_gu[e], w_dn[e], s_dn[e]) for e in range(E)]
    out = moe_ffn(x, ids, w, w_gu, s_gu, w_dn, s_dn)
    for r in range(R):
        exp = sum((float(w[r, j]) * dense[e][r] for j, e in enumerate(ids[r]) if 0 <= e < E), np.zeros(d))
        assert np.allclose(out[r], exp, rtol=1e-12, atol=1e-12)
    assert not out[3].any()
