"""Projections and routed experts in 8-bit integers.  TEST INFRASTRUCTURE: the
plain statement of what the library's 8-bit entries compute.

Codes are defined by float32 arithmetic (two divisions, a product, a rounding to
the nearest integer with halves to even) and reproduced as such; everything
behind them is float64, with the roundings to bf16 that the definition has:
hidden activations, and each expert's result before the weighted sum.  Results
that are stored in bf16 by the caller's choice are left unrounded.

Pins (tests/test_oracle_int8.py): closed forms and hand examples of the codes,
the error of a code and its scale (at most half a step), integer products in
Python integers, the expert layer against one dense layer per expert.
"""
import numpy as np

from workload.gen import bf16_bits_from_f32, f32_from_bf16_bits

TINY = np.float32(2.0 ** -119)     # rows below it have scale 0


def round_bf16(x):
    return f32_from_bf16_bits(bf16_bits_from_f32(np.asarray(x, dtype=np.float32)))


def quantize_rows(x):
    """x float32 [rows][cols] -> codes int8, scales float32."""
    x = np.asarray(x, dtype=np.float32)
    q = np.zeros(x.shape, dtype=np.int8)
    scale = np.zeros(x.shape[0], dtype=np.float32)
    for r in range(x.shape[0]):
        if not np.isfinite(x[r]).all():
            scale[r] = np.nan
            continue
        a = np.abs(x[r]).max()
        if a < TINY:
            continue
        scale[r] = a / np.float32(127)
        q[r] = np.rint(x[r] * (np.float32(127) / a)).astype(np.int8)
    return q, scale


def silu(x):
    with np.errstate(over="ignore"):
        return x / (1.0 + np.exp(-x))


def swiglu(c):
    """silu(gate) * up of columns interleaved in groups of 16."""
    f = np.arange(c.shape[-1] // 2)
    g = f // 16 * 32 + f % 16
    return silu(c[..., g]) * c[..., g + 16]


def product(a, a_scale, w, w_scale):
    """float64 [M][N]: the integer sums are exact in float64."""
    acc = a.astype(np.float64) @ w.astype(np.float64).T
    return acc * a_scale.astype(np.float64)[:, None] * w_scale.astype(np.float64)[None, :]


def expert(x, w_gu, s_gu, w_down, s_down):
    """One expert's rows: x float32 (bf16 values) -> float64 (bf16 values)."""
    h = round_bf16(swiglu(product(*quantize_rows(x), w_gu, s_gu)))
    return round_bf16(product(*quantize_rows(h), w_down, s_down)).astype(np.float64)


def moe_ffn(x, ids, weights, w_gu, s_gu, w_down, s_down):
    out = np.zeros(x.shape, dtype=np.float64)
    for e in range(w_gu.shape[0]):
        row, slot = np.nonzero(ids == e)
        if len(row):
            y = expert(x[row], w_gu[e], s_gu[e], w_down[e], s_down[e])
            np.add.at(out, row, y * weights[row, slot].astype(np.float64)[:, None])
    return out
