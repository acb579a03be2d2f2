"""8-bit codes, products and expert layers against the float64 oracle, and the
whole set as an expert layer uses it: router, experts, projections.

Tolerances.  Codes and their scales are defined in float32 and have to be equal
bit for bit.  A product's sum is exact; its float32 result has three roundings
(conversion, two scales), 3 * 2^-24 of the value, the residual add one more of
the sum.  A bf16 result is off by half a step, 2^-8.  SwiGLU: exp of |g| has a
relative error of (|g| + 4) * 2^-23 in float32, and so has silu; with the other
products' roundings (|g| + 12) * 2^-23, and the bf16 step."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"

from oracle import int8 as O


def _b():
    from paper_2605_30859_amd import binding
    binding.load_library()
    return binding


def _gen(*seed):
    return torch.Generator(device=DEV).manual_seed(sum(int(s) * 1009 ** i for i, s in enumerate(seed)) % (1 << 31))


def _np(t):
    return t.float().cpu().numpy()


def _dt(B, t):
    return B.DARTS_BF16 if t.dtype == torch.bfloat16 else B.DARTS_F32


def quantize(x):
    B = _b()
    q = torch.full((x.shape[0] + 1, x.shape[1]), 99, dtype=torch.int8, device=DEV)
    s = torch.full((x.shape[0] + 1,), 99.0, device=DEV)
    B.darts_quantize_rows(x, _dt(B, x), q, s)
    torch.cuda.synchronize()
    assert bool((q[-1] == 99).all()) and float(s[-1]) == 99.0
    return q[:-1].contiguous(), s[:-1].contiguous()


def same_codes(x):
    q, s = quantize(x)
    eq, es = O.quantize_rows(_np(x))
    assert (q.cpu().numpy() == eq).all()
    assert np.array_equal(s.cpu().numpy(), es, equal_nan=True)


# ---------------------------------------------------------------------- codes
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 16), (1, 4096), (33, 768), (17, 2064), (4, 12288), (9, 1000),
                                       (2, 40000), (300, 128), (1030, 72)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_codes(rows, cols, dtype):
    print(f"codes {rows} {cols} {dtype}", flush=True)
    x = torch.empty(rows, cols, device=DEV).normal_(0, 2, generator=_gen(rows, cols)).to(dtype)
    same_codes(x)
    wide = torch.full((rows, cols + 5), float("nan"), dtype=dtype, device=DEV)     # strided rows, addresses of any alignment
    wide[:, 3:cols + 3] = x
    same_codes(wide[:, 3:cols + 3])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_codes_of_special_rows(dtype):
    x = torch.empty(14, 100, device=DEV).normal_(generator=_gen(5))
    x[0] = 0
    x[1, 99] = float("nan")
    x[2, 50] = float("inf")
    x[3, 0] = -float("inf")
    x[4] *= 2.0 ** -130
    x[5] *= 2.0 ** -119
    x[6] = 2.0 ** -120
    x[7] = 2.0 ** -119
    x[8] *= 3e37
    x[9] = torch.finfo(dtype).max
    x[10] = -0.0
    x[11] = torch.arange(100, device=DEV) * 0.5
    x[11, 99] = 127.0
    x[12, :99] = 0
    x[12, 99] = -5.0
    same_codes(x.to(dtype))


# ------------------------------------------------------------------- products
def _operands(M, N, K, seed=0):
    g = _gen(M, N, K, seed)
    a = torch.randint(-127, 128, (M, K), dtype=torch.int8, device=DEV, generator=g)
    w = torch.randint(-127, 128, (N, K), dtype=torch.int8, device=DEV, generator=g)
    sa = torch.rand(M, device=DEV, generator=g) * 0.02 + 0.001
    sw = (torch.rand(N, device=DEV, generator=g) + 0.1) / (5000.0 * K ** 0.5 * 0.01)
    return a, sa, w, sw


def _i64(a, w):
    """Exact integer product, in float64 (|sum| < 2^53)."""
    return a.double() @ w.double().t()


def _swiglu64(c):
    f = torch.arange(c.shape[1] // 2, device=DEV)
    g, u = c[:, f // 16 * 32 + f % 16], c[:, f // 16 * 32 + 16 + f % 16]
    return g, u, g * torch.special.expit(g) * u


def product(a, sa, w, sw, epi, stream=None):
    B = _b()
    (M, K), N = a.shape, w.shape[0]
    cols = N // 2 if epi == 3 else N
    out = torch.full((M + 70, cols), 3.0, dtype=torch.float32 if epi in (0, 2) else torch.bfloat16, device=DEV)
    ws = torch.full((B.darts_gemm_i8_workspace_bytes(M, N, K) + 256,), 0x5a, dtype=torch.uint8, device=DEV)
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())       # for what was just filled
    B.darts_gemm_i8(a, sa, w, sw, out, M, N, K, epi, ws[:-256], stream=stream)
    torch.cuda.synchronize()
    assert bool((out[M:] == 3.0).all()) and bool((ws[-256:] == 0x5a).all())
    return out[:M]


def check_product(a, sa, w, sw, epi):
    got = product(a, sa, w, sw, epi).double()
    c = _i64(a, w) * sa.double()[:, None] * sw.double()[None, :]
    u24 = 2.0 ** -24 * (1 + 1e-6)
    if epi == 0:
        ref, tol = c, 3 * u24 * c.abs()
    elif epi == 1:
        ref, tol = c, (2.0 ** -8 + 4 * u24) * c.abs()
    elif epi == 2:
        ref = c + 3.0
        tol = 3 * u24 * c.abs() + u24 * ref.abs()
    else:
        g, u, ref = _swiglu64(c)
        tol = (2.0 ** -8 + (g.abs() + 12) * 2.0 ** -23) * ref.abs() + 1e-30
    bad = (got - ref).abs() > tol + 2.0 ** -140
    assert not bool(bad.any()), (torch.nonzero(bad)[:4].tolist(), float(((got - ref).abs() - tol).max()))


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 31, 33, 48, 64, 65, 100, 128, 129, 200, 257, 300, 513])
def test_product_all_batch_sizes(M):
    print(f"product M={M}", flush=True)
    for N, K, epi in ((1536, 1024, 0), (2048, 4096, 1), (1024, 768, 3)):
        check_product(*_operands(M, N, K), epi)


@pytest.mark.parametrize("M,N,K", [(1, 16, 16), (5, 32, 48), (17, 96, 80), (64, 64, 64), (65, 160, 144), (130, 272, 272),
                                   (3, 4112, 2064), (777, 4112, 2064), (300, 528, 1040), (1000, 1056, 272), (257, 5664, 1456),
                                   (1300, 1552, 720), (2049, 288, 4000)])
@pytest.mark.parametrize("epi", [0, 1, 2, 3])
def test_product_sizes_that_divide_no_tile(M, N, K, epi):
    print(f"product {M} {N} {K} epi={epi}", flush=True)
    if epi == 3 and N % 32:
        N += 16
    check_product(*_operands(M, N, K), epi)


@pytest.mark.parametrize("M,N,K,epi", [(1, 6144, 4096, 0), (45, 4096, 12288, 2), (389, 24576, 4096, 3), (12, 4096, 12288, 1),
                                       (64, 6144, 4096, 0), (128, 24576, 4096, 3), (200, 4096, 12288, 2), (350, 5120, 2048, 0),
                                       (512, 2048, 4096, 2), (1024, 6144, 4096, 1), (4133, 4096, 4096, 2), (8203, 6144, 512, 1),
                                       (2049, 4096, 12288, 0), (4100, 24576, 1024, 3), (1030, 8192, 256, 0)])
def test_product_decoder_shapes(M, N, K, epi):
    print(f"product {M} {N} {K} epi={epi}", flush=True)
    check_product(*_operands(M, N, K), epi)


@pytest.mark.parametrize("M,N", [(1, 64), (40, 128), (300, 256)])
def test_product_of_the_largest_codes(M, N):
    """K = 131072 codes of +-127: sums of 2.1e9, just inside 32 bits."""
    K = 131072
    a = torch.full((M, K), 127, dtype=torch.int8, device=DEV)
    w = torch.full((N, K), 127, dtype=torch.int8, device=DEV)
    w[1::2] = -127
    check_product(a, torch.ones(M, device=DEV), w, torch.full((N,), 1e-6, device=DEV), 0)


def test_product_scales_that_are_zero_or_nan():
    for M, N, K in ((5, 64, 128), (300, 1024, 2048)):
        a, sa, w, sw = _operands(M, N, K)
        sa[0], sa[M - 1] = 0.0, float("nan")
        out = product(a, sa, w, sw, 0)
        assert bool((out[0] == 0).all()) and bool(out[M - 1].isnan().all()) and bool(out[1:M - 1].isfinite().all())


def test_product_is_the_same_every_time_and_on_any_stream():
    a, sa, w, sw = _operands(45, 4096, 12288)
    one = product(a, sa, w, sw, 0)
    st = torch.cuda.Stream()
    assert torch.equal(one, product(a, sa, w, sw, 0, stream=st)) and torch.equal(one, product(a, sa, w, sw, 0))


def test_results_beyond_32_bit_offsets():
    """More than 2^31 bytes of results, and of codes."""
    M, N, K = 70000, 8192, 64
    a, sa, w, sw = _operands(M, N, K)
    out = torch.empty(M, N, device=DEV)
    B = _b()
    ws = torch.empty(max(B.darts_gemm_i8_workspace_bytes(M, N, K), 16), dtype=torch.uint8, device=DEV)
    B.darts_gemm_i8(a, sa, w, sw, out, M, N, K, 0, ws)
    rows = torch.tensor([0, 255, 65535, 65536, 69999], device=DEV)
    ref = _i64(a[rows], w) * sa[rows].double()[:, None] * sw.double()
    assert bool(((out[rows].double() - ref).abs() <= 3.01 * 2.0 ** -24 * ref.abs()).all())


def test_more_channels_than_a_launch_of_strips_has():
    """One row and 2^28 + 32 channels, 4 GB of codes."""
    N, K = (1 << 28) + 32, 16
    g = _gen(1, 1, K)
    a = torch.randint(-127, 128, (1, K), dtype=torch.int8, device=DEV, generator=g)
    w = torch.randint(-127, 128, (N, K), dtype=torch.int8, device=DEV, generator=g)
    sa, sw = torch.full((1,), 0.5, device=DEV), torch.full((N,), 2.0, device=DEV)
    out = torch.full((N + 16,), 3.0, device=DEV)
    _b().darts_gemm_i8(a, sa, w, sw, out, 1, N, K, 0, None)
    # sums below 2^24, and scales of powers of two: exact in float32
    for at in range(0, N, 1 << 24):
        rows = w[at:at + (1 << 24)]
        ref = torch.zeros(rows.shape[0], device=DEV)
        for j in range(K):
            ref += rows[:, j].float() * a[0, j].float()
        assert torch.equal(out[at:at + rows.shape[0]], ref)
    assert bool((out[N:] == 3.0).all())


# -------------------------------------------------------------------- experts
def _layer(E, d, F, seed=0):
    g = _gen(E, d, F, seed)
    gu = torch.randint(-127, 128, (E, 2 * F, d), dtype=torch.int8, device=DEV, generator=g)
    dn = torch.randint(-127, 128, (E, d, F), dtype=torch.int8, device=DEV, generator=g)
    s_gu = (torch.rand(E, 2 * F, device=DEV, generator=g) + 0.5) / (75.0 * d ** 0.5)
    s_dn = (torch.rand(E, d, device=DEV, generator=g) + 0.5) / (75.0 * F ** 0.5)
    return gu, s_gu, dn, s_dn


def _routed(R, E, k, seed=0):
    g = _gen(R, E, k, seed)
    ids = torch.randint(0, E, (R, k), dtype=torch.int32, device=DEV, generator=g)      # some ids twice in a row
    return ids, torch.rand(R, k, device=DEV, generator=g)


def _rows(R, d, seed=0):
    return torch.empty(R, d, device=DEV).normal_(generator=_gen(R, d, seed)).bfloat16()


def ffn(x, ids, w, layer, epi=1, stream=None):
    B = _b()
    R, d = x.shape
    E, F2, _ = layer[0].shape
    out = torch.full((R + 3, d), 2.0, dtype=torch.bfloat16 if epi == 1 else torch.float32, device=DEV)
    ws = torch.full((B.darts_moe_ffn_i8_workspace_bytes(R, d, E, ids.shape[1], F2 // 2) + 256,), 0xff, dtype=torch.uint8,
                    device=DEV)
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    B.darts_moe_ffn_i8(x, ids, w, E, F2 // 2, *layer, out, epi, ws[:-256], stream=stream)
    torch.cuda.synchronize()
    assert bool((out[R:] == 2.0).all()) and bool((ws[-256:] == 0xff).all())
    return out[:R]


def by_parts(x, ids, w, layer):
    """The definition with the library's other calls: y of every pair (bf16), and
    the weighted sum and the sum of magnitudes in float64."""
    gu, s_gu, dn, s_dn = layer
    R, d = x.shape
    out = torch.zeros(R, d, dtype=torch.float64, device=DEV)
    mag = torch.zeros_like(out)
    for e in torch.unique(ids).tolist():
        if not 0 <= e < gu.shape[0]:
            continue
        row, slot = torch.nonzero(ids == e, as_tuple=True)
        h = product(*quantize(x[row]), gu[e].contiguous(), s_gu[e].contiguous(), 3)
        y = product(*quantize(h.contiguous()), dn[e].contiguous(), s_dn[e].contiguous(), 1).double()
        t = y * w[row, slot].double()[:, None]
        out.index_add_(0, row, t)
        mag.index_add_(0, row, t.abs())
    return out, mag


def check_ffn(R, E, k, d, F, ids=None, w=None, epi=1):
    """Against the library's own parts: k float32 roundings of the sum, the
    residual's, and half a bf16 step.  Where the parts run another tile, their
    SwiGLU may differ in a last digit, never here: both use the same function."""
    x, layer = _rows(R, d), _layer(E, d, F)
    rid, rw = _routed(R, E, k)
    ids, w = rid if ids is None else ids, rw if w is None else w
    got = ffn(x, ids, w, layer, epi).double()
    ref, mag = by_parts(x, ids, w, layer)
    tol = (ids.shape[1] + 1) * 2.0 ** -24 * mag
    if epi == 1:
        tol = tol + 2.0 ** -8 * ref.abs()
    else:
        ref = ref + 2.0
        tol = tol + 2.0 ** -24 * (ref.abs() + mag)
    bad = (got - ref).abs() > tol + 1e-37
    assert not bool(bad.any()), (torch.nonzero(bad)[:4].tolist(), float(((got - ref).abs() - tol).max()))
    return got


@pytest.mark.parametrize("R,E,k,d,F", [(1, 128, 8, 2048, 768), (1, 1, 1, 16, 16), (3, 4, 2, 48, 32), (61, 128, 8, 2048, 768),
                                       (17, 60, 4, 1456, 720), (200, 16, 4, 1024, 512), (130, 8, 2, 272, 144),
                                       (700, 12, 3, 528, 1040), (5, 1024, 8, 64, 32), (40, 8, 64, 128, 64),
                                       (2500, 7, 2, 256, 256), (3000, 16, 8, 512, 256), (2, 64, 6, 1024, 1408)])
@pytest.mark.parametrize("epi", [1, 2])
def test_experts_against_their_parts(R, E, k, d, F, epi):
    print(f"experts {R} {E} {k} {d} {F} epi={epi}", flush=True)
    check_ffn(R, E, k, d, F, epi=epi)


@pytest.mark.parametrize("R", [1, 9, 150, 1500])
def test_experts_with_places_left_empty(R):
    """Ids outside the experts, rows with none at all, one expert for everybody,
    an id twice in a row."""
    E, k, d, F = 16, 4, 256, 128
    ids, w = _routed(R, E, k)
    ids[:, 1] = -1
    ids[R // 2] = -1
    ids[R - 1, 0] = 1 << 30
    ids[0] = -(1 << 31)
    check_ffn(R, E, k, d, F, ids, w)
    check_ffn(R, E, k, d, F, torch.full_like(ids, -1), w, epi=2)
    check_ffn(R, E, k, d, F, torch.full_like(ids, E - 1), w)
    check_ffn(R, E, k, d, F, ids.fill_(3).index_fill(1, torch.tensor([2], device=DEV), 0), w, epi=2)


@pytest.mark.parametrize("R", [4, 300])
def test_experts_with_poisoned_rows(R):
    """A row that the router could not read (weights NaN), and one whose
    activations hold an infinity, come out NaN; the others are as without them."""
    E, k, d, F = 16, 4, 256, 128
    x, layer = _rows(R, d), _layer(E, d, F)
    ids, w = _routed(R, E, k)
    clean = ffn(x, ids, w, layer)
    ids[1], w[1] = -1, float("nan")
    x[2, 7] = float("inf")
    got = ffn(x, ids, w, layer)
    assert bool(got[1:3].isnan().all())
    keep = torch.ones(R, dtype=torch.bool, device=DEV)
    keep[1:3] = False
    assert torch.equal(got[keep], clean[keep])


@pytest.mark.parametrize("R,E,k,d,F", [(1, 8, 2, 256, 128), (37, 8, 2, 256, 128), (600, 12, 3, 272, 144)])
def test_experts_against_the_oracle(R, E, k, d, F):
    """In the 2-norm: the stored result and y are rounded to bf16, half a step
    (2^-8) of each; h is rounded to bf16 on both sides, and where the last digit of
    SwiGLU turns that rounding or a code, by a step of 2^-7 of a few elements."""
    x, layer = _rows(R, d), _layer(E, d, F)
    ids, w = _routed(R, E, k)
    got = _np(ffn(x, ids, w, layer)).astype(np.float64)
    ref = O.moe_ffn(_np(x), ids.cpu().numpy(), w.cpu().numpy(), *(t.cpu().numpy() for t in layer))
    assert np.linalg.norm(got - ref) <= 3 * 2.0 ** -8 * np.linalg.norm(ref)


# ------------------------------------------------------------- the set together
def _run_layer(B, x, router, bias, layer, proj, buf):
    """A decoder's expert layer in 8 bits: the router's logits, routing, experts
    added to the residual, and a projection of the result."""
    R = x.shape[0]
    E, F2, d = layer[0].shape
    B.darts_quantize_rows(x, B.DARTS_BF16, buf["q"], buf["s"])
    B.darts_gemm_i8(buf["q"], buf["s"], router[0], router[1], buf["logits"], R, router[0].shape[0], d, 0, buf["ws"])
    B.darts_moe_route(buf["logits"][:, :E], B.DARTS_F32, buf["ids"], buf["w"], score=B.SCORE_SIGMOID, bias=bias,
                      n_groups=4, top_groups=2, group_best=2, factor=2.5)
    B.darts_moe_ffn_i8(x, buf["ids"], buf["w"], E, F2 // 2, *layer, buf["res"], 2, buf["ws"])
    B.darts_quantize_rows(buf["res"], B.DARTS_F32, buf["q"], buf["s"])
    B.darts_gemm_i8(buf["q"], buf["s"], proj[0], proj[1], buf["out"], R, proj[0].shape[0], d, 1, buf["ws"])


@pytest.mark.parametrize("R", [1, 50, 700])
def test_layer_eager_and_replayed(R):
    B = _b()
    E, k, d, F, N = 32, 4, 512, 256, 1024
    layer = _layer(E, d, F)
    g = _gen(R, 9)
    router = (torch.randint(-127, 128, (128, d), dtype=torch.int8, device=DEV, generator=g),
              torch.full((128,), 1e-3, device=DEV))
    proj = (torch.randint(-127, 128, (N, d), dtype=torch.int8, device=DEV, generator=g),
            torch.full((N,), 1e-3, device=DEV))
    bias = torch.empty(E, device=DEV).normal_(0, 0.05, generator=g)
    nb = max(B.darts_moe_ffn_i8_workspace_bytes(R, d, E, k, F), B.darts_gemm_i8_workspace_bytes(R, N, d),
             B.darts_gemm_i8_workspace_bytes(R, 128, d))

    def buffers():
        return dict(q=torch.empty(R, d, dtype=torch.int8, device=DEV), s=torch.empty(R, device=DEV),
                    logits=torch.empty(R, 128, device=DEV), ids=torch.empty(R, k, dtype=torch.int32, device=DEV),
                    w=torch.empty(R, k, device=DEV), res=torch.zeros(R, d, device=DEV),
                    out=torch.empty(R, N, dtype=torch.bfloat16, device=DEV),
                    ws=torch.empty(nb, dtype=torch.uint8, device=DEV))

    x = _rows(R, d)
    one, two = buffers(), buffers()
    _run_layer(B, x, router, bias, layer, proj, one)
    torch.cuda.synchronize()
    # the parts against the oracle, each on the values that it got
    from oracle.routing import route
    ids, w = route(one["logits"][:, :E].cpu().numpy(), k, score="sigmoid", bias=bias.cpu().numpy(), n_groups=4,
                   top_groups=2, group_best=2, factor=2.5)
    assert (one["ids"].cpu().numpy() == ids).all()
    ref = O.moe_ffn(_np(x), ids, w, *(t.cpu().numpy() for t in layer))
    assert np.linalg.norm(_np(one["res"]) - ref) <= 2 * 2.0 ** -8 * np.linalg.norm(ref)
    ref = O.product(*O.quantize_rows(_np(one["res"])), *(t.cpu().numpy() for t in proj))
    assert (np.abs(_np(one["out"]) - ref) <= (2.0 ** -8 + 2.0 ** -22) * np.abs(ref) + 1e-30).all()
    # two captured graphs with workspaces of their own, replayed beside eager work
    graphs = []
    for buf in (one, two):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            buf["res"].zero_()
            _run_layer(B, x, router, bias, layer, proj, buf)
        graphs.append(graph)
    for i in range(3):
        x.copy_(_rows(R, d, seed=i + 1))
        eager = buffers()
        _run_layer(B, x, router, bias, layer, proj, eager)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for buf in (one, two):
            assert torch.equal(buf["ids"], eager["ids"]) and torch.equal(buf["w"], eager["w"])
            assert torch.equal(buf["res"], eager["res"]) and torch.equal(buf["out"], eager["out"])
