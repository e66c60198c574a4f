"""int8 linear operators on the GPU against their definitions in 64 bits.

Quantisation: of bf16 rows every integer is the definition's (the quotient is rounded as if exact). Of fp32 rows a
quotient carries the rounding of 127 x and of the division, |q - 127 x / max| <= 1/2 + 127 3 2^-24; after an RMSNorm
also the norm's, whose fp32 sum of d squares, root, quotient and two products are off by less than (d / 2 + 8) 2^-24.

Products: the int32 sum is exact, so y = s_m w_n sum is off by three roundings, 3 2^-24 |y| (the sum's conversion, s_m w_n,
the product). A residual adds one of |y| + |r|; SwiGLU on the hardware exp2 and reciprocal (a few fp32 steps each, the
exponent's argument rounded at |gate| 1.44) is off by (|gate| + 16) 2^-23 of the result, and the halves' 6 2^-24 (1 + |gate|).
A bf16 result is rounded once more, 2^-8 |result|.
"""
import numpy as np
import pytest

from oracle import layer as O
from synth import gen
from tests import helpers as H

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2608_21719_amd import binding as B  # noqa: E402

CODE = {"f32": B.PS_F32, "bf16": B.PS_BF16}
EPI = {"store": B.PS_EPI_STORE, "residual": B.PS_EPI_RESIDUAL, "swiglu": B.PS_EPI_SWIGLU}


def store(a, dtype):
    return gen.to_storage(np.asarray(a, np.float32), dtype)


def quant(x, dt, g=None, gdt="bf16", eps=1e-5):
    rows, d = x.shape
    q = torch.full((rows, d), 99, dtype=torch.int8, device="cuda")
    s = torch.full((rows,), -1.0, dtype=torch.float32, device="cuda")
    if g is None:
        B.op_quant_rows(CODE[dt], rows, d, H.to_dev(x, dt), q, s)
    else:
        B.op_rmsnorm_quant(CODE[dt], CODE[gdt], rows, d, H.to_dev(x, dt), H.to_dev(g, gdt), eps, q, s)
    torch.cuda.synchronize()
    return q, s


# ---------------------------------------------------------------- quantisation
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 7), (5, 64), (64, 4096), (33, 8192), (7, 14336), (2, 28672), (2, 40000), (600, 200)])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_quant_rows(rows, d, dt):
    rng = np.random.default_rng(d)
    x = store(rng.standard_normal((rows, d)) * 10.0 ** rng.integers(-20, 21, (rows, 1)), dt)
    q, s = quant(x, dt)
    xf = gen.widen(x, dt)
    top = np.abs(xf).max(1, keepdims=True)
    exact = 127.0 * xf / top
    got = q.cpu().numpy().astype(np.float64)
    if dt == "bf16":
        assert np.array_equal(got, np.round(exact))
    else:
        assert (np.abs(got - exact) <= 0.5 + 127 * 3 * 2.0 ** -24).all()
    assert np.array_equal(np.abs(got).max(1), np.full(rows, 127.0))
    assert (np.abs(s.cpu().numpy().astype(np.float64)[:, None] - top / 127) <= 2.0 ** -24 * top / 127).all()


def test_quant_rows_on_the_border_between_integers():
    """Rows of multiples of amax / 254: every second quotient ends in one half."""
    n = np.arange(-254, 255, dtype=np.float32)
    x = np.stack([n, n * 2.0 ** -60, n * 0.5])
    q, s = quant(store(np.pad(x, ((0, 0), (0, 3))), "f32"), "f32")
    assert np.array_equal(q.cpu().numpy()[:, :509], np.round(np.stack([n / 2] * 3)))


def test_quant_rows_special():
    x = np.zeros((7, 72), np.float32)
    x[1, 5], x[2, 9], x[3, 70] = np.nan, np.inf, -np.inf
    x[1:4, 0] = 1.0
    x[4, 3] = 2.0 ** -110
    x[5, :] = np.linspace(-3e38, 3e38, 72)
    x[6, :] = np.linspace(-1, 1, 72) * 2.0 ** -99
    for dt in ("f32", "bf16"):
        q, s = quant(store(x, dt), dt)
        q, s = q.cpu().numpy(), s.cpu().numpy()
        assert s[0] == 0 and s[4] == 0 and np.isnan(s[1:4]).all() and (q[:5] == 0).all()
        assert np.isfinite(s[5:]).all() and (np.abs(q[5:]).max(1) == 127).all()


@pytest.mark.parametrize("rows,d", [(1, 64), (9, 4096), (3, 8192), (4, 200), (3, 77), (2, 20000)])
@pytest.mark.parametrize("dt,gdt", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32"), ("bf16", "f32")])
def test_rmsnorm_quant(rows, d, dt, gdt):
    rng = np.random.default_rng(d + 1)
    x = store(rng.standard_normal((rows, d)) * 3, dt)
    g = store(1 + 0.1 * rng.standard_normal(d), gdt)
    q, s = quant(x, dt, g, gdt)
    y = O.rmsnorm(gen.widen(x, dt), gen.widen(g, gdt), 1e-5)
    top = np.abs(y).max(1, keepdims=True)
    err = (d / 2 + 8) * 2.0 ** -24
    assert (np.abs(q.cpu().numpy() - 127 * y / top) <= 0.5 + 127 * (3 * 2.0 ** -24 + 2 * err)).all()
    assert (np.abs(s.cpu().numpy().astype(np.float64)[:, None] * 127 / top - 1) <= err + 2.0 ** -23).all()


# ---------------------------------------------------------------- products
def product(rng, M, N, K, epi, r, c, a=None, w=None):
    if a is None:
        a = rng.integers(-127, 128, (M, K)).astype(np.int8)
    if w is None:
        w = rng.integers(-127, 128, (N, K)).astype(np.int8)
    sa = (rng.uniform(0.5, 2, M) / 127).astype(np.float32)
    sw = (rng.uniform(0.5, 2, N) / 127 / np.sqrt(K)).astype(np.float32)
    cols = N // 2 if epi == "swiglu" else N
    R = store(rng.standard_normal((M, N)), r) if epi == "residual" else None
    W = torch.from_numpy(B.tile_weight_i8(w)).cuda()
    A, SA, SW = (torch.from_numpy(x).cuda() for x in (a, sa, sw))
    C = torch.full((M + 1, cols), float("nan"), dtype=torch.bfloat16 if c == "bf16" else torch.float32, device="cuda")
    Rd = H.to_dev(R, r) if R is not None else None
    n = B.op_gemm_i8_workspace_bytes(M, N, K)
    ws = torch.full((max(n, 16),), 255, dtype=torch.uint8, device="cuda")
    call = lambda: B.op_gemm_i8(CODE[r], CODE[c], EPI[epi], M, N, K, A, SA, W, SW, Rd, C, ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    got = H.to_f64(C)
    assert np.isnan(got[M]).all()  # the row behind the last is not written
    y = (a.astype(np.float64) @ w.astype(np.float64).T) * (sa.astype(np.float64)[:, None] * sw.astype(np.float64))
    u = 2.0 ** -24
    if epi == "store":
        ref, b = y, 3 * u * np.abs(y)
    elif epi == "residual":
        rf = gen.widen(R, r)
        ref, b = y + rf, 3 * u * np.abs(y) + u * (np.abs(y) + np.abs(rf))
    else:
        y = y.reshape(M, -1, 2, 32)
        gate, up = y[:, :, 0].reshape(M, -1), y[:, :, 1].reshape(M, -1)
        ref = O.silu(gate) * up
        b = np.abs(ref) * ((np.abs(gate) + 16) * 2.0 ** -23 + 6 * u * (1 + np.abs(gate)))
    b = b * 1.01 + (2.0 ** -8 * np.abs(ref) if c == "bf16" else 0) + 1e-38
    bad = ~(np.abs(got[:M] - ref) <= b)
    assert not bad.any(), f"{bad.sum()} of {bad.size}, worst {np.nanmax(np.abs(got[:M] - ref) / b):.2f} of the bound"
    first = H.bits(C[:M])
    call()
    torch.cuda.synchronize()
    assert np.array_equal(first, H.bits(C[:M]))


SHAPES = [(1, 64, 64), (1, 6144, 4096), (5, 128, 192), (16, 320, 4160), (17, 64, 14336), (33, 4096, 4096), (64, 640, 1024),
          (64, 32768, 256), (40, 57344, 128),                    # one, two and four weight blocks, split and not
          (65, 64, 64), (100, 192, 320), (130, 320, 1088), (389, 1024, 512), (257, 4096, 1024), (300, 576, 4096),
          (1000, 2048, 192), (700, 28672, 256), (2500, 512, 704),
          (2600, 8192, 512), (4400, 6208, 768), (4400, 6208, 640),  # several rounds of 256x256 tiles, and of two launches
          (97, 320, 16448), (300, 576, 14400), (130, 1024, 9280),  # K splits of tiles
          (2, 6208, 4032), (9, 4096, 1088), (16, 8192, 1536), (7, 2048, 8192), (8, 16384, 1984), (3, 192, 3200)]  # narrow


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("epi,r,c", [("store", "f32", "bf16"), ("store", "f32", "f32"), ("residual", "bf16", "f32"),
                                     ("residual", "f32", "bf16"), ("residual", "bf16", "bf16"), ("residual", "f32", "f32"),
                                     ("swiglu", "f32", "bf16"), ("swiglu", "f32", "f32")])
def test_gemm_i8(M, N, K, epi, r, c):
    if M * N * K > 3e9 and (epi, r, c) not in (("store", "f32", "f32"), ("swiglu", "f32", "bf16")):
        pytest.skip("the large shapes are held in one exact and one fused form")
    product(np.random.default_rng(M + N + K), M, N, K, epi, r, c)


@pytest.mark.parametrize("M", [2, 70])
def test_longest_sums(M):
    """K at its limit with every operand at -128: the sum is 2^31 - 2^20, the largest a call can reach."""
    K, N = 131008, 64
    a, w = np.full((M, K), -128, np.int8), np.full((N, K), -128, np.int8)
    a[1::2] = 127
    product(np.random.default_rng(1), M, N, K, "store", "f32", "f32", a, w)


def test_rows_of_nan_scale_are_nan_and_no_others():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((6, 256)).astype(np.float32)
    x[2, 9], x[4, 1] = np.inf, np.nan
    q, s = quant(store(x, "f32"), "f32")
    w = rng.integers(-127, 128, (128, 256)).astype(np.int8)
    W, sw = torch.from_numpy(B.tile_weight_i8(w)).cuda(), torch.ones(128, device="cuda")
    C = H.empty((6, 128), "bf16")
    ws = H.workspace(B.op_gemm_i8_workspace_bytes(6, 128, 256))
    B.op_gemm_i8(0, B.PS_BF16, B.PS_EPI_STORE, 6, 128, 256, q, s, W, sw, None, C, ws)
    torch.cuda.synchronize()
    bad = np.isnan(H.to_f64(C))
    assert bad[[2, 4]].all() and not bad[[0, 1, 3, 5]].any()


def test_residual_in_place_and_device_tiling():
    rng = np.random.default_rng(3)
    for M in (20, 200):
        N, K = 320, 448
        a, w = rng.integers(-127, 128, (M, K)).astype(np.int8), rng.integers(-127, 128, (N, K)).astype(np.int8)
        A, W0 = torch.from_numpy(a).cuda(), torch.from_numpy(w).cuda()
        W = torch.full((B.tiled_weight_i8_bytes(N, K),), 7, dtype=torch.int8, device="cuda")
        B.op_tile_weight_i8(N, K, W0, W)
        assert np.array_equal(W.cpu().numpy(), B.tile_weight_i8(w))
        sa, sw = torch.full((M,), 0.01, device="cuda"), torch.full((N,), 0.01, device="cuda")
        r = torch.randn((M, N), device="cuda", generator=torch.Generator("cuda").manual_seed(1))
        out, ws = torch.empty_like(r), H.workspace(B.op_gemm_i8_workspace_bytes(M, N, K))
        B.op_gemm_i8(0, 0, B.PS_EPI_RESIDUAL, M, N, K, A, sa, W, sw, r, out, ws)
        B.op_gemm_i8(0, 0, B.PS_EPI_RESIDUAL, M, N, K, A, sa, W, sw, r, r, ws)
        torch.cuda.synchronize()
        assert np.array_equal(H.bits(r), H.bits(out))


def test_a_captured_linear_layer_replays():
    """Norm, quantisation and product in a graph, replayed on new rows with eager calls between."""
    rng = np.random.default_rng(4)
    M, N, K = 24, 6144, 4096
    g = H.to_dev(store(1 + 0.1 * rng.standard_normal(K), "bf16"), "bf16")
    w = rng.integers(-127, 128, (N, K)).astype(np.int8)
    W, sw = torch.from_numpy(B.tile_weight_i8(w)).cuda(), torch.full((N,), 1e-4, device="cuda")
    x = H.to_dev(store(rng.standard_normal((M, K)), "bf16"), "bf16")

    def make():
        q, s, C = (torch.empty((M, K), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda"), H.empty((M, N), "bf16"))
        ws = H.workspace(B.op_gemm_i8_workspace_bytes(M, N, K))

        def call():
            B.op_rmsnorm_quant(B.PS_BF16, B.PS_BF16, M, K, x, g, 1e-5, q, s)
            B.op_gemm_i8(0, B.PS_BF16, B.PS_EPI_STORE, M, N, K, q, s, W, sw, None, C, ws)
        return call, C
    eager, ce = make()
    eager()
    torch.cuda.synchronize()
    captured, cg = make()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured()
    for _ in range(4):
        x.copy_(H.to_dev(store(rng.standard_normal((M, K)), "bf16"), "bf16"))
        cg.zero_()
        graph.replay()
        torch.cuda.synchronize()
        eager()
        torch.cuda.synchronize()
        assert np.array_equal(H.bits(cg), H.bits(ce)) and np.isfinite(H.to_f64(cg)).all()
