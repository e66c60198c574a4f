"""Every form of the int8 product on the GPU: tile shapes, K splits of tiles, launches in two column parts, epilogues.

Which form a size takes follows from the cost model of gemm_tile_plan for 256 compute units (int8 counts as half the K);
the lists name it. The sums are exact in int32, so the reference is the 64-bit product of the integers, and a result is
off by the roundings behind it alone: the sum's conversion, s_m w_n and their product, 3 2^-24 |y|; a residual adds one
of |y| + |r|; SwiGLU on the hardware exp2 and reciprocal (a few fp32 steps each, the exponent's argument rounded at
|gate| 1.44) (|gate| + 16) 2^-23 of the result and the halves' 6 2^-24 (1 + |gate|); a bf16 result half a step, 2^-8.
"""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2608_21719_amd import binding as B  # noqa: E402
from tests import helpers as H  # noqa: E402

CODE = {"f32": B.PS_F32, "bf16": B.PS_BF16}
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
EPI = {"store": B.PS_EPI_STORE, "residual": B.PS_EPI_RESIDUAL, "swiglu": B.PS_EPI_SWIGLU}
FORMS = [("store", "f32", "bf16"), ("store", "f32", "f32"), ("residual", "bf16", "f32"), ("residual", "f32", "bf16"),
         ("residual", "bf16", "bf16"), ("residual", "f32", "f32"), ("swiglu", "f32", "bf16"), ("swiglu", "f32", "f32")]


class Product:
    """Operands of one size on the device."""

    def __init__(self, M, N, K, seed=0):
        g = torch.Generator("cuda").manual_seed(seed + M + N + K)
        self.M, self.N, self.K = M, N, K
        self.a, self.w = (torch.randint(-127, 128, (n, K), dtype=torch.int8, device="cuda", generator=g) for n in (M, N))
        self.sa = (0.5 + torch.rand(M, device="cuda", generator=g)) / 127
        self.sw = (0.5 + torch.rand(N, device="cuda", generator=g)) / 127 / K ** 0.5
        self.r = torch.randn((M, N), device="cuda", generator=g)
        self.W = torch.empty(B.tiled_weight_i8_bytes(N, K), dtype=torch.int8, device="cuda")
        B.op_tile_weight_i8(N, K, self.w, self.W)

    def run(self, epi, r, c, M=None):
        M = M or self.M
        cols = self.N // 2 if epi == "swiglu" else self.N
        out = torch.full((M + 1, cols), float("nan"), dtype=TYPE[c], device="cuda")
        R = self.r.to(TYPE[r]) if epi == "residual" else None
        ws = torch.full((max(16, B.op_gemm_i8_workspace_bytes(M, self.N, self.K)),), 255, dtype=torch.uint8, device="cuda")
        B.op_gemm_i8(CODE[r], CODE[c], EPI[epi], M, self.N, self.K, self.a, self.sa, self.W, self.sw, R, out, ws)
        torch.cuda.synchronize()
        assert torch.isnan(out[M]).all()  # the row behind the last is not written
        return out[:M]

    def check(self, epi, r, c):
        got = self.run(epi, r, c).double()
        y = (self.a.double() @ self.w.double().t()) * (self.sa.double()[:, None] * self.sw.double())
        u = 2.0 ** -24
        if epi == "store":
            ref, b = y, 3 * u * y.abs()
        elif epi == "residual":
            rf = self.r.to(TYPE[r]).double()
            ref, b = y + rf, 3 * u * y.abs() + u * (y.abs() + rf.abs())
        else:
            y = y.reshape(self.M, -1, 2, 32)
            gate, up = y[:, :, 0].reshape(self.M, -1), y[:, :, 1].reshape(self.M, -1)
            ref = gate / (1 + torch.exp(-gate)) * up
            b = ref.abs() * ((gate.abs() + 16) * 2.0 ** -23 + 6 * u * (1 + gate.abs()))
        b = b * 1.01 + (2.0 ** -8 * ref.abs() if c == "bf16" else 0) + 1e-38
        bad = ~((got - ref).abs() <= b)
        assert not bad.any(), f"{int(bad.sum())} of {bad.numel()}, worst {((got - ref).abs() / b).nan_to_num(1e30).max():.2f} of the bound"


# Tile shape of store and residual ("nt": weights by non-temporal loads); K below a tile's 128, of a few stages, of many.
SHAPES = [(129, 8448, 64), (70, 16576, 192), (129, 10240, 128), (129, 8448, 1664), (65, 18240, 1536),  # 128x128, nt from 65
          (193, 16896, 64), (70, 33984, 64), (389, 14336, 128), (193, 16832, 1728),                     # 128x256, the second nt
          (129, 5568, 64), (65, 9216, 1536), (129, 5824, 1600),                                         # 128x64, the second nt
          (257, 14336, 128), (129, 18112, 64), (390, 8384, 64), (257, 13120, 1536),                     # 192x128, the second nt
          (389, 17088, 64), (129, 35520, 64), (390, 17408, 1536),                                       # 192x256, the second nt
          (389, 14336, 2048), (193, 17088, 1856), (390, 10816, 1920),                                   # 256x128, the second nt
          (1000, 10880, 64), (193, 34432, 64), (193, 34304, 1536)]                                      # 256x256, nt from 193
# K splits of tiles, with a reduction: 64x64 in 2, 3, 4; 128x64 in 3, 4; 128x128 in 2, 3, 4; 192x128 in 2, 3, 4
SPLIT = [(65, 64, 4416), (65, 192, 6080), (70, 320, 8384), (520, 1024, 8192), (1500, 64, 9024), (65, 10816, 14784),
         (520, 2048, 8192), (3500, 64, 12352), (129, 11328, 7488), (129, 8256, 6080), (257, 3840, 9216)]
# Two launches, the columns of whole rounds of one shape and the rest of another (store and residual; SwiGLU)
TWO = [(257, 34304, 64),   # 192x256 + 64x64
       (520, 22016, 64),   # 192x256 + 64x64
       (1000, 34304, 64),  # 256x256 + 128x64; 128x128
       (2600, 14080, 64),  # 256x256 + 192x128 both
       (3500, 14336, 192), (2048, 10240, 8192)]  # 256x256 + 128x64, 128x128; 128x128 both


@pytest.mark.parametrize("M,N,K", SHAPES + SPLIT + TWO)
def test_forms(M, N, K):
    p = Product(M, N, K)
    for form in FORMS:
        p.check(*form)


@pytest.mark.parametrize("N,K", [(2048, 8192), (6144, 1088), (33024, 320), (4160, 6080)])
@pytest.mark.parametrize("form", FORMS)
def test_a_row_does_not_depend_on_how_many_share_the_call(N, K, form):
    """Narrow, skinny (whole and split), tiles of every shape, splits and two launches: the same bits."""
    p = Product(2600, N, K)
    whole = H.bits(p.run(*form))
    for M in (1, 9, 17, 40, 64, 65, 129, 193, 389, 1000):
        assert (H.bits(p.run(*form, M=M)) == whole[:M]).all(), M
