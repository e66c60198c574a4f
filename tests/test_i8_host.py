"""The int8 linear operators without a GPU: tiled layout, sizes, refusals."""
import numpy as np
import pytest

from paper_2608_21719_amd import binding as B

OK, BAD = 0x20000, 0x20008  # never dereferenced: every call below is refused first


@pytest.mark.parametrize("N,K", [(64, 128), (70, 192), (1, 64), (256, 1024)])
def test_tiled_layout(N, K):
    w = np.random.default_rng(1).integers(-128, 128, (N, K)).astype(np.int8)
    t = B.tile_weight_i8(w)
    kt = (K + 127) // 128
    assert t.size == B.tiled_weight_i8_bytes(N, K) == (N + 63) // 64 * kt * 8192
    n, k = np.meshgrid(np.arange(N), np.arange(K), indexing="ij")
    at = ((n // 64) * kt + k // 128) * 8192 + (n % 64) * 128 + k % 128
    assert np.array_equal(t[at], w)
    rest = np.ones(t.size, bool)
    rest[at.ravel()] = False
    assert (t[rest] == 0).all()


def test_sizes():
    assert B.tiled_weight_i8_bytes(64, 100) == 0 and B.tiled_weight_i8_bytes(0, 128) == 0
    assert B.op_gemm_i8_workspace_bytes(65, 256, 256) == 0 and B.op_gemm_i8_workspace_bytes(0, 256, 256) == 0
    assert B.op_gemm_i8_workspace_bytes(64, 256, 4096) >= 64 * 256 * 4
    assert B.op_gemm_i8_workspace_bytes(64, 100, 4096) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(epi=3), B.PS_E_INVALID), (dict(M=-1), B.PS_E_INVALID), (dict(N=0), B.PS_E_INVALID), (dict(A=None), B.PS_E_INVALID),
    (dict(a_scale=None), B.PS_E_INVALID), (dict(w_scale=None), B.PS_E_INVALID), (dict(W=BAD), B.PS_E_INVALID),
    (dict(a_scale=BAD), B.PS_E_INVALID), (dict(epi=1, R=None), B.PS_E_INVALID), (dict(C=None), B.PS_E_INVALID),
    (dict(ws=0, ws_bytes=0), B.PS_E_INVALID), (dict(ws_bytes=16), B.PS_E_INVALID),
    (dict(N=100), B.PS_E_UNSUPPORTED), (dict(K=96), B.PS_E_UNSUPPORTED), (dict(K=131072), B.PS_E_UNSUPPORTED),
    (dict(c_dt=2), B.PS_E_UNSUPPORTED), (dict(epi=1, r_dt=0, c_dt=0, M=100, R=BAD), B.PS_E_INVALID)])
def test_gemm_refusals(kw, code):
    a = dict(r_dt=1, c_dt=1, epi=0, M=4, N=256, K=256, A=OK, a_scale=OK, W=OK, w_scale=OK, R=OK, C=OK, ws=OK, ws_bytes=1 << 30)
    a.update(kw)
    rc = B.lib.ps_op_gemm_i8(a["r_dt"], a["c_dt"], a["epi"], a["M"], a["N"], a["K"], a["A"], a["a_scale"], a["W"], a["w_scale"],
                             a["R"], a["C"], a["ws"], a["ws_bytes"], None)
    assert rc == code, B.last_error()


def test_quant_refusals():
    q = B.lib.ps_op_quant_rows
    n = B.lib.ps_op_rmsnorm_quant
    assert q(2, 4, 64, OK, OK, OK, None) == B.PS_E_INVALID
    assert q(1, -1, 64, OK, OK, OK, None) == B.PS_E_INVALID
    assert q(1, 4, 0, OK, OK, OK, None) == B.PS_E_INVALID
    assert q(1, 4, 64, None, OK, OK, None) == B.PS_E_INVALID
    assert q(1, 4, 64, OK, BAD, OK, None) == B.PS_E_INVALID
    assert n(1, 1, 4, 64, OK, None, 1e-5, OK, OK, None) == B.PS_E_INVALID
    assert n(1, 3, 4, 64, OK, OK, 1e-5, OK, OK, None) == B.PS_E_INVALID
    assert n(1, 1, 4, 64, OK, OK, -1.0, OK, OK, None) == B.PS_E_INVALID
    assert q(1, 0, 64, None, None, None, None) == B.PS_OK  # no rows: nothing to do


def test_tile_refusals():
    w = np.zeros((64, 96), np.int8)
    with pytest.raises(B.PsError) as e:
        B.tile_weight_i8(w)
    assert e.value.code == B.PS_E_UNSUPPORTED
    assert B.lib.ps_op_tile_weight_i8(64, 96, OK, OK, None) == B.PS_E_UNSUPPORTED
    assert B.lib.ps_op_tile_weight_i8(64, 128, None, OK, None) == B.PS_E_INVALID
    assert B.lib.ps_op_tile_weight_i8(64, 128, OK, BAD, None) == B.PS_E_INVALID
