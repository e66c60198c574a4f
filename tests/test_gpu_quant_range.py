"""ps_op_rmsnorm_quant where the fp32 sum of a row's squares is infinite or loses the row (GPU).

The mean square is then taken of the row times a power of two, so the bound is that of ordinary rows: an fp32 sum of d
squares, root, quotient and two products are off by less than (d / 2 + 8) 2^-24, a quotient by 3 2^-24 more.
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


def run(x, g, dt, gdt, eps):
    rows, d = x.shape
    q = torch.full((rows, d), 99, dtype=torch.int8, device="cuda")
    s = torch.full((rows,), -1.0, dtype=torch.float32, device="cuda")
    B.op_rmsnorm_quant(CODE[dt], CODE[gdt], rows, d, H.to_dev(x, dt), H.to_dev(g, gdt), eps, q, s)
    torch.cuda.synchronize()
    return q.cpu().numpy(), s.cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("d", [8, 77, 4096, 8192, 16384, 28672, 40000])
@pytest.mark.parametrize("dt,gdt", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("eps", [1e-5, 0.0])
def test_rows_far_from_one(d, dt, gdt, eps):
    """Magnitudes of 2^-125 to 2^125 among ordinary ones; eps counts for the small rows, or is 0."""
    rng = np.random.default_rng(d)
    mag = 2.0 ** np.array([0, 62, 64, 67, 100, 125, -20, -49, -52, -66, -80, -100, -125, 3.0])
    x = gen.to_storage((rng.uniform(0.5, 1.0, (mag.size, d)) * rng.choice([-1, 1], (mag.size, d)) * mag[:, None]).astype(np.float32), dt)
    g = gen.to_storage((1 + 0.1 * rng.standard_normal(d)).astype(np.float32), gdt)
    q, s = run(x, g, dt, gdt, eps)
    y = O.rmsnorm(gen.widen(x, dt), gen.widen(g, gdt), eps)
    top = np.abs(y).max(1, keepdims=True)
    err = (d / 2 + 8) * 2.0 ** -24
    live = top[:, 0] >= 2.0 ** -99  # rows below 2^-100 throughout are zero
    assert live[:8].all() and (live.all() if eps == 0 else not live[-2])
    assert (np.abs(q - 127 * y / top) <= 0.5 + 127 * (3 * 2.0 ** -24 + 2 * err))[live].all()
    assert (np.abs(s[:, None] * 127 / top - 1) <= err + 2.0 ** -23)[live].all()
    assert (q[~live] == 0).all() and (s[~live] == 0).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [72, 77])
def test_largest_values_and_non_finite_ones(dt, d):
    """One large value in a row, a row of the largest numbers, and rows that no scaling saves."""
    x = np.ones((6, d), np.float32)
    x[0, 5] = 3e38
    x[1, :] = np.where(np.arange(d) % 2, 3.3e38, -3.3e38)
    x[2, 7], x[3, 9], x[4, d - 1] = np.inf, np.nan, -np.inf
    g = np.ones(d, np.float32)
    x, g = gen.to_storage(x, dt), gen.to_storage(g, dt)
    q, s = run(x, g, dt, dt, 1e-5)
    assert np.isnan(s[2:5]).all() and (q[2:5] == 0).all()
    y = O.rmsnorm(gen.widen(x[:2], dt), gen.widen(g, dt), 1e-5)
    top = np.abs(y).max(1)
    assert (np.abs(s[:2] * 127 / top - 1) <= (d / 2 + 8) * 2.0 ** -24 + 2.0 ** -23).all()
    assert np.array_equal(q[:2], np.round(127 * y / top[:, None])) and (q[5] == 127).all()
