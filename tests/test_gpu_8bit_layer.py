"""A decoder layer made of the 8-bit operators, as a serving loop runs it (GPU): int8 projections, an e4m3 KV pool and
attention over it, prompts and then decode steps. Every stage is held against its definition in 64 bits on what the stage
before it left on the device, with the stage's own bound."""
import numpy as np
import pytest

from oracle import layer as O
from synth import gen
from tests import helpers as H
from tests.test_gpu_kv8 import Pool8, check
from tests.kv8_helpers import shape

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2608_21719_amd import binding as B  # noqa: E402


class Int8Layer:
    def __init__(self, shp, rng):
        self.s, d = shp, shp.hidden
        dq, dkv = shp.n_q * shp.head_dim, shp.n_kv * shp.head_dim
        self.w = {}
        for name, n, k in (("qkv", dq + 2 * dkv, d), ("o", d, dq), ("gu", 2 * shp.ffn, d), ("down", d, shp.ffn)):
            w = H.to_dev((rng.standard_normal((n, k)) / np.sqrt(k)).astype(np.float32), "f32")
            q, s = torch.empty((n, k), dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
            B.op_quant_rows(B.PS_F32, n, k, w, q, s)  # a weight's channels are quantised as rows are
            t = torch.empty(B.tiled_weight_i8_bytes(n, k), dtype=torch.int8, device="cuda")
            B.op_tile_weight_i8(n, k, q, t)
            self.w[name] = (n, k, t, s, q.double().cpu().numpy())
        self.g = [H.to_dev(gen.to_storage((1 + 0.1 * rng.standard_normal(d)).astype(np.float32), "bf16"), "bf16") for _ in range(2)]
        self.ws = H.workspace(max(B.op_gemm_i8_workspace_bytes(64, n, k) for n, k, *_ in self.w.values()))

    def linear(self, name, x, epi, c, r=None, gain=None):
        """One product with its quantisation; returns C after checking it against 64 bits on the same int8 rows."""
        n, k, t, sw, wi = self.w[name]
        M = x.shape[0]
        code = {torch.float32: B.PS_F32, torch.bfloat16: B.PS_BF16}
        q, s = torch.empty((M, k), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
        if gain is None:
            B.op_quant_rows(code[x.dtype], M, k, x, q, s)
        else:
            B.op_rmsnorm_quant(code[x.dtype], B.PS_BF16, M, k, x, gain, 1e-5, q, s)
        C = torch.empty((M, n // 2 if epi == B.PS_EPI_SWIGLU else n), dtype=c, device="cuda")
        B.op_gemm_i8(code[r.dtype] if r is not None else 0, code[c], epi, M, n, k, q, s, t, sw, r, C, self.ws)
        torch.cuda.synchronize()
        # the rows: half an integer step of the rounding, and the norm's error where there is one
        y = H.to_f64(x) if gain is None else O.rmsnorm(H.to_f64(x), H.to_f64(gain), 1e-5)
        ai, sa = q.double().cpu().numpy(), s.double().cpu().numpy()[:, None]
        assert (np.abs(ai * sa - y) <= np.abs(y).max(1, keepdims=True) * (0.5 / 127 + 2 * (k / 2 + 16) * 2.0 ** -24)).all(), name
        # the product: relative 3 2^-24 of the terms behind the exact sum; SwiGLU and the output's rounding
        # (the integers' sums are exact in 64 bits too, zeros among them)
        z = (ai @ wi.T) * sa * sw.double().cpu().numpy()
        if epi == B.PS_EPI_SWIGLU:
            z = z.reshape(M, -1, 2, 32)
            gate, up = z[:, :, 0].reshape(M, -1), z[:, :, 1].reshape(M, -1)
            ref = O.silu(gate) * up
            b = np.abs(ref) * (np.abs(gate) + 24) * 2.0 ** -22
        elif r is not None:
            ref = z + H.to_f64(r)
            b = 5 * 2.0 ** -24 * (np.abs(z) + np.abs(ref) + np.abs(H.to_f64(r)))
        else:
            ref, b = z, 4 * 2.0 ** -24 * np.abs(z)
        b = b + (2.0 ** -8 * np.abs(ref) if c == torch.bfloat16 else 0) + 1e-30
        assert (np.abs(H.to_f64(C) - ref) <= b).all(), name
        return C

    def step(self, pool, seqs, new, x, decode):
        s, rows = self.s, x.shape[0]
        bf = torch.bfloat16
        qkv = self.linear("qkv", x, B.PS_EPI_STORE, bf, gain=self.g[0])
        q, o = H.empty((rows, s.n_q, s.head_dim), "bf16"), H.empty((rows, s.n_q * s.head_dim), "bf16")
        B.op_rope_kvwrite(pool.kv, 0, seqs, new, qkv, q, pool.ws)
        if decode:
            B.op_decode_attention(pool.kv, 0, seqs, q, o, pool.ws)
        else:
            B.op_attention(pool.kv, 0, seqs, new, q, o, pool.ws)
        pool.kv.commit(seqs, new)
        torch.cuda.synchronize()
        r0 = 0
        for i, n in zip(seqs, new):
            k, v = pool.gather(i)
            pos = np.arange(len(k) - n, len(k))
            x3 = H.to_f64(qkv)[r0:r0 + n].reshape(n, -1, s.head_dim)
            qf = O.rope(x3[:, :s.n_q], pos, s.theta)
            m = np.abs(x3[:, :s.n_q])
            assert (np.abs(H.to_f64(q)[r0:r0 + n] - qf) <= 2.0 ** -8 * np.abs(qf) + 2.0 ** -22 * (m + np.roll(m, s.head_dim // 2, -1))).all()
            # what the pool holds: half an e4m3 step, or a whole one of the last scale where it grew later
            kf = O.rope(x3[:, s.n_q:s.n_q + s.n_kv], pos, s.theta)
            for have, want in ((k[pos], kf), (v[pos], x3[:, s.n_q + s.n_kv:])):
                assert (np.abs(have - want) <= 2.0 ** -3 * np.abs(want) + 2.0 ** -9 * np.abs(have).max() / 224).all()
            check(H.to_f64(o)[r0:r0 + n].reshape(n, s.n_q, -1), H.to_f64(q)[r0:r0 + n], k, v, pos, "attention")
            r0 += n
        h = self.linear("o", o, B.PS_EPI_RESIDUAL, torch.float32, r=x)
        m = self.linear("gu", h, B.PS_EPI_SWIGLU, bf, gain=self.g[1])
        return self.linear("down", m, B.PS_EPI_RESIDUAL, bf, r=h)


@pytest.mark.parametrize("n_q,n_kv,hd,ffn", [(8, 2, 128, 512), (12, 4, 64, 704)])
def test_prompts_then_decode_steps(n_q, n_kv, hd, ffn):
    rng = np.random.default_rng(21)
    shp = shape(n_q, n_kv, hd, ffn=ffn)
    layer, pool = Int8Layer(shp, rng), Pool8(shp, 32, max_pages=16)
    new = [70, 33, 1]
    seqs = pool.seqs([n + 8 for n in new])
    x = H.to_dev(gen.to_storage(rng.standard_normal((sum(new), shp.hidden)).astype(np.float32), "bf16"), "bf16")
    y = layer.step(pool, seqs, new, x, decode=False)
    last = y[[69, 102, 103]].contiguous()
    for _ in range(3):
        last = layer.step(pool, seqs, [1] * 3, last, decode=True)
    assert torch.isfinite(last.float()).all()
