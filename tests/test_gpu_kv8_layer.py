"""Layer, mixed and model calls over an e4m3 KV pool (GPU), run as a serving loop runs them.

The reference evaluates the layer in 64 bits with the keys and values that the pool holds after the call (ps_kv_gather,
whose numbers tests/test_gpu_kv8.py pins), so what is left is the bf16 layer's own rounding: the normwise bound of the
16-bit layer tests. The keys and values themselves are held against the oracle's: half a step of e4m3 is 2^-4 of a value
(2^-10 2^e below the normal numbers), less than a whole step of the last scale where a page's scale grew; bf16 rounding
on the way to them is 2e-2 + 1e-2 of a value, the bound of the bf16 stages.
"""
import numpy as np
import pytest

from oracle import layer as O
from synth import gen
from synth.configs import CONFIGS, LayerShape, Workload
from tests import helpers as H

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2608_21719_amd import binding as B  # noqa: E402

SHAPES = {
    "8b": CONFIGS["llama8b_prefill"].shape,
    "g4": LayerShape(512, 4, 1, 128, 1024, 1e-5, 500000.0, "bf16"),
    "g3_hd64": LayerShape(768, 12, 4, 64, 512, 1e-5, 10000.0, "bf16"),
    "g1": LayerShape(512, 4, 4, 128, 1024, 1e-5, 10000.0, "bf16"),
}


class Loop:
    """One layer over an e4m3 pool, with the inputs' 64-bit values on the side."""

    def __init__(self, name, n_pages=160, max_seqs=12, max_pages=80, max_rows=1024):
        self.shape = SHAPES[name]
        self.wl = Workload("kv8_" + name, 41, self.shape, prefill_seqs=1, prefill_tokens=16)
        w = gen.layer_weights(self.wl, 0)
        self.wf, self.dev = H.weights_f64(w, "bf16"), H.DeviceLayer(w, "bf16")
        cfg = B.make_cfg(self.shape)
        self.mem = H.nan_filled_bytes(B.KV8.pool_bytes(cfg, 1, n_pages))
        self.kv = B.KV8(cfg, 1, n_pages, max_seqs, max_pages, self.mem, 11)
        self.layer = B.Layer(cfg)
        self.ws = H.workspace(B.Layer.workspace_bytes(cfg, max_rows, max_seqs, max_pages))
        self.step = 0

    def open(self, n):
        s = self.kv.open()
        self.kv.alloc(s, n)
        return s

    def rows(self, n):
        self.step += 1
        return gen.prefill_input(self.wl, n, step=self.step)

    def gather(self, s):
        n = self.kv.seq_len(s)
        k, v = (H.empty((n, self.shape.n_kv, self.shape.head_dim), "bf16") for _ in range(2))
        self.kv.gather(0, s, k, v, self.ws)
        torch.cuda.synchronize()
        return H.to_f64(k), H.to_f64(v)

    def check(self, got, x, seqs, n_tok, what):
        """After the call's commit: the outputs from the pool's numbers, and the new numbers from the layer's keys."""
        sh, w, r0 = self.shape, self.wf, 0
        for s, n in zip(seqs, n_tok):
            xs = gen.widen(x, "bf16")[r0:r0 + n]
            K, V = self.gather(s)
            pos = np.arange(len(K) - n, len(K))
            xn = O.rmsnorm(xs, w["attn_norm"], sh.eps)
            q = O.rope(O.linear(xn, w["wq"]).reshape(n, sh.n_q, sh.head_dim), pos, sh.theta)
            for have, want in ((K, O.rope(O.linear(xn, w["wk"]).reshape(n, sh.n_kv, sh.head_dim), pos, sh.theta)),
                               (V, O.linear(xn, w["wv"]).reshape(n, sh.n_kv, sh.head_dim))):
                top = np.abs(have).max()
                assert (np.abs(have[pos] - want) <= 2.0 ** -3 * np.abs(want) + 2.0 ** -9 * 2 * top / 256 + 2e-2).all(), what
            o = O.attention(q, K, V, pos).reshape(n, -1)
            h = xs + O.linear(o, w["wo"])
            hn = O.rmsnorm(h, w["ffn_norm"], sh.eps)
            ref = h + O.linear(O.silu(O.linear(hn, w["wg"])) * O.linear(hn, w["wu"]), w["wd"])
            mx, rms = H.normwise(got[r0:r0 + n], ref)
            assert mx <= H.NORMWISE_TOL and rms <= H.NORMWISE_TOL, f"{what}, sequence {s}: {mx:.2e} {rms:.2e}"
            r0 += n

    def prefill(self, seqs, n_tok, what):
        x = self.rows(sum(n_tok))
        out = H.empty((sum(n_tok), self.shape.hidden), "bf16")
        self.layer.prefill(self.dev.w, self.kv, 0, seqs, n_tok, H.to_dev(x, "bf16"), out, self.ws)
        self.kv.commit(seqs, n_tok)
        self.check(H.to_f64(out), x, seqs, n_tok, what)

    def decode(self, seqs, what):
        x = self.rows(len(seqs))
        out = H.empty((len(seqs), self.shape.hidden), "bf16")
        self.layer.decode_step(self.dev.w, self.kv, 0, B.PS_PHASE_THINK, seqs, H.to_dev(x, "bf16"), out, self.ws)
        self.kv.commit(seqs, [1] * len(seqs))
        self.check(H.to_f64(out), x, seqs, [1] * len(seqs), what)

    def mixed(self, chunk, tok, dec, what):
        n = sum(tok) + len(dec)
        x = self.rows(n)
        out = H.empty((n, self.shape.hidden), "bf16")
        self.layer.mixed_step(self.dev.w, self.kv, 0, chunk, tok, dec, H.to_dev(x, "bf16"), out, self.ws)
        seqs, new = chunk + dec, tok + [1] * len(dec)
        self.kv.commit(seqs, new)
        self.check(H.to_f64(out), x, seqs, new, what)


@pytest.mark.parametrize("name", sorted(SHAPES))
def test_a_serving_loop(name):
    """Prompts, decode steps, a chunk behind a cached prefix, a mixed step, and a handoff to another pool."""
    t = Loop(name)
    a, b, c = t.open(120), t.open(60), t.open(400)
    t.prefill([a, b], [70, 33], "prompts")
    for i in range(3):
        t.decode([a, b], f"decode step {i}")
    t.prefill([c], [90], "first chunk")
    t.prefill([c], [37], "second chunk")
    t.mixed([c], [100], [b, a], "mixed step")
    t.decode([c], "decode after chunks")
    dst = B.KV8(t.kv.cfg, 1, 40, 4, 40, H.nan_filled_bytes(B.KV8.pool_bytes(t.kv.cfg, 1, 40)), 5)
    s = dst.open()
    dst.alloc(s, 260)
    B.kv_transfer(t.kv, c, dst, s, t.ws)
    t.kv.free(c)
    t.kv, t.pool_before = dst, t.kv
    t.decode([s], "decode after the handoff")


def test_a_forked_mixed_step():
    """Decode rows on the second stream beside the chunk rows."""
    t = Loop("8b", n_pages=420, max_rows=2200, max_pages=140)
    dec = [t.open(40) for _ in range(4)]
    t.prefill(dec, [20, 17, 33, 16], "contexts")
    c = t.open(2100)
    plan = t.layer.step_plan(t.kv, [c], [2048], dec, t.ws.numel())
    x = t.rows(2052)
    out = H.empty((2052, t.shape.hidden), "bf16")
    t.layer.mixed_step(t.dev.w, t.kv, 0, [c], [2048], dec, H.to_dev(x, "bf16"), out, t.ws)
    t.kv.commit([c] + dec, [2048, 1, 1, 1, 1])
    assert plan.forks == 1
    t.check(H.to_f64(out)[2048:], x[2048:], dec, [1] * 4, "forked decode rows")


def test_model_over_an_e4m3_pool():
    """Two layers with embedding and LM head: logits from the pool's numbers, prompt then greedy decode."""
    sh, vocab, n_layers = SHAPES["g4"], 512, 2
    wl = Workload("kv8_model", 42, sh, prefill_seqs=1, prefill_tokens=16, n_layers=n_layers, vocab=vocab)
    ws_ = [gen.layer_weights(wl, i) for i in range(n_layers)]
    wf = [H.weights_f64(w, "bf16") for w in ws_]
    dev = [H.DeviceLayer(w, "bf16") for w in ws_]
    rng = np.random.default_rng(4)
    emb, head = (gen.to_storage((rng.standard_normal((vocab, sh.hidden)) * s).astype(np.float32), "bf16") for s in (1.0, 0.05))
    fn = gen.to_storage((1 + 0.02 * rng.standard_normal(sh.hidden)).astype(np.float32), "bf16")
    cfg = B.make_cfg(sh)
    emb_d, fn_d, head_d = H.to_dev(emb, "bf16"), H.to_dev(fn, "bf16"), H.to_dev_w(head, "bf16")
    model = B.Model(cfg, [d.w for d in dev], vocab, emb_d, fn_d, head_d)
    kv = B.KV8(cfg, n_layers, 32, 4, 16, H.nan_filled_bytes(B.KV8.pool_bytes(cfg, n_layers, 32)), 9)
    ws = H.workspace(B.Model.workspace_bytes(cfg, vocab, 128, 4, 16))
    lens = [50, 21]
    seqs = []
    for n in lens:
        seqs.append(kv.open())
        kv.alloc(seqs[-1], n + 4)
    tokens = [rng.integers(0, vocab, n).astype(np.int32) for n in lens]
    nxt = torch.empty(2, dtype=torch.int32, device="cuda")
    logits = H.empty((2, vocab), "f32")

    def reference(i, step_tok):
        x = O.embed(gen.widen(emb, "bf16"), step_tok)
        n = len(step_tok)
        for layer in range(n_layers):
            L = kv.seq_len(seqs[i])
            k, v = (H.empty((L, sh.n_kv, sh.head_dim), "bf16") for _ in range(2))
            kv.gather(layer, seqs[i], k, v, ws)
            torch.cuda.synchronize()
            K, V, pos, w = H.to_f64(k), H.to_f64(v), np.arange(L - n, L), wf[layer]
            q = O.rope(O.linear(O.rmsnorm(x, w["attn_norm"], sh.eps), w["wq"]).reshape(n, sh.n_q, sh.head_dim), pos, sh.theta)
            h = x + O.linear(O.attention(q, K, V, pos).reshape(n, -1), w["wo"])
            hn = O.rmsnorm(h, w["ffn_norm"], sh.eps)
            x = h + O.linear(O.silu(O.linear(hn, w["wg"])) * O.linear(hn, w["wu"]), w["wd"])
        return O.lm_logits(x[-1:], gen.widen(fn, "bf16"), gen.widen(head, "bf16"), sh.eps)

    def check(step_tokens, what):
        got = H.to_f64(logits)
        for i in range(2):
            ref = reference(i, step_tokens[i])
            mx, rms = H.normwise(got[i:i + 1], ref)
            assert mx <= 2 * H.NORMWISE_TOL and rms <= 2 * H.NORMWISE_TOL, f"{what} {i}: {mx:.2e} {rms:.2e}"  # two layers

    model.prefill(kv, seqs, lens, torch.from_numpy(np.concatenate(tokens)).cuda(), nxt, ws, logits)
    kv.commit(seqs, lens)
    check(tokens, "prompt")
    for step in range(3):
        cur = nxt.clone()
        model.decode_step(kv, B.PS_PHASE_ANSWER, seqs, cur, nxt, ws, logits)
        kv.commit(seqs, [1, 1])
        check([cur.cpu().numpy()[i:i + 1] for i in range(2)], f"step {step}")
