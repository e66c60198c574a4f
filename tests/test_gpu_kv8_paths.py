"""Paths of the e4m3 KV pool that take many splits, many pages or long contexts (GPU).

References and bounds are those of tests/test_gpu_kv8.py (storage and attention) and tests/test_gpu_kv8_layer.py (layer
calls, on the numbers that ps_kv_gather returns).
"""
import numpy as np
import pytest

from oracle import kv8 as K
from oracle import layer as O
from synth import gen
from synth.configs import LayerShape
from tests import helpers as H
from tests.kv8_helpers import bf16, shape, wide

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2608_21719_amd import binding as B  # noqa: E402
from tests import test_gpu_kv8_layer as TL  # noqa: E402
from tests.test_gpu_kv8 import Pool8, check  # noqa: E402


# ---------------------------------------------------------------- decode over many splits
@pytest.mark.parametrize("n_q,n_kv,hd", [(8, 2, 128), (3, 1, 64), (20, 1, 128)])
@pytest.mark.parametrize("n,split", [(2047, 2), (2048, 2), (9000, 2), (9000, 1)])  # 64, 65, 282 and 563 splits
@pytest.mark.parametrize("peak,height", [("none", 0), ("first", 1), ("middle", 1), ("last", 1), ("first", 4), ("last", 4)])
def test_more_splits_than_a_batch_of_the_combine(n_q, n_kv, hd, n, split, peak, height):
    """The row's maximum in the first, a later or the last batch of 64 splits: as heavy as all others, or far above them."""
    rng = np.random.default_rng(n + split)
    p = Pool8(shape(n_q, n_kv, hd), n // 16 + 3, max_seqs=2, max_pages=n // 16 + 2, rows=64)
    (s,) = p.seqs([n + 1])
    q = wide(bf16(rng, (1, n_q, hd)))
    k = rng.standard_normal((n + 1, n_kv, hd)).astype(np.float32) * 0.3
    if peak != "none":
        at, G = {"first": 5, "middle": n // 2, "last": n - 3}[peak], n_q // n_kv
        k[at] = q.reshape(n_kv, G, hd).mean(1) * G * height * np.log(n) / np.sqrt(hd)  # scores near height ln n
    kv = [gen.to_storage(k, "bf16"), bf16(rng, (n + 1, n_kv, hd))]
    p.append([s], [n + 1], *kv)
    pool = p.gather(s)
    p.kv.truncate(s, n)
    o = H.empty((1, n_q * hd), "bf16")
    B.op_decode_attention(p.kv, 0, [s], H.to_dev(gen.to_storage(q.astype(np.float32), "bf16"), "bf16"), o,
                          H.workspace(1 << 24), split)
    torch.cuda.synchronize()
    check(H.to_f64(o).reshape(1, n_q, hd), q, *pool, np.array([n]), f"{n} tokens by {split} pages, {peak} {height}")


# ---------------------------------------------------------------- writes of more than 128 pages
def mixed_lengths(rng, n):
    return [int(x) for x in rng.integers(1, 32, n)], [int(x) for x in rng.integers(1, 41, n)]


@pytest.mark.parametrize("n_kv,hd", [(2, 64), (3, 128)])
def test_append_of_many_pages_is_the_oracle_bit_for_bit(n_kv, hd):
    """140 sequences a call, starting inside pages, of mixed lengths and of one row each, with magnitudes that grow."""
    rng = np.random.default_rng(31)
    n = 140
    past, new = mixed_lengths(rng, n)
    calls = [past, new, [1] * n, [1] * n, new[::-1]]
    total = [sum(c[i] for c in calls) for i in range(n)]
    p = Pool8(shape(n_kv, n_kv, hd), sum((t + 15) // 16 for t in total) + 2, max_seqs=n, max_pages=16)
    seqs = p.seqs(total)
    ref = [[K.Sequence(n_kv, hd) for _ in range(2)] for _ in range(n)]
    for step, c in enumerate(calls):
        mag = 2.0 ** (rng.integers(-6, 7, (2, sum(c), n_kv, 1)) + 3 * step)
        kv = [gen.to_storage((wide(bf16(rng, (sum(c), n_kv, hd))) * m).astype(np.float32), "bf16") for m in mag]
        p.append(seqs, c, *kv)
        at = np.cumsum([0] + c)
        for i in range(n):
            for j in (0, 1):
                ref[i][j].append(wide(kv[j][at[i]:at[i + 1]]))
    for s, r in zip(seqs, ref):
        k, v = p.gather(s)
        assert np.array_equal(k, r[0].values()) and np.array_equal(v, r[1].values())


@pytest.mark.parametrize("n_q,n_kv,hd", [(8, 2, 128), (6, 3, 64), (20, 1, 128)])
def test_rope_write_of_many_pages_is_that_of_few(n_q, n_kv, hd):
    """One call of 140 sequences against calls of 20, whose work lists are kernel arguments: the same bytes and rows."""
    rng = np.random.default_rng(32)
    n = 140
    past, new = mixed_lengths(rng, n)
    shp = shape(n_q, n_kv, hd)
    pools = [Pool8(shp, 6 * n, max_seqs=n, max_pages=6, seed=seed) for seed in (1, 2)]
    seqs = [p.seqs([a + b + 2 for a, b in zip(past, new)]) for p in pools]
    kv = [bf16(rng, (sum(past), n_kv, hd), 0.05) for _ in range(2)]
    for p, s in zip(pools, seqs):
        p.append(s, past, *kv)
    for step, c in enumerate((new, [1] * n, [1] * n)):  # the last two: a row each, growing
        qkv = H.to_dev(bf16(rng, (sum(c), n_q + 2 * n_kv, hd), 2.0 ** (3 * step)), "bf16")
        at = [int(x) for x in np.cumsum([0] + c)]
        q = [H.empty((sum(c), n_q, hd), "bf16") for _ in range(2)]
        B.op_rope_kvwrite(pools[0].kv, 0, seqs[0], c, qkv, q[0], pools[0].ws)
        for i in range(0, n, 20):
            B.op_rope_kvwrite(pools[1].kv, 0, seqs[1][i:i + 20], c[i:i + 20], qkv[at[i]:], q[1][at[i]:], pools[1].ws)
        for p, s in zip(pools, seqs):
            p.kv.commit(s, c)
        torch.cuda.synchronize()
        assert np.array_equal(H.bits(q[0]), H.bits(q[1]))
        for a, b in zip(*seqs):
            for x, y in zip(pools[0].gather(a), pools[1].gather(b)):
                assert np.array_equal(x, y)


# ---------------------------------------------------------------- layer calls
SHAPES = {**TL.SHAPES, "g3_hd64": LayerShape(768, 12, 4, 64, 4096, 1e-5, 10000.0, "bf16")}


class Loop(TL.Loop):
    def __init__(self, name, **kw):
        before, TL.SHAPES = TL.SHAPES, SHAPES
        try:
            super().__init__(name, **kw)
        finally:
            TL.SHAPES = before

    def context(self, n, room):
        """A sequence of n random tokens in the pool, with room for more."""
        sh, s = self.shape, self.open(n + room)
        rng = np.random.default_rng(n)
        self.kv.append(0, [s], [n], *(H.to_dev(bf16(rng, (n, sh.n_kv, sh.head_dim)), "bf16") for _ in range(2)), self.ws)
        self.kv.commit([s], [n])
        return s

    def check_rows(self, got, x, s, pos, what):
        """Rows of one sequence at the positions `pos` of those that the call added, as `check`."""
        sh, w = self.shape, self.wf
        xs = gen.widen(x, "bf16")
        Kp, V = self.gather(s)
        q = O.rope(O.linear(O.rmsnorm(xs, w["attn_norm"], sh.eps), w["wq"]).reshape(len(pos), sh.n_q, sh.head_dim), pos, sh.theta)
        h = xs + O.linear(O.attention(q, Kp, V, pos).reshape(len(pos), -1), w["wo"])
        hn = O.rmsnorm(h, w["ffn_norm"], sh.eps)
        ref = h + O.linear(O.silu(O.linear(hn, w["wg"])) * O.linear(hn, w["wu"]), w["wd"])
        mx, rms = H.normwise(got, ref)
        assert mx <= H.NORMWISE_TOL and rms <= H.NORMWISE_TOL, f"{what}: {mx:.2e} {rms:.2e}"


@pytest.mark.parametrize("name", ["8b", "g4", "g1", "g3_hd64"])
@pytest.mark.parametrize("n", [37, 64])
def test_a_chunk_whose_walk_is_cut(name, n):
    """A layer call behind 6000 tokens: partial results of several workgroups a row, laid over the call's own buffers."""
    t = Loop(name, n_pages=420, max_pages=400, max_rows=128)
    s, other = t.context(6000, n), t.open(60)
    assert t.layer.step_plan(t.kv, [s], [n], [], t.ws.numel()).split_walks > 0
    t.prefill([s], [n], "cut")
    t.prefill([other], [20], "whole")
    t.kv.truncate(s, 6000)
    plan = t.layer.step_plan(t.kv, [s], [n], [other], t.ws.numel())
    assert plan.split_walks > 0
    t.mixed([s], [n], [other], "cut beside a decode row")


def test_a_forked_step_with_cut_walks():
    """Chunk rows behind a long context beside decode rows on the second stream: every row of the step."""
    t = Loop("8b", n_pages=1000, max_rows=1100, max_seqs=40, max_pages=460)
    dec = [t.context(30 + 7 * i, 1) for i in range(32)]
    long, fresh = t.context(7000, 200), t.open(824)
    seqs, new = [long, fresh], [200, 824]
    plan = t.layer.step_plan(t.kv, seqs, new, dec, t.ws.numel())
    assert plan.forks == 1 and plan.split_walks > 0
    x = t.rows(1024 + 32)
    out = H.empty((1024 + 32, t.shape.hidden), "bf16")
    t.layer.mixed_step(t.dev.w, t.kv, 0, seqs, new, dec, H.to_dev(x, "bf16"), out, t.ws)
    t.kv.commit(seqs + dec, new + [1] * 32)
    got = H.to_f64(out)
    t.check_rows(got[:200], x[:200], long, np.arange(7000, 7200), "rows behind the long context")
    t.check_rows(got[200:1024], x[200:1024], fresh, np.arange(824), "rows of the new prompt")
    t.check(got[1024:], x[1024:], dec, [1] * 32, "decode rows")


def test_a_forked_step_of_many_chunk_rows():
    t = Loop("8b", n_pages=420, max_rows=2200, max_pages=140)
    dec = [t.context(n, 1) for n in (20, 17, 33, 16)]
    c = t.open(2048)
    assert t.layer.step_plan(t.kv, [c], [2048], dec, t.ws.numel()).forks == 1
    x = t.rows(2052)
    out = H.empty((2052, t.shape.hidden), "bf16")
    t.layer.mixed_step(t.dev.w, t.kv, 0, [c], [2048], dec, H.to_dev(x, "bf16"), out, t.ws)
    t.kv.commit([c] + dec, [2048, 1, 1, 1, 1])
    got, pos = H.to_f64(out), np.r_[0:70, 1000:1064, 1984:2048]
    t.check_rows(got[pos], x[pos], c, pos, "chunk rows")
    t.check(got[2048:], x[2048:], dec, [1] * 4, "decode rows")
