"""The e4m3 KV pool on the GPU: what is stored, and attention over it, against 64-bit definitions.

Storage (oracle/kv8.py). ps_kv_append rounds bf16 values that the oracle has exactly, so gather has to return the
oracle's numbers bit for bit. ps_op_rope_kvwrite rotates in fp32 first: each product and sum of y = x1 c - x2 s is off by
at most 3 half steps of fp32 of |x1| + |x2| (two roundings, and the cosine's), so a stored number may be the oracle's
neighbour where the value lies within that of a border. The pool's scale can then differ only where the maximum does.

Attention is checked on the numbers that gather returns. With P rounded to bf16 (half a step is 2^-8 of a value) both in
the product and the normaliser, and the result rounded once more:
  |o - ref| <= 2^-8 (S + 2 |ref|) (1 + 2^-6) + d S,  S = sum p |v|,
d = 2 x the relative error of an exponential: fp32 sums of hd products, hd 2^-24 max |q| (sum |k|) / sqrt(hd), and 2^-20
for the exponential and the rescales.
"""
import numpy as np
import pytest

from oracle import kv8 as K
from oracle import layer as O
from synth import gen
from tests import helpers as H
from tests.kv8_helpers import PAGE, bf16, shape, wide

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2608_21719_amd import binding as B  # noqa: E402


class Pool8:
    """An e4m3 pool full of NaN bytes, page order shuffled, with its workspace."""

    def __init__(self, shp, n_pages, max_seqs=8, max_pages=None, n_layers=1, seed=3, rows=4096):
        self.shape, self.cfg = shp, B.make_cfg(shp)
        self.mem = H.nan_filled_bytes(B.KV8.pool_bytes(self.cfg, n_layers, n_pages))
        self.kv = B.KV8(self.cfg, n_layers, n_pages, max_seqs, max_pages or n_pages, self.mem, seed)
        self.ws = H.workspace(B.Layer.workspace_bytes(self.cfg, rows, max_seqs, max_pages or n_pages))

    def seqs(self, capacities):
        out = []
        for n in capacities:
            s = self.kv.open()
            if n:
                self.kv.alloc(s, n)
            out.append(s)
        return out

    def gather(self, seq, layer=0):
        n = self.kv.seq_len(seq)
        k, v = (H.empty((max(n, 1), self.shape.n_kv, self.shape.head_dim), "bf16") for _ in range(2))
        self.kv.gather(layer, seq, k, v, self.ws)
        torch.cuda.synchronize()
        return H.to_f64(k)[:n], H.to_f64(v)[:n]

    def append(self, seqs, ns, k, v, layer=0, commit=True):
        self.kv.append(layer, seqs, ns, H.to_dev(k, "bf16"), H.to_dev(v, "bf16"), self.ws)
        if commit:
            self.kv.commit(seqs, ns)


HEADS = [(32, 8, 128), (8, 8, 64), (4, 1, 128), (6, 2, 64), (20, 1, 128)]


# ---------------------------------------------------------------- storage
@pytest.mark.parametrize("n_q,n_kv,hd", [(8, 8, 128), (6, 3, 64), (4, 1, 128)])
@pytest.mark.parametrize("calls", [
    [[1], [1], [1], [1]], [[16], [16]], [[5], [30], [1], [12]], [[40, 3, 17], [1, 1, 1], [9, 20, 15]],
    [[1] * 70, [15] * 70, [1] * 70]])
def test_append_and_gather_are_the_oracle_bit_for_bit(n_q, n_kv, hd, calls):
    rng = np.random.default_rng(5)
    n = len(calls[0])
    total = [sum(c[i] for c in calls) for i in range(n)]
    p = Pool8(shape(n_q, n_kv, hd), sum((t + 15) // 16 for t in total) + 2, max_seqs=n, max_pages=16)
    seqs = p.seqs(total)
    ref = [[K.Sequence(n_kv, hd) for _ in range(2)] for _ in range(n)]
    for c in calls:
        # magnitudes that wander over 2^-12 .. 2^12, so that scales grow inside pages
        kv = [bf16(rng, (sum(c), n_kv, hd)) for _ in range(2)]
        mag = 2.0 ** rng.integers(-12, 13, (2, sum(c), n_kv, 1))
        kv = [gen.to_storage((wide(x) * m).astype(np.float32), "bf16") for x, m in zip(kv, mag)]
        p.append(seqs, c, *kv)
        r0 = 0
        for i, t in enumerate(c):
            for j in (0, 1):
                ref[i][j].append(wide(kv[j])[r0:r0 + t])
            r0 += t
    for i, s in enumerate(seqs):
        k, v = p.gather(s)
        assert np.array_equal(k, ref[i][0].values()) and np.array_equal(v, ref[i][1].values())


def test_special_values():
    """Zeros, the largest and smallest bf16 numbers, infinities and NaN: stored as documented, each in its own page."""
    hd, n_kv = 64, 2
    p = Pool8(shape(4, n_kv, hd), 16)
    x = np.zeros((6 * 16, n_kv, hd), dtype=np.float32)
    x[16:32] = 3.3895314e38
    x[32:48] = 1e-38
    x[48:64, :, ::2] = 5.0
    x[50, 0, 3], x[51, 0, 4], x[52, 0, 5] = np.inf, -np.inf, np.nan
    x[64:80] = np.linspace(-448, 448, hd, dtype=np.float32)
    x[80:96, :, 0], x[80:96, :, 1] = 1.0, 2.0 ** -18
    bits = gen.to_storage(x, "bf16")
    (s,) = p.seqs([96])
    p.append([s], [96], bits, bits)
    ref = K.Sequence(n_kv, hd)
    ref.append(wide(bits))
    for got in p.gather(s):
        assert np.array_equal(got, ref.values(), equal_nan=True)
        assert np.isnan(got[50, 0, 3]) and np.isnan(got[51, 0, 4]) and np.isnan(got[52, 0, 5])
        assert np.isnan(got).sum() == 3 and (got[48:64, 1, ::2] == 5.0).all()


def test_truncate_then_append_keeps_the_scale_of_what_stays():
    rng = np.random.default_rng(6)
    p = Pool8(shape(4, 2, 128), 8)
    (s,) = p.seqs([40])
    ref = [K.Sequence(2, 128) for _ in range(2)]
    for n, keep in ((20, 18), (10, 16), (9, None)):
        kv = [bf16(rng, (n, 2, 128), 2.0 ** rng.integers(-4, 5)) for _ in range(2)]
        p.append([s], [n], *kv)
        for r, x in zip(ref, kv):
            r.append(wide(x))
        if keep:
            p.kv.truncate(s, keep)
            for r in ref:
                r.truncate(keep)
    for got, r in zip(p.gather(s), ref):
        assert np.array_equal(got, r.values())


def test_slots_and_pages_outside_the_call_stay_as_they_are():
    rng = np.random.default_rng(7)
    n_kv, hd = 2, 128
    p = Pool8(shape(8, n_kv, hd), 12)
    a, b = p.seqs([37, 64])
    p.append([b], [50], bf16(rng, (50, n_kv, hd)), bf16(rng, (50, n_kv, hd)))
    before = p.mem.clone()
    p.append([a], [37], bf16(rng, (37, n_kv, hd)), bf16(rng, (37, n_kv, hd)))
    torch.cuda.synchronize()
    blocks = 12 * n_kv * 2 * PAGE * hd
    mine = set(p.kv.block_table(a))
    old, new = (m[:blocks].view(12, n_kv, 2, PAGE * hd).cpu().numpy() for m in (before, p.mem))
    for page in range(12):
        if page not in mine:
            assert np.array_equal(old[page], new[page])
    # of a's last page, tokens 5 .. 15 are not written
    last = p.kv.block_table(a)[2]
    tok = np.arange(PAGE)[:, None]
    dim = np.arange(hd)[None]
    off = (dim // 16 * 256 + tok * 16 + dim % 16,
           dim // 64 * 1024 + (tok // 4 * 16 + dim % 16) * 16 + dim % 64 // 16 * 4 + tok % 4)
    for i in (0, 1):
        assert (new[last][:, i][:, off[i][5:]] == 255).all()
        assert (new[last][:, i][:, off[i][:5]] != 255).all()


@pytest.mark.parametrize("n_q,n_kv,hd", HEADS)
@pytest.mark.parametrize("past,new", [([0], [1]), ([0, 0], [33, 16]), ([5, 31, 16, 0], [1, 1, 1, 1]),
                                      ([7, 0, 40], [60, 100, 5]), ([1000], [3])])
def test_rope_write(n_q, n_kv, hd, past, new):
    rng = np.random.default_rng(8)
    shp = shape(n_q, n_kv, hd)
    p = Pool8(shp, sum((a + b + 15) // 16 for a, b in zip(past, new)) + 1, max_pages=80)
    seqs = p.seqs([a + b for a, b in zip(past, new)])
    ref = [[K.Sequence(n_kv, hd) for _ in range(2)] for _ in seqs]
    for s, n, r in zip(seqs, past, ref):
        if n:
            kv = [bf16(rng, (n, n_kv, hd), 0.3) for _ in range(2)]
            p.append([s], [n], *kv)
            for x, y in zip(r, kv):
                x.append(wide(y))
    rows = sum(new)
    qkv = bf16(rng, (rows, n_q + 2 * n_kv, hd))
    q = H.empty((rows, n_q, hd), "bf16")
    B.op_rope_kvwrite(p.kv, 0, seqs, new, H.to_dev(qkv, "bf16"), q, p.ws)
    p.kv.commit(seqs, new)
    torch.cuda.synchronize()
    x = wide(qkv)
    q = H.to_f64(q)
    r0 = 0
    for s, a, n, r in zip(seqs, past, new, ref):
        pos = np.arange(a, a + n)
        rot = O.rope(x[r0:r0 + n, :n_q + n_kv], pos, shp.theta)
        mag = np.abs(x[r0:r0 + n, :n_q + n_kv])
        mag = mag + np.roll(mag, hd // 2, axis=-1)   # |x1| + |x2|
        err = 3 * 2.0 ** -24 * mag
        assert (np.abs(q[r0:r0 + n] - rot[:, :n_q]) <= 2.0 ** -8 * np.abs(rot[:, :n_q]) + 1.01 * err[:, :n_q]).all()
        k, v = p.gather(s)
        r[1].append(x[r0:r0 + n, n_q + n_kv:])
        assert np.array_equal(v, r[1].values())
        # keys: the oracle's numbers for the exact rotation, or for one moved by the rounding error
        stored = []
        for off in (-1, 0, 1):
            t = K.Sequence(n_kv, hd)
            t.len, t.pages = r[0].len, [[_copy(y) for y in pg] for pg in r[0].pages]
            t.append(rot[:, n_q:] + off * err[:, n_q:] * np.sign(rot[:, n_q:]))
            stored.append(t.values())
        lo, near, hi = stored
        assert ((k == near) | (k == lo) | (k == hi)).all()
        assert (k != near).mean() < 1e-3
        r0 += n


def _copy(p):
    q = K.Page(p.hd)
    q.e, q.x = p.e, p.x.copy()
    return q


def test_transfer_moves_bytes_and_scales():
    rng = np.random.default_rng(9)
    shp = shape(8, 4, 64)
    src, dst = Pool8(shp, 20, n_layers=3, seed=1), Pool8(shp, 33, n_layers=3, seed=2)
    (s,) = src.seqs([100])
    for layer in range(3):
        src.append([s], [90], bf16(rng, (90, 4, 64), 10.0 ** layer), bf16(rng, (90, 4, 64)), layer, commit=layer == 2)
    (d,) = dst.seqs([128])
    B.kv_transfer(src.kv, s, dst.kv, d, dst.ws)
    assert dst.kv.seq_len(d) == 90
    for layer in range(3):
        for a, b in zip(src.gather(s, layer), dst.gather(d, layer)):
            assert np.array_equal(a, b)


# ---------------------------------------------------------------- attention
def bound(q, k, v, pos):
    """Reference output and the bound of the module's docstring. q [T, n_q, hd], k, v [L, n_kv, hd]."""
    hd = q.shape[-1]
    o, prob = O.attention(q, k, v, pos, return_probs=True)
    G = q.shape[1] // k.shape[1]
    S = np.stack([prob[:, h] @ np.abs(v[:, h // G]) for h in range(q.shape[1])], axis=1)
    qk = np.abs(q).max() * np.abs(k).sum(-1).max() / np.sqrt(hd)
    d = 2 * (hd * 2.0 ** -24 * qk + 2.0 ** -20)
    return o, 2.0 ** -8 * (S + 2 * np.abs(o)) * (1 + 2.0 ** -6) + d * S


def check(got, q, k, v, pos, what):
    ref, b = bound(q, k, v, pos)
    bad = ~(np.abs(got - ref) <= b)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, worst {np.nanmax(np.abs(got - ref) / b):.2f} of the bound"


def filled(shp, lens, extra, rng, **kw):
    """A pool with `lens` committed tokens for each sequence and `extra` more written behind them."""
    cap = [a + b for a, b in zip(lens, extra)]
    p = Pool8(shp, sum((c + 15) // 16 for c in cap) + 3, max_seqs=max(8, len(lens)), max_pages=max((c + 15) // 16 for c in cap), **kw)
    seqs = p.seqs(cap)
    gains = np.exp(0.5 * rng.standard_normal((1, shp.n_kv, shp.head_dim)))
    for s, n, e in zip(seqs, lens, extra):
        k = gen.to_storage((rng.standard_normal((n + e, shp.n_kv, shp.head_dim)) * gains).astype(np.float32), "bf16")
        v = bf16(rng, (n + e, shp.n_kv, shp.head_dim))
        p.append([s], [n + e], k, v)
    kv = [p.gather(s) for s in seqs]
    for s, n in zip(seqs, lens):
        p.kv.truncate(s, n)
    return p, seqs, kv


@pytest.mark.parametrize("n_q,n_kv,hd", HEADS + [(16, 1, 64), (40, 2, 64), (5, 5, 128)])
@pytest.mark.parametrize("lens", [[0], [15, 16, 17], [31, 0, 100, 300, 1], [1000]])
@pytest.mark.parametrize("split", [0, 2, 3])
def test_decode_attention(n_q, n_kv, hd, lens, split):
    rng = np.random.default_rng(10)
    p, seqs, kv = filled(shape(n_q, n_kv, hd), lens, [1] * len(lens), rng)
    q = bf16(rng, (len(lens), n_q, hd))
    o = torch.full((len(lens), n_q * hd), float("nan"), dtype=torch.bfloat16, device="cuda")
    B.op_decode_attention(p.kv, 0, seqs, H.to_dev(q, "bf16"), o, p.ws, split)
    torch.cuda.synchronize()
    got = H.to_f64(o).reshape(len(lens), n_q, hd)
    for i, n in enumerate(lens):
        check(got[i:i + 1], wide(q)[i:i + 1], *kv[i], np.array([n]), f"sequence {i} of {n} tokens")


@pytest.mark.parametrize("lens", [[5000, 40, 3001], [9000]])
def test_decode_attention_long(lens):
    rng = np.random.default_rng(11)
    p, seqs, kv = filled(shape(8, 2, 128), lens, [1] * len(lens), rng, rows=9100)
    q = bf16(rng, (len(lens), 8, 128))
    o = H.empty((len(lens), 8 * 128), "bf16")
    B.op_decode_attention(p.kv, 0, seqs, H.to_dev(q, "bf16"), o, p.ws)
    torch.cuda.synchronize()
    for i, n in enumerate(lens):
        check(H.to_f64(o).reshape(-1, 8, 128)[i:i + 1], wide(q)[i:i + 1], *kv[i], np.array([n]), f"{n} tokens")


@pytest.mark.parametrize("n_q,n_kv,hd", HEADS + [(3, 1, 64), (40, 2, 64)])
@pytest.mark.parametrize("past,new", [([0], [1]), ([0], [33]), ([0, 0, 0], [64, 15, 100]), ([17, 160, 3], [40, 1, 70]),
                                      ([1500], [9])])
def test_prefill_attention(n_q, n_kv, hd, past, new):
    rng = np.random.default_rng(12)
    p, seqs, kv = filled(shape(n_q, n_kv, hd), past, new, rng)
    rows = sum(new)
    q = bf16(rng, (rows, n_q, hd))
    o = torch.full((rows + 1, n_q * hd), float("nan"), dtype=torch.bfloat16, device="cuda")
    B.op_attention(p.kv, 0, seqs, new, H.to_dev(q, "bf16"), o, p.ws)
    torch.cuda.synchronize()
    got = H.to_f64(o)
    assert np.isnan(got[rows]).all()  # the row behind the last sequence is not written
    got = got[:rows].reshape(rows, n_q, hd)
    r0 = 0
    for i, (a, n) in enumerate(zip(past, new)):
        check(got[r0:r0 + n], wide(q)[r0:r0 + n], *kv[i], np.arange(a, a + n), f"sequence {i}: {a} + {n}")
        r0 += n


@pytest.mark.parametrize("n_q,n_kv,hd", [(8, 2, 128), (3, 1, 64)])
def test_prefill_split_walk(n_q, n_kv, hd):
    """Few rows behind a long prefix: walked by several workgroups where the workspace has room, by one where not."""
    rng = np.random.default_rng(13)
    past, new = [6000, 30], [37, 5]
    p, seqs, kv = filled(shape(n_q, n_kv, hd, ffn=28672), past, new, rng, rows=6100)
    q = H.to_dev(bf16(rng, (42, n_q, hd)), "bf16")
    layer = B.Layer(p.cfg)
    assert layer.step_plan(p.kv, seqs, new, [], 1 << 40).split_walks > 0
    small = H.workspace(16384)
    for ws in (p.ws, small):
        o = H.empty((42, n_q * hd), "bf16")
        B.op_attention(p.kv, 0, seqs, new, q, o, ws)
        torch.cuda.synchronize()
        got = H.to_f64(o).reshape(42, n_q, hd)
        check(got[:37], H.to_f64(q)[:37], *kv[0], np.arange(6000, 6037), "long")
        check(got[37:], H.to_f64(q)[37:], *kv[1], np.arange(30, 35), "short")


def test_capped_run_and_other_streams_give_the_same_bits():
    rng = np.random.default_rng(14)
    lens = [700, 33, 1200, 5]
    p, seqs, kv = filled(shape(32, 8, 128), lens, [1] * 4, rng)
    q = H.to_dev(bf16(rng, (4, 32, 128)), "bf16")
    o = [H.empty((4, 32 * 128), "bf16") for _ in range(3)]
    B.op_decode_plan(p.kv, seqs, p.ws)
    B.op_decode_run(p.kv, 0, q, o[0], p.ws)
    B.op_decode_run_capped(p.kv, 0, q, o[1], p.ws, 16)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    B.op_decode_run(p.kv, 0, q, o[2], p.ws, stream=st)
    st.synchronize()
    for x in o[1:]:
        assert np.array_equal(H.bits(x), H.bits(o[0]))


def test_decode_run_in_a_graph():
    """A planned run captured once and replayed on new queries, with eager work between the replays."""
    rng = np.random.default_rng(15)
    lens = [300, 77]
    p, seqs, kv = filled(shape(8, 2, 64), lens, [1, 1], rng)
    q = H.to_dev(bf16(rng, (2, 8, 64)), "bf16")
    o, eager = H.empty((2, 512), "bf16"), H.empty((2, 512), "bf16")
    B.op_decode_plan(p.kv, seqs, p.ws, split_pages=4)
    B.op_decode_run(p.kv, 0, q, eager, p.ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.op_decode_run(p.kv, 0, q, o, p.ws)
    for i in range(4):
        q.copy_(H.to_dev(bf16(rng, (2, 8, 64)), "bf16"))
        o.zero_()
        g.replay()
        torch.cuda.synchronize()
        B.op_decode_run(p.kv, 0, q, eager, p.ws)
        torch.cuda.synchronize()
        assert np.array_equal(H.bits(o), H.bits(eager))
        check(H.to_f64(o).reshape(2, 8, 64)[:1], H.to_f64(q)[:1], *kv[0], np.array([300]), f"replay {i}")


def test_non_finite_keys_reach_only_the_rows_that_see_them():
    rng = np.random.default_rng(16)
    shp = shape(4, 1, 128)
    p = Pool8(shp, 16)
    k = wide(bf16(rng, (60, 1, 128))).astype(np.float32)
    k[40, 0, 7] = np.inf
    a, b = p.seqs([60, 60])
    kb, vb = gen.to_storage(k, "bf16"), bf16(rng, (60, 1, 128))
    clean = bf16(rng, (60, 1, 128))
    p.append([a, b], [60, 60], np.concatenate([kb, clean]), np.concatenate([vb, clean]))
    p.kv.truncate(a, 0)
    p.kv.truncate(b, 0)
    q = H.to_dev(bf16(rng, (120, 4, 128)), "bf16")
    o = H.empty((120, 512), "bf16")
    B.op_attention(p.kv, 0, [a, b], [60, 60], q, o, p.ws)
    torch.cuda.synchronize()
    got = H.to_f64(o)
    assert np.isnan(got[40:60]).all() and np.isfinite(got[:40]).all() and np.isfinite(got[60:]).all()


@pytest.mark.parametrize("hd,past,bad", [(128, 0, (40, 7)), (64, 0, (31, 63)), (128, 21, (0, 127)), (128, 16, (33, 64))])
def test_non_finite_values_reach_only_the_rows_that_see_them(hd, past, bad):
    """An infinity among the values, in the same tile as rows before it; earlier calls' tokens are finite."""
    rng = np.random.default_rng(18)
    n, (at, dim) = 70, bad
    p = Pool8(shape(4, 1, hd), 32)
    k, v = wide(bf16(rng, (past + n, 1, hd))).astype(np.float32), wide(bf16(rng, (past + n, 1, hd))).astype(np.float32)
    outs = []
    for x in (0.0, np.inf, -np.inf, np.nan):
        v[past + at, 0, dim] = x
        s, = p.seqs([past + n])
        kb, vb = gen.to_storage(k, "bf16"), gen.to_storage(v, "bf16")
        if past:
            p.append([s], [past], kb[:past], vb[:past])
        p.append([s], [n], kb[past:], vb[past:])
        p.kv.truncate(s, past)
        q = H.to_dev(bf16(np.random.default_rng(19), (n, 4, hd)), "bf16")
        o = H.empty((n, 4 * hd), "bf16")
        B.op_attention(p.kv, 0, [s], [n], q, o, p.ws)
        torch.cuda.synchronize()
        outs.append(H.to_f64(o).reshape(n, 4, hd))
        p.kv.free(s)
    clean = outs[0]
    for got in outs[1:]:
        assert np.isnan(got[at:, :, dim]).all()
        assert np.isfinite(got[:at]).all() and np.array_equal(got[:at], clean[:at])
        assert np.array_equal(np.delete(got, dim, 2), np.delete(clean, dim, 2))


def test_results_repeat_bit_for_bit():
    rng = np.random.default_rng(17)
    p, seqs, kv = filled(shape(32, 8, 128), [4000, 50], [1, 1], rng)
    q = H.to_dev(bf16(rng, (2, 32, 128)), "bf16")
    outs = []
    for _ in range(3):
        o = H.empty((2, 4096), "bf16")
        B.op_decode_attention(p.kv, 0, seqs, q, o, p.ws)
        torch.cuda.synchronize()
        outs.append(H.bits(o))
    assert all(np.array_equal(x, outs[0]) for x in outs[1:])


def test_writes_of_128_and_of_more_pages_are_the_same():
    """A call's work list as a kernel argument or through the workspace: the same bytes and rows."""
    rng = np.random.default_rng(20)
    n = 129 * PAGE
    p = Pool8(shape(4, 2, 64), 4 * 130, max_pages=129)
    qkv = H.to_dev(bf16(rng, (n, 8, 64)), "bf16")
    got = []
    for calls in ([n], [n - PAGE, PAGE], [PAGE, n - PAGE]):
        s, = p.seqs([n])
        q = H.empty((n, 4, 64), "bf16")
        r0 = 0
        for t in calls:
            B.op_rope_kvwrite(p.kv, 0, [s], [t], qkv[r0:], q[r0:], p.ws)
            p.kv.commit([s], [t])
            r0 += t
        torch.cuda.synchronize()
        got.append((H.to_f64(q), *p.gather(s)))
    for other in got[1:]:
        assert all(np.array_equal(a, b) for a, b in zip(got[0], other))
    # many sequences: 129 one-page prompts against one at a time
    seqs = Pool8(shape(4, 2, 64), 260, max_seqs=130, max_pages=1)
    one = seqs.seqs([PAGE] * 129)
    q = H.empty((n, 4, 64), "bf16")
    B.op_rope_kvwrite(seqs.kv, 0, one, [PAGE] * 129, qkv, q, seqs.ws)
    seqs.kv.commit(one, [PAGE] * 129)
    for i in (0, 63, 128):
        s, = p.seqs([PAGE])
        alone = H.empty((PAGE, 4, 64), "bf16")
        B.op_rope_kvwrite(p.kv, 0, [s], [PAGE], qkv[i * PAGE:], alone, p.ws)
        p.kv.commit([s], [PAGE])
        torch.cuda.synchronize()
        assert np.array_equal(H.bits(q)[i * PAGE:(i + 1) * PAGE], H.bits(alone))
        assert all(np.array_equal(a, b) for a, b in zip(seqs.gather(one[i]), p.gather(s)))


@pytest.mark.parametrize("new", [[5] * 16, [5] * 17, [40, 3] * 10, [128 * 32], [128 * 32 + 1], [700] * 9])
def test_prefill_work_lists_of_either_kind_give_the_same_bits(new):
    """Rows of a sequence do not depend on which others share the call, nor on how the work list travels."""
    rng = np.random.default_rng(21)
    p, seqs, _ = filled(shape(2, 1, 64), [0] * len(new), new, rng)
    rows = sum(new)
    q = H.to_dev(bf16(rng, (rows, 2, 64)), "bf16")
    small = H.workspace(32768)  # no room for parts: whole walks
    together, alone = H.empty((rows, 128), "bf16"), H.empty((rows, 128), "bf16")
    B.op_attention(p.kv, 0, seqs, new, q, together, small)
    r0 = 0
    for s, n in zip(seqs, new):
        for c0 in range(0, n, 2048):  # chunks of whole tiles
            n_c = min(2048, n - c0)
            B.op_attention(p.kv, 0, [s], [n_c], q[r0 + c0:], alone[r0 + c0:], small)
            p.kv.commit([s], [n_c])
        r0 += n
    torch.cuda.synchronize()
    assert np.array_equal(H.bits(together), H.bits(alone))


@pytest.mark.parametrize("at", [0, 13, 36])
def test_non_finite_values_in_split_walks(at):
    rng = np.random.default_rng(22)
    past, n = 6000, 37
    p = Pool8(shape(4, 1, 128, ffn=28672), 2 * 380, max_pages=380, rows=6100)
    k, v = (wide(bf16(rng, (past + n, 1, 128))).astype(np.float32) for _ in range(2))
    v[past + at, 0, 100] = np.inf
    s, = p.seqs([past + n])
    p.append([s], [past], *(gen.to_storage(x[:past], "bf16") for x in (k, v)))
    p.append([s], [n], *(gen.to_storage(x[past:], "bf16") for x in (k, v)))
    p.kv.truncate(s, past)
    q = H.to_dev(bf16(rng, (n, 4, 128)), "bf16")
    for ws in (p.ws, H.workspace(16384)):
        o = H.empty((n, 512), "bf16")
        B.op_attention(p.kv, 0, [s], [n], q, o, ws)
        torch.cuda.synchronize()
        bad = np.isnan(H.to_f64(o).reshape(n, 4, 128))
        want = np.zeros_like(bad)
        want[at:, :, 100] = True
        assert np.array_equal(bad, want)


def test_a_pool_past_four_gib():
    """Pages whose bytes lie past 32-bit offsets: written, gathered, read by both attentions, copied."""
    rng = np.random.default_rng(23)
    n = 2000
    p = Pool8(shape(2, 1, 128), 1_300_000, max_seqs=2, max_pages=130, rows=2048)
    s, = p.seqs([n])
    assert max(p.kv.block_table(s)) * 4096 > 2 ** 32
    k, v = bf16(rng, (n, 1, 128)), bf16(rng, (n, 1, 128))
    p.append([s], [n], k, v)
    ref = [K.Sequence(1, 128) for _ in range(2)]
    for r, x in zip(ref, (k, v)):
        r.append(wide(x))
    got = p.gather(s)
    assert all(np.array_equal(a, r.values()) for a, r in zip(got, ref))
    t = Pool8(shape(2, 1, 128), 130, max_seqs=2, max_pages=130)
    d, = t.seqs([n])
    B.kv_transfer(p.kv, s, t.kv, d, t.ws)
    assert all(np.array_equal(a, b) for a, b in zip(t.gather(d), got))
    p.kv.truncate(s, n - 40)
    q = bf16(rng, (40, 2, 128))
    o = H.empty((40, 256), "bf16")
    B.op_attention(p.kv, 0, [s], [40], H.to_dev(q, "bf16"), o, p.ws)
    torch.cuda.synchronize()
    check(H.to_f64(o).reshape(40, 2, 128), wide(q), *got, np.arange(n - 40, n), "prefill")
    p.kv.truncate(s, n - 41)
    B.op_decode_attention(p.kv, 0, [s], H.to_dev(q[:1], "bf16"), o[:1], p.ws)
    torch.cuda.synchronize()
    check(H.to_f64(o[:1]).reshape(1, 2, 128), wide(q[:1]), got[0][:n - 40], got[1][:n - 40], np.array([n - 41]), "decode")
