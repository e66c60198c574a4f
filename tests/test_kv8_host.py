"""The e4m3 KV pool without a GPU: its definition (oracle/kv8.py) against independent statements, sizes, refusals."""
import numpy as np
import pytest

from oracle import kv8 as K
from paper_2608_21719_amd import binding as B
from synth.configs import CONFIGS, LayerShape

FAKE_POOL = 0x10000  # never dereferenced by host-only calls
S8 = CONFIGS["llama8b_decode"].shape


def _kv(cfg=None, n_layers=2, n_pages=64, max_seqs=4, max_pages=16, pool=FAKE_POOL):
    return B.KV8(cfg or B.make_cfg(S8), n_layers, n_pages, max_seqs, max_pages, pool)


def test_table_has_the_format_s_landmarks():
    t = K.table()
    assert t[0x7e] == 448 and t[0x01] == 2.0 ** -9 and t[0x08] == 2.0 ** -6 and t[0x38] == 1.0 and t[0xb8] == -1.0
    assert np.isnan(t[[0x7f, 0xff]]).all() and np.isfinite(np.delete(t, [0x7f, 0xff])).all()


def test_table_agrees_with_torch():
    torch = pytest.importorskip("torch")
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t, K.table(), equal_nan=True)


def test_nearest_is_the_closest_number_with_ties_to_even():
    t = np.unique(K.table()[np.isfinite(K.table())])
    pos = t[t >= 0]
    x = np.concatenate([np.random.default_rng(1).uniform(0, 448, 4000), np.random.default_rng(2).uniform(0, 0.03, 4000),
                        pos, (pos[:-1] + pos[1:]) / 2])
    y = K.nearest(x)
    d = np.abs(x[:, None] - pos[None]).min(1)
    assert np.isin(y, pos).all() and np.array_equal(np.abs(x - y), d)
    mid = K.nearest((pos[:-1] + pos[1:]) / 2)
    byte = {v: i for i, v in enumerate(K.table()) if i < 127}
    assert all(byte[v] % 2 == 0 for v in mid)
    assert np.array_equal(K.nearest(-x), -y) and np.isnan(K.nearest(np.array([np.inf, np.nan]))).all()


def test_exponent_is_the_smallest_that_fits():
    for a in (1e-20, 0.013, 1.0, 448.0, np.nextafter(448.0, 1e9), 449.0, 3.0e38):
        e = K.exponent(a)
        assert e == 119 or a <= 448 * 2.0 ** e
        assert e == -100 or a > 448 * 2.0 ** (e - 1)
    assert K.exponent(0.0) == -100


def test_growing_scale_costs_less_than_one_step():
    rng = np.random.default_rng(3)
    p = K.Page(8)
    rows = rng.standard_normal((16, 8)) * 2.0 ** rng.integers(-6, 10, (16, 1))
    for r in rows:
        p.append(r[None])
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(rows) * 2.0 ** -p.e, 2.0 ** -6))) - 3) * 2.0 ** p.e
    assert (np.abs(p.values() - rows) < step).all()


def test_pool_bytes():
    cfg = B.make_cfg(S8)
    assert B.KV8.pool_bytes(cfg, 3, 10) == 3 * 10 * 8 * (2 * 16 * 128 + 8)
    assert B.KV8.pool_bytes(cfg, 0, 10) == 0 and B.KV8.pool_bytes(cfg, 1, 0) == 0
    assert B.KV8.pool_bytes(cfg, 1, 1 << 20) < 0.51 * B.KV.pool_bytes(cfg, 1, 1 << 20)


@pytest.mark.parametrize("change,code", [
    (dict(dtype="f32"), B.PS_E_UNSUPPORTED), (dict(head_dim=96), B.PS_E_UNSUPPORTED), (dict(head_dim=32), B.PS_E_UNSUPPORTED),
    (dict(head_dim=0), B.PS_E_INVALID), (dict(n_kv=3), B.PS_E_INVALID)])
def test_refused_configurations(change, code):
    d = dict(hidden=512, n_q=8, n_kv=4, head_dim=64, ffn=256, eps=1e-5, theta=1e4, dtype="bf16")
    d.update(change)
    with pytest.raises(B.PsError) as e:
        _kv(B.make_cfg(LayerShape(**d)))
    assert e.value.code == code


def test_refused_pools_and_sizes():
    for kw in (dict(pool=None), dict(pool=FAKE_POOL + 8), dict(n_pages=0), dict(n_layers=0), dict(max_seqs=-1)):
        with pytest.raises(B.PsError) as e:
            _kv(**kw)
        assert e.value.code == B.PS_E_INVALID


def test_transfer_needs_pools_stored_alike():
    a, b = _kv(), B.KV(B.make_cfg(S8), 2, 64, 4, 16, FAKE_POOL)
    sa, sb = a.open(), b.open()
    ws = np.zeros(1024, dtype=np.uint8)
    for src, s, dst, d in ((a, sa, b, sb), (b, sb, a, sa)):
        rc = B.lib.ps_kv_transfer(src.h, s, dst.h, d, B.ptr(ws), ws.nbytes, None)
        assert rc == B.PS_E_INVALID and "differently" in B.last_error()


def test_calls_check_their_arguments_before_any_work():
    """Refusals on an e4m3 handle, none of which reaches the device."""
    kv = _kv()
    s = kv.open()
    kv.alloc(s, 20)
    one, n1 = B.ints([s]), B.ints([1])
    ok, bad = 0x20000, 0x20008
    calls = {
        "layer out of range": (B.lib.ps_op_rope_kvwrite(kv.h, 2, 1, one, n1, ok, ok, ok, 1 << 20, None), B.PS_E_INVALID),
        "null rows": (B.lib.ps_op_rope_kvwrite(kv.h, 0, 1, one, n1, None, ok, ok, 1 << 20, None), B.PS_E_INVALID),
        "unaligned rows": (B.lib.ps_op_rope_kvwrite(kv.h, 0, 1, one, n1, bad, ok, ok, 1 << 20, None), B.PS_E_INVALID),
        "past the reservation": (B.lib.ps_op_rope_kvwrite(kv.h, 0, 1, one, B.ints([33]), ok, ok, ok, 1 << 20, None),
                                 B.PS_E_CAPACITY),
        "no rows": (B.lib.ps_kv_append(kv.h, 0, 1, one, B.ints([0]), ok, ok, ok, 1 << 20, None), B.PS_E_INVALID),
        "twice": (B.lib.ps_kv_append(kv.h, 0, 2, B.ints([s, s]), B.ints([1, 1]), ok, ok, ok, 1 << 20, None), B.PS_E_INVALID),
        "small workspace": (B.lib.ps_op_attention(kv.h, 0, 1, one, n1, ok, ok, ok, 16, None), B.PS_E_INVALID),
        "null q": (B.lib.ps_op_decode_attention(kv.h, 0, 1, one, None, ok, 0, ok, 1 << 20, None), B.PS_E_INVALID),
        "run without a plan": (B.lib.ps_op_decode_run(kv.h, 0, ok, ok, ok, 1 << 20, None), B.PS_E_INVALID),
        "negative split": (B.lib.ps_op_decode_plan(kv.h, 1, one, -1, ok, 1 << 20, None), B.PS_E_INVALID),
        "sequence not open": (B.lib.ps_kv_gather(kv.h, 0, s + 1, ok, ok, ok, 1 << 20, None), B.PS_E_INVALID),
    }
    assert {k: rc for k, (rc, _) in calls.items()} == {k: want for k, (_, want) in calls.items()}
    assert kv.seq_len(s) == 0 and kv.capacity(s) == 32


def test_layer_and_plan_take_the_handle():
    """The planning calls see an e4m3 pool as any other; a layer of another configuration is refused."""
    kv = _kv(max_pages=64, n_pages=256)
    layer = B.Layer(B.make_cfg(S8))
    s = [kv.open() for _ in range(2)]
    kv.alloc(s[0], 300)
    kv.alloc(s[1], 40)
    p = layer.step_plan(kv, [s[0]], [300], [s[1]], 1 << 30)
    assert p.o_splits >= 1
    other = B.Layer(B.make_cfg(LayerShape(2048, 16, 8, 128, 1024, 1e-5, 1e4, "bf16")))
    with pytest.raises(B.PsError) as e:
        other.step_plan(kv, [s[0]], [10], [], 1 << 30)
    assert e.value.code == B.PS_E_INVALID
