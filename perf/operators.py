"""Performance cases of the 8-bit serving operators: what is timed, on which inputs, and what the results should be.

Three operators that replace their bf16 forms in a serving loop:

* ``linear``: C = epilogue(A W^T) in 8-bit integers. The rows of x (after an RMSNorm, or as they are) get a scale each
  and are rounded to int8, the weight has one scale for each output channel, the sums are int32.
* ``write``: RoPE, and the new keys and values into a paged KV pool held in e4m3 with one power-of-two scale for each
  page of 16 tokens, KV head, and keys or values. Where a page holds earlier tokens and the new ones need a larger
  scale, the earlier ones are encoded anew.
* ``decode`` and ``prefill``: attention over such a pool, one row for each sequence, or a prompt's (or chunk's) rows
  behind a cached prefix.

Layer shapes are those of the benchmark (8B- and 70B-shaped); head layouts beside them (one KV head for each query
head, one for all, three query heads on each, heads of 64) are generic. Lengths follow the benchmark's laws, batch
sizes run from one chat user to the largest batch of the phase sweep.

Inputs come from the seed alone: activations N(0, 1) with a few channels ten times as large (as in trained layers),
weights N(0, 0.02^2), keys with channel gains of their own, values N(0, 1). Pages are handed out in turn to sequences
that grow side by side, so that a sequence's pages lie scattered over the pool.
"""
import math
import random

import torch

own = False
PAGE = 16

# query heads, KV heads, head dim
HEADS = {
    "8b": (32, 8, 128),
    "70b": (64, 8, 128),
    "mha": (16, 16, 128),
    "mqa": (32, 1, 128),
    "three": (12, 4, 128),
    "hd64": (32, 8, 64),
}
THETA = 500000.0
EPS = 1e-5


def linear_case(name, m, n, k, epi="store", norm=False, x="bf16", r="bf16", c="bf16"):
    return {"name": name, "op": "linear", "m": m, "n": n, "k": k, "epi": epi, "norm": norm, "x": x, "r": r, "c": c}


def kv_case(name, op, heads, seqs, new_lo=1, new_hi=1, past_lo=0, past_hi=0, median=0, len_seed=1):
    """new_lo..new_hi rows for each of `seqs` sequences behind past_lo..past_hi cached tokens (log-normal around `median`
    with sigma 0.5, clipped to that range, where median > 0)."""
    return {"name": name, "op": op, "heads": heads, "seqs": seqs, "new_lo": new_lo, "new_hi": new_hi, "past_lo": past_lo,
            "past_hi": past_hi, "median": median, "len_seed": len_seed}


def listed():
    return [
        # one chat user's step: the attention norm and the QKV projection of one row (latency)
        linear_case("linear_8b_qkv_m1", 1, 6144, 4096, norm=True),
        # the answer-phase batch: the down projection onto the fp32 residual
        linear_case("linear_8b_down_m64", 64, 4096, 14336, "residual", x="bf16", r="f32", c="bf16"),
        # one user's question of an odd length: the O projection of the large layer onto its input, into fp32
        linear_case("linear_70b_o_m389", 389, 8192, 8192, "residual", r="bf16", c="f32"),
        # eight long prompts at once: the FFN norm of the fp32 residual, gate and up projections, SwiGLU
        linear_case("linear_8b_gate_up_m16384", 16384, 28672, 4096, "swiglu", norm=True, x="f32"),
        # a decode step's new tokens, answers early in their life
        kv_case("write_8b_b64", "write", "8b", 64, past_lo=16, past_hi=512),
        # the prompts of the benchmark's prefill
        kv_case("write_8b_8x2048", "write", "8b", 8, 2048, 2048),
        # one chat user: latency of the smallest attention call
        kv_case("decode_8b_b1", "decode", "8b", 1, past_lo=2048, past_hi=2048),
        # the benchmark's answer-phase batch
        kv_case("decode_8b_b64", "decode", "8b", 64, past_lo=1024, past_hi=4096),
        # the benchmark's reasoning batch: long log-normal contexts
        kv_case("decode_8b_think_b32", "decode", "8b", 32, past_lo=4096, past_hi=32768, median=12288),
        # one user's question of an odd length
        kv_case("prefill_8b_1x389", "prefill", "8b", 1, 389, 389),
        # the benchmark's prefill
        kv_case("prefill_8b_8x2048", "prefill", "8b", 8, 2048, 2048),
        # follow-up turns over long cached conversations
        kv_case("prefill_8b_3x512_past", "prefill", "8b", 3, 300, 512, 6000, 12000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear", "write", "decode", "decode", "prefill", "prefill"])
    if op == "linear":
        k = 64 * _log_int(rng, 4, 224)
        n = 64 * _log_int(rng, 4, 448)
        m = _log_int(rng, 1, min(16384, 16384 * 28672 * 4096 // (n * k)))
        epi = rng.choice(["store", "residual", "swiglu"])
        r, c = {"store": ("f32", rng.choice(["bf16", "f32"])), "swiglu": ("f32", "bf16"),
                "residual": rng.choice([("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16")])}[epi]
        norm, x = rng.random() < 0.5, rng.choice(["bf16", "f32"])
        if c == "f32":  # a border case of a computed row is one of 254 steps either way: no fp32 result holds that still
            norm, x = False, "bf16"
        c = linear_case("", m, n, k, epi, norm, x, r, c)
    else:
        heads = rng.choice(["8b", "8b", "70b", "mha", "mqa", "three", "hd64"])
        seed = rng.randrange(1, 1 << 30)
        if op == "decode":
            seqs = _log_int(rng, 1, 128)
            lo = _log_int(rng, 1, max(2, min(16384, 300000 // seqs)))
            hi = lo + _log_int(rng, 1, lo)
            if heads == "mha":
                lo, hi = (lo + 1) // 2, (hi + 1) // 2
            c = kv_case("", op, heads, seqs, 1, 1, lo, hi, 0, seed)
        else:
            rows = _log_int(rng, 2, 16384 if op == "write" else 6000)
            seqs = rng.randint(1, min(64 if op == "write" else 8, rows))
            hi = rows // seqs
            past = _log_int(rng, 1, 4000 if hi < 1000 else 500) if rng.random() < 0.6 else 0
            if op == "prefill":
                hi = min(hi, 2500)  # rows x keys within the largest listed case
            c = kv_case("", op, heads, seqs, max(1, int(hi * rng.uniform(0.3, 1.0))), hi, past // 2, past, 0, seed)
    del c["name"]
    return c


# ---------------------------------------------------------------- lengths, pages and the pool
class Lengths:
    """Cached tokens and new rows of each sequence, and the sequence each page of the pool goes to."""

    def __init__(self, c):
        r = random.Random(c["len_seed"])
        self.past, self.new = [], []
        for _ in range(c["seqs"]):
            if c["median"]:
                x = math.exp(math.log(c["median"]) + 0.5 * r.gauss(0.0, 1.0))
                self.past.append(min(max(int(round(x)), c["past_lo"]), c["past_hi"]))
            else:
                self.past.append(r.randint(c["past_lo"], c["past_hi"]))
            self.new.append(r.randint(c["new_lo"], c["new_hi"]))
        self.rows = sum(self.new)
        self.pages = [(p + n + PAGE - 1) // PAGE for p, n in zip(self.past, self.new)]
        self.n_pages = sum(self.pages)
        self.owner = [s for s, n in enumerate(self.pages) for _ in range(n)]
        r.shuffle(self.owner)
        self.table = [[] for _ in self.pages]
        for page, s in enumerate(self.owner):
            self.table[s].append(page)


def blocks_of(pool, n_pages, n_kv, hd):
    """The pool's bytes as [page, KV head, K or V, 16 hd]."""
    return pool[:n_pages * n_kv * 2 * PAGE * hd].view(n_pages, n_kv, 2, PAGE * hd)


def scales_of(pool, n_pages, n_kv, hd):
    """The pool's scales as [KV head, page, K or V]."""
    return pool[n_pages * n_kv * 2 * PAGE * hd:].view(torch.float32).view(n_kv, n_pages, 2)


def to_k_block(x):
    """[..., 16 tokens, hd] bytes -> a K block: [hd / 16][16 tokens][16 dims]."""
    hd = x.shape[-1]
    return x.unflatten(-1, (hd // 16, 16)).transpose(-3, -2).reshape(*x.shape[:-2], PAGE * hd)


def from_k_block(b):
    hd = b.shape[-1] // PAGE
    return b.unflatten(-1, (hd // 16, PAGE, 16)).transpose(-3, -2).flatten(-2)


def to_v_block(x):
    """[..., 16 tokens, hd] bytes -> a V block: [hd / 64][4 token quads][16 dims][4 blocks of 16 dims][4 tokens]."""
    hd = x.shape[-1]
    y = x.unflatten(-1, (hd // 64, 4, 16)).unflatten(-4, (4, 4))  # [..., quad, tok, big, blk, dim]
    n = y.dim() - 5
    return y.permute(*range(n), n + 2, n, n + 4, n + 3, n + 1).reshape(*x.shape[:-2], PAGE * hd)


def from_v_block(b):
    hd = b.shape[-1] // PAGE
    y = b.unflatten(-1, (hd // 64, 4, 16, 4, 4))  # [..., big, quad, dim, blk, tok]
    n = y.dim() - 5
    return y.permute(*range(n), n + 1, n + 4, n, n + 3, n + 2).flatten(-3).flatten(-3, -2)


def exponent(amax):
    """The smallest e with amax <= 448 2^e, from -100 to 119."""
    m, x = torch.frexp(amax)
    return (x - 9 + (m > 0.875).to(x.dtype)).masked_fill(amax == 0, -100).clamp(-100, 119)


def encode(x, e):
    """x 2^-e as e4m3 bytes."""
    return (x * torch.ldexp(torch.ones((), device=x.device), -e)).to(torch.float8_e4m3fn).view(torch.uint8)


def decode_bytes(b):
    return b.view(torch.float8_e4m3fn).float()


class State:
    pass


def normal(g, *shape, std=1.0, mean=0.0, dtype=torch.bfloat16):
    t = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    if std != 1.0:
        t.mul_(std)
    if mean:
        t.add_(mean)
    return t.to(dtype)


DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------- what a serving program holds before the call
def prepare(case, seed):
    c, s = case, State()
    s.case = c
    g = torch.Generator(device="cuda").manual_seed(seed)
    if c["op"] == "linear":
        prepare_linear(c, s, g)
    else:
        prepare_kv(c, s, g)
    return s


def prepare_linear(c, s, g):
    m, n, k = c["m"], c["n"], c["k"]
    x = torch.randn((m, k), generator=g, device="cuda", dtype=torch.float32)
    gain = torch.ones(k, device="cuda")
    gain[torch.randperm(k, generator=g, device="cuda")[:max(1, k // 512)]] = 10.0
    s.x = (x * gain).to(DTYPE[c["x"]])
    s.g = normal(g, k, std=0.02, mean=1.0) if c["norm"] else None
    w = torch.randn((n, k), generator=g, device="cuda", dtype=torch.float32).mul_(0.02)
    s.w_scale = w.abs().amax(1) / 127.0
    s.w = torch.round(w / s.w_scale[:, None]).to(torch.int8)  # SwiGLU: rows in 32s, gate and up in turn
    s.r = normal(g, m, n, dtype=DTYPE[c["r"]]) if c["epi"] == "residual" else None
    cols = n // 2 if c["epi"] == "swiglu" else n
    s.out = torch.empty((m, cols), dtype=DTYPE[c["c"]], device="cuda")
    if own:
        from paper_2608_21719_amd import binding as B
        s.lib = B
        tiled = torch.empty(B.tiled_weight_i8_bytes(n, k), dtype=torch.int8, device="cuda")
        B.op_tile_weight_i8(n, k, s.w, tiled)
        s.w = tiled
        s.a = torch.empty((m, k), dtype=torch.int8, device="cuda")
        s.a_scale = torch.empty(m, dtype=torch.float32, device="cuda")
        s.ws = torch.empty(max(256, B.op_gemm_i8_workspace_bytes(m, n, k)), dtype=torch.uint8, device="cuda")
        code = {"bf16": B.PS_BF16, "f32": B.PS_F32}
        s.x_dt, s.r_dt, s.c_dt = code[c["x"]], code[c["r"]], code[c["c"]]
        s.epi = {"store": B.PS_EPI_STORE, "residual": B.PS_EPI_RESIDUAL, "swiglu": B.PS_EPI_SWIGLU}[c["epi"]]


def prepare_kv(c, s, g):
    n_q, n_kv, hd = HEADS[c["heads"]]
    L = Lengths(c)
    s.n_q, s.n_kv, s.hd, s.lengths = n_q, n_kv, hd, L
    P = L.n_pages
    s.pool = torch.zeros(P * n_kv * (2 * PAGE * hd + 8), dtype=torch.uint8, device="cuda")
    blocks, scales = blocks_of(s.pool, P, n_kv, hd), scales_of(s.pool, P, n_kv, hd)
    write = c["op"] == "write"
    # tokens of each page that hold keys before the call: the cached ones, and the call's own where attention follows
    held = torch.zeros(P, dtype=torch.int64)
    for t, p, n in zip(L.table, L.past, L.new):
        length = p if write else p + n
        for i, page in enumerate(t):
            held[page] = min(max(length - PAGE * i, 0), PAGE)
    live = (torch.arange(PAGE)[None] < held[:, None]).to("cuda")[:, None, :, None]
    if bool(live.any()):
        gains = torch.exp(0.5 * torch.randn((1, n_kv, 1, hd), generator=g, device="cuda"))
        for i, lay in ((0, to_k_block), (1, to_v_block)):
            x = torch.randn((P, n_kv, PAGE, hd), generator=g, device="cuda")
            if i == 0:
                x.mul_(gains)
            x.mul_(live)
            e = exponent(x.abs().amax((2, 3)))
            blocks[:, :, i] = lay(encode(x, e[:, :, None, None]))
            scales[:, :, i] = torch.ldexp(torch.ones((), device="cuda"), e).T
            del x
    if write:
        s.qkv = normal(g, L.rows, (n_q + 2 * n_kv) * hd)
        s.q_out = torch.empty((L.rows, n_q * hd), dtype=torch.bfloat16, device="cuda")
    else:
        s.q = normal(g, L.rows, n_q, hd)
        s.o = torch.empty((L.rows, n_q * hd), dtype=torch.bfloat16, device="cuda")
    # the batch's tables on the GPU, as any paged implementation keeps them
    width = max(L.pages)
    s.table = torch.tensor([t + [0] * (width - len(t)) for t in L.table], device="cuda")
    s.past = torch.tensor(L.past, device="cuda")
    s.new = torch.tensor(L.new, device="cuda")
    if own:
        from paper_2608_21719_amd import binding as B
        s.lib = B
        s.cfg = B.LayerCfg(n_q * hd, n_q, n_kv, hd, 4 * n_q * hd, EPS, THETA, B.PS_BF16)
        s.kv = B.KV8(s.cfg, 1, P, len(L.new), width, s.pool)
        s.seqs = [s.kv.open() for _ in L.new]
        have = [0] * len(L.new)
        for q in L.owner:  # page i of the pool to the sequence that owns it
            have[q] += 1
            s.kv.alloc(s.seqs[q], have[q] * PAGE)
        if any(L.past):
            at = [i for i, p in enumerate(L.past) if p]
            s.kv.commit([s.seqs[i] for i in at], [L.past[i] for i in at])
        s.ws = torch.empty(B.Layer.workspace_bytes(s.cfg, L.rows, len(L.new), width), dtype=torch.uint8, device="cuda")
        if c["op"] == "decode":  # a step plans once and runs every layer's attention from it
            B.op_decode_plan(s.kv, s.seqs, s.ws)


# ---------------------------------------------------------------- one pass
def run(state):
    op = state.case["op"]
    if own:
        return {"linear": own_linear, "write": own_write, "decode": own_decode, "prefill": own_prefill}[op](state.lib, state)
    if op == "linear":
        return plain_linear(state)
    if op == "write":
        return plain_write(state)
    return plain_attention(state)


def own_linear(B, s):
    c = s.case
    if c["norm"]:
        B.op_rmsnorm_quant(s.x_dt, B.PS_BF16, c["m"], c["k"], s.x, s.g, EPS, s.a, s.a_scale)
    else:
        B.op_quant_rows(s.x_dt, c["m"], c["k"], s.x, s.a, s.a_scale)
    B.op_gemm_i8(s.r_dt, s.c_dt, s.epi, c["m"], c["n"], c["k"], s.a, s.a_scale, s.w, s.w_scale, s.r, s.out, s.ws)
    return s.out


def own_write(B, s):
    B.op_rope_kvwrite(s.kv, 0, s.seqs, s.lengths.new, s.qkv, s.q_out, s.ws)
    return written(s)


def own_decode(B, s):
    B.op_decode_run(s.kv, 0, s.q, s.o, s.ws)
    return s.o


def own_prefill(B, s):
    B.op_attention(s.kv, 0, s.seqs, s.lengths.new, s.q, s.o, s.ws)
    return s.o


def written(s):
    P = s.lengths.n_pages
    return {"q": s.q_out, "kv": blocks_of(s.pool, P, s.n_kv, s.hd).view(torch.float8_e4m3fn),
            "scales": scales_of(s.pool, P, s.n_kv, s.hd)}


def plain_linear(s):
    c = s.case
    x = s.x.float()
    if c["norm"]:
        x = x * torch.rsqrt(x.square().mean(1, keepdim=True) + EPS) * s.g.float()
    amax = x.abs().amax(1, keepdim=True)
    # the quotient in 64 bits: bf16 rows often lie on or next to a border between two integers
    a = torch.round(torch.where(amax > 0, 127.0 * x.double() / amax.double(), 0.0)).float()
    y = (a @ s.w.float().T) * (amax / 127.0) * s.w_scale
    if c["epi"] == "residual":
        y = y + s.r.float()
    elif c["epi"] == "swiglu":
        y = y.view(c["m"], -1, 2, 32)
        gate, up = y[:, :, 0], y[:, :, 1]
        y = (gate / (1.0 + torch.exp(-gate)) * up).reshape(c["m"], -1)
    return y.to(s.out.dtype)


def row_places(s):
    """Of each row: its sequence and its position in it."""
    seq = torch.repeat_interleave(torch.arange(len(s.new), device="cuda"), s.new, output_size=s.lengths.rows)
    start = torch.cumsum(s.new, 0) - s.new
    return seq, s.past[seq] + torch.arange(s.lengths.rows, device="cuda") - start[seq]


def plain_write(s):
    n_q, n_kv, hd, rows, P = s.n_q, s.n_kv, s.hd, s.lengths.rows, s.lengths.n_pages
    seq, pos = row_places(s)
    page, slot = s.table[seq, pos // PAGE], pos % PAGE
    angle = pos.double()[:, None] * THETA ** (-2.0 * torch.arange(hd // 2, device="cuda", dtype=torch.float64) / hd)
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    x = s.qkv.view(rows, n_q + 2 * n_kv, hd).float()
    x1, x2 = x[:, :n_q + n_kv, :hd // 2], x[:, :n_q + n_kv, hd // 2:]
    turned = torch.cat([x1 * cos - x2 * sin, x2 * cos + x1 * sin], 2)
    s.q_out.copy_(turned[:, :n_q].reshape(rows, -1))
    blocks, scales = blocks_of(s.pool, P, n_kv, hd), scales_of(s.pool, P, n_kv, hd)
    # the touched pages, the first new slot of each, and whether a slot is new
    touched, at = torch.unique(page, return_inverse=True)
    T = touched.numel()
    first = torch.full((T,), PAGE, device="cuda").scatter_reduce_(0, at, slot, "amin")
    fresh = torch.zeros((T, PAGE), dtype=torch.bool, device="cuda")
    fresh[at, slot] = True
    earlier = torch.arange(PAGE, device="cuda")[None] < first[:, None]
    for i, new, to, back in ((0, turned[:, n_q:], to_k_block, from_k_block),
                             (1, x[:, n_q + n_kv:], to_v_block, from_v_block)):
        was = back(blocks[touched, :, i]).contiguous()                # [T, n_kv, 16, hd] bytes
        old_scale = scales[:, touched, i].T                            # [T, n_kv]
        old_scale = torch.where((first > 0)[:, None], old_scale, 0.0)
        full = torch.zeros((T, PAGE, n_kv, hd), device="cuda")
        full[at, slot] = new
        full = full.transpose(1, 2)
        e = exponent(full.abs().amax((2, 3)))
        e = torch.where(old_scale > 0, torch.maximum(e, torch.frexp(old_scale)[1] - 1), e)
        full = torch.where(earlier[:, None, :, None], decode_bytes(was) * old_scale[:, :, None, None], full)
        now = encode(full, e[:, :, None, None])
        keep = (earlier | fresh)[:, None, :, None]
        blocks[touched, :, i] = to(torch.where(keep, now, was))
        scales[:, touched, i] = torch.ldexp(torch.ones((), device="cuda"), e).T
    return written(s)



def plain_attention(s):
    n_q, n_kv, hd, L = s.n_q, s.n_kv, s.hd, s.lengths
    G, B = n_q // n_kv, len(L.new)
    blocks, scales = blocks_of(s.pool, L.n_pages, n_kv, hd), scales_of(s.pool, L.n_pages, n_kv, hd)
    width = s.table.shape[1]
    keys = width * PAGE

    def cached(i, back):  # [B, n_kv, keys, hd]
        x = decode_bytes(back(blocks[s.table, :, i]).contiguous())      # [B, width, n_kv, 16, hd]
        x = x * scales[:, s.table, i].permute(1, 2, 0)[..., None, None]
        return x.transpose(1, 2).reshape(B, n_kv, keys, hd)

    most = max(L.new)
    seq, pos = row_places(s)
    row = pos - s.past[seq]
    q = torch.zeros((B, most, n_q, hd), device="cuda")
    q[seq, row] = s.q.float()
    q = q.view(B, most, n_kv, G, hd).permute(0, 2, 3, 1, 4).reshape(B, n_kv, G * most, hd)
    score = torch.matmul(q, cached(0, from_k_block).transpose(2, 3)).view(B, n_kv, G, most, keys)
    score *= hd ** -0.5
    last = s.past[:, None] + torch.minimum(torch.arange(most, device="cuda")[None], s.new[:, None] - 1)
    hidden = torch.arange(keys, device="cuda")[None, None] > last[:, :, None]
    score.masked_fill_(hidden[:, None, None], -math.inf)
    score -= score.amax(-1, keepdim=True)
    score.exp_()
    total = score.sum(-1, keepdim=True)
    o = torch.matmul(score.view(B, n_kv, G * most, keys), cached(1, from_v_block)).view(B, n_kv, G, most, hd) / total
    return o.permute(0, 3, 1, 2, 4)[seq, row].reshape(L.rows, n_q * hd).to(torch.bfloat16)


# ---------------------------------------------------------------- the same from the definitions in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"linear": exact_linear, "write": exact_write, "decode": exact_attention,
            "prefill": exact_attention}[case["op"]](s)


def exact_linear(s):
    c = s.case
    out = torch.empty(s.out.shape, dtype=torch.float64, device="cuda")
    for r0 in range(0, c["m"], 2048):
        x = s.x[r0:r0 + 2048].double()
        if s.g is not None:
            x = x / (x.pow(2).sum(1, keepdim=True) / c["k"] + EPS).sqrt() * s.g.double()
        most = x.abs().max(1, keepdim=True).values
        a = torch.where(most > 0, (x * 127 / most).round(), 0.0) * (most / 127)
        for n0 in range(0, c["n"], 4096):
            y = a @ (s.w[n0:n0 + 4096].double() * s.w_scale[n0:n0 + 4096, None].double()).T.contiguous()
            if c["epi"] == "swiglu":
                gate = torch.cat([y[:, i:i + 32] for i in range(0, y.shape[1], 64)], 1)
                up = torch.cat([y[:, i + 32:i + 64] for i in range(0, y.shape[1], 64)], 1)
                out[r0:r0 + 2048, n0 // 2:n0 // 2 + gate.shape[1]] = gate * torch.sigmoid(gate) * up
            else:
                if c["epi"] == "residual":
                    y += s.r[r0:r0 + 2048, n0:n0 + 4096].double()
                out[r0:r0 + 2048, n0:n0 + 4096] = y
    return out


def exact_write(s):
    L, n_q, n_kv, hd = s.lengths, s.n_q, s.n_kv, s.hd
    P = L.n_pages
    blocks = blocks_of(s.pool, P, n_kv, hd).view(torch.float8_e4m3fn).double()
    scales = scales_of(s.pool, P, n_kv, hd).double()
    q_out = torch.empty((L.rows, n_q * hd), dtype=torch.float64, device="cuda")
    tok, dim = torch.meshgrid(torch.arange(PAGE, device="cuda"), torch.arange(hd, device="cuda"), indexing="ij")
    place = (dim // 16 * 256 + tok * 16 + dim % 16,                                                     # K
             dim // 64 * 1024 + (tok // 4 * 16 + dim % 16) * 16 + dim % 64 // 16 * 4 + tok % 4)           # V
    freq = torch.tensor([THETA ** (-2.0 * j / hd) for j in range(hd // 2)], dtype=torch.float64, device="cuda")
    r0 = 0
    for b, (past, n) in enumerate(zip(L.past, L.new)):
        x = s.qkv[r0:r0 + n].double().view(n, n_q + 2 * n_kv, hd)
        z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                        torch.arange(past, past + n, device="cuda").double()[:, None] * freq)[:, None]
        z = torch.complex(x[:, :n_q + n_kv, :hd // 2], x[:, :n_q + n_kv, hd // 2:]) * z
        x = torch.cat([torch.cat([z.real, z.imag], 2), x[:, n_q + n_kv:]], 1)
        q_out[r0:r0 + n] = x[:, :n_q].reshape(n, -1)
        p0 = past // PAGE
        count = (past + n - 1) // PAGE + 1 - p0
        ids = torch.tensor(L.table[b][p0:p0 + count], device="cuda")
        lead = past - p0 * PAGE  # tokens of the first page from before
        for i in (0, 1):
            new = torch.zeros((count * PAGE, n_kv, hd), dtype=torch.float64, device="cuda")
            new[lead:lead + n] = x[:, n_q + i * n_kv:n_q + (i + 1) * n_kv]
            new = new.view(count, PAGE, n_kv, hd).transpose(1, 2)          # [pages, n_kv, 16, hd]
            e = torch.ceil(torch.log2(new.abs().amax((2, 3)).clamp_min(2.0 ** -100) / 448)).clamp_min(-100)
            was = blocks[ids, :, i][:, :, place[i]]
            if lead:
                e[0] = torch.maximum(e[0], torch.log2(scales[:, ids[0], i]))
                new[0, :, :lead] = (was[0] * scales[:, ids[0], i, None, None])[:, :lead]
            y = new / torch.exp2(e)[:, :, None, None]
            # half to even onto e4m3: three bits behind the leading one, steps of 2^-9 below 2^-6
            step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
            y = (y / step).round() * step
            end = lead + n - (count - 1) * PAGE
            y[-1, :, end:] = was[-1, :, end:]  # slots behind the last token stay
            back = torch.empty((count, n_kv, PAGE * hd), dtype=torch.float64, device="cuda")
            back[:, :, place[i].flatten()] = y.flatten(2)
            blocks[ids, :, i] = back
            scales[:, ids, i] = torch.exp2(e).T
        r0 += n
    return {"q": q_out, "kv": blocks, "scales": scales}


def exact_attention(s):
    L, n_q, n_kv, hd = s.lengths, s.n_q, s.n_kv, s.hd
    blocks, scales = blocks_of(s.pool, L.n_pages, n_kv, hd), scales_of(s.pool, L.n_pages, n_kv, hd)
    out = torch.empty((L.rows, n_q, hd), dtype=torch.float64, device="cuda")
    tok, dim = torch.meshgrid(torch.arange(PAGE, device="cuda"), torch.arange(hd, device="cuda"), indexing="ij")
    place = (dim // 16 * 256 + tok * 16 + dim % 16,
             dim // 64 * 1024 + (tok // 4 * 16 + dim % 16) * 16 + dim % 64 // 16 * 4 + tok % 4)
    r0 = 0
    for b, (past, n) in enumerate(zip(L.past, L.new)):
        ids = torch.tensor(L.table[b], device="cuda")
        kv = []
        for i in (0, 1):  # [n_kv, keys, hd]
            x = blocks[ids, :, i].view(torch.float8_e4m3fn).double()[:, :, place[i]] * scales[:, ids, i].T.double()[:, :, None, None]
            kv.append(x.transpose(0, 1).reshape(n_kv, -1, hd)[:, :past + n])
        seen = torch.arange(past + n, device="cuda")[None] <= torch.arange(past, past + n, device="cuda")[:, None]
        for h in range(n_q):
            k, v = kv[0][h // (n_q // n_kv)], kv[1][h // (n_q // n_kv)]
            score = s.q[r0:r0 + n, h].double() @ k.T.contiguous() / math.sqrt(hd)
            out[r0:r0 + n, h] = torch.softmax(score.masked_fill(~seen, -math.inf), 1) @ v
        r0 += n
    return out.view(L.rows, n_q * hd)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    size = {"bf16": 2, "f32": 4}
    if c["op"] == "linear":
        m, n, k = c["m"], c["n"], c["k"]
        b = m * k * size[c["x"]] + (2 * k if c["norm"] else 0) + n * k + 4 * n
        b += m * n * size[c["r"]] if c["epi"] == "residual" else 0
        b += m * (n // 2 if c["epi"] == "swiglu" else n) * size[c["c"]]
        return {"bytes": b, "flops": 2 * m * n * k}
    n_q, n_kv, hd = HEADS[c["heads"]]
    L = Lengths(c)
    if c["op"] == "write":
        pages = sum((p + n - 1) // PAGE + 1 - p // PAGE for p, n in zip(L.past, L.new))
        return {"bytes": L.rows * hd * ((n_q + 2 * n_kv) * 2 + n_q * 2 + 2 * n_kv) + pages * n_kv * 8,
                "flops": L.rows * hd * (n_q + n_kv) * 3}
    seen = sum(n * p + n * (n + 1) // 2 for p, n in zip(L.past, L.new))
    held = sum(p + n for p, n in zip(L.past, L.new))
    return {"bytes": held * n_kv * 2 * hd + L.n_pages * n_kv * 8 + 4 * L.rows * n_q * hd, "flops": 4 * hd * n_q * seen}
