"""Measured work of the operators of a transformer's layers on 8-bit integers: matrices held in 8 bits with a scale for each row,
linear layers on them, the gated feed-forward block's two projections with activation and product, its backward pass, and the norms
of queries and keys with the rotation by position.

A matrix in 8 bits is whole numbers from -127 to 127, times its row's scale: the row's largest magnitude divided by 127 in fp32 (2^-126 at
least, 0 for a row of zeros).  An element is divided by the scale and rounded to nearest, ties to even.  What is held is the
magnitude, from which a reader has the scale.

`run` with own = False computes the operators with elementary torch operations, with own = True through the package's API.
"""
import math

import numpy as np
import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


# ---- cases --------------------------------------------------------------------------------------

def listed():
    return [
        # a slice of a wider fp32 matrix, its rows on no 16-byte boundary, kept in 8 bits until it is wanted
        dict(name="save_restore_odd", op="save", rows=4099, cols=1000, ld=1003, dtype="f32", both=False),
        # a gradient for both products of a linear layer's backward pass: a scale for each token and for each channel
        dict(name="save_restore_gradient", op="save", rows=8192, cols=4096, ld=4096, dtype="bf16", both=True),
        # one token through a linear layer: into 8 bits, then the product
        dict(name="linear_token", op="linear", m=1, n=8192, k=8192, dtype="bf16", alpha=1.0, accumulate=False),
        # a training batch through a linear layer, the largest product
        dict(name="linear_large", op="linear", m=8192, n=8192, k=4096, dtype="bf16", alpha=1.0, accumulate=False),
        # one token through the gated block's projections
        dict(name="gated_token", op="gated", m=1, f=8192, k=4096, dtype="bf16", activation="silu", keep=False),
        # a training batch, with what the backward pass needs
        dict(name="gated_batch", op="gated", m=4096, f=8192, k=4096, dtype="bf16", activation="silu", keep=True),
        # the backward pass of odd sizes
        dict(name="gated_backward_odd", op="gated_backward", m=1001, f=1111, k=777, dtype="f32", activation="gelu"),
        # the backward pass of a training batch.  (The input's and the weights' gradients are sent on in bf16: behind whole numbers that a last
        # place of what was rounded to them may turn over, fp32 has no more to say.)
        dict(name="gated_backward_batch", op="gated_backward", m=4096, f=8192, k=4096, dtype="bf16", activation="silu"),
        # one token's queries and keys, far along in its text
        dict(name="heads_token", op="heads", tokens=1, q_heads=32, k_heads=8, dim=128, rotary=128, pairs="halves", kind="rms", dtype="bf16",
             weights="bf16", far=100000),
        # a batch of texts of different lengths
        dict(name="heads_batch", op="heads", tokens=16384, q_heads=32, k_heads=8, dim=128, rotary=128, pairs="halves", kind="rms", dtype="bf16",
             weights="bf16", far=8192),
        # the backward pass of odd sizes: part of a head is rotated, neighbours are a pair
        dict(name="heads_backward_odd", op="heads_backward", tokens=2049, q_heads=6, k_heads=6, dim=100, rotary=50, pairs="neighbours", kind="layer",
             dtype="f32", weights="f32", far=4000),
        # the backward pass of a training batch
        dict(name="heads_backward_batch", op="heads_backward", tokens=16384, q_heads=32, k_heads=8, dim=128, rotary=128, pairs="halves", kind="rms",
             dtype="bf16", weights="f32", far=8192),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["save", "linear", "gated", "gated_backward", "heads", "heads_backward"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "save":
        rows = _log(rng, 1, 16384)
        cols = _log(rng, 1, min(16384, 8192 * 4096 // rows))
        return dict(op=op, rows=rows, cols=cols, ld=cols + rng.choice([0, 0, 1, 8, 100]), dtype=dtype, both=rng.random() < 0.4)
    if op == "linear":
        m, n = _log(rng, 1, 8192), _log(rng, 8, 8192)
        return dict(op=op, m=m, n=n, k=_log(rng, 32, min(16384, 8192 * 8192 * 4096 // (m * n))), dtype=dtype, alpha=rng.choice([1.0, 0.5, 0.37]),
                    accumulate=rng.random() < 0.3)
    if op in ("gated", "gated_backward"):
        m, f = _log(rng, 1, 4096), _log(rng, 16, 8192)
        c = dict(op=op, m=m, f=f, k=_log(rng, 16, 4096), dtype=dtype, activation=rng.choice(["silu", "gelu", "gelu_tanh", "relu"]))
        return c | dict(keep=rng.random() < 0.5) if op == "gated" else c
    dim = rng.choice([32, 64, 64, 80, 100, 128, 128, 128, 192, 256])
    kv = rng.choice([1, 2, 4, 8])
    q = kv * rng.choice([1, 2, 4, 7])
    return dict(op=op, tokens=_log(rng, 1, min(16384, 16384 * 40 * 128 // ((q + kv) * dim))), q_heads=q, k_heads=kv, dim=dim,
                rotary=rng.choice([dim, dim, dim // 4 * 2]), pairs=rng.choice(["halves", "neighbours"]), kind=rng.choice(["rms", "rms", "layer"]),
                dtype=dtype, weights=rng.choice(["f32", "bf16"]), far=_log(rng, 4096, 200000))


def _i8_bytes(rows, cols):
    """What a matrix in 8 bits cannot do without: its codes and a magnitude for each row."""
    return rows * cols + 4 * rows


def work(case):
    op, es = case["op"], 4 if case["dtype"] == "f32" else 2
    if op == "save":
        r, c = case["rows"], case["cols"]
        moved = 2 * es * r * c + 2 * _i8_bytes(r, c) + (es * r * c + 2 * _i8_bytes(c, r) if case["both"] else 0)
        return {"bytes": moved, "flops": 0}
    if op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": es * m * k + 2 * _i8_bytes(m, k) + _i8_bytes(n, k) + es * m * n * (1 + case["accumulate"]), "flops": 2 * m * n * k}
    if op == "gated":
        m, f, k = case["m"], case["f"], case["k"]
        return {"bytes": es * m * k + 2 * _i8_bytes(m, k) + 2 * _i8_bytes(f, k) + es * m * f * (3 if case["keep"] else 1), "flops": 4 * m * f * k}
    if op == "gated_backward":
        m, f, k = case["m"], case["f"], case["k"]
        moved = es * m * f * 5 + 2 * _i8_bytes(m, 2 * f) + 2 * _i8_bytes(2 * f, m) + _i8_bytes(k, 2 * f) + _i8_bytes(k, m) + 2 * m * k + 2 * 2 * f * k
        return {"bytes": moved, "flops": 8 * m * f * k}
    t, h, d, ws = case["tokens"], case["q_heads"] + case["k_heads"], case["dim"], 4 if case["weights"] == "f32" else 2
    small = t * (4 + 4 * case["rotary"])
    if op == "heads":
        return {"bytes": 2 * es * t * h * d + small + 2 * ws * d, "flops": 8 * t * h * d}
    return {"bytes": 3 * es * t * h * d + small + 4 * ws * d, "flops": 16 * t * h * d}


# ---- matrices in 8 bits, in plain operations -----------------------------------------------------

def _scale(magnitude):
    s = (magnitude / 127).clamp(min=2.0 ** -126)
    return torch.where(magnitude == 0, torch.zeros_like(s), s)


def _quantise(x):
    """(whole numbers as fp32, magnitudes) of x, a scale for each row.  (Quotients in 64 bits: in 32 they may be rounded to a tie.)"""
    x = x.float()
    a = x.abs().amax(dim=1)
    s = _scale(a)[:, None]
    q = torch.round(x.double() / torch.where(s == 0, 1.0, s).double())
    return q.float(), a


def _restored(x):
    """What a matrix is after it was held in 8 bits, in fp32."""
    q, a = _quantise(x)
    return q * _scale(a)[:, None]


# ---- the container: 128 bytes of header, codes, magnitudes ---------------------------------------
# Codes: blocks of 128 rows (the last one: as many as there are, to a multiple of 8), in each the columns in chunks of 16, in each chunk 16
# bytes a row; columns padded to a multiple of 32.  Magnitudes: fp32, rows padded to a multiple of 8.

def _pack(x):
    rows, cols = x.shape
    r8, kp = -(-rows // 8) * 8, -(-cols // 32) * 32
    q, a = _quantise(x)
    codes = torch.nn.functional.pad(q.to(torch.int8), (0, kp - cols, 0, r8 - rows)).view(torch.uint8).reshape(r8, kp // 16, 16)
    full = r8 // 128 * 128
    a = torch.nn.functional.pad(a, (0, r8 - rows)).view(torch.uint8)
    head = np.zeros(128, dtype=np.uint8)
    head[:4] = np.frombuffer(b"FHI8", dtype=np.uint8)
    head[4] = 1
    head[8:16] = np.array([rows, cols], dtype=np.int32).view(np.uint8)
    head[24:32] = np.array([128 + r8 * kp + 4 * r8], dtype=np.uint64).view(np.uint8)
    return torch.cat([torch.from_numpy(head).to(x.device), codes[:full].reshape(-1, 128, kp // 16, 16).transpose(1, 2).reshape(-1),
                      codes[full:].transpose(0, 1).reshape(-1), a])


def _unpack(buf, rows, cols, to=torch.float32):
    r8, kp = -(-rows // 8) * 8, -(-cols // 32) * 32
    full, c = r8 // 128 * 128, buf[128:128 + r8 * kp]
    codes = torch.cat([c[:full * kp].reshape(-1, kp // 16, 128, 16).transpose(1, 2).reshape(full, kp),
                       c[full * kp:].reshape(kp // 16, r8 - full, 16).transpose(0, 1).reshape(r8 - full, kp)])
    a = buf[128 + r8 * kp:].view(torch.float32)[:rows]
    return codes.view(torch.int8)[:rows, :cols].to(to) * _scale(a).to(to)[:, None]


# ---- inputs ---------------------------------------------------------------------------------------

def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + salt)
    return g


def _values(seed, salt, rows, cols, scale):
    """Normal values whose columns differ in size, one in 64 of them eight times larger, as activations have them."""
    g = _gen(seed, salt)
    x = torch.randn(rows, cols, device="cuda", generator=g)
    size = torch.exp(0.3 * torch.randn(cols, device="cuda", generator=g))
    size = torch.where(torch.rand(cols, device="cuda", generator=g) < 1 / 64, 8 * size, size)
    return x * (size * scale)


def _table(rows, rotary):
    """Cosine and sine of position times 10000^(-2i / rotary), the angles in 64 bits."""
    at = torch.arange(rows, device="cuda", dtype=torch.float64)
    angle = at[:, None] * 10000.0 ** (-torch.arange(0, rotary, 2, device="cuda", dtype=torch.float64) / rotary)
    return torch.stack([torch.cos(angle), torch.sin(angle)], dim=2).float()


def _positions(seed, tokens, far):
    """Places of tokens of several texts in a row; a single token's is the last."""
    if tokens == 1:
        return torch.full((1,), far - 1 - seed % 7, dtype=torch.int32, device="cuda")
    g = _gen(seed, 9)
    starts = torch.rand(tokens, device="cuda", generator=g) < 1 / 1000
    at = torch.arange(tokens, device="cuda")
    begin = torch.cummax(torch.where(starts, at, torch.zeros_like(at)), dim=0).values
    return ((at - begin + seed % 7) % far).to(torch.int32)


def _make(case, seed):
    """The inputs of a case, from the seed alone."""
    op, dt = case["op"], DT[case["dtype"]]
    if op == "save":
        r, c = case["rows"], case["cols"]
        wide = torch.zeros(r, case["ld"], dtype=dt, device="cuda")
        wide[:, :c] = _values(seed, 1, r, c, 1.0)
        return dict(x=wide[:, :c])
    if op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        s = dict(x=_values(seed, 1, m, k, 1.0).to(dt), w=_pack(_values(seed, 2, n, k, 0.03)))
        if case["accumulate"]:
            s["c"] = torch.randn(m, n, device="cuda", generator=_gen(seed, 3)).to(dt)
        return s
    if op == "gated":
        m, f, k = case["m"], case["f"], case["k"]
        return dict(x=_values(seed, 1, m, k, 1.0).to(dt), gate=_pack(_values(seed, 2, f, k, 0.7 * k ** -0.5)), up=_pack(_values(seed, 3, f, k, 0.7 * k ** -0.5)))
    if op == "gated_backward":
        m, f, k = case["m"], case["f"], case["k"]
        return dict(pre=_values(seed, 1, m, 2 * f, 1.0).to(dt), dh=_values(seed, 2, m, f, 0.1).to(dt), w=_pack(_values(seed, 3, 2 * f, k, 0.03).t()),
                    x=_pack(_values(seed, 4, m, k, 1.0).t()))
    t, hq, hk, d, wt = case["tokens"], case["q_heads"], case["k_heads"], case["dim"], DT[case["weights"]]
    g = _gen(seed, 6)
    qkv = (_values(seed, 1, t, (hq + 2 * hk) * d, 1.0)).to(dt)
    s = dict(qkv=qkv, gq=(1 + 0.2 * torch.randn(d, device="cuda", generator=g)).to(wt), gk=(1 + 0.2 * torch.randn(d, device="cuda", generator=g)).to(wt),
             table=_table(case["far"], case["rotary"]), at=_positions(seed, t, case["far"]))
    if op == "heads_backward":
        s |= dict(dq=_values(seed, 7, t, hq * d, 0.1).to(dt).view(t, hq, d), dk=_values(seed, 8, t, hk * d, 0.1).to(dt).view(t, hk, d))
    return s


def prepare(case, seed):
    return dict(case=case, **_make(case, seed))


# ---- one pass -------------------------------------------------------------------------------------

def run(state):
    return globals()[("_own_" if own else "_plain_") + state["case"]["op"]](state["case"], state)


def _plain_save(case, s):
    x, dt = s["x"], DT[case["dtype"]]
    out = [_restored(x).to(dt)]
    if case["both"]:
        out.append(_restored(x.t().contiguous()).to(dt))
    return out


def _plain_linear(case, s):
    c = (_restored(s["x"]) @ _unpack(s["w"], case["n"], case["k"]).t()) * case["alpha"]
    return (s["c"].float() + c if case["accumulate"] else c).to(DT[case["dtype"]])


def _act(g, kind):
    """(activation, its derivative) of g."""
    if kind == "silu":
        p = 1 / (1 + torch.exp(-g))
        return g * p, p * (1 + g * (1 - p))
    if kind == "gelu":
        p = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * p, p + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    if kind == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (g + 0.044715 * g * g * g))
        return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * (c * (1 + 3 * 0.044715 * g * g))
    on = (g > 0).to(g.dtype)
    return g * on, on


def _plain_gated(case, s):
    x, dt = _restored(s["x"]), DT[case["dtype"]]
    g, u = x @ _unpack(s["gate"], case["f"], case["k"]).t(), x @ _unpack(s["up"], case["f"], case["k"]).t()
    h = (_act(g, case["activation"])[0] * u).to(dt)
    return [h, torch.cat([g, u], dim=1).to(dt)] if case["keep"] else [h]


def _plain_gated_backward(case, s):
    m, f, k, dt = case["m"], case["f"], case["k"], DT[case["dtype"]]
    g, u, dh = s["pre"][:, :f].float(), s["pre"][:, f:].float(), s["dh"].float()
    a, da = _act(g, case["activation"])
    dpre = torch.cat([dh * u * da, dh * a], dim=1).to(dt)
    dx = _restored(dpre) @ _unpack(s["w"], k, 2 * f).t()
    dw = _restored(dpre.t().contiguous()) @ _unpack(s["x"], k, m).t()
    return [dpre, dx.bfloat16(), dw.bfloat16()]


def _heads(case, s):
    """Queries and keys in the packed rows."""
    t, hq, hk, d = case["tokens"], case["q_heads"], case["k_heads"], case["dim"]
    x = s["qkv"].view(t, hq + 2 * hk, d)
    return x[:, :hq], x[:, hq:hq + hk]


def _pairs(z, rotary, pairs):
    """First and second of each pair, and what is not rotated."""
    if pairs == "halves":
        return z[..., :rotary // 2], z[..., rotary // 2:rotary], z[..., rotary:]
    return z[..., 0:rotary:2], z[..., 1:rotary:2], z[..., rotary:]


def _joined(a, b, rest, pairs):
    return torch.cat(([a, b] if pairs == "halves" else [torch.stack([a, b], dim=-1).flatten(-2)]) + [rest], dim=-1)


def _unit(x, kind):
    if kind == "layer":
        x = x - x.mean(dim=-1, keepdim=True)
    rstd = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS)
    return x * rstd, rstd


def _plain_heads_one(case, s, x, gamma):
    z = _unit(x.float(), case["kind"])[0] * gamma.float()
    a, b, rest = _pairs(z, case["rotary"], case["pairs"])
    row = s["table"][s["at"].long()][:, None]
    c, n = row[..., 0], row[..., 1]
    return _joined(a * c - b * n, b * c + a * n, rest, case["pairs"]).to(x.dtype)


def _plain_heads(case, s):
    q, k = _heads(case, s)
    return [_plain_heads_one(case, s, q, s["gq"]), _plain_heads_one(case, s, k, s["gk"])]


def _plain_heads_backward_one(case, s, x, gamma, dy):
    xhat, rstd = _unit(x.float(), case["kind"])
    a, b, rest = _pairs(dy.float(), case["rotary"], case["pairs"])
    row = s["table"][s["at"].long()][:, None]
    c, n = row[..., 0], row[..., 1]
    dz = _joined(a * c + b * n, b * c - a * n, rest, case["pairs"])
    g = dz * gamma.float()
    dx = g - xhat * (g * xhat).mean(dim=-1, keepdim=True)
    if case["kind"] == "layer":
        dx = dx - g.mean(dim=-1, keepdim=True)
    return (dx * rstd).to(x.dtype), (dz * xhat).sum(dim=(0, 1)).to(gamma.dtype)


def _plain_heads_backward(case, s):
    q, k = _heads(case, s)
    (dq, gq), (dk, gk) = _plain_heads_backward_one(case, s, q, s["gq"], s["dq"]), _plain_heads_backward_one(case, s, k, s["gk"], s["dk"])
    return [dq, dk, gq, gk]


# ---- the package's calls --------------------------------------------------------------------------

def _check(api, rc):
    if rc != api.FH_OK:
        raise api.FhError(rc, "operators on 8-bit matrices and heads")


def _kind(api, name):
    return api.FH_F32 if name == "f32" else api.FH_BF16


def _room(api, rows, cols):
    return torch.empty(api.i8_bytes(rows, cols), dtype=torch.uint8, device="cuda")


def _own_save(case, s):
    from paper_2510_11400_b200 import api
    x, kind = s["x"], _kind(api, case["dtype"])
    rows, cols = x.shape
    by_rows, by_cols = _room(api, rows, cols), _room(api, cols, rows) if case["both"] else None
    _check(api, api.fh_i8_compress(api.matrix(rows, cols, kind, x.stride(0)), x, by_rows, by_cols))
    out = [torch.empty(rows, cols, dtype=x.dtype, device=x.device)]
    _check(api, api.fh_i8_decompress(by_rows, api.matrix(rows, cols, kind), out[0]))
    if case["both"]:
        out.append(torch.empty(cols, rows, dtype=x.dtype, device=x.device))
        _check(api, api.fh_i8_decompress(by_cols, api.matrix(cols, rows, kind), out[1]))
    return out


def _own_linear(case, s):
    from paper_2510_11400_b200 import api
    m, n, k, x, kind = case["m"], case["n"], case["k"], s["x"], _kind(api, case["dtype"])
    x8 = _room(api, m, k)
    _check(api, api.fh_i8_compress(api.matrix(m, k, kind), x, x8))
    c = s["c"].clone() if case["accumulate"] else torch.empty(m, n, dtype=x.dtype, device=x.device)
    _check(api, api.fh_i8_product(api.i8_product_desc(m, n, k, kind, alpha=case["alpha"], accumulate=case["accumulate"]), x8, s["w"], c))
    return c


def _gated_desc(api, case):
    act = {"silu": api.FH_SILU, "gelu": api.FH_GELU, "gelu_tanh": api.FH_GELU_TANH, "relu": api.FH_RELU}[case["activation"]]
    return api.gated_desc(case["m"], case["f"], case["k"], act, _kind(api, case["dtype"]))


def _own_gated(case, s):
    from paper_2510_11400_b200 import api
    m, f, k, x = case["m"], case["f"], case["k"], s["x"]
    x8 = _room(api, m, k)
    _check(api, api.fh_i8_compress(api.matrix(m, k, _kind(api, case["dtype"])), x, x8))
    h = torch.empty(m, f, dtype=x.dtype, device=x.device)
    pre = torch.empty(m, 2 * f, dtype=x.dtype, device=x.device) if case["keep"] else None
    _check(api, api.fh_i8_gated(_gated_desc(api, case), x8, s["gate"], s["up"], h, pre))
    return [h, pre] if case["keep"] else [h]


def _own_gated_backward(case, s):
    from paper_2510_11400_b200 import api
    m, f, k, pre, kind = case["m"], case["f"], case["k"], s["pre"], _kind(api, case["dtype"])
    dpre, by_rows, by_cols = torch.empty_like(pre), _room(api, m, 2 * f), _room(api, 2 * f, m)
    _check(api, api.fh_gated_backward(_gated_desc(api, case), s["dh"], pre, dpre, by_rows))
    _check(api, api.fh_i8_compress(api.matrix(m, 2 * f, kind), dpre, None, by_cols))
    dx, dw = (torch.empty(rows, k, dtype=torch.bfloat16, device=pre.device) for rows in (m, 2 * f))
    _check(api, api.fh_i8_product(api.i8_product_desc(m, k, 2 * f, api.FH_BF16), by_rows, s["w"], dx))
    _check(api, api.fh_i8_product(api.i8_product_desc(2 * f, k, m, api.FH_BF16), by_cols, s["x"], dw))
    return [dpre, dx, dw]


def _heads_desc(api, case, q, k):
    return api.heads_desc(case["tokens"], case["q_heads"], case["k_heads"], case["dim"], case["rotary"], _kind(api, case["dtype"]), _kind(api, case["weights"]),
                          kind=api.FH_HEADS_RMS if case["kind"] == "rms" else api.FH_HEADS_LAYER,
                          pairs=api.FH_PAIRS_HALVES if case["pairs"] == "halves" else api.FH_PAIRS_NEIGHBOURS, eps=EPS, positions=case["far"],
                          q_strides=q.stride()[:2], k_strides=k.stride()[:2])


def _own_heads(case, s):
    from paper_2510_11400_b200 import api
    q, k = _heads(case, s)
    out = [torch.empty(q.shape, dtype=q.dtype, device=q.device), torch.empty(k.shape, dtype=k.dtype, device=k.device)]
    _check(api, api.fh_head_norm(_heads_desc(api, case, q, k), q, k, s["gq"], s["gk"], s["table"], s["at"], out[0], out[1]))
    return out


def _own_heads_backward(case, s):
    from paper_2510_11400_b200 import api
    q, k = _heads(case, s)
    d = _heads_desc(api, case, q, k)
    # (the gradients of queries and keys lie as these do, in rows of the packed matrix's width)
    grad = torch.empty_like(s["qkv"])
    dq, dk = _heads(case, dict(qkv=grad))
    gq, gk = torch.empty_like(s["gq"]), torch.empty_like(s["gk"])
    room = torch.empty(api.heads_work_bytes(d), dtype=torch.uint8, device="cuda")
    _check(api, api.fh_head_norm_backward(d, s["dq"], s["dk"], q, k, s["gq"], s["gk"], s["table"], s["at"], dq, dk, gq, gk, room))
    return [dq, dk, gq, gk]


# ---- the definition in 64 bits --------------------------------------------------------------------

def _exact_held(x):
    """x, in its own type, after it was held in 8 bits."""
    a = x.abs().max(dim=1).values.float()
    s = torch.where(a > 0, torch.maximum(a / 127, a.new_tensor(2.0 ** -126)), a).double()[:, None]
    t = x.double() / torch.where(s > 0, s, torch.ones_like(s))
    low = torch.floor(t)
    up = (t - low > 0.5) | ((t - low == 0.5) & (low % 2 != 0))
    return (low + up.double()) * s


def _exact_act(g, kind):
    if kind == "silu":
        p = torch.sigmoid(g)
        return g * p, p + g * p * torch.sigmoid(-g)
    if kind == "gelu":
        p = torch.special.ndtr(g)
        return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        w = c * (g + 0.044715 * g ** 3)
        p = torch.sigmoid(2 * w)                                    # (1 + tanh w) / 2
        return g * p, p + g * 2 * p * torch.sigmoid(-2 * w) * c * (1 + 3 * 0.044715 * g * g)
    return torch.relu(g), torch.heaviside(g, torch.zeros((), dtype=g.dtype, device=g.device))


def _exact_turn(case, s):
    """The rotation of a token's head as complex numbers, and back."""
    row = s["table"].double()[s["at"].long()]
    return torch.complex(row[..., 0], row[..., 1])[:, None, :]


def _exact_rotated(case, z, turn):
    r = case["rotary"]
    if case["pairs"] == "halves":
        w = torch.complex(z[..., :r // 2], z[..., r // 2:r]) * turn
        return torch.cat([w.real, w.imag, z[..., r:]], dim=-1)
    w = torch.view_as_complex(z[..., :r].reshape(*z.shape[:-1], r // 2, 2).contiguous()) * turn
    return torch.cat([torch.view_as_real(w).flatten(-2), z[..., r:]], dim=-1)


def _exact_unit(case, x):
    x = x.double()
    if case["kind"] == "layer":
        x = x - x.sum(dim=-1, keepdim=True) / x.shape[-1]
    size = torch.sqrt(torch.einsum("thd,thd->th", x, x) / x.shape[-1] + EPS)[..., None]
    return x / size, size


def exact(case, seed):
    s, op = _make(case, seed), case["op"]
    if op == "save":
        return [_exact_held(x) for x in [s["x"]] + ([s["x"].t().contiguous()] if case["both"] else [])]
    if op == "linear":
        c = case["alpha"] * (_exact_held(s["x"]) @ _unpack(s["w"], case["n"], case["k"], torch.float64).t())
        return c + s["c"].double() if case["accumulate"] else c
    if op == "gated":
        x = _exact_held(s["x"])
        g, u = x @ _unpack(s["gate"], case["f"], case["k"], torch.float64).t(), x @ _unpack(s["up"], case["f"], case["k"], torch.float64).t()
        h = _exact_act(g, case["activation"])[0] * u
        return [h, torch.cat([g, u], dim=1)] if case["keep"] else [h]
    if op == "gated_backward":
        m, f, k = case["m"], case["f"], case["k"]
        g, u = s["pre"].double().split(f, dim=1)
        a, da = _exact_act(g, case["activation"])
        dpre = torch.cat([s["dh"].double() * u * da, s["dh"].double() * a], dim=1)
        kept = dpre.to(DT[case["dtype"]])
        dx = _exact_held(kept) @ _unpack(s["w"], k, 2 * f, torch.float64).t()
        return [dpre, dx, _exact_held(kept.t().contiguous()) @ _unpack(s["x"], k, m, torch.float64).t()]
    turn, q, k = _exact_turn(case, s), *_heads(case, s)
    if op == "heads":
        return [_exact_rotated(case, _exact_unit(case, x)[0] * g.double(), turn) for x, g in ((q, s["gq"]), (k, s["gk"]))]
    out = []
    for x, gamma, dy in ((q, s["gq"], s["dq"]), (k, s["gk"], s["dk"])):
        unit, size = _exact_unit(case, x)
        dz = _exact_rotated(case, dy.double(), turn.conj())
        g = dz * gamma.double()
        dx = g - unit * torch.einsum("thd,thd->th", g, unit)[..., None] / case["dim"]
        if case["kind"] == "layer":
            dx = dx - g.sum(dim=-1, keepdim=True) / case["dim"]
        out.append((dx / size, torch.einsum("thd,thd->d", dz, unit)))
    return [out[0][0], out[1][0], out[0][1], out[1][1]]
