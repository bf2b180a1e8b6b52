"""Measured work of the microscaled 4-bit operators: saving and restoring matrices, products of matrices held in 4 bits, and
the layer norm that writes its output in 4 bits and whose backward pass reads its saved input from them.

A value in 4 bits is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign (E2M1), times the scale of its block: consecutive elements of
a row, the last block of a row padded with zeros.  Format 0: blocks of 32, the scale a power of two (E8M0).  Format 1: blocks of 16,
the scale an E4M3 number times 2^exponent, the exponent given for the whole matrix.  The scale is the smallest of its type that
is at least a sixth of the block's largest magnitude (2^125 and 448 at most, a block of zeros: the smallest); values are rounded
to nearest, ties to even, or at random.

`run` with own = False computes the operators with elementary torch operations, with own = True through the package's API.
"""
import math

import numpy as np
import torch

own = False

BLOCK = (32, 16)
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- cases --------------------------------------------------------------------------------------

def listed():
    return [
        # one token's activation, kept in 4 bits until it is wanted: two launches and little else
        dict(name="save_restore_token", op="save", rows=1, cols=4096, ld=4096, dtype="bf16", format=0, exponent=0, rounding=0, both=False),
        # a slice of a wider fp32 matrix, its rows on no 16-byte boundary, its last blocks short
        dict(name="save_restore_odd", op="save", rows=4099, cols=1000, ld=1003, dtype="f32", format=1, exponent=-6, rounding=0, both=False),
        # a saved activation of a large batch
        dict(name="save_restore_large", op="save", rows=16384, cols=8192, ld=8192, dtype="bf16", format=0, exponent=0, rounding=0, both=False),
        # a gradient for both products of a linear layer's backward pass: blocks along rows and along columns, random rounding
        dict(name="save_restore_gradient", op="save", rows=8192, cols=4096, ld=4096, dtype="bf16", format=1, exponent=-12, rounding=1, both=True),
        # one token through a linear layer
        dict(name="product_token", op="product", m=1, n=8192, k=8192, dtype="bf16", format=1, ea=0, eb=-4, alpha=1.0, accumulate=False),
        # a prompt or a training batch through a linear layer
        dict(name="product_linear", op="product", m=4096, n=4096, k=4096, dtype="bf16", format=1, ea=0, eb=-4, alpha=1.0, accumulate=False),
        # a weight's gradient added to the sum so far: few tiles, a long axis of tokens, odd sizes
        dict(name="product_weight_gradient", op="product", m=1000, n=777, k=16384, dtype="f32", format=0, ea=0, eb=0, alpha=0.5, accumulate=True),
        # the largest product
        dict(name="product_large", op="product", m=8192, n=16384, k=8192, dtype="bf16", format=0, ea=0, eb=0, alpha=1.0, accumulate=False),
        # layer norm straight into 4 bits and the linear layer that reads them, for a few tokens
        dict(name="norm_linear", op="norm_linear", rows=16, cols=4096, n=4096, dtype="bf16", weights="bf16", format=1, exponent=0, eb=-4),
        # layer norm of a training batch
        dict(name="norm_forward", op="norm", rows=16384, cols=4096, dtype="bf16", weights="f32", affine=True),
        # its backward pass from dense inputs, odd sizes, fp32
        dict(name="norm_backward_odd", op="norm_backward", rows=5001, cols=1111, dtype="f32", weights="f32", packed=False, format=0),
        # its backward pass from an input that was saved in 4 bits
        dict(name="norm_backward_packed", op="norm_backward", rows=16384, cols=4096, dtype="bf16", weights="bf16", packed=True, format=0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["save", "product", "norm_linear", "norm", "norm_backward"])
    dtype, fmt = rng.choice(["f32", "bf16"]), rng.choice([0, 1])
    if op == "save":
        rows = _log(rng, 1, 16384)
        cols = _log(rng, 1, min(16384, 8192 * 8192 // rows))
        return dict(op=op, rows=rows, cols=cols, ld=cols + rng.choice([0, 0, 1, 8, 100]), dtype=dtype, format=fmt,
                    exponent=rng.choice([-12, -6, 0]) if fmt else 0, rounding=rng.choice([0, 0, 1]), both=rng.random() < 0.4)
    if op == "product":
        m, n, k = _log(rng, 1, 8192), _log(rng, 8, 8192), _log(rng, 32, 16384)
        return dict(op=op, m=m, n=n, k=k, dtype=dtype, format=fmt, ea=rng.choice([0, -6]) if fmt else 0, eb=-4 if fmt else 0,
                    alpha=rng.choice([1.0, 0.5, 0.37]), accumulate=rng.random() < 0.3)
    if op == "norm_linear":
        return dict(op=op, rows=_log(rng, 1, 4096), cols=_log(rng, 32, 8192), n=_log(rng, 8, 4096), dtype="bf16",
                    weights=rng.choice(["f32", "bf16"]), format=fmt, exponent=0, eb=-4 if fmt else 0)
    rows = _log(rng, 1, 16384)
    cols = _log(rng, 32, min(20000, 4096 * 16384 // rows))
    if op == "norm":
        return dict(op=op, rows=rows, cols=cols, dtype=dtype, weights=rng.choice(["f32", "bf16"]), affine=rng.random() < 0.8)
    return dict(op=op, rows=rows, cols=cols, dtype=dtype, weights=rng.choice(["f32", "bf16"]), packed=rng.random() < 0.5, format=fmt)


def _mx_bytes(rows, cols, fmt):
    """What a matrix in 4 bits cannot do without: its codes and its scales."""
    return rows * (cols / 2 + math.ceil(cols / BLOCK[fmt]))


def work(case):
    op, es = case["op"], 4 if case["dtype"] == "f32" else 2
    if op == "save":
        r, c, f = case["rows"], case["cols"], case["format"]
        moved = es * r * c * (2 + case["both"]) + 2 * _mx_bytes(r, c, f) + (2 * _mx_bytes(c, r, f) if case["both"] else 0)
        return {"bytes": moved, "flops": 0}
    if op == "product":
        m, n, k, f = case["m"], case["n"], case["k"], case["format"]
        return {"bytes": _mx_bytes(m, k, f) + _mx_bytes(n, k, f) + es * m * n * (1 + case["accumulate"]), "flops": 2 * m * n * k}
    r, c, ws = case["rows"], case["cols"], 4 if case["weights"] == "f32" else 2
    if op == "norm_linear":
        n, f = case["n"], case["format"]
        return {"bytes": es * r * c + 2 * ws * c + 8 * r + 2 * _mx_bytes(r, c, f) + _mx_bytes(n, c, f) + es * r * n, "flops": 2 * r * n * c}
    if op == "norm":
        return {"bytes": 2 * es * r * c + (2 * ws * c if case["affine"] else 0) + 8 * r, "flops": 8 * r * c}
    x = _mx_bytes(r, c, case["format"]) if case["packed"] else es * r * c
    return {"bytes": 2 * es * r * c + x + 3 * ws * c + 8 * r, "flops": 12 * r * c}


# ---- matrices in 4 bits, in plain operations -----------------------------------------------------

def _blocks(x, fmt):
    """[rows, cols] as [rows, blocks, block], zeros behind the last column."""
    b = BLOCK[fmt]
    return torch.nn.functional.pad(x, (0, -x.shape[1] % b)).reshape(x.shape[0], -1, b)


def _pow2(k):
    """2^k for whole k, exact, in 64 bits."""
    return ((k.to(torch.int64) + 1023) << 52).view(torch.float64)


def _scales(top, fmt):
    """The smallest scale of the format that is at least top / 6, and its byte."""
    if fmt == 0:
        m, e = torch.frexp(top)                                     # top = m 2^e, m in [0.5, 1): 6 2^k = 0.75 2^(k+3)
        k = torch.where(m > 0.75, e - 2, e - 3)
        k = torch.where(top == 0, -127, k).clamp(-127, 125)
        return _pow2(k).float(), k + 127
    t = top / 6
    _, e = torch.frexp(t)
    unit = _pow2(e.clamp(min=-5) - 4).float()                       # distance of neighbouring E4M3 numbers around t
    s = (torch.ceil(t / unit) * unit).clamp(2.0 ** -9, 448.0)
    m, e = torch.frexp(s)
    return s, torch.where(s < 2.0 ** -6, s * 512, (e + 6) * 8 + (m * 16 - 8)).to(torch.int32)


def _mulhilo(a, b):
    p, q = a * (b >> 16), a * (b & 0xFFFF)
    return (p + (q >> 16)) >> 16, ((p << 16) + q) & 0xFFFFFFFF


def _draws(rows, cols, seed, tensor_id, device):
    """16 uniform bits for each element: Philox-4x32-10, key = seed, counter = (col / 8, row, tensor id), eight draws a call."""
    c0 = torch.arange((cols + 7) // 8, device=device)[None, :].expand(rows, -1)
    c1 = torch.arange(rows, device=device)[:, None].expand_as(c0)
    c2, c3 = torch.full_like(c0, tensor_id & 0xFFFFFFFF), torch.full_like(c0, tensor_id >> 32)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        h0, l0 = _mulhilo(0xD2511F53, c0)
        h1, l1 = _mulhilo(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    w = torch.stack([c0, c1, c2, c3], dim=-1)
    return torch.stack([w & 0xFFFF, w >> 16], dim=-1).reshape(rows, -1)[:, :cols]


def _quantise(x, fmt, exponent, draws=None):
    """(values of the codes, scales without the factor 2^exponent, scale bytes) of x, blocks along its rows."""
    b = _blocks(x.float(), fmt) * 2.0 ** -exponent
    s, code = _scales(b.abs().amax(dim=2), fmt)
    # (quotients by a scale of four bits are inexact; a nearest value is the right one all the same, a drawn one needs 64 bits)
    to = torch.float64 if fmt == 1 and draws is not None else torch.float32
    a = b.abs().to(to) / s[:, :, None].to(to)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).to(to)
    if draws is None:
        q = (torch.round(a / step) * step).clamp(max=6.0)
    else:
        r = _blocks(draws, fmt).to(to)
        low = torch.floor(a / step)
        q = ((low + (a / step - low > (r + 0.5) / 65536)) * step).clamp(max=6.0)
    return torch.copysign(q.float(), b), s, code


def _restored(x, fmt, exponent, draws=None):
    """What a matrix is after it was held in 4 bits."""
    q, s, _ = _quantise(x, fmt, exponent, draws)
    return (q * s[:, :, None] * 2.0 ** exponent).reshape(x.shape[0], -1)[:, :x.shape[1]]


# ---- the container: 128 bytes of header, codes, scales -------------------------------------------
# Codes: blocks of 128 rows (the last one: as many as there are, to a multiple of 8), in each the columns in chunks of 32, in each chunk 16
# bytes a row; columns padded to a multiple of 64.  Scales: for 128 rows and 4 blocks 512 bytes, row r's at 16 (r % 32) + 4 (r / 32).

def _sizes(rows, cols, fmt):
    r8, kp = -(-rows // 8) * 8, -(-cols // 64) * 64
    atoms = -(-rows // 128) * -(-kp // (4 * BLOCK[fmt]))
    return r8, kp, r8 * kp // 2, atoms * 512


def _pack(x, fmt, exponent):
    rows, cols = x.shape
    r8, kp, nc, ns = _sizes(rows, cols, fmt)
    q, _, byte = _quantise(x, fmt, exponent)
    a = q.abs()
    idx = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) | (torch.signbit(q).to(torch.uint8) << 3)
    idx = torch.nn.functional.pad(idx.reshape(rows, -1)[:, :cols], (0, kp - cols, 0, r8 - rows))
    codes = (idx[:, 0::2] | (idx[:, 1::2] << 4)).reshape(r8, kp // 32, 16)
    full = r8 // 128 * 128
    parts = [codes[:full].reshape(-1, 128, kp // 32, 16).transpose(1, 2).reshape(-1), codes[full:].transpose(0, 1).reshape(-1)]
    nb4 = -(-kp // (4 * BLOCK[fmt])) * 4
    byte = torch.nn.functional.pad(byte.to(torch.uint8), (0, nb4 - byte.shape[1], 0, -rows % 128))
    parts.append(byte.reshape(-1, 4, 32, nb4 // 4, 4).permute(0, 3, 2, 1, 4).reshape(-1))
    head = np.zeros(128, dtype=np.uint8)
    head[:4] = np.frombuffer(b"FHM4", dtype=np.uint8)
    head[4:8] = np.array([1, 0, fmt, 0], dtype=np.uint8)
    head[8:20] = np.array([rows, cols, exponent], dtype=np.int32).view(np.uint8)
    head[24:32] = np.array([128 + nc + ns], dtype=np.uint64).view(np.uint8)
    return torch.cat([torch.from_numpy(head).to(x.device)] + parts)


def _unpack(buf, rows, cols, fmt, exponent, to=torch.float32):
    r8, kp, nc, ns = _sizes(rows, cols, fmt)
    full, c = r8 // 128 * 128, buf[128:128 + nc]
    codes = torch.cat([c[:full * kp // 2].reshape(-1, kp // 32, 128, 16).transpose(1, 2).reshape(full, kp // 2),
                       c[full * kp // 2:].reshape(kp // 32, r8 - full, 16).transpose(0, 1).reshape(r8 - full, kp // 2)])
    idx = torch.stack([codes & 15, codes >> 4], dim=-1).reshape(r8, kp)[:rows]
    level = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=to, device=buf.device)
    bs = BLOCK[fmt]
    byte = buf[128 + nc:128 + nc + ns].reshape(-(-rows // 128), -1, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-(-rows // 128) * 128, -1)
    byte = byte[:rows, :kp // bs].to(torch.int32)
    if fmt == 0:
        s = _pow2(byte - 127).to(to)
    else:
        s = torch.where(byte < 8, byte, 8 + byte % 8).to(to) * _pow2((byte // 8).clamp(min=1) - 10 + exponent).to(to)
    return (level[idx.int()].reshape(rows, -1, bs) * s[:, :, None]).reshape(rows, kp)[:, :cols]


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


def _make(case, seed):
    """The inputs of a case, from the seed alone."""
    op, dt = case["op"], DT[case["dtype"]]
    if op == "save":
        r, c = case["rows"], case["cols"]
        wide = torch.zeros(r, case["ld"], dtype=dt, device="cuda")
        wide[:, :c] = _values(seed, 1, r, c, 2.0 ** case["exponent"])
        return dict(x=wide[:, :c], draw_seed=(seed * 2654435761 + 12345) & 0xFFFFFFFFFFFF, tensor_id=seed + (5 << 32))
    if op == "product":
        f = case["format"]
        a, b = _values(seed, 1, case["m"], case["k"], 2.0 ** case["ea"]), _values(seed, 2, case["n"], case["k"], 0.03 if not f else 2.0 ** case["eb"])
        s = dict(a=_pack(a, f, case["ea"]), b=_pack(b, f, case["eb"]))
        if case["accumulate"]:
            s["c"] = torch.randn(case["m"], case["n"], device="cuda", generator=_gen(seed, 3)).to(dt)
        return s
    r, c, wt = case["rows"], case["cols"], DT[case["weights"]]
    x = (_values(seed, 1, r, c, 1.0) + 0.5).to(dt)
    g = _gen(seed, 4)
    s = dict(gamma=(1 + 0.2 * torch.randn(c, device="cuda", generator=g)).to(wt), beta=(0.2 * torch.randn(c, device="cuda", generator=g)).to(wt))
    if op == "norm_linear":
        s["w"] = _pack(_values(seed, 2, case["n"], c, 0.03 if not case["format"] else 2.0 ** case["eb"]), case["format"], case["eb"])
    if op == "norm_backward":
        d = x.double()
        mean, var = d.mean(dim=1), d.var(dim=1, unbiased=False)
        s |= dict(dy=_values(seed, 5, r, c, 0.1).to(dt), mean=mean.float(), rstd=torch.rsqrt(var + EPS).float())
        if case["packed"]:
            return s | dict(x=_pack(x, case["format"], 0))
    return s | dict(x=x)


EPS = 1e-5


def prepare(case, seed):
    return dict(case=case, **_make(case, seed))


# ---- one pass -------------------------------------------------------------------------------------

def run(state):
    return globals()[("_own_" if own else "_plain_") + state["case"]["op"]](state["case"], state)


def _plain_save(case, s):
    x, f, e, dt = s["x"], case["format"], case["exponent"], DT[case["dtype"]]
    rows, cols = x.shape
    d = _draws(rows, cols, s["draw_seed"], s["tensor_id"], x.device) if case["rounding"] else None
    out = [_restored(x, f, e, d).to(dt)]
    if case["both"]:
        d = _draws(cols, rows, s["draw_seed"], s["tensor_id"], x.device) if case["rounding"] else None
        out.append(_restored(x.t().contiguous(), f, e, d).to(dt))
    return out


def _plain_product(case, s):
    m, n, k, f = case["m"], case["n"], case["k"], case["format"]
    c = _unpack(s["a"], m, k, f, case["ea"]) @ _unpack(s["b"], n, k, f, case["eb"]).t()
    c = c * case["alpha"]
    return (s["c"].float() + c if case["accumulate"] else c).to(DT[case["dtype"]])


def _norm(x, gamma, beta):
    x = x.float()
    mean = x.mean(dim=1)
    d = x - mean[:, None]
    rstd = torch.rsqrt((d * d).mean(dim=1) + EPS)
    y = d * rstd[:, None]
    return (y if gamma is None else y * gamma.float() + beta.float()), mean, rstd


def _plain_norm(case, s):
    y, mean, rstd = _norm(s["x"], *((s["gamma"], s["beta"]) if case["affine"] else (None, None)))
    return [y.to(s["x"].dtype), mean, rstd]


def _plain_norm_linear(case, s):
    y, mean, rstd = _norm(s["x"], s["gamma"], s["beta"])
    y = _restored(y.to(s["x"].dtype), case["format"], case["exponent"]).float()
    w = _unpack(s["w"], case["n"], case["cols"], case["format"], case["eb"])
    return [(y @ w.t()).to(s["x"].dtype), mean, rstd]


def _plain_norm_backward(case, s):
    x = _unpack(s["x"], case["rows"], case["cols"], case["format"], 0) if case["packed"] else s["x"].float()
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xhat = (x - s["mean"][:, None]) * rstd
    g = dy * s["gamma"].float()
    dx = rstd * (g - g.mean(dim=1, keepdim=True) - xhat * (g * xhat).mean(dim=1, keepdim=True))
    return [dx.to(s["dy"].dtype), (dy * xhat).sum(dim=0).to(s["gamma"].dtype), dy.sum(dim=0).to(s["gamma"].dtype)]


# ---- the package's calls --------------------------------------------------------------------------

def _check(api, rc):
    if rc != api.FH_OK:
        raise api.FhError(rc, "microscaled operators")


def _own_save(case, s):
    from paper_2510_11400_b200 import api
    x, f, dt = s["x"], case["format"], DT[case["dtype"]]
    rows, cols = x.shape
    p = api.mx_params(f, case["exponent"], case["rounding"], s["draw_seed"], s["tensor_id"])
    m = api.matrix(rows, cols, api.FH_F32 if dt == torch.float32 else api.FH_BF16, x.stride(0))
    by_rows = torch.empty(api.mx_bytes(rows, cols, f), dtype=torch.uint8, device=x.device)
    by_cols = torch.empty(api.mx_bytes(cols, rows, f), dtype=torch.uint8, device=x.device) if case["both"] else None
    _check(api, api.fh_mx_compress(m, p, x, by_rows, by_cols))
    out = [torch.empty(rows, cols, dtype=dt, device=x.device)]
    _check(api, api.fh_mx_decompress(by_rows, api.matrix(rows, cols, m.dtype), f, out[0]))
    if case["both"]:
        out.append(torch.empty(cols, rows, dtype=dt, device=x.device))
        _check(api, api.fh_mx_decompress(by_cols, api.matrix(cols, rows, m.dtype), f, out[1]))
    return out


def _own_product(case, s):
    from paper_2510_11400_b200 import api
    m, n, k, dt = case["m"], case["n"], case["k"], DT[case["dtype"]]
    c = s["c"].clone() if case["accumulate"] else torch.empty(m, n, dtype=dt, device="cuda")
    d = api.mx_product_desc(m, n, k, case["format"], api.FH_F32 if dt == torch.float32 else api.FH_BF16, alpha=case["alpha"],
                            accumulate=case["accumulate"])
    _check(api, api.fh_mx_product(d, s["a"], s["b"], c))
    return c


def _norm_desc(api, case):
    kind = {"f32": api.FH_F32, "bf16": api.FH_BF16}
    return api.norm_desc(case["rows"], case["cols"], kind[case["dtype"]], kind[case["weights"]], EPS)


def _own_norm(case, s):
    from paper_2510_11400_b200 import api
    x = s["x"]
    y, mean, rstd = torch.empty_like(x), torch.empty(x.shape[0], device=x.device), torch.empty(x.shape[0], device=x.device)
    gamma, beta = (s["gamma"], s["beta"]) if case["affine"] else (None, None)
    _check(api, api.fh_layer_norm(_norm_desc(api, case), x, gamma, beta, y, mean, rstd))
    return [y, mean, rstd]


def _own_norm_linear(case, s):
    from paper_2510_11400_b200 import api
    x, f = s["x"], case["format"]
    rows, cols = x.shape
    mean, rstd = torch.empty(rows, device=x.device), torch.empty(rows, device=x.device)
    packed = torch.empty(api.mx_bytes(rows, cols, f), dtype=torch.uint8, device=x.device)
    d = _norm_desc(api, case)
    _check(api, api.fh_layer_norm(d, x, s["gamma"], s["beta"], None, mean, rstd, packed=packed, params=api.mx_params(f, case["exponent"])))
    c = torch.empty(rows, case["n"], dtype=x.dtype, device=x.device)
    _check(api, api.fh_mx_product(api.mx_product_desc(rows, case["n"], cols, f, d.dtype), packed, s["w"], c))
    return [c, mean, rstd]


def _own_norm_backward(case, s):
    from paper_2510_11400_b200 import api
    dy, gamma = s["dy"], s["gamma"]
    dx, dgamma, dbeta = torch.empty_like(dy), torch.empty_like(gamma), torch.empty_like(gamma)
    d = _norm_desc(api, case)
    work_ = torch.empty(api.norm_work_bytes(d), dtype=torch.uint8, device=dy.device)
    _check(api, api.fh_layer_norm_backward(d, dy, s["x"], gamma, s["mean"], s["rstd"], dx, dgamma, dbeta, work_,
                                           packed=case["format"] if case["packed"] else None))
    return [dx, dgamma, dbeta]


# ---- the definition in 64 bits --------------------------------------------------------------------

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_scale_table(fmt, device):
    if fmt == 0:
        return torch.tensor([2.0 ** k for k in range(-127, 126)], dtype=torch.float64, device=device)
    return torch.tensor([m * 2.0 ** -9 for m in range(1, 8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1],
                        dtype=torch.float64, device=device)


def _exact_draws(rows, cols, seed, tensor_id):
    """The draws from a Philox-4x32-10 of its own, in unsigned 64-bit integers."""
    g, low = (cols + 7) // 8, np.uint64(0xFFFFFFFF)
    c = [np.tile(np.arange(g, dtype=np.uint64), rows), np.repeat(np.arange(rows, dtype=np.uint64), g),
         np.full(rows * g, tensor_id & 0xFFFFFFFF, dtype=np.uint64), np.full(rows * g, tensor_id >> 32, dtype=np.uint64)]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for i in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64((key[0] + i * 0x9E3779B9) & 0xFFFFFFFF), b & low,
             (a >> np.uint64(32)) ^ c[3] ^ np.uint64((key[1] + i * 0xBB67AE85) & 0xFFFFFFFF), a & low]
    return np.stack(c, axis=1).astype(np.uint32).view(np.uint16).reshape(rows, g * 8)[:, :cols]


def _exact_held(x, fmt, exponent, draws=None):
    """x after it was held in 4 bits: neighbours in the table of levels, and which of them is nearer or drawn."""
    rows, cols = x.shape
    out = torch.empty(rows, cols, dtype=torch.float64, device=x.device)
    table, levels = _exact_scale_table(fmt, x.device), torch.tensor(LEVELS, dtype=torch.float64, device=x.device)
    bs = BLOCK[fmt]
    for r in range(0, rows, 2048):
        v = x[r:r + 2048].double() * 2.0 ** -exponent
        v = torch.cat([v, v.new_zeros(v.shape[0], (bs - cols % bs) % bs)], dim=1)
        mag = v.abs().view(v.shape[0], -1, bs)
        top = mag.max(dim=2).values
        s = table[torch.searchsorted(6 * table, top).clamp(max=table.numel() - 1)][:, :, None]
        below = (torch.searchsorted(levels, (mag / s).contiguous(), right=True) - 1).clamp(0, 6)
        lo, hi = levels[below] * s, levels[below + 1] * s
        if draws is None:
            d = (mag - lo) - (hi - mag)
            up = (d > 0) | ((d == 0) & (below % 2 == 1))
        else:
            t = torch.from_numpy(draws[r:r + 2048].astype(np.int32)).to(x.device).double()
            t = torch.cat([t, t.new_zeros(t.shape[0], (bs - cols % bs) % bs)], dim=1).view_as(mag)
            up = (mag - lo) * 65536 > (hi - lo) * (t + 0.5)
        got = torch.where(up | (mag >= hi), hi, lo).view_as(v) * torch.sign(v)
        out[r:r + 2048] = got[:, :cols] * 2.0 ** exponent
    return out


def exact(case, seed):
    s, op = _make(case, seed), case["op"]
    if op == "save":
        rows, cols = s["x"].shape
        out = []
        for x in [s["x"]] + ([s["x"].t().contiguous()] if case["both"] else []):
            d = _exact_draws(x.shape[0], x.shape[1], s["draw_seed"], s["tensor_id"]) if case["rounding"] else None
            out.append(_exact_held(x, case["format"], case["exponent"], d))
        return out
    if op == "product":
        m, n, k, f = case["m"], case["n"], case["k"], case["format"]
        c = case["alpha"] * (_unpack(s["a"], m, k, f, case["ea"], torch.float64) @ _unpack(s["b"], n, k, f, case["eb"], torch.float64).t())
        return c + s["c"].double() if case["accumulate"] else c
    r, c = case["rows"], case["cols"]
    g, b = s["gamma"].double(), s["beta"].double()
    if op in ("norm", "norm_linear"):
        x = s["x"].double()
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = 1 / torch.sqrt(var + EPS)
        y = (x - mean[:, None]) * rstd[:, None]
        if op == "norm":
            return [g * y + b if case["affine"] else y, mean, rstd]
        y = _exact_held((g * y + b).to(s["x"].dtype), case["format"], case["exponent"])
        return [y @ _unpack(s["w"], case["n"], c, case["format"], case["eb"], torch.float64).t(), mean, rstd]
    x = _unpack(s["x"], r, c, case["format"], 0, torch.float64) if case["packed"] else s["x"].double()
    dy, rstd = s["dy"].double(), s["rstd"].double()
    xhat = torch.einsum("rc,r->rc", x - s["mean"].double()[:, None], rstd)
    p, q = dy @ g / c, torch.einsum("rc,rc,c->r", dy, xhat, g) / c
    dx = rstd[:, None] * (dy * g - p[:, None] - xhat * q[:, None])
    return [dx, torch.einsum("rc,rc->c", dy, xhat), dy.sum(dim=0)]
