"""Norms of queries and keys with the rotation by position, and their backward pass, against the plain definition in 64 bits."""
import numpy as np
import pytest

from oracle import i8
from paper_2510_11400_b200 import api, build

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U = 2.0 ** -24                                                       # half a step of fp32, relative
HALF = {api.FH_F32: U, api.FH_BF16: 2.0 ** -8}
TYPES = {api.FH_F32: torch.float32, api.FH_BF16: torch.bfloat16}
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build()
    api.lib()


def held(x, dtype):
    """fp32 values that the type holds."""
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(TYPES[dtype]).float().numpy()


class Rows:
    """[tokens, heads, dim] somewhere in a buffer that is 7 elsewhere."""

    def __init__(self, tokens, heads, dim, dtype, layout, values=None):
        strides = {"plain": (heads * dim, dim), "packed": ((heads + 3) * dim, dim), "turned": (dim, tokens * dim), "odd": (heads * (dim + 3) + 1, dim + 3),
                   "wide": (heads * (dim + 8) + 16, dim + 8)}[layout]
        start = 5 if layout == "odd" else 0
        self.strides = strides
        n = start + (tokens - 1) * strides[0] + (heads - 1) * strides[1] + dim if heads else 0
        self.flat = torch.full((n + 64,), 7.0, dtype=TYPES[dtype], device="cuda")
        self.view = self.flat.as_strided((tokens, heads, dim), (*strides, 1), start)
        if values is not None:
            self.view.copy_(torch.from_numpy(values))

    def read(self):
        torch.cuda.synchronize()
        got = self.view.float().cpu().numpy().copy()
        self.view.fill_(7.0)
        assert (self.flat == 7.0).all()
        return got


def setup(tokens, hq, hk, dim, rotary, dtype, wdtype, seed=0):
    rng = np.random.default_rng([seed, tokens, hq, hk, dim])
    rows = lambda h, s: held(rng.standard_normal((tokens, h, dim)) * s * np.exp(rng.standard_normal((tokens, h, 1))), dtype)  # noqa: E731
    positions = 37 + tokens
    at = rng.integers(0, positions, size=tokens).astype(np.int32)
    tab = i8.table(positions, max(rotary, 2)).astype(np.float32)
    gq, gk = (held(1 + 0.3 * rng.standard_normal(dim), wdtype) for _ in range(2))
    return dict(x=(rows(hq, 1.0), rows(hk, 3.0)), dy=(rows(hq, 0.1), rows(hk, 1.0)), g=(gq, gk), at=at, table=tab, positions=positions)


def cuda(x, dtype=None):
    t = torch.from_numpy(x).cuda()
    return t if dtype is None else t.to(TYPES[dtype])


def sums_slack(dim):
    """Relative error of a sum of `dim` numbers of one sign, and of what rstd is made of it, which halves it: chains of at most dim / 32 + 16 additions to a lane,
    five across lanes, one for the division, one for the addition, four for a reciprocal root within two places."""
    return (dim / 32 + 32) * U


def summed(z, cs, rotary, pairs):
    """Magnitudes z of pairs that are turned, summed up."""
    c, n = cs[:, None, :, 0], cs[:, None, :, 1]
    a = slice(0, rotary // 2) if pairs == i8.HALVES else slice(0, rotary, 2)
    b = slice(rotary // 2, rotary) if pairs == i8.HALVES else slice(1, rotary, 2)
    out = z.copy()
    out[..., a] = z[..., a] * c + z[..., b] * n
    out[..., b] = z[..., b] * c + z[..., a] * n
    return out


def forward_bound(x, g, cs, rotary, kind, pairs, dtype):
    """(the value, how far from it a result may be)."""
    want = i8.head_norm(x, g, cs, rotary, kind, pairs, EPS)
    unit, rstd = i8._unit(x, kind, EPS)
    rel = sums_slack(x.shape[-1])
    off = rel * np.abs(x).mean(axis=-1, keepdims=True) * rstd if kind == i8.LAYER else 0.0   # of the mean
    z = (np.abs(unit) * (rel + 6 * U) + 2 * off) * np.abs(g)
    z = summed(z + 3 * U * np.abs(unit * g), np.abs(cs), rotary, pairs) if rotary else z
    return want, z + HALF[dtype] * (1 + 1e-6) * np.abs(want)


def backward_bound(dy, x, g, cs, rotary, kind, pairs, dtype):
    dx, dg = i8.head_norm_backward(dy, x, g, cs, rotary, kind, pairs, EPS)
    unit, rstd = i8._unit(x, kind, EPS)
    rel = sums_slack(x.shape[-1])
    dz = i8._turned(dy.astype(np.float64), cs, rotary, pairs, True) if rotary else dy.astype(np.float64)
    size = summed(np.abs(dy), np.abs(cs), rotary, pairs) if rotary else np.abs(dy)          # of dz, ahead of cancelling
    off = rel * np.abs(x).mean(axis=-1, keepdims=True) * rstd if kind == i8.LAYER else 0.0  # of a unit's element
    eg, gs = 3 * U * size * np.abs(g), np.abs(dz * g)                                        # g and its error
    mean = lambda v: v.mean(axis=-1, keepdims=True)  # noqa: E731
    along, e_along = np.abs(mean(dz * g * unit)), mean(eg * np.abs(unit) + gs * ((rel + 6 * U) * np.abs(unit) + off)) + rel * mean(gs * np.abs(unit))
    e = eg + 2 * U * gs + np.abs(unit) * e_along + along * ((rel + 6 * U) * np.abs(unit) + 2 * off)
    if kind == i8.LAYER:
        e = e + mean(eg) + (rel + 4 * U) * mean(gs)
    inner = np.abs(dx) / rstd
    e_dx = rstd * (e + (rel + 6 * U) * inner) + HALF[dtype] * (1 + 1e-6) * np.abs(dx)
    n = x.shape[0] * x.shape[1]
    terms = np.abs(dz * unit)
    e_dg = (3 * U * size * np.abs(unit) + np.abs(dz) * ((rel + 6 * U) * np.abs(unit) + 2 * off) + (min(n, 4096) + 64) * U * terms).sum(axis=(0, 1))
    return dx, e_dx, dg, e_dg


CASES = [(1, 1, 0, 1, 0), (1, 0, 2, 2, 2), (1, 32, 8, 128, 128), (3, 5, 1, 128, 64), (2, 4, 4, 64, 64), (7, 3, 2, 80, 80), (5, 6, 6, 100, 50), (4, 2, 1, 256, 256),
         (3, 2, 2, 512, 512), (2, 1, 1, 8192, 4096), (9, 2, 1, 33, 32), (300, 7, 1, 96, 32), (2000, 8, 2, 64, 64), (513, 12, 12, 16, 8), (1500, 3, 1, 40, 10)]


@pytest.mark.parametrize("layout", ["plain", "packed", "turned", "odd", "wide"])
@pytest.mark.parametrize("kind", [i8.RMS, i8.LAYER])
@pytest.mark.parametrize("pairs", [i8.HALVES, i8.NEIGHBOURS])
@pytest.mark.parametrize("dtype,wdtype", [(api.FH_F32, api.FH_F32), (api.FH_BF16, api.FH_BF16), (api.FH_BF16, api.FH_F32)])
@pytest.mark.parametrize("case", CASES)
def test_both_passes(case, dtype, wdtype, pairs, kind, layout):
    tokens, hq, hk, dim, rotary = case
    s = setup(*case, dtype, wdtype)
    cs = s["table"][s["at"]].astype(np.float64)
    other = "plain" if layout != "plain" else "wide"                  # (inputs and outputs lie differently)
    q, k = (Rows(tokens, h, dim, dtype, layout, v) for h, v in ((hq, s["x"][0]), (hk, s["x"][1])))
    oq, ok = (Rows(tokens, h, dim, dtype, other) for h in (hq, hk))
    gq, gk = (cuda(g, wdtype) for g in s["g"])
    table, at = cuda(s["table"]) if rotary else None, cuda(s["at"])
    d = api.heads_desc(tokens, hq, hk, dim, rotary, dtype, wdtype, kind, pairs, EPS, s["positions"], q.strides, k.strides, oq.strides, ok.strides)
    pick = lambda t, h: t if h else None  # noqa: E731
    status = torch.full((1,), 99, dtype=torch.int64, device="cuda")
    assert api.fh_head_norm(d, pick(q.view, hq), pick(k.view, hk), gq, None, table, at, pick(oq.view, hq), pick(ok.view, hk), status) == api.FH_OK
    for h, out, x, g in ((hq, oq, s["x"][0], s["g"][0]), (hk, ok, s["x"][1], np.ones(dim))):
        if not h:
            continue
        want, bound = forward_bound(x, g, cs, rotary, kind, pairs, dtype)
        assert (np.abs(out.read() - want) <= bound + 1e-30).all()
    assert int(status.item()) == api.FH_OK
    yq, yk = (Rows(tokens, h, dim, dtype, other, v) for h, v in ((hq, s["dy"][0]), (hk, s["dy"][1])))
    dq, dk = (Rows(tokens, h, dim, dtype, layout) for h in (hq, hk))
    wq, wk = (torch.full((dim + 8,), 7.0, dtype=TYPES[wdtype], device="cuda") for _ in range(2))
    n = api.heads_work_bytes(d)
    work = torch.full((n + 64,), 0xA5, dtype=torch.uint8, device="cuda")

    def back(**kw):
        given = dict(dq=pick(dq.view, hq), dk=pick(dk.view, hk), dgamma_q=pick(wq[:dim], hq), dgamma_k=pick(wk[:dim], hk)) | kw
        assert api.fh_head_norm_backward(d, pick(yq.view, hq), pick(yk.view, hk), pick(q.view, hq), pick(k.view, hk), gq, gk, table, at, work=work[:n], status=status,
                                         **given) == api.FH_OK
    back()
    got = [(dq.read(), wq.clone()), (dk.read(), wk.clone())]
    assert int(status.item()) == api.FH_OK and (work[n:] == 0xA5).all()
    for h, (gx, gw), x, dy, g in ((hq, got[0], s["x"][0], s["dy"][0], s["g"][0]), (hk, got[1], s["x"][1], s["dy"][1], s["g"][1])):
        if not h:
            assert (gw == 7.0).all()
            continue
        dx, e_dx, dg, e_dg = backward_bound(dy, x, g, cs, rotary, kind, pairs, dtype)
        assert (np.abs(gx - dx) <= e_dx + 1e-30).all()
        assert (np.abs(gw[:dim].double().cpu().numpy() - dg) <= e_dg + HALF[wdtype] * (1 + 1e-6) * np.abs(dg) + 1e-30).all() and (gw[dim:] == 7.0).all()
    # each alone: the same bits
    back(dgamma_q=None, dgamma_k=None)
    assert np.array_equal(dq.read(), got[0][0]) and np.array_equal(dk.read(), got[1][0])
    wq.fill_(7.0)
    wk.fill_(7.0)
    back(dq=None, dk=None)
    assert torch.equal(wq, got[0][1]) and torch.equal(wk, got[1][1])
    dq.read(), dk.read()


@pytest.mark.parametrize("dim,rotary", [(128, 128), (128, 32), (90, 50)])
@pytest.mark.parametrize("pairs", [i8.HALVES, i8.NEIGHBOURS])
@pytest.mark.parametrize("alternate", [False, True])
def test_in_place_in_rows_of_queries_keys_and_values(alternate, pairs, dim, rotary):
    """q, k and v in one matrix, one after the other or head by head; everything over its own input, v untouched."""
    tokens, h = 50, 4
    s = setup(tokens, h, h, dim, rotary, api.FH_BF16, api.FH_F32)
    table, at, gq, gk = cuda(s["table"]), cuda(s["at"]), *(cuda(g) for g in s["g"])

    def fused(a, b):
        m = torch.full((tokens, 3 * h * dim), 7.0, dtype=torch.bfloat16, device="cuda")
        views = [m.view(tokens, h, 3, dim)[:, :, i] for i in range(3)] if alternate else [m.view(tokens, 3, h, dim)[:, i] for i in range(3)]
        views[0].copy_(torch.from_numpy(a))
        views[1].copy_(torch.from_numpy(b))
        return m, views
    m, (q, k, v) = fused(*s["x"])
    st = q.stride()[:2]
    apart = api.heads_desc(tokens, h, h, dim, rotary, api.FH_BF16, api.FH_F32, pairs=pairs, positions=s["positions"], q_strides=st, k_strides=st)
    inside = api.heads_desc(tokens, h, h, dim, rotary, api.FH_BF16, api.FH_F32, pairs=pairs, positions=s["positions"], q_strides=st, k_strides=st, q_out_strides=st,
                            k_out_strides=st)
    want = [torch.empty(tokens, h, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    assert api.fh_head_norm(apart, q, k, gq, gk, table, at, *want) == api.FH_OK
    mi, (qi, ki, vi) = fused(*s["x"])
    assert api.fh_head_norm(inside, qi, ki, gq, gk, table, at, qi, ki) == api.FH_OK
    assert torch.equal(qi, want[0]) and torch.equal(ki, want[1]) and (vi == 7.0).all()
    dy = [cuda(y, api.FH_BF16) for y in s["dy"]]
    md, (dq, dk, dv) = fused(*(np.zeros_like(x) for x in s["x"]))
    assert api.fh_head_norm_backward(apart, *dy, q, k, gq, gk, table, at, dq, dk) == api.FH_OK
    mi, (qi, ki, vi) = fused(*s["x"])                                 # over q and k
    assert api.fh_head_norm_backward(apart, *dy, qi, ki, gq, gk, table, at, qi, ki) == api.FH_OK
    assert torch.equal(qi, dq) and torch.equal(ki, dk) and (vi == 7.0).all()
    my, (yq, yk, yv) = fused(*s["dy"])                                # over the gradients
    assert api.fh_head_norm_backward(inside, yq, yk, q, k, gq, gk, table, at, yq, yk) == api.FH_OK
    assert torch.equal(yq, dq) and torch.equal(yk, dk) and (yv == 7.0).all()


@pytest.mark.parametrize("dim", [128, 100])
@pytest.mark.parametrize("tokens", [1, 6, 1000])
def test_positions_that_the_table_does_not_have(tokens, dim):
    """Such tokens are left out and the status says so; the others are as they are without them."""
    hq, hk = 4, 2
    s = setup(tokens, hq, hk, dim, dim, api.FH_F32, api.FH_F32)
    q, k, yq, yk = (cuda(v) for v in (*s["x"], *s["dy"]))
    gq, gk, table = *(cuda(g) for g in s["g"]), cuda(s["table"])
    d = api.heads_desc(tokens, hq, hk, dim, positions=s["positions"], eps=EPS)
    bad = s["at"].copy()
    out = np.arange(tokens) % 3 == 0
    bad[out] = np.array([-1, s["positions"], 2 ** 31 - 1, -2 ** 31])[np.arange(out.sum()) % 4]
    status = torch.full((1,), 99, dtype=torch.int64, device="cuda")
    res = {}
    for name, at in (("good", s["at"]), ("bad", bad)):
        o = [torch.full((tokens, h, dim), 7.0, device="cuda") for h in (hq, hk, hq, hk)]
        w = [torch.full((dim,), 7.0, device="cuda") for _ in range(2)]
        work = torch.empty(api.heads_work_bytes(d), dtype=torch.uint8, device="cuda")
        assert api.fh_head_norm(d, q, k, gq, gk, table, cuda(at), *o[:2], status) == api.FH_OK
        first = int(status.item())
        status.fill_(99)
        assert api.fh_head_norm_backward(d, yq, yk, q, k, gq, gk, table, cuda(at), *o[2:], *w, work, status) == api.FH_OK
        assert first == int(status.item()) == (api.FH_OK if name == "good" else api.FH_ERR_CORRUPT)
        res[name] = (o, w)
    for a, b in zip(res["good"][0], res["bad"][0]):
        assert (b[out] == 7.0).all() and torch.equal(b[~out], a[~out])
    cs = s["table"][s["at"]].astype(np.float64)[~out]
    for w, x, dy, g in zip(res["bad"][1], s["x"], s["dy"], s["g"]):
        if (~out).any():
            _, _, dg, e_dg = backward_bound(dy[~out], x[~out], g, cs, dim, i8.RMS, i8.HALVES, api.FH_F32)
            assert (np.abs(w.cpu().numpy() - dg) <= e_dg + U * np.abs(dg) + 1e-30).all()
        else:
            assert (w == 0).all()


def test_positions_in_order_and_rows_without_spread():
    d = api.heads_desc(5, 2, 0, 16, positions=5, eps=0.0)
    x = torch.randn(5, 2, 16, device="cuda")
    x[1, 1] = 0
    x[2, 0, 3] = float("nan")
    x[3, 1, 0] = float("inf")
    table = api.rotation_table(5, 16)
    out, same = torch.empty_like(x), torch.empty_like(x)
    assert api.fh_head_norm(d, x, None, None, None, table, None, out, None) == api.FH_OK
    assert api.fh_head_norm(d, x, None, None, None, table, torch.arange(5, dtype=torch.int32, device="cuda"), same, None) == api.FH_OK
    bad = torch.zeros(5, 2, dtype=torch.bool, device="cuda")
    bad[1, 1] = bad[2, 0] = True
    assert out[bad].isnan().all() and torch.equal(out[~bad].isnan(), same[~bad].isnan())
    fine = ~bad
    fine[3, 1] = False
    assert torch.equal(out[fine], same[fine]) and out[fine].isfinite().all()


@pytest.mark.parametrize("positions,rotary,base,scale", [(1, 2, 10000.0, 1.0), (300, 128, 10000.0, 1.0), (131072, 64, 500000.0, 0.25), (7, 10, 2.0, -1.5)])
def test_tables(positions, rotary, base, scale):
    got = api.rotation_table(positions, rotary, base, scale).cpu().numpy()
    want = i8.table(positions, rotary, base, scale)
    # angles up to 1e5 carry 1e5 * 2^-51 into the cosine; rounded once to fp32
    assert got.shape == want.shape and (np.abs(got - want) <= U * np.abs(want) + 1e-10).all()


def test_captured_and_on_another_stream():
    tokens, hq, hk, dim = 700, 8, 2, 64
    s = setup(tokens, hq, hk, dim, dim, api.FH_BF16, api.FH_F32)
    q, k, yq, yk = (cuda(v, api.FH_BF16) for v in (*s["x"], *s["dy"]))
    gq, gk, table, at = *(cuda(g) for g in s["g"]), cuda(s["table"]), cuda(s["at"])
    d = api.heads_desc(tokens, hq, hk, dim, dtype=api.FH_BF16, positions=s["positions"])

    def outputs():
        return [torch.zeros_like(t) for t in (q, k, q, k, gq, gk)] + [torch.empty(api.heads_work_bytes(d), dtype=torch.uint8, device="cuda"),
                                                                       torch.full((1,), 99, dtype=torch.int64, device="cuda")]

    def step(o, stream=None):
        assert api.fh_head_norm(d, q, k, gq, gk, table, at, o[0], o[1], o[7], stream) == api.FH_OK
        assert api.fh_head_norm_backward(d, yq, yk, q, k, gq, gk, table, at, *o[2:7], o[7], stream) == api.FH_OK

    want, side, graphed = outputs(), outputs(), outputs()
    step(want)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    step(side, stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(graphed)
    graph.replay()
    torch.cuda.synchronize()
    for o in (side, graphed):
        assert all(torch.equal(a, b) for a, b in zip(o[:6], want[:6])) and int(o[7].item()) == 0
    q.mul_(-0.5)
    yk.mul_(2)
    step(want)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(graphed[:6], want[:6]))
