"""Refusals of the functions on 8-bit matrices, of the gated block and of norms of heads, and their size formulas: host-side, before any CUDA call.  And
what the binding refuses before the library is called."""
import ctypes as C
import types

import pytest

from oracle import i8
from paper_2510_11400_b200 import api, build

A, B = 4096, 1 << 30    # aligned addresses that nothing reads
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    build.build()
    return api.lib()


ARG, CAP, UNS = api.FH_ERR_ARG, api.FH_ERR_CAPACITY, api.FH_ERR_UNSUPPORTED


def test_struct_sizes_match_the_header():
    assert C.sizeof(api.fh_i8_product_desc) == 32 and C.sizeof(api.fh_gated_desc) == 40 and C.sizeof(api.fh_heads_desc) == 112


@pytest.mark.parametrize("shape", [(1, 1), (8, 32), (9, 33), (128, 256), (129, 257), (2 ** 31 - 1, 1), (1, 2 ** 31 - 1), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_sizes(lib, shape):
    assert api.i8_bytes(*shape) == i8.sizes(*shape)[2]


def test_sizes_of_nothing(lib):
    assert api.i8_bytes(0, 5) == api.i8_bytes(5, 0) == api.i8_bytes(-1, 5) == 0


def changed(d, **kw):
    c = type(d).from_buffer_copy(d)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_compress_refuses(lib):
    def call(m, src=A, rows=B, rcap=BIG, cols=2 * B, ccap=BIG):
        return lib.fh_i8_compress(m, src, rows, rcap, cols, ccap, None)
    m = api.matrix(10, 40)
    for bad in (None, api.matrix(0, 40), api.matrix(10, 0), api.matrix(10, 40, 2), api.matrix(10, 40, 0, 39), api.matrix(2 ** 31 - 1, 40, 0, 2 ** 40),
                changed(m, reserved=1)):
        assert call(bad) == ARG
    for kw in (dict(src=None), dict(rows=None, cols=None), dict(src=A + 2), dict(rows=B + 8), dict(cols=2 * B + 4)):
        assert call(m, **kw) == ARG, kw
    assert call(api.matrix(10, 40, api.FH_BF16), src=A + 1) == ARG
    assert call(m, rcap=api.i8_bytes(10, 40) - 1) == CAP and call(m, ccap=api.i8_bytes(40, 10) - 1) == CAP
    n = api.i8_bytes(10, 40)
    for kw in (dict(rows=B, cols=B), dict(rows=B, cols=B + n - 16), dict(src=B + n - 4), dict(src=2 * B - 1596)):
        assert call(m, **kw) == ARG, kw


def test_decompress_refuses(lib):
    def call(m, src=A, n=BIG, dst=B, status=None):
        return lib.fh_i8_decompress(src, n, m, dst, status, None)
    m = api.matrix(10, 40)
    assert call(None) == call(m, src=None) == call(m, dst=None) == call(m, src=A + 8) == call(m, dst=B + 2) == call(m, dst=A) == call(m, status=A + 4) == ARG
    assert call(m, status=A + 8) == call(m, status=B + 1592) == call(api.matrix(10, 40, 3)) == call(api.matrix(10, 40, 0, 8)) == ARG


def test_product_refuses(lib):
    def call(d, a=A, b=A, c=B, status=None):
        return lib.fh_i8_product(d, a, BIG, b, BIG, c, status, None)
    good = api.i8_product_desc(5, 6, 7)
    assert call(None) == ARG
    for bad in (dict(m=0), dict(n=0), dict(k=-1), dict(dtype=2), dict(ldc=5), dict(alpha=float("nan")), dict(alpha=float("inf")), dict(ldc=2 ** 62),
                dict(accumulate=2)):
        assert call(changed(good, **bad)) == ARG, bad
    assert call(changed(good, k=api.FH_I8_MAX_K + 1)) == UNS
    for kw in (dict(a=None), dict(b=None), dict(c=None), dict(a=A + 8), dict(b=A + 8), dict(c=B + 2), dict(c=A), dict(c=A + 128), dict(status=A), dict(status=B + 112),
               dict(status=B + 1004)):
        assert call(good, **kw) == ARG, kw
    assert call(api.i8_product_desc(2 ** 28, 2 ** 28, 7), a=16, b=1 << 40, c=1 << 59) == UNS


def test_gated_refuses(lib):
    def forward(d, x=A, gate=B, up=2 * B, h=3 * B, pre=4 * B, status=None):
        return lib.fh_i8_gated(d, x, BIG, gate, BIG, up, BIG, h, pre, status, None)

    def backward(d, dh=A, pre=B, dpre=2 * B, packed=3 * B, cap=BIG):
        return lib.fh_gated_backward(d, dh, pre, dpre, packed, cap, None)
    good = api.gated_desc(5, 6, 7)
    for f in (forward, backward):
        assert f(None) == ARG
        for bad in (dict(rows=0), dict(width=0), dict(width=2 ** 30), dict(activation=4), dict(activation=-1), dict(dtype=2), dict(reserved=1), dict(ldh=5),
                    dict(ldp=11), dict(ldh=2 ** 62), dict(ldp=2 ** 62)):
            assert f(changed(good, **bad)) == ARG, bad
    assert forward(changed(good, k=0)) == ARG and forward(changed(good, k=api.FH_I8_MAX_K + 1)) == UNS
    for kw in (dict(x=None), dict(gate=None), dict(up=None), dict(h=None, pre=None), dict(x=A + 8), dict(gate=B + 4), dict(up=2 * B + 2), dict(h=3 * B + 2),
               dict(pre=4 * B + 1), dict(status=4), dict(h=A), dict(h=B + 16), dict(pre=2 * B), dict(h=4 * B + 4), dict(status=3 * B), dict(status=4 * B + 8),
               dict(status=B)):
        assert forward(good, **kw) == ARG, kw
    for kw in (dict(dh=None), dict(pre=None), dict(dpre=None, packed=None), dict(dh=A + 2), dict(pre=B + 1), dict(dpre=2 * B + 2), dict(packed=3 * B + 8),
               dict(dpre=A), dict(dpre=B + 4), dict(packed=A), dict(packed=B), dict(packed=2 * B + 16)):
        assert backward(good, **kw) == ARG, kw
    assert backward(good, cap=api.i8_bytes(5, 12) - 1) == CAP


Q, K, QO, KO, GQ, GK, T, P = (i << 30 for i in range(1, 9))


def test_heads_refuse(lib):
    def forward(d, q=Q, k=K, gq=GQ, gk=GK, table=T, at=P, qo=QO, ko=KO, status=None):
        return lib.fh_head_norm(d, q, k, gq, gk, table, at, qo, ko, status, None)

    def backward(d, yq=QO, yk=KO, q=Q, k=K, gq=GQ, gk=GK, table=T, at=P, dq=9 << 30, dk=10 << 30, wq=11 << 30, wk=12 << 30, work=13 << 30, n=BIG, status=None):
        return lib.fh_head_norm_backward(d, yq, yk, q, k, gq, gk, table, at, dq, dk, wq, wk, work, n, status, None)
    good = api.heads_desc(5, 4, 2, 16, 8, positions=5)
    n = api.heads_work_bytes(good)
    assert n >= 2 * 16 * 4 and api.heads_work_bytes(changed(good, tokens=0)) == 0
    for f in (forward, backward):
        assert f(None) == ARG
        for bad in (dict(dtype=2), dict(wdtype=-1), dict(kind=2), dict(pairs=2), dict(tokens=0), dict(dim=0), dict(rotary=7), dict(rotary=18), dict(rotary=-2), dict(positions=0),
                    dict(q_heads=-1), dict(q_heads=0, k_heads=0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(reserved=1),
                    dict(q_token=63), dict(q_head=15), dict(k_out_token=-1), dict(q_out_head=-16), dict(k_token=2 ** 61), dict(q_token=16, q_head=16),
                    dict(q_token=16, q_head=79), dict(q_head=17)):
            assert f(changed(good, **bad)) == ARG, bad
        assert f(changed(api.heads_desc(1, 1, 0, 8194), positions=1)) == UNS
        for kw in (dict(q=None), dict(k=None), dict(table=None), dict(q=Q + 2), dict(gq=GQ + 1), dict(table=T + 4), dict(at=P + 2), dict(status=P - 4)):
            assert f(good, **kw) == ARG, kw
        assert f(changed(good, positions=4), at=None) == ARG         # positions 0 ... 4 are not all in the table
    # outputs that meet an input, one another, or something smaller
    for kw in (dict(qo=None), dict(ko=None), dict(qo=Q + 4), dict(qo=K), dict(ko=Q), dict(ko=QO), dict(qo=GQ), dict(ko=T + 64), dict(qo=P - 16), dict(status=Q), dict(status=QO + 8),
               dict(status=GK + 8), dict(status=T), dict(status=P)):
        assert forward(good, **kw) == ARG, kw
    for kw in (dict(yq=None), dict(yk=None), dict(dq=None, dk=None, wq=None, wk=None), dict(work=None), dict(work=(13 << 30) + 8), dict(dq=Q + 4), dict(dq=K), dict(dk=Q), dict(dq=KO),
               dict(dk=9 << 30), dict(wq=Q), dict(wk=GQ), dict(wq=12 << 30), dict(work=QO), dict(work=9 << 30), dict(work=11 << 30), dict(dq=GK), dict(dk=T), dict(status=9 << 30),
               dict(status=13 << 30), dict(status=11 << 30), dict(status=Q), dict(wq=P), dict(wk=T)):
        assert backward(good, **kw) == ARG, kw
    assert backward(good, n=n - 1) == CAP
    only_q = api.heads_desc(5, 4, 0, 16, 8, positions=5)
    assert backward(only_q) == ARG                                    # a gradient of keys that there are none of
    # in place with other strides
    assert forward(changed(good, q_out_token=80), qo=Q) == ARG and backward(changed(good, q_out_token=80), dq=QO) == ARG


def test_tables_refuse(lib):
    f = lambda *a, p=A: lib.fh_rotation_table(*a, p, None)  # noqa: E731
    nan, inf = float("nan"), float("inf")
    for a in ((0, 2, 10.0, 1.0), (1, 0, 10.0, 1.0), (1, 3, 10.0, 1.0), (1, 2, 0.0, 1.0), (1, 2, -1.0, 1.0), (1, 2, nan, 1.0), (1, 2, inf, 1.0), (1, 2, 10.0, nan), (1, 2, 10.0, inf)):
        assert f(*a) == ARG, a
    assert f(1, 2, 10.0, 1.0, p=None) == ARG and f(1, 2, 10.0, 1.0, p=A + 4) == ARG


torch = pytest.importorskip("torch")
STREAM = types.SimpleNamespace(cuda_stream=0)
U8 = torch.uint8


@pytest.fixture
def calls(monkeypatch):
    """The library's calls: host tensors stand for CUDA tensors and a list for the library."""
    build.build()
    real, made = api.lib(), []

    class Library:
        def __getattr__(self, name):
            if name.endswith("bytes"):
                return getattr(real, name)
            return lambda *a: made.append(name) or api.FH_OK

    monkeypatch.setattr(api, "_device", lambda: -1)    # (where host tensors are)
    monkeypatch.setattr(api, "lib", lambda: Library())
    return made


def taken(calls, call):
    calls.clear()
    assert call() == api.FH_OK and len(calls) == 1


def refused(calls, call):
    calls.clear()
    with pytest.raises(ValueError):
        call()
    assert not calls


def test_the_binding_takes_matrices_as_they_are_described(calls):
    buf, wide = torch.zeros(1 << 16, dtype=U8), torch.zeros(64, 96)
    m, p, g = api.matrix(10, 40, api.FH_F32, 96), api.i8_product_desc(10, 40, 32, ldc=96), api.gated_desc(10, 40, 8, ldh=96, ldp=96)

    def each(x):
        return [lambda: api.fh_i8_compress(m, x, buf, None, STREAM), lambda: api.fh_i8_decompress(buf, m, x, None, STREAM),
                lambda: api.fh_i8_product(p, buf, buf, x, None, STREAM), lambda: api.fh_i8_gated(g, buf, buf, buf, x, None, None, STREAM),
                lambda: api.fh_gated_backward(g, x, wide, wide, None, STREAM)]
    for call in each(wide[:, :40]) + each(wide[3:20, 7:47]):
        taken(calls, call)
    for x in (wide[:, :40].t(), wide[:, ::2], torch.zeros(10, 40), wide[:, :40].double(), wide[:, :40].half(), wide[:5, :40].contiguous()):
        for call in each(x):
            refused(calls, call)
    for bad in (torch.zeros(1, dtype=torch.int32), torch.zeros(2)):
        refused(calls, lambda: api.fh_i8_product(p, buf, buf, wide, bad, STREAM))
        refused(calls, lambda: api.fh_i8_gated(g, buf, buf, buf, wide, None, bad, STREAM))
        refused(calls, lambda: api.fh_i8_decompress(buf, m, wide, bad, STREAM))
    refused(calls, lambda: api.fh_i8_product(p, buf[::2], buf, wide, None, STREAM))


def test_the_binding_takes_heads_as_they_are_described(calls):
    t, hq, hk, dim = 6, 4, 2, 16
    packed = torch.zeros(t, (hq + 2 * hk) * dim).view(t, hq + 2 * hk, dim)
    q, k = packed[:, :hq], packed[:, hq:hq + hk]
    d = api.heads_desc(t, hq, hk, dim, 8, positions=9, q_strides=q.stride()[:2], k_strides=k.stride()[:2])
    oq, ok, gamma, table, at = torch.zeros(t, hq, dim), torch.zeros(t, hk, dim), torch.zeros(dim), torch.zeros(9, 4, 2), torch.zeros(t, dtype=torch.int32)
    work = torch.zeros(api.heads_work_bytes(d), dtype=U8)

    def both(**kw):
        a = dict(q=q, k=k, gq=gamma, gk=gamma, table=table, at=at, oq=oq, ok=ok) | kw
        return [lambda: api.fh_head_norm(d, a["q"], a["k"], a["gq"], a["gk"], a["table"], a["at"], a["oq"], a["ok"], None, STREAM),
                lambda: api.fh_head_norm_backward(d, a["oq"], a["ok"], a["q"], a["k"], a["gq"], a["gk"], a["table"], a["at"], a["q"], a["k"], a["gq"], a["gk"], work, None,
                                                  STREAM)]
    for kw in ({}, dict(at=None), dict(gq=None), dict(oq=torch.zeros(t * hq * dim)), dict(at=torch.zeros(t, dtype=torch.uint32))):
        for call in both(**kw):
            taken(calls, call)
    for kw in (dict(q=k), dict(k=q), dict(q=torch.zeros(t, hq, dim)), dict(oq=q), dict(oq=torch.zeros(t, hq, dim, dtype=torch.float64)), dict(oq=torch.zeros(t, hq, dim).half()),
               dict(gq=torch.zeros(dim - 1)), dict(table=torch.zeros(8, 4, 2)), dict(at=torch.zeros(t, dtype=torch.int64)), dict(at=torch.zeros(t)),
               dict(at=torch.zeros(t - 1, dtype=torch.int32)), dict(oq=torch.zeros(t * hq * dim - 1)), dict(q=packed[:, :hq].transpose(0, 1))):
        for call in both(**kw):
            refused(calls, call)
