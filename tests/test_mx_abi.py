"""Refusals of the microscaled matrices' functions and their size formula: host-side, before any CUDA call."""
import ctypes as C

import pytest

from oracle import mx
from paper_2510_11400_b200 import api, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return api.lib()


A = 4096    # an aligned address that nothing reads


def test_struct_sizes_match_the_header():
    assert C.sizeof(api.fh_matrix) == 24 and C.sizeof(api.fh_mx_params) == 32 and C.sizeof(api.fh_mx_product_desc) == 40


@pytest.mark.parametrize("fmt", [mx.B32, mx.B16])
@pytest.mark.parametrize("shape", [(1, 1), (8, 64), (9, 65), (128, 256), (129, 257), (1000, 40), (2 ** 31 - 1, 1), (1, 2 ** 31 - 1),
                                   (2 ** 31 - 1, 2 ** 31 - 1)])
def test_sizes(lib, shape, fmt):
    assert api.mx_bytes(*shape, fmt) == mx.sizes(*shape, fmt)[3]


def test_sizes_of_nothing(lib):
    assert api.mx_bytes(0, 5, 0) == api.mx_bytes(5, 0, 0) == api.mx_bytes(-1, 5, 0) == api.mx_bytes(5, 5, 2) == api.mx_bytes(5, 5, -1) == 0


def compress(lib, m, p, src=A, rows=A << 20, rcap=1 << 40, cols=A << 30, ccap=1 << 40):
    return lib.fh_mx_compress(C.byref(m) if m is not None else None, C.byref(p) if p is not None else None, src, rows, rcap, cols, ccap, None)


def test_compress_refuses(lib):
    m, p, ARG = api.matrix(10, 40), api.mx_params(), api.FH_ERR_ARG
    assert compress(lib, None, p) == ARG and compress(lib, m, None) == ARG
    for bad in (api.matrix(0, 40), api.matrix(10, 0), api.matrix(10, -4), api.matrix(10, 40, 2), api.matrix(10, 40, 0, 39),
                api.matrix(2 ** 31 - 1, 40, 0, 2 ** 40), api.matrix(2 ** 31 - 1, 2 ** 31 - 1), api.fh_matrix(0, 10, 40, 1, 40)):
        assert compress(lib, bad, p) == ARG
    for bad in (api.mx_params(2), api.mx_params(-1), api.mx_params(mx.B32, 1), api.mx_params(mx.B16, 65), api.mx_params(mx.B16, -65),
                api.fh_mx_params(0, 0, 0, 1, 0, 0)):
        assert compress(lib, m, bad) == ARG
    assert compress(lib, m, api.mx_params(rounding=2)) == api.FH_ERR_UNSUPPORTED
    assert compress(lib, m, p, src=None) == ARG and compress(lib, m, p, rows=None, cols=None) == ARG
    assert compress(lib, m, p, src=A + 2) == ARG and compress(lib, m, p, rows=(A << 20) + 8) == ARG and compress(lib, m, p, cols=(A << 30) + 8) == ARG
    assert compress(lib, api.matrix(10, 40, api.FH_BF16), p, src=A + 1) == ARG
    assert compress(lib, m, p, rcap=api.mx_bytes(10, 40, 0) - 1) == api.FH_ERR_CAPACITY
    assert compress(lib, m, p, ccap=api.mx_bytes(40, 10, 0) - 1) == api.FH_ERR_CAPACITY
    assert compress(lib, api.matrix(2 ** 29, 2 ** 29), p, src=16, rows=1 << 61, rcap=1 << 62, cols=1 << 62, ccap=1 << 62) == api.FH_ERR_UNSUPPORTED
    # containers that overlap one another, or the matrix
    n = api.mx_bytes(10, 40, 0)
    for kw in (dict(rows=A << 20, cols=A << 20), dict(rows=A << 20, cols=(A << 20) + n - 16), dict(src=(A << 20) + n - 4), dict(src=(A << 30) - 1596)):
        assert compress(lib, m, p, **kw) == ARG, kw


def test_decompress_refuses(lib):
    def call(m, fmt=0, src=A, n=1 << 40, dst=A << 20, status=None):
        return lib.fh_mx_decompress(src, n, C.byref(m) if m is not None else None, fmt, dst, status, None)
    m, ARG = api.matrix(10, 40), api.FH_ERR_ARG
    assert call(None) == ARG and call(m, 2) == ARG and call(m, src=None) == ARG and call(m, dst=None) == ARG
    assert call(m, src=A + 8) == ARG and call(m, dst=(A << 20) + 2) == ARG and call(m, dst=A) == ARG and call(m, status=A + 4) == ARG
    assert call(api.matrix(10, 40, 3)) == ARG and call(api.matrix(10, 40, 0, 8)) == ARG and call(api.matrix(0, 1)) == ARG


def test_product_refuses(lib):
    def call(d, a=A, b=A, c=A << 20, status=None):
        return lib.fh_mx_product(C.byref(d) if d is not None else None, a, 1 << 40, b, 1 << 40, c, status, None)
    ARG, good = api.FH_ERR_ARG, api.mx_product_desc(5, 6, 7)
    assert call(None) == ARG
    for bad in (dict(m=0), dict(n=0), dict(k=-1), dict(format=2), dict(dtype=2), dict(ldc=5), dict(alpha=float("nan")), dict(alpha=float("inf")),
                dict(ldc=2 ** 62)):
        kw = dict(m=5, n=6, k=7) | bad
        assert call(api.mx_product_desc(**kw)) == ARG, bad
    for field in ("accumulate", "reserved"):
        d = api.mx_product_desc(5, 6, 7)
        setattr(d, field, 2)
        assert call(d) == ARG
    assert call(good, a=None) == ARG and call(good, b=None) == ARG and call(good, c=None) == ARG
    assert call(good, a=A + 8) == ARG and call(good, b=A + 8) == ARG and call(good, c=(A << 20) + 2) == ARG and call(good, c=A) == ARG and call(good, status=A + 4) == ARG


def test_layer_norm_refuses(lib):
    assert C.sizeof(api.fh_norm_desc) == 40
    ARG, good, p = api.FH_ERR_ARG, api.norm_desc(10, 40), api.mx_params()

    def fwd(d=good, x=A, g=A, b=A, y=A, mean=A, rstd=A, prm=None, packed=None, cap=0):
        return lib.fh_layer_norm(C.byref(d) if d is not None else None, x, g, b, y, mean, rstd, C.byref(prm) if prm is not None else None, packed, cap, None)

    def bwd(d=good, dy=A, x=A, xb=0, xf=0, g=A, mean=A, rstd=A, dx=A, dg=A << 10, db=A << 11, work=A << 20, wb=1 << 40, status=None):
        return lib.fh_layer_norm_backward(C.byref(d) if d is not None else None, dy, x, xb, xf, g, mean, rstd, dx, dg, db, work, wb, status, None)

    bad = [None, api.norm_desc(0, 40), api.norm_desc(10, 0), api.norm_desc(10, 40, 2), api.norm_desc(10, 40, 0, 2), api.norm_desc(10, 40, eps=-1.0),
           api.norm_desc(10, 40, eps=float("nan")), api.norm_desc(10, 40, eps=float("inf")), api.norm_desc(10, 40, ldx=39), api.norm_desc(10, 40, ldy=39),
           api.norm_desc(2 ** 31 - 1, 40, ldx=2 ** 40), api.fh_norm_desc(0, 0, 10, 40, 0.0, 1, 40, 40)]
    for d in bad:
        assert fwd(d) == ARG and bwd(d) == ARG
        assert lib.fh_layer_norm_work_bytes(C.byref(d) if d is not None else None) == 0
    assert fwd(api.norm_desc(10, 28673)) == bwd(api.norm_desc(10, 28673)) == api.FH_ERR_UNSUPPORTED
    assert fwd(x=None) == ARG and fwd(y=None) == ARG
    for name in ("x", "g", "b", "y", "mean", "rstd"):
        assert fwd(**{name: A + 2}) == ARG, name
    assert fwd(packed=A << 20) == ARG and fwd(prm=p, packed=A, cap=1 << 40) == ARG and fwd(prm=p, packed=A + 8, cap=1 << 40) == ARG and fwd(prm=api.mx_params(3), packed=A << 20, cap=1 << 40) == ARG
    assert fwd(prm=api.mx_params(rounding=1), packed=A << 20, cap=1 << 40) == api.FH_ERR_UNSUPPORTED
    assert fwd(prm=p, packed=A << 20, cap=api.mx_bytes(10, 40, 0) - 1) == api.FH_ERR_CAPACITY
    for name in ("dy", "x", "mean", "rstd"):
        assert bwd(**{name: None}) == ARG, name
    for name in ("dy", "x", "g", "mean", "rstd", "dx", "dg", "db"):
        assert bwd(**{name: (A << 12) + 2}) == ARG, name
    assert bwd(dg=A << 10, db=(A << 10) + 156) == ARG and bwd(x=A, xb=1 << 20, dx=A + 16) == ARG
    assert bwd(dx=None, dg=None, db=None) == ARG and bwd(x=A + 8, xb=1 << 20) == ARG and bwd(xb=1 << 20, xf=2) == ARG and bwd(status=A + 4) == ARG
    assert bwd(work=None) == ARG and bwd(work=(A << 20) + 8) == ARG and bwd(wb=api.norm_work_bytes(good) - 1) == api.FH_ERR_CAPACITY
    assert api.norm_work_bytes(api.norm_desc(10 ** 6, 4096)) == 296 * 2 * 4096 * 4 and api.norm_work_bytes(api.norm_desc(1, 1)) == 8


class Tensor:
    """What the binding asks of a tensor."""
    shape, dtype, device = (4, 5), "torch.float32", "cuda:1"

    def __init__(self, device=0, esize=4, numel=20, contiguous=True, storage=80, offset=0):
        self.d, self.e, self.n, self.c, self.s, self.o = device, esize, numel, contiguous, storage, offset

    def get_device(self): return self.d
    def element_size(self): return self.e
    def numel(self): return self.n
    def is_contiguous(self): return self.c
    def storage_offset(self): return self.o
    def data_ptr(self): return 4096
    def untyped_storage(self): return type("S", (), {"nbytes": lambda _: self.s})()


def test_the_binding_takes_no_tensor_that_is_too_small_or_elsewhere():
    assert api._ptr(None, 0, 5, 4) is None and api._ptr(Tensor(), 0, 20, 4) == 4096
    assert api._ptr(Tensor(contiguous=False, numel=12, storage=100, offset=3), 0, 22, 4) == 4096    # a slice of a wider matrix
    for bad in (Tensor(device=1), Tensor(device=-1), Tensor(esize=2), Tensor(numel=19, storage=76), Tensor(contiguous=False, numel=40, storage=76),
                Tensor(contiguous=False, numel=12, storage=80, offset=1)):
        with pytest.raises(ValueError):
            api._ptr(bad, 0, 20, 4)
    with pytest.raises(ValueError):
        api._ptr(Tensor(contiguous=False), 0)    # a container, or a workspace
