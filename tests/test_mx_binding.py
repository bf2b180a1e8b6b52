"""What the binding of the matrix functions refuses before the library is called, which takes addresses and cannot see what they belong to.
Host tensors stand for CUDA tensors and a list of calls for the library."""
import types

import pytest

from paper_2510_11400_b200 import api, build

torch = pytest.importorskip("torch")
STREAM = types.SimpleNamespace(cuda_stream=0)
U8 = torch.uint8


@pytest.fixture(params=[False, True], ids=["first call", "later"])
def calls(monkeypatch, request):
    """The library's calls; torch's types are known to the binding from its first call on."""
    monkeypatch.setattr(api, "_types", {api.FH_F32: torch.float32, api.FH_BF16: torch.bfloat16} if request.param else {})
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


def with_status(status):
    """Every call that has a status."""
    buf, m = torch.zeros(1 << 14, dtype=U8), torch.zeros(8, 40)
    one = torch.zeros(8)
    d = api.norm_desc(8, 40)
    return [lambda: api.fh_mx_decompress(buf, api.matrix(8, 40), api.FH_MX_B32, m, status, STREAM),
            lambda: api.fh_mx_product(api.mx_product_desc(8, 8, 40), buf, buf, torch.zeros(8, 8), status, STREAM),
            lambda: api.fh_layer_norm_backward(d, m, buf, None, one, one, m, packed=api.FH_MX_B32, status=status, stream=STREAM)]


def test_a_status_is_64_bits(calls):
    for good in (None, torch.zeros(1, dtype=torch.int64), torch.zeros(1, dtype=torch.uint64), torch.zeros(9, dtype=torch.int64)[3:]):
        for call in with_status(good):
            taken(calls, call)
    for bad in (torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(4), torch.zeros(8, dtype=U8), torch.zeros(1, dtype=torch.complex64), torch.zeros(1, dtype=torch.float64),
                torch.zeros(0, dtype=torch.int64),
                torch.zeros(4, dtype=torch.int64)[::2]):
        for call in with_status(bad):
            refused(calls, call)


def with_matrix(x, rows, cols, ld):
    """Every call that has a dense matrix, with `x` in each place that `rows`, `cols` and `ld` describe."""
    buf, m, d = torch.zeros(1 << 16, dtype=U8), api.matrix(rows, cols, api.FH_F32, ld), api.norm_desc(rows, cols, ldx=ld, ldy=ld)
    other, one = torch.zeros(rows * ld), torch.zeros(rows)
    return [lambda: api.fh_mx_compress(m, api.mx_params(), x, buf, None, STREAM),
            lambda: api.fh_mx_decompress(buf, m, api.FH_MX_B32, x, None, STREAM),
            lambda: api.fh_mx_product(api.mx_product_desc(rows, cols, 32, ldc=ld), buf, buf, x, None, STREAM),
            lambda: api.fh_layer_norm(d, x, None, None, other, stream=STREAM),
            lambda: api.fh_layer_norm(d, other, None, None, x, stream=STREAM),
            lambda: api.fh_layer_norm_backward(d, x, other, None, one, one, other, stream=STREAM),
            lambda: api.fh_layer_norm_backward(d, other, x, None, one, one, other, stream=STREAM),
            lambda: api.fh_layer_norm_backward(d, other, other, None, one, one, x, stream=STREAM)]


def test_a_matrix_lies_as_it_is_described(calls):
    wide, deep = torch.zeros(64, 96), torch.zeros(4, 16, 96)
    for x, rows, cols, ld in ((torch.zeros(8, 40), 8, 40, 40), (torch.zeros(320), 8, 40, 40), (torch.zeros(2, 4, 40), 8, 40, 40), (torch.zeros(4, 80), 8, 40, 40),
                              (wide[:, :40], 64, 40, 96), (wide[8:, 5:45], 56, 40, 96), (wide[:, :40], 10, 30, 96), (wide[::2, :40], 32, 40, 192),
                              (deep[:, :, 30:70], 64, 40, 96), (wide[3:4, :40], 1, 40, 96), (wide[3:4, :40], 1, 40, 40), (wide[:, 7], 64, 1, 96),
                              (wide[:, 7:8], 64, 1, 96), (wide[:, 7:9], 64, 1, 96), (wide[0, :40], 1, 40, 40)):
        for call in with_matrix(x, rows, cols, ld):
            taken(calls, call)
    for x, rows, cols, ld in ((wide[:, :40], 32, 40, 40),                  # rows 96 apart, described as 40 apart
                              (wide[:, :40], 32, 40, 41), (torch.zeros(40, 8).t(), 8, 40, 40),
                              (wide[:, :80:2], 20, 40, 96), (wide[:, :80:2], 20, 40, 192), (torch.zeros(2000)[::2], 8, 40, 40),
                              (torch.zeros(4000)[:40].expand(8, 40), 8, 40, 40), (deep[:, :10, :40], 40, 40, 96),
                              (wide[:, 7], 32, 1, 1), (wide[0, ::2], 1, 40, 40), (wide[:, :40].t(), 40, 64, 96)):
        for call in with_matrix(x, rows, cols, ld):
            refused(calls, call)


def test_vectors_have_their_elements_side_by_side(calls):
    x, y, d = torch.zeros(8, 40), torch.zeros(8, 40), api.norm_desc(8, 40)
    work = torch.zeros(api.norm_work_bytes(d), dtype=U8)

    def each(v, r):
        return [lambda: api.fh_layer_norm(d, x, v, None, y, stream=STREAM), lambda: api.fh_layer_norm(d, x, None, v, y, stream=STREAM),
                lambda: api.fh_layer_norm(d, x, None, None, y, r, None, stream=STREAM), lambda: api.fh_layer_norm(d, x, None, None, y, None, r, stream=STREAM),
                lambda: api.fh_layer_norm_backward(d, x, y, v, r, r, None, v, v, work, stream=STREAM)]

    for v, r in ((torch.zeros(40), torch.zeros(8)), (torch.zeros(1, 40), torch.zeros(8, 1)), (torch.zeros(100)[7:47], torch.zeros(4, 8)[1]),
                 (torch.zeros(3, 100)[1:2, 5:45], torch.zeros(1, 8, 1))):
        for call in each(v, r):
            taken(calls, call)
    fine_v, fine_r = torch.zeros(40), torch.zeros(8)
    for v, r in ((torch.zeros(200)[::2], torch.zeros(64)[::2]), (torch.zeros(40, 40)[:, 3], torch.zeros(8, 8)[:, 3]),
                 (torch.zeros(4000)[:1].expand(40), torch.zeros(4000)[:1].expand(8))):
        for call in each(v, fine_r)[:2] + each(fine_v, r)[2:]:
            refused(calls, call)


def test_fp16_is_not_taken_for_bf16(calls):
    """Both have two bytes."""
    buf, work = torch.zeros(1 << 16, dtype=U8), torch.zeros(1 << 16, dtype=U8)
    m, d = api.matrix(8, 40, api.FH_BF16), api.norm_desc(8, 40, api.FH_BF16, api.FH_BF16)
    r = torch.zeros(8)

    def each(x, w):
        return [lambda: api.fh_mx_compress(m, api.mx_params(), x, buf, None, STREAM), lambda: api.fh_mx_decompress(buf, m, api.FH_MX_B32, x, None, STREAM),
                lambda: api.fh_mx_product(api.mx_product_desc(8, 40, 32, dtype=api.FH_BF16), buf, buf, x, None, STREAM),
                lambda: api.fh_layer_norm(d, x, w, w, x, r, r, stream=STREAM),
                lambda: api.fh_layer_norm_backward(d, x, x, w, r, r, x, w, w, work, stream=STREAM)]

    bf = dict(dtype=torch.bfloat16)
    for t in (torch.bfloat16, torch.uint16, torch.int16):    # (bits, as the plane codec's callers hold them)
        for call in each(torch.zeros(8, 40, dtype=t), torch.zeros(40, dtype=t)):
            taken(calls, call)
    for call in each(torch.zeros(8, 40, dtype=torch.float16), torch.zeros(40, **bf)) + each(torch.zeros(8, 40, **bf), torch.zeros(40, dtype=torch.float16))[3:]:
        refused(calls, call)
