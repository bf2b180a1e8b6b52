"""Microscaled 4-bit matrices on the GPU: containers and restored matrices against the plain definition, byte for byte."""
import numpy as np
import pytest

from oracle import mx
from paper_2510_11400_b200 import api, build

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build()
    api.lib()


def values(rows, cols, seed=0, scale=1.0):
    rng = np.random.default_rng([seed, rows, cols])
    x = rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal(cols)) * scale
    x[rng.random((rows, cols)) < 0.05] = 0.0
    return x.astype(np.float32)


def dense(x, dtype, ld=None, offset=0):
    """(a CUDA tensor that holds x at `offset` elements with rows `ld` apart, NaN elsewhere; x as it is held)."""
    rows, cols = x.shape
    ld = cols if ld is None else ld
    t = torch.float32 if dtype == api.FH_F32 else torch.bfloat16
    flat = torch.full((offset + rows * ld + 64,), float("nan"), dtype=t, device="cuda")
    view = flat.as_strided((rows, cols), (ld, 1), offset)
    view.copy_(torch.from_numpy(x).cuda())
    return view, view.float().cpu().numpy()


def compress(view, m, p, guard=64):
    """Both containers of a matrix; their ends are watched."""
    out = []
    for r, c in ((m.rows, m.cols), (m.cols, m.rows)):
        n = api.mx_bytes(r, c, p.format)
        out.append(torch.full((n + guard,), 0xA5, dtype=torch.uint8, device="cuda"))
    assert api.fh_mx_compress(m, p, view, out[0][:-guard], out[1][:-guard]) == api.FH_OK
    torch.cuda.synchronize()
    for t in out:
        assert (t[-guard:] == 0xA5).all()
    return [t[:-guard] for t in out]


def restore(buf, rows, cols, dtype, fmt, ld=None):
    ld = cols if ld is None else ld
    t = torch.float32 if dtype == api.FH_F32 else torch.bfloat16
    flat = torch.full((rows * ld + 64,), -7.0, dtype=t, device="cuda")
    status = torch.full((1,), 99, dtype=torch.int64, device="cuda")
    assert api.fh_mx_decompress(buf, api.matrix(rows, cols, dtype, ld), fmt, flat, status) == api.FH_OK
    torch.cuda.synchronize()
    view = flat[:rows * ld].view(rows, ld)
    assert (flat[rows * ld:] == -7.0).all() and (view[:, cols:] == -7.0).all()
    return int(status.item()), view[:, :cols].float().cpu().numpy()


SHAPES = [(1, 1), (1, 32), (1, 4096), (5, 31), (7, 33), (8, 64), (9, 65), (127, 100), (128, 128), (129, 127), (130, 257), (200, 16),
          (256, 512), (300, 1000), (1000, 40)]


@pytest.mark.parametrize("rounding", [0, 1])
@pytest.mark.parametrize("fmt,exponent", [(mx.B32, 0), (mx.B16, 0), (mx.B16, -7)])
@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("shape", SHAPES)
def test_containers_and_restored_matrices(shape, dtype, fmt, exponent, rounding):
    rows, cols = shape
    view, x = dense(values(rows, cols, 1, 2.0 ** exponent), dtype)
    p = api.mx_params(fmt, exponent, rounding, seed=0x123456789ABCDEF, tensor_id=(9 << 32) + 5)
    kw = dict(exponent=exponent, rounding=rounding, seed=0x123456789ABCDEF, tensor_id=(9 << 32) + 5)
    for buf, a in zip(compress(view, api.matrix(rows, cols, dtype), p), (x, x.T)):
        want = mx.compress(a, fmt, **kw)
        assert np.array_equal(buf.cpu().numpy(), want)
        st, got = restore(buf, *a.shape, dtype, fmt)
        assert st == api.FH_OK and np.array_equal(got, mx.restore(want, *a.shape, fmt))


@pytest.mark.parametrize("fmt", [mx.B32, mx.B16])
@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("ld,offset", [(139, 0), (139, 1), (144, 0), (144, 8), (144, 3)])
def test_strides_and_alignments(dtype, fmt, ld, offset):
    rows, cols = 150, 137
    view, x = dense(values(rows, cols, 2), dtype, ld, offset)
    bufs = compress(view, api.matrix(rows, cols, dtype, ld), api.mx_params(fmt))
    for buf, a in zip(bufs, (x, x.T)):
        assert np.array_equal(buf.cpu().numpy(), mx.compress(a, fmt))
    st, got = restore(bufs[0], rows, cols, dtype, fmt, ld)
    assert st == api.FH_OK and np.array_equal(got, mx.restore(bufs[0].cpu().numpy(), rows, cols, fmt))


@pytest.mark.parametrize("rounding", [0, 1])
@pytest.mark.parametrize("fmt,exponent", [(mx.B32, 0), (mx.B16, 0), (mx.B16, 64), (mx.B16, -64)])
@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
def test_edges_of_the_formats(dtype, fmt, exponent, rounding):
    """A row of blocks for each: zeros of both signs, NaN and infinities, the smallest and largest numbers, ties, and largest
    magnitudes around each scale's border."""
    one = 2.0 ** exponent
    rows = [np.zeros(32), -np.zeros(32), np.full(32, 2.0 ** -149), np.full(32, 3.4028235e38), np.full(32, -3.3e38)]
    for bad in (np.nan, np.inf, -np.inf):
        r = np.linspace(-3, 3, 32)
        r[17] = bad
        rows.append(r)
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    for f in (1.0, 1 + 2.0 ** -7, 1 - 2.0 ** -8, 1 + 2.0 ** -23, 1 - 2.0 ** -24):
        for s in (1.0, 1.125, 1.875, 2.0 ** -9, 3 * 2.0 ** -9, 2.0 ** -6, 240.0, 448.0):
            # (whole and broken, so that the largest magnitude is six scales and a little more or less)
            rows.append(np.tile(np.concatenate([ties * s * f, -ties * s * f]), 2) * one)
            rows.append(np.tile(np.concatenate([ties * s * f, [6 * s] * 8]), 2) * one)
    with np.errstate(over="ignore"):
        x = np.array(rows).astype(np.float32)
    x[np.isinf(x) & ~np.isinf(np.array(rows))] = 1.0
    view, x = dense(x, dtype)
    kw = dict(rounding=rounding, seed=77, tensor_id=3)
    bufs = compress(view, api.matrix(*x.shape, dtype), api.mx_params(fmt, exponent, **kw))
    for buf, a in zip(bufs, (x, x.T)):
        want = mx.compress(a, fmt, exponent, **kw)
        assert np.array_equal(buf.cpu().numpy(), want)
        st, got = restore(buf, *a.shape, dtype, fmt)
        assert st == api.FH_OK and np.array_equal(got, mx.restore(want, *a.shape, fmt), equal_nan=True)


def test_one_form_alone_is_the_same():
    view, x = dense(values(260, 300, 4), api.FH_BF16)
    m, p = api.matrix(260, 300, api.FH_BF16), api.mx_params(mx.B16)
    both = compress(view, m, p)
    for i in range(2):
        out = [None, None]
        out[i] = torch.zeros_like(both[i])
        assert api.fh_mx_compress(m, p, view, *out) == api.FH_OK
        assert torch.equal(out[i], both[i])


@pytest.mark.parametrize("change", ["magic", "version", "format", "rows", "cols", "exponent", "total", "short"])
def test_another_header_is_reported_and_nothing_written(change):
    view, _ = dense(values(40, 70, 5), api.FH_F32)
    buf = compress(view, api.matrix(40, 70), api.mx_params(mx.B16, 3))[0].clone()
    at = dict(magic=0, version=4, format=6, rows=8, cols=12, exponent=17, total=24)
    if change == "short":
        buf = buf[:-16]
    else:
        buf[at[change]] += 1
    st, got = restore(buf, 40, 70, api.FH_F32, mx.B16)
    assert st == api.FH_ERR_CORRUPT and (got == -7.0).all()


def test_captured_calls_and_other_streams():
    """A capture of both directions, replayed on other values; on a stream of its own and next to calls on another stream."""
    rows, cols, fmt = 300, 260, mx.B32
    m, p = api.matrix(rows, cols), api.mx_params(fmt)
    view, _ = dense(values(rows, cols, 6), api.FH_F32)
    buf = torch.empty(api.mx_bytes(rows, cols, fmt), dtype=torch.uint8, device="cuda")
    out = torch.empty(rows, cols, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        assert api.fh_mx_compress(m, p, view, buf) == api.FH_OK
        assert api.fh_mx_decompress(buf, m, fmt, out) == api.FH_OK
    for seed in (7, 8):
        x = values(rows, cols, seed)
        view.copy_(torch.from_numpy(x).cuda())
        graph.replay()
        with torch.cuda.stream(side):
            other = torch.from_numpy(values(64, 64, seed)).cuda()
            mine, back = torch.empty(api.mx_bytes(64, 64, fmt), dtype=torch.uint8, device="cuda"), torch.empty(64, 64, device="cuda")
            assert api.fh_mx_compress(api.matrix(64, 64), p, other, mine) == api.FH_OK
            assert api.fh_mx_decompress(mine, api.matrix(64, 64), fmt, back) == api.FH_OK
        torch.cuda.synchronize()
        assert np.array_equal(out.cpu().numpy(), mx.restore(mx.compress(x, fmt), rows, cols, fmt))
        assert np.array_equal(back.cpu().numpy(), mx.restore(mx.compress(values(64, 64, seed), fmt), 64, 64, fmt))


def test_calls_next_to_the_plane_codec():
    """Both codecs on one stream, in turn: each container is what it is alone."""
    from oracle import fho
    from paper_2510_11400_b200 import synth
    spec = synth.TensorSpec("mixed", (4, 16, 28, 28), synth.F32, "spiky_relu", 3)
    raw = synth.make(spec)
    planes = torch.from_numpy(raw).cuda()
    want = fho.compress(raw, fho.desc(spec.shape, spec.dtype), fho.params(bits=2))[1]
    x = values(64, 784, 9)
    view, _ = dense(x, api.FH_F32)
    for _ in range(3):
        st, packed, total = api.compress_tensor(planes, spec.shape, spec.dtype, api.default_params(bits=2))
        buf = torch.empty(api.mx_bytes(64, 784, mx.B32), dtype=torch.uint8, device="cuda")
        assert api.fh_mx_compress(api.matrix(64, 784), api.mx_params(), view, buf) == api.FH_OK
        assert st == api.FH_OK and np.array_equal(packed[:total].cpu().numpy(), want)
        assert np.array_equal(buf.cpu().numpy(), mx.compress(x, mx.B32))


def test_a_long_matrix_passes_32_bit_offsets():
    """2^31 elements and more: the last rows are read, kept and restored where they belong."""
    rows, cols, fmt = 131_200, 16_416, mx.B32
    m = api.matrix(rows, cols, api.FH_BF16)
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    tail = torch.from_numpy(values(300, cols, 10)).cuda().to(torch.bfloat16)
    x[-300:] = tail
    buf = torch.empty(api.mx_bytes(rows, cols, fmt), dtype=torch.uint8, device="cuda")
    assert api.fh_mx_compress(m, api.mx_params(fmt), x, buf) == api.FH_OK
    want = mx.restore(mx.compress(tail.float().cpu().numpy(), fmt), 300, cols, fmt)
    x.fill_(9.0)
    assert api.fh_mx_decompress(buf, m, fmt, x) == api.FH_OK
    assert np.array_equal(x[-300:].float().cpu().numpy(), want)
    assert not x[:-300].any()
