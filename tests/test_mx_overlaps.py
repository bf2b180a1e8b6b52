"""Memory that a call of the matrix functions would write while it, or another of its threads, reads or writes it: refused on the host.  Addresses are
made up, so that this runs only where nothing can be launched: a call that is not refused ends with FH_ERR_CUDA there."""
import ctypes as C

import pytest

from oracle import mx
from paper_2510_11400_b200 import api, build

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: only without a device")
OK, ARG = api.FH_ERR_CUDA, api.FH_ERR_ARG
MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    build.build()
    return api.lib()


ROWS, COLS = 12, 40
FWD = dict(x=1 * MB, gamma=2 * MB, beta=3 * MB, y=4 * MB, mean=5 * MB, rstd=6 * MB, packed=7 * MB)
BWD = dict(dy=1 * MB, x=2 * MB, gamma=3 * MB, mean=4 * MB, rstd=5 * MB, dx=6 * MB, dgamma=7 * MB, dbeta=8 * MB, work=9 * MB, status=10 * MB)


def forward(lib, ldx=COLS, ldy=COLS, rows=ROWS, **at):
    p = FWD | at
    d, prm = api.norm_desc(rows, COLS, ldx=ldx, ldy=ldy), api.mx_params()
    return lib.fh_layer_norm(C.byref(d), p["x"], p["gamma"], p["beta"], p["y"], p["mean"], p["rstd"], C.byref(prm), p["packed"], 1 << 40, None)


def backward(lib, ldx=COLS, ldy=COLS, rows=ROWS, packed=False, **at):
    p = BWD | at
    d = api.norm_desc(rows, COLS, ldx=ldx, ldy=ldy)
    return lib.fh_layer_norm_backward(C.byref(d), p["dy"], p["x"], 1 << 16 if packed else 0, 0, p["gamma"], p["mean"], p["rstd"], p["dx"], p["dgamma"],
                                      p["dbeta"], p["work"], 1 << 40, p["status"], None)


SIZE = dict(x=ROWS * COLS * 4, y=ROWS * COLS * 4, dy=ROWS * COLS * 4, dx=ROWS * COLS * 4, gamma=COLS * 4, beta=COLS * 4, dgamma=COLS * 4, dbeta=COLS * 4,
            mean=ROWS * 4, rstd=ROWS * 4, packed=mx.sizes(ROWS, COLS, 0)[3], work=2 * COLS * 4, status=8)


def first_and_last(call, lib, names, out, other, **kw):
    """What a call says with `out` over the last 16-byte piece of `other`, with its own last one over the first, and with neither."""
    at = names[other]
    over = (SIZE[other] - 1) // 16 * 16, -((SIZE[out] - 1) // 16 * 16)
    return [call(lib, **{out: at + o}, **kw) for o in over], [call(lib, **{out: at + o}, **kw) for o in ((SIZE[other] + 15) // 16 * 16, -((SIZE[out] + 15) // 16 * 16))]


@pytest.mark.parametrize("out,other", [(o, i) for o in ("y", "mean", "rstd", "packed") for i in FWD if i != o])
def test_outputs_of_the_forward_pass(lib, out, other):
    assert forward(lib) == OK
    over, beside = first_and_last(forward, lib, FWD, out, other)
    assert over == [ARG, ARG] and beside == [OK, OK]


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("out,other", [("dx", i) for i in BWD if i != "dx"] + [("work", i) for i in BWD if i not in ("work", "dx")] +
                         [("status", i) for i in BWD if i != "status"] + [("dgamma", "dbeta")])
def test_outputs_of_the_backward_pass(lib, out, other, packed):
    if packed and other == "x":
        pytest.skip("another size: below")
    assert backward(lib, packed=packed) == OK
    over, beside = first_and_last(backward, lib, BWD, out, other, packed=packed)
    assert over == [ARG, ARG] and beside == [OK, OK]


@pytest.mark.parametrize("out", ["dx", "dgamma", "dbeta", "work", "status"])
def test_the_container_that_the_backward_pass_reads(lib, out):
    n = mx.sizes(ROWS, COLS, 0)[3]
    for o in (0, 64, n - 16):
        assert backward(lib, packed=True, **{out: BWD["x"] + o}) == ARG
    assert backward(lib, packed=True, **{out: BWD["x"] + n}) == OK


def test_in_place(lib):
    assert forward(lib, y=FWD["x"]) == OK and forward(lib, y=FWD["x"], ldx=48, ldy=48) == OK
    assert forward(lib, y=FWD["x"], ldx=48, ldy=44) == ARG and forward(lib, y=FWD["x"] + 16) == ARG
    assert forward(lib, y=FWD["x"], ldx=48, ldy=44, rows=1) == OK
    assert backward(lib, dx=BWD["dy"]) == OK and backward(lib, dx=BWD["x"]) == OK and backward(lib, dx=BWD["x"], ldx=48, ldy=44) == OK
    assert backward(lib, dx=BWD["dy"], ldx=48, ldy=44) == ARG and backward(lib, dx=BWD["dy"], ldx=48, ldy=44, rows=1) == OK
    assert backward(lib, dx=BWD["dy"] + 16) == ARG and backward(lib, dx=BWD["x"] - 16) == ARG
    # (the weights' gradients are written when everything has been read)
    for name in ("gamma", "dy", "x", "mean"):
        assert backward(lib, dgamma=BWD[name]) == OK


def test_matrices_side_by_side_in_a_wider_one(lib):
    """Rows that lie between one another's are not over one another."""
    ld = 3 * COLS
    for shift, want in ((COLS, OK), (2 * COLS, OK), (COLS - 1, ARG), (2 * COLS + 1, ARG), (ld, ARG), (ld + COLS, OK), ((ROWS - 1) * ld, ARG), (ROWS * ld, OK),
                        (-COLS, OK), (-COLS + 1, ARG), (-2 * COLS, OK), (-ld, ARG), (-ROWS * ld, OK), (-(ROWS - 1) * ld, ARG), (-ROWS * ld + COLS - 1, OK)):
        assert forward(lib, ldx=ld, ldy=ld, y=FWD["x"] + 4 * shift) == want, shift
        assert backward(lib, ldx=ld, ldy=ld, dx=BWD["dy"] + 4 * shift) == want, shift
    # rows of different distances: 120 and 240 elements meet at every second one
    assert forward(lib, ldx=ld, ldy=2 * ld, y=FWD["x"] + 4 * COLS) == OK and forward(lib, ldx=2 * ld, ldy=ld, y=FWD["x"] - 4 * COLS) == OK
    assert forward(lib, ldx=ld, ldy=2 * ld, y=FWD["x"] + 4 * COLS - 4) == ARG and forward(lib, ldx=ld, ldy=ld + 1, y=FWD["x"] + 4 * 2 * COLS - 8) == ARG
    # a row of statistics between the rows of x
    assert forward(lib, ldx=ld, mean=FWD["x"] + 4 * COLS) == OK and forward(lib, ldx=ld, mean=FWD["x"] + 4 * (ld - 11)) == ARG


def test_status_words_of_the_other_calls(lib):
    n = mx.sizes(ROWS, COLS, 0)[3]
    m, d = api.matrix(ROWS, COLS), api.mx_product_desc(ROWS, ROWS, COLS)

    def restore(status):
        return lib.fh_mx_decompress(MB, 1 << 40, C.byref(m), 0, 2 * MB, status, None)

    def product(status):
        return lib.fh_mx_product(C.byref(d), MB, 1 << 40, 2 * MB, 1 << 40, 3 * MB, status, None)

    for call, at, sizes in ((restore, (MB, 2 * MB), (n, ROWS * COLS * 4)), (product, (MB, 2 * MB, 3 * MB), (n, n, ROWS * ROWS * 4))):
        assert call(4 * MB) not in (api.FH_OK, ARG)
        for p, size in zip(at, sizes):
            assert call(p) == call(p + size - 8) == ARG
            assert call(p + size) != ARG and call(p - 8) != ARG
