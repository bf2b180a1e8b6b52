"""Norms of heads with as many rows as every rule of their launches asks for, against the plain definition in 64 bits: one, two and four heads to a team,
teams of every size that go on to further rows, warps of the loose kernels that do."""
import numpy as np
import pytest

from oracle import i8
from paper_2510_11400_b200 import api, build
from tests.test_gpu_heads import EPS, HALF, TYPES, Rows, backward_bound, cuda, forward_bound, setup

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build()
    api.lib()


def both_passes(tokens, hq, hk, dim, rotary, dtype, wdtype, pairs, kind, layout="packed", outside="plain"):
    s = setup(tokens, hq, hk, dim, rotary, dtype, wdtype)
    cs = s["table"][s["at"]].astype(np.float64)
    q, k = (Rows(tokens, h, dim, dtype, layout, v) for h, v in ((hq, s["x"][0]), (hk, s["x"][1])))
    oq, ok = (Rows(tokens, h, dim, dtype, outside) for h in (hq, hk))
    (gq, gk), table, at = (cuda(g, wdtype) for g in s["g"]), cuda(s["table"]), cuda(s["at"])
    d = api.heads_desc(tokens, hq, hk, dim, rotary, dtype, wdtype, kind, pairs, EPS, s["positions"], q.strides, k.strides, oq.strides, ok.strides)
    assert api.fh_head_norm(d, q.view, k.view, gq, gk, table, at, oq.view, ok.view) == api.FH_OK
    for out, x, g in ((oq, s["x"][0], s["g"][0]), (ok, s["x"][1], s["g"][1])):
        want, bound = forward_bound(x, g, cs, rotary, kind, pairs, dtype)
        assert (np.abs(out.read() - want) <= bound + 1e-30).all()
    yq, yk = (Rows(tokens, h, dim, dtype, outside, v) for h, v in ((hq, s["dy"][0]), (hk, s["dy"][1])))
    dq, dk = (Rows(tokens, h, dim, dtype, layout) for h in (hq, hk))
    wq, wk = (torch.full((dim,), 7.0, dtype=TYPES[wdtype], device="cuda") for _ in range(2))
    work = torch.full((api.heads_work_bytes(d),), 0xA5, dtype=torch.uint8, device="cuda")
    assert api.fh_head_norm_backward(d, yq.view, yk.view, q.view, k.view, gq, gk, table, at, dq.view, dk.view, wq, wk, work) == api.FH_OK
    for gx, gw, x, dy, g in ((dq, wq, s["x"][0], s["dy"][0], s["g"][0]), (dk, wk, s["x"][1], s["dy"][1], s["g"][1])):
        dx, e_dx, dg, e_dg = backward_bound(dy, x, g, cs, rotary, kind, pairs, dtype)
        assert (np.abs(gx.read() - dx) <= e_dx + 1e-30).all()
        assert (np.abs(gw.double().cpu().numpy() - dg) <= e_dg + HALF[wdtype] * (1 + 1e-6) * np.abs(dg) + 1e-30).all()


# lanes to a row: a 16-byte vector's elements twice to a lane
@pytest.mark.parametrize("pairs,kind", [(i8.HALVES, i8.RMS), (i8.NEIGHBOURS, i8.LAYER)])
@pytest.mark.parametrize("dtype,wdtype", [(api.FH_F32, api.FH_F32), (api.FH_BF16, api.FH_F32), (api.FH_BF16, api.FH_BF16)])
@pytest.mark.parametrize("heads", [(9, 2), (2, 1), (5, 5)])
@pytest.mark.parametrize("lanes", [4, 8, 16, 32])
def test_heads_to_a_team(lanes, heads, dtype, wdtype, pairs, kind):
    """Four heads to a team where rows / (32 / lanes) / 4 is eight warps an SM, two where half as many are, or no more heads there."""
    dim = lanes * (8 if dtype == api.FH_F32 else 16)
    four = 4 * 8 * torch.cuda.get_device_properties(0).multi_processor_count * (32 // lanes)      # rows
    for rows in (four, four // 2) if heads != (2, 1) else (four,):
        both_passes(-(-rows // sum(heads)) + 1, *heads, dim, dim // 2 if kind == i8.LAYER else dim, dtype, wdtype, pairs, kind)


@pytest.mark.parametrize("pairs,kind", [(i8.HALVES, i8.LAYER), (i8.NEIGHBOURS, i8.RMS)])
@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("tokens,dim,rotary", [(1100, 33, 32), (1100, 100, 50), (1100, 201, 100), (1100, 300, 300), (400, 1100, 550), (130, 8192, 8192)])
def test_loose_rows(tokens, dim, rotary, dtype, pairs, kind):
    """More rows than the backward pass has warps: four to each of 8 CTAs an SM, or one an SM for rows of more than 1024 elements."""
    both_passes(tokens, 3, 2, dim, rotary, dtype, api.FH_F32, pairs, kind, "odd", "wide")
