"""What the binding takes as the place of a rotation table.  Host tensors stand for CUDA tensors and a list of calls for the library."""
import types

import pytest

from paper_2510_11400_b200 import api, build

torch = pytest.importorskip("torch")
STREAM = types.SimpleNamespace(cuda_stream=0)


@pytest.fixture(params=[False, True], ids=["first call", "later"])
def made(monkeypatch, request):
    monkeypatch.setattr(api, "_types", {api.FH_F32: torch.float32, api.FH_BF16: torch.bfloat16} if request.param else {})
    build.build()
    calls = []
    monkeypatch.setattr(api, "_device", lambda: -1)    # (where host tensors are)
    monkeypatch.setattr(api, "lib", lambda: types.SimpleNamespace(fh_rotation_table=lambda *a: calls.append(a) or (api.FH_OK if a[0] > 0 else api.FH_ERR_ARG)))
    return calls


def test_places_side_by_side(made):
    for out in (torch.zeros(9, 4, 2), torch.zeros(72), torch.zeros(100), torch.zeros(9, 8), torch.zeros(20, 8)[3:12]):
        assert api.rotation_table(9, 8, out=out, stream=STREAM) is out
        assert made.pop()[4] == out.data_ptr() and not made


@pytest.mark.parametrize("out", [torch.zeros(9, 16)[:, :8], torch.zeros(9, 16)[:, ::2], torch.zeros(18, 4, 2)[::2], torch.zeros(200)[::2], torch.zeros(8, 9).t(),
                                 torch.zeros(4, 9, 2).transpose(0, 1)], ids=lambda t: str(tuple(t.stride())))
def test_places_that_are_not(made, out):
    """Views whose storage has room enough: the table would be written between their elements."""
    with pytest.raises(ValueError):
        api.rotation_table(9, 8, out=out, stream=STREAM)
    assert not made


def test_what_is_no_place_for_it(made):
    for out in (torch.zeros(71), torch.zeros(72, dtype=torch.float64), torch.zeros(72, dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            api.rotation_table(9, 8, out=out, stream=STREAM)
    assert not made


def test_refusals_are_the_librarys(made):
    for positions in (0, -1):
        with pytest.raises(api.FhError):
            api.rotation_table(positions, 8, out=torch.zeros(72), stream=STREAM)
