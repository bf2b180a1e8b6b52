"""What the binding of the matrix functions refuses before the library is called, which takes addresses and cannot see what they belong to.
Host tensors stand for CUDA tensors and a list of calls for the library."""
import types

import pytest

from paper_2510_11400_b200 import api, build

torch = pytest.importorskip("torch")
STREAM = types.SimpleNamespace(cuda_stream=0)
U8 = torch.uint8


@pytest.fixture
def calls(monkeypatch):
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
