"""Calls of the 4-bit cache that move or see no rows: pointers may be NULL, and the binding
takes None for them."""
import pytest

from gpu_util import need_gpu
from paper_2502_12085_amd import apb

NAMES = ("k_codes", "k_scales", "v_codes", "v_scales")


def _rows(n_rows):
    return apb.Cache4Problem(2, 64, 100, 10, n_rows, 40, 5)


@pytest.mark.parametrize("cache", [None, dict.fromkeys(NAMES)])
def test_no_rows(cache):
    apb.cache4_write(_rows(0), None, None, cache, stream=0)
    apb.cache4_read(_rows(0), cache, None, None, stream=0)
    for call in (lambda p: apb.cache4_write(p, None, None, cache, stream=0),
                 lambda p: apb.cache4_read(p, cache, None, None, stream=0)):
        with pytest.raises(apb.ApbError, match="NULL_POINTER"):
            call(_rows(1))
        with pytest.raises(apb.ApbError) as e:
            call(apb.Cache4Problem(2, 64, 100, 101, 0, 40, 5))
        assert e.value.status == 2


def test_some_tensors_of_no_rows():
    torch = pytest.importorskip("torch")
    cache = dict.fromkeys(NAMES, None)
    cache["v_codes"] = torch.zeros(2, 100, 32, dtype=torch.uint8)  # not the device's
    with pytest.raises(ValueError, match="device tensor"):
        apb.cache4_write(_rows(0), None, None, cache, stream=0)


@pytest.mark.gpu
@pytest.mark.parametrize("cache", [None, dict.fromkeys(NAMES)])
def test_no_keys(cache):
    torch = need_gpu()
    q = torch.ones(8, 3, 64, dtype=torch.bfloat16, device="cuda")
    o, lse = torch.ones(8, 3, 64, device="cuda"), torch.ones(8, 3, device="cuda")
    ws = torch.empty(16, dtype=torch.uint8, device="cuda")
    apb.decode4_attention(apb.Decode4Problem(8, 2, 64, 100, 0, 3, 0), q, cache, o, lse, ws)
    assert not o.any() and torch.isneginf(lse).all()
    with pytest.raises(apb.ApbError, match="NULL_POINTER"):
        apb.decode4_attention(apb.Decode4Problem(8, 2, 64, 100, 1, 3, 0), q, cache, o, lse, ws)
