"""Refusals of the 4-bit cache's entry points, all raised on the host before any
HIP call (fake device addresses are never dereferenced)."""
import ctypes

import pytest

from paper_2502_12085_amd import apb

A = 0x7F0000000000
K, V, KC, KS, VC, VS, Q, O, LSE, WS = (A + i * (1 << 36) for i in range(10))


def _cache(kc=KC, ks=KS, vc=VC, vs=VS):
    return apb.Cache4(kc, ks, vc, vs)


def _rows(**kw):
    base = dict(n_kv_heads=2, head_dim=64, capacity=100, first_row=10, n_rows=20, bf16_rows=40,
                bf16_first=5)
    base.update(kw)
    return apb.Cache4Problem(**base)


def _step(**kw):
    base = dict(n_q_heads=8, n_kv_heads=2, head_dim=64, capacity=100, cache_len=60, n_new=3,
                causal=1)
    base.update(kw)
    return apb.Decode4Problem(**base)


@pytest.mark.parametrize("kw,code", [
    (dict(), 0),
    (dict(n_rows=0), 0),
    (dict(first_row=80), 0),
    (dict(first_row=81), 2),
    (dict(bf16_first=20), 0),
    (dict(bf16_first=21), 2),
    (dict(first_row=-1), 2),
    (dict(bf16_first=-1), 2),
    (dict(n_rows=-1), 2),
    (dict(capacity=0, first_row=0, n_rows=0), 2),
    (dict(capacity=(1 << 30) + 1), 2),
    (dict(bf16_rows=(1 << 30) + 1), 2),
    (dict(bf16_rows=-1, bf16_first=0, n_rows=0), 2),
    (dict(n_rows=2147483647), 2),            # sums past 32 bits
    (dict(first_row=2147483647, n_rows=1), 2),
    (dict(n_kv_heads=0), 2),
    (dict(n_kv_heads=65537), 2),
    (dict(head_dim=0), 2),
    (dict(head_dim=96), 3),
    (dict(head_dim=256), 3),
    # more threads than a launch can have: 64 rows of d = 64 a workgroup, K and V
    (dict(n_kv_heads=1 << 13, capacity=1 << 17, n_rows=1 << 16, first_row=0, bf16_rows=1 << 17,
          bf16_first=0), 2),
    (dict(n_kv_heads=(1 << 13) - 1, capacity=1 << 17, n_rows=1 << 16, first_row=0,
          bf16_rows=1 << 17, bf16_first=0), 0),
    (dict(n_kv_heads=65536, capacity=1 << 30, n_rows=1 << 30, first_row=0, bf16_rows=1 << 30,
          bf16_first=0), 2),
])
def test_validate_cache4(kw, code):
    assert apb.validate_cache4(_rows(**kw)) == code


@pytest.mark.parametrize("kw,code", [
    (dict(), 0),
    (dict(cache_len=0, causal=0), 0),
    (dict(cache_len=100), 0),
    (dict(cache_len=101), 2),
    (dict(cache_len=-1, causal=0), 2),
    (dict(cache_len=3), 0),
    (dict(cache_len=2), 2),                  # the new tokens' rows are missing
    (dict(cache_len=2, causal=0), 0),
    (dict(n_new=0), 2),
    (dict(causal=2), 2),
    (dict(causal=-1), 2),
    (dict(n_q_heads=7), 2),
    (dict(n_q_heads=0), 2),
    (dict(n_kv_heads=0), 2),
    (dict(n_q_heads=65537, n_kv_heads=65537), 2),
    (dict(n_new=1 << 28, causal=0), 2),
    (dict(n_new=1 << 21, causal=0), 2),      # more rows than a launch can have
    (dict(n_new=(1 << 21) - 1, causal=0), 0),
    (dict(capacity=0, cache_len=0, causal=0), 2),
    (dict(capacity=(1 << 30) + 1), 2),
    (dict(head_dim=0), 2),
    (dict(head_dim=32), 3),
])
def test_validate_decode4(kw, code):
    assert apb.validate_decode4(_step(**kw)) == code
    n = ctypes.c_uint64(77)
    assert apb.lib().apb_decode4_workspace_size(ctypes.byref(_step(**kw)), ctypes.byref(n)) == code
    assert (n.value == 77) if code else (n.value > 0)


def test_null_problems():
    L, n = apb.lib(), ctypes.c_uint64()
    assert L.apb_validate_cache4(None) == 1
    assert L.apb_validate_decode4(None) == 1
    assert L.apb_decode4_workspace_size(None, ctypes.byref(n)) == 1
    assert L.apb_decode4_workspace_size(ctypes.byref(_step()), None) == 1
    assert L.apb_cache4_write(None, K, V, ctypes.byref(_cache()), None) == 1
    assert L.apb_cache4_read(None, ctypes.byref(_cache()), K, V, None) == 1
    assert L.apb_decode4_attention(None, Q, ctypes.byref(_cache()), O, LSE, 0.0, WS, 1 << 30,
                                   None) == 1


@pytest.mark.parametrize("write", [True, False])
def test_rows_error_paths(write):
    def call(p=None, k=K, v=V, cache=None, null=False):
        p = ctypes.byref(p or _rows())
        c = None if null else ctypes.byref(cache or _cache())
        L = apb.lib()
        return L.apb_cache4_write(p, k, v, c, None) if write else L.apb_cache4_read(p, c, k, v, None)
    assert call(null=True) == 1
    assert call(k=None) == 1
    assert call(v=None) == 1
    for name in ("kc", "ks", "vc", "vs"):
        assert call(cache=_cache(**{name: None})) == 1
    assert call(k=K + 8) == 4
    assert call(v=V + 2) == 4
    assert call(cache=_cache(kc=KC + 8)) == 4
    assert call(cache=_cache(vc=VC + 4)) == 4
    # 2 heads: bf16 10240 bytes, codes 6400, scales 400
    assert call(cache=_cache(vc=KC)) == 6
    assert call(cache=_cache(vc=KC + 6384)) == 6
    assert call(cache=_cache(ks=KC + 6396)) == 6
    assert call(cache=_cache(vs=KS + 396)) == 6
    assert call(k=KC - 10240 + 16) == 6
    assert call(v=VS - 16) == 6
    assert call(_rows(first_row=81)) == 2
    assert call(_rows(head_dim=96)) == 3
    if not write:
        assert call(v=K + 16) == 6           # outputs overlap each other
    # no rows: valid, and launches nothing
    assert call(_rows(n_rows=0), k=None, v=None, null=True) == 0


def test_decode4_error_paths():
    long = _step(capacity=4000, cache_len=3000)
    need = apb.decode4_workspace_size(long)
    assert need >= 2 * 8 * 3 * 66 * 4 and apb.decode4_workspace_size(_step()) == 16

    def call(p=long, q=Q, cache=None, o=O, lse=LSE, ws=WS, n=1 << 30, null=False):
        c = None if null else ctypes.byref(cache or _cache())
        return apb.lib().apb_decode4_attention(ctypes.byref(p), q, c, o, lse, 0.0, ws,
                                               n, None)
    assert call(null=True) == 1
    assert call(q=None) == 1
    assert call(o=None) == 1
    assert call(lse=None) == 1
    assert call(ws=None) == 1
    for name in ("kc", "ks", "vc", "vs"):
        assert call(cache=_cache(**{name: None})) == 1
    assert call(q=Q + 8) == 4
    assert call(o=O + 4) == 4
    assert call(lse=LSE + 2) == 4
    assert call(ws=WS + 8) == 4
    assert call(cache=_cache(kc=KC + 8)) == 4
    assert call(n=need - 1) == 2
    assert call(_step(), n=15) == 2          # one split needs next to nothing, but not nothing
    assert call(o=Q) == 6
    assert call(o=KC + 16) == 6
    assert call(lse=VS + 396) == 6
    assert call(lse=O + 8) == 6
    assert call(ws=Q) == 6
    assert call(ws=VC - 16) == 6
    assert call(ws=O) == 6
    assert call(_step(cache_len=2)) == 2
    assert call(_step(head_dim=96)) == 3


def test_binding_checks_its_tensors():
    torch = pytest.importorskip("torch")
    p = _rows()
    k = torch.zeros(2, 40, 64, dtype=torch.bfloat16)
    cache = {n: torch.zeros(2, 100, w, dtype=torch.uint8)
             for n, w in (("k_codes", 32), ("k_scales", 2), ("v_codes", 32), ("v_scales", 2))}
    with pytest.raises(ValueError, match="device tensor"):
        apb.cache4_write(p, k, k, cache)
    with pytest.raises(ValueError, match="device tensor"):
        apb.cache4_read(p, cache, k, k)
    with pytest.raises(apb.ApbError) as e:
        apb.cache4_write(_rows(first_row=90), k, k, cache)
    assert e.value.status == 2
    with pytest.raises(apb.ApbError, match="apb_cache4_read: APB_ERR_NULL_POINTER"):
        apb.cache4_read(p, dict(cache, k_codes=None), k, k)
    with pytest.raises(ValueError, match="workspace"):
        apb.decode4_attention(_step(), k, cache, None, None, None)
    with pytest.raises(apb.ApbError):
        apb.decode4_attention(_step(cache_len=101), k, cache, None, None, None)
