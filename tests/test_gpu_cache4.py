"""GPU parity of the KV cache in 4 bits against the fp64 oracle: codes and scale
bytes bit for bit, values read back exactly, and the rows beside a call's own
left as they were."""
import numpy as np
import pytest

import oracle
from paper_2502_12085_amd import inputs
from gpu_util import dev_bf16, host_bf16_to_f64, host_bits, need_gpu, say

pytestmark = pytest.mark.gpu

FILL = 0xA5


def _device(a):
    import torch
    return torch.from_numpy(np.array(a)).cuda()  # a copy: writable and contiguous


def new_cache(n_kv, capacity, d, fill=FILL):
    import torch
    return {n: torch.full((n_kv, capacity, w), fill, dtype=torch.uint8, device="cuda")
            for n, w in (("k_codes", d // 2), ("k_scales", d // 32), ("v_codes", d // 2),
                         ("v_scales", d // 32))}


def bf16_rows(n_kv, rows, d, seed, wide=True):
    """N(0, 1) rows; with ``wide`` also powers of two over most of bf16's range."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n_kv, rows, d))
    if wide:
        x *= np.exp2(rng.integers(-100, 100, (n_kv, rows, 1)).astype(np.float64))
    return inputs.f32_to_bf16_bits(x.astype(np.float32))


def _write(p, k, v, cache):
    import torch
    from paper_2502_12085_amd import apb
    apb.cache4_write(p, dev_bf16(k), dev_bf16(v), cache)
    torch.cuda.synchronize()


@pytest.mark.parametrize("d", [64, 128])
def test_every_bf16_number(d):
    need_gpu()
    from paper_2502_12085_amd import apb
    say(f"[cache4 every number] {d}")
    rng = np.random.default_rng(d)
    every = np.arange(65536, dtype=np.uint16)
    groups = [
        every.reshape(-1, 32),                                  # neighbours share a group
        rng.permutation(every).reshape(-1, 32),                 # and strangers
    ]
    # every number under a scale near its own: beside a largest element up to 16
    # times as large (in the high exponents the largest there is)
    near = every.copy()
    top = np.minimum((near & 0x7FFF).astype(np.int32) + rng.integers(0, 4 * 128, 65536), 0x7F7F)
    g = np.zeros((65536, 32), np.uint16)
    g[:, 0], g[:, 1], g[:, 2] = near, top, near ^ 0x8000
    groups.append(g)
    bits = np.concatenate(groups).reshape(1, -1, d)
    rows = bits.shape[1]
    cache = new_cache(1, rows, d)
    p = apb.Cache4Problem(1, d, rows, 0, rows, rows, 0)
    _write(p, bits, bits[:, ::-1], cache)
    for n, x in (("k", bits), ("v", bits[:, ::-1])):
        codes, scales = oracle.quantise4_ref(x)
        assert np.array_equal(cache[n + "_scales"].cpu().numpy(), scales)
        assert np.array_equal(cache[n + "_codes"].cpu().numpy(), codes)


@pytest.mark.parametrize("shape", [
    # n_kv, d, capacity, first_row, n_rows, bf16_rows, bf16_first
    (1, 64, 1, 0, 1, 1, 0),            # one row, no more
    (3, 64, 7, 3, 1, 5, 4),            # one row inside
    (2, 128, 1021, 515, 1, 1, 0),
    (2, 64, 1021, 130, 127, 300, 173),  # rows off every block
    (2, 64, 1021, 0, 128, 128, 0),
    (2, 128, 777, 1, 65, 66, 1),
    (5, 128, 64, 0, 64, 64, 0),
    (1, 128, 5000, 999, 3001, 4000, 7),
    (7, 64, 4099, 1, 4098, 4100, 2),
    (8, 128, 16400, 11, 16384, 20480, 4096),
])
def test_write_and_read(shape):
    torch = need_gpu()
    from paper_2502_12085_amd import apb
    say(f"[cache4 rows] {shape}")
    n_kv, d, cap, first, n, src, src_first = shape
    k, v = (bf16_rows(n_kv, src, d, s) for s in (1, 2))
    cache = new_cache(n_kv, cap, d)
    p = apb.Cache4Problem(n_kv, d, cap, first, n, src, src_first)
    _write(p, k, v, cache)
    k_out = torch.full((n_kv, src, d), 7.0, dtype=torch.bfloat16, device="cuda")
    v_out = k_out.clone()
    apb.cache4_read(p, cache, k_out, v_out)
    torch.cuda.synchronize()
    for name, x, out in (("k", k, k_out), ("v", v, v_out)):
        ref_codes, ref_scales = oracle.quantise4_ref(x[:, src_first:src_first + n])
        for got, ref in ((cache[name + "_codes"], ref_codes), (cache[name + "_scales"], ref_scales)):
            want = np.full(got.shape, FILL, np.uint8)
            want[:, first:first + n] = ref
            assert np.array_equal(got.cpu().numpy(), want)
        want = np.full((n_kv, src, d), 7.0)
        want[:, src_first:src_first + n] = oracle.values4_ref(ref_codes, ref_scales)
        assert np.array_equal(host_bf16_to_f64(out), want)


def test_read_not_a_number():
    torch = need_gpu()
    from paper_2502_12085_amd import apb
    k = bf16_rows(2, 9, 64, 5, wide=False)
    k[0, 3, 5], k[1, 8, 40], k[1, 0, 63] = 0x7F80, 0xFF80, 0x7FC1  # inf, -inf, NaN
    cache = new_cache(2, 9, 64)
    p = apb.Cache4Problem(2, 64, 9, 0, 9, 9, 0)
    _write(p, k, k, cache)
    out = torch.zeros(2, 9, 64, dtype=torch.bfloat16, device="cuda")
    apb.cache4_read(p, cache, out, torch.zeros_like(out))
    ref = oracle.values4_ref(*oracle.quantise4_ref(k))
    assert np.isnan(ref).sum() == 3 * 32
    assert np.array_equal(host_bf16_to_f64(out), ref, equal_nan=True)


def test_memory_of_zeros_reads_as_zeros():
    torch = need_gpu()
    from paper_2502_12085_amd import apb
    cache = new_cache(2, 33, 128, fill=0)
    out = torch.full((2, 33, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    v = out.clone()
    apb.cache4_read(apb.Cache4Problem(2, 128, 33, 0, 33, 33, 0), cache, out, v)
    assert not host_bits(out).any() and not host_bits(v).any()


def test_every_code_under_every_scale():
    torch = need_gpu()
    from paper_2502_12085_amd import apb
    say("[cache4 every code and scale]")
    cache = new_cache(1, 256, 64, fill=0)
    codes = np.tile(np.arange(16, dtype=np.uint8), 4)
    cache["k_codes"][:] = _device(codes[0::2] | (codes[1::2] << 4))
    b = np.arange(256, dtype=np.uint8)
    b = np.where((b < 7) | ((b > 252) & (b < 255)), 7, b).astype(np.uint8)
    cache["k_scales"][:] = _device(np.repeat(b[:, None], 2, 1)[None])
    out = torch.zeros(1, 256, 64, dtype=torch.bfloat16, device="cuda")
    apb.cache4_read(apb.Cache4Problem(1, 64, 256, 0, 256, 256, 0), cache, out, torch.zeros_like(out))
    ref = oracle.values4_ref(cache["k_codes"].cpu().numpy(), cache["k_scales"].cpu().numpy())
    assert np.array_equal(host_bf16_to_f64(out), ref, equal_nan=True)


def test_appending_token_by_token_is_one_write():
    need_gpu()
    from paper_2502_12085_amd import apb
    k, v = (bf16_rows(3, 40, 64, s) for s in (8, 9))
    whole, grown = new_cache(3, 50, 64), new_cache(3, 50, 64)
    _write(apb.Cache4Problem(3, 64, 50, 5, 40, 40, 0), k, v, whole)
    for i in range(40):
        _write(apb.Cache4Problem(3, 64, 50, 5 + i, 1, 40, i), k, v, grown)
    for n in whole:
        assert np.array_equal(whole[n].cpu().numpy(), grown[n].cpu().numpy())


def test_on_another_stream_and_in_a_graph():
    torch = need_gpu()
    from paper_2502_12085_amd import apb
    k, v = (dev_bf16(bf16_rows(2, 33, 64, s)) for s in (3, 4))
    whole = new_cache(2, 40, 64)
    p = apb.Cache4Problem(2, 64, 40, 7, 33, 33, 0)
    apb.cache4_write(p, k, v, whole)
    torch.cuda.synchronize()
    side, other = torch.cuda.Stream(), new_cache(2, 40, 64)
    out = [torch.zeros_like(k) for _ in range(4)]
    torch.cuda.synchronize()
    apb.cache4_write(p, k, v, other, stream=side)
    apb.cache4_read(p, other, out[0], out[1], stream=side)
    side.synchronize()
    with torch.cuda.stream(side):  # the current stream, which is not the default
        apb.cache4_read(p, whole, out[2], out[3])
    side.synchronize()
    assert all(torch.equal(whole[n], other[n]) for n in whole)
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3])
    graph, grown = torch.cuda.CUDAGraph(), new_cache(2, 40, 64)
    with torch.cuda.graph(graph):
        apb.cache4_write(p, k, v, grown)
    for _ in range(3):
        grown["k_codes"].fill_(FILL)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(whole[n], grown[n]) for n in whole)


def test_offsets_past_32_bits():
    # the last head's codes start 4.3 GB into the tensor, its bf16 rows past 2^32 bytes
    torch = need_gpu()
    from paper_2502_12085_amd import apb
    say("[cache4 long]")
    n_kv, d, cap = 3, 128, (1 << 25) + 5
    cache = new_cache(n_kv, cap, d, fill=0)
    rows = 1 << 24
    k = torch.zeros(n_kv, rows, d, dtype=torch.bfloat16, device="cuda")
    tail = bf16_rows(n_kv, 70, d, 6)
    k[:, -70:] = dev_bf16(tail)
    apb.cache4_write(apb.Cache4Problem(n_kv, d, cap, cap - 70, 70, rows, rows - 70), k, k, cache)
    codes, scales = oracle.quantise4_ref(tail)
    assert np.array_equal(cache["v_codes"][:, -70:].cpu().numpy(), codes)
    assert np.array_equal(cache["k_scales"][:, -70:].cpu().numpy(), scales)
    assert not cache["k_codes"][:, -200:-70].any() and not cache["k_codes"][:, :200].any()
    out = torch.zeros_like(k)
    apb.cache4_read(apb.Cache4Problem(n_kv, d, cap, cap - 70, 70, rows, rows - 70), cache, out,
                    k)
    assert np.array_equal(host_bf16_to_f64(out[:, -70:].contiguous()),
                          oracle.values4_ref(codes, scales))
    assert not out[:, :-70].any()
