"""Decoding attention over a KV cache in 4 bits where probabilities of every size count:
one key far above the rest whose values are zero (an attention sink), so that o is made
of probabilities that are tiny beside the largest.

Bound of an element of o: that of ``test_gpu_decode4``, relative to sum p |v|, without its
absolute term.  A probability enters the value product with its 24 bits whatever its size,
down to where fp32 itself ends: 2^-126 of the largest, times max |v|, for each key, twice
over.

Norm of o's error, shapes of N(0, 1): a logit of a few units is a sum of d terms whose
partial sums are rounded to 2^-24 of themselves, 2e-7 of a probability at d = 128; its
base-2 exponent, 8 to 16 in magnitude, is rounded to half of 2^-20, 3.3e-7; the
exponential, the parts and the sums are 2e-7 together.  Of independent signs over the keys
they are below 1e-6 of o's norm.  Behind a sink of g nats the exponent is up to 128 in
magnitude, rounded to half of 2^-17 (2.6e-6 of a probability): 1e-5.
"""
import numpy as np
import pytest

import oracle
import test_gpu_decode4 as base
from paper_2502_12085_amd import inputs
from gpu_util import dev_bf16, need_gpu, say
from test_gpu_cache4 import bf16_rows, new_cache

pytestmark = pytest.mark.gpu

ORDINARY = list(dict.fromkeys(
    s for f in (base.test_matches_oracle, base.test_forms) for m in f.pytestmark
    if m.name == "parametrize" for s in m.args[1]))

# every form of the kernel: head size, 16 or 32 rows a wave, four or eight waves, one split
# or several (a CPU test holds that)
SINKS = [
    # n_q, n_kv, d, capacity, cache_len, n_new, causal
    (4, 1, 64, 130, 128, 4, 1),
    (4, 1, 64, 1021, 515, 3, 1),
    (8, 2, 128, 120, 100, 3, 1),
    (8, 2, 128, 500, 400, 3, 0),
    (4, 1, 64, 100, 97, 7, 1),
    (8, 1, 128, 100, 90, 6, 1),
    (4, 1, 64, 300, 300, 5, 1),
    (8, 1, 128, 300, 290, 4, 0),
    (8, 2, 64, 2100, 2000, 1, 1),
    (8, 8, 128, 1000, 1000, 1, 1),
    (32, 8, 128, 4500, 4097, 1, 1),
    (8, 2, 64, 30000, 29000, 1, 1),
    (32, 8, 128, 16390, 16385, 1, 1),
    (4, 1, 64, 2000, 1999, 7, 1),
    (8, 1, 128, 2000, 1777, 4, 0),
    (7, 1, 128, 1810, 1800, 1, 1),
    (8, 1, 64, 50000, 49000, 5, 1),
    (8, 1, 128, 50000, 49000, 5, 0),
    (32, 8, 128, 2200, 2112, 64, 1),
    (120, 120, 64, 1700, 1650, 17, 1),
    (120, 120, 128, 1700, 1650, 17, 0),
    (300, 300, 64, 200, 199, 1, 1),
    (260, 260, 64, 140, 131, 70, 1),
]


def check(what, got, ref, keys, d, norm_bound):
    (o, lse), (ro, rl, pv, qk) = got, ref
    _, bl = base.bounds(keys, d, rl, pv, qk)
    logit, add = 2 * (d + 8) * 2.0 ** -24 * qk, 2 * (keys / 32 + 64) * 2.0 ** -24
    bo = pv * (2 * logit + 2.0 ** -21 + 2.0 ** -24 + 2 * add)[..., None]
    bo = bo + 2 * keys * 2.0 ** -126 * base.V_MAX
    assert np.isfinite(o).all() and np.isfinite(lse).all(), what
    eo, el = np.abs(o - ro), np.abs(lse - rl)
    norm = np.linalg.norm(o - ro) / np.linalg.norm(ro)
    say(f"  {what}: o {norm:.2e} of its norm, worst {(eo / bo).max():.3f} of its bound, lse "
        f"{(el / bl).max():.3f} of its")
    assert norm <= norm_bound, what
    assert np.all(eo <= bo) and np.all(el <= bl), what


@pytest.mark.parametrize("shape", ORDINARY)
def test_ordinary_logits(shape):
    need_gpu()
    say(f"[decode4 range] {shape}")
    n_q, n_kv, d, cap, keys, n_new, causal = shape
    q, cache = base.make(n_q, n_kv, d, cap, keys, n_new, seed=keys + 1)
    k, v = base.held(cache, keys)
    got = base.run(q, cache, n_kv, cap, keys, causal)
    check(f"ordinary {shape}", got, oracle.decode4_ref(q, k, v, causal=causal, bound=True), keys,
          d, 1e-6)


@pytest.mark.parametrize("every", [0, 97])
@pytest.mark.parametrize("shape", SINKS)
def test_sinks(shape, every):
    """Key 0 (and with ``every`` each 97th) g nats above the others, its values zero: 32
    elements of q are equal, and those of the others' K zero."""
    torch = need_gpu()
    from paper_2502_12085_amd import apb
    say(f"[decode4 sinks] {shape} {every}")
    n_q, n_kv, d, cap, keys, n_new, causal = shape
    q = inputs.bf16_bits_to_f32(bf16_rows(n_q, n_new, d, 1, wide=False)).copy()
    k, v = (inputs.bf16_bits_to_f32(bf16_rows(n_kv, keys, d, s, wide=False)).copy()
            for s in (2, 3))
    at = slice(0, keys, every) if every else slice(0, 1)
    k[:, :, :32] = 0
    k[:, at] = 0
    k[:, at, :32] = 4
    v[:, at] = 0
    cache = new_cache(n_kv, cap, d, fill=0xFF)
    apb.cache4_write(apb.Cache4Problem(n_kv, d, cap, 0, keys, keys, 0),
                     *(dev_bf16(inputs.f32_to_bf16_bits(x)) for x in (k, v)), cache)
    cache["v_scales"][:, at] = 127  # zeros of an ordinary scale
    torch.cuda.synchronize()
    hk, hv = base.held(cache, keys)
    for g in (10, 14, 18, 22, 50):
        q[:, :, :32] = g * d ** 0.5 / (32 * 4)
        bits = inputs.f32_to_bf16_bits(q)
        ref = oracle.decode4_ref(bits, hk, hv, causal=causal, bound=True)
        got = base.run(bits, cache, n_kv, cap, keys, causal)
        check(f"{g} nats {shape} {every}", got, ref, keys, d, 1e-5)


@pytest.mark.parametrize("rows", base.ROWS)
def test_values_of_one_group_behind_a_sink(rows):
    """The sink's values are zero in the first 32 elements and large in the others: the
    small probabilities count in the first alone."""
    torch = need_gpu()
    from paper_2502_12085_amd import apb
    say(f"[decode4 group behind a sink] {rows}")
    n_q, n_kv, d, n_new = rows
    keys = 1300
    q = inputs.bf16_bits_to_f32(bf16_rows(n_q, n_new, d, 1, wide=False)).copy()
    k, v = (inputs.bf16_bits_to_f32(bf16_rows(n_kv, keys, d, s, wide=False)).copy()
            for s in (2, 3))
    k[:, :, :32], k[:, 0], k[:, 0, :32] = 0, 0, 4
    v[:, 0], v[:, 0, 32:] = 0, 6
    q[:, :, :32] = 20 * d ** 0.5 / (32 * 4)
    cache = new_cache(n_kv, keys, d, fill=0xFF)
    apb.cache4_write(apb.Cache4Problem(n_kv, d, keys, 0, keys, keys, 0),
                     *(dev_bf16(inputs.f32_to_bf16_bits(x)) for x in (k, v)), cache)
    cache["v_scales"][:, 0, 0] = 127
    torch.cuda.synchronize()
    bits = inputs.f32_to_bf16_bits(q)
    ref = oracle.decode4_ref(bits, *base.held(cache, keys), causal=1, bound=True)
    o, lse = base.run(bits, cache, n_kv, keys, keys, 1)
    for dims in (slice(0, 32), slice(32, None)):
        check(f"group {rows} {dims}", (o[..., dims], lse),
              (ref[0][..., dims], ref[1], ref[2][..., dims], ref[3]), keys, d, 1e-5)


@pytest.mark.parametrize("rows", [(4, 1, 64, 6), (8, 2, 128, 3), (8, 2, 128, 20), (4, 2, 64, 70)])
def test_unseen_rows_of_any_bytes(rows):
    """Every scale byte and the largest codes in a row among the new tokens' own, of K, of V
    and of both: the tokens before it are as if it were not there.  Scale bytes past 252 in V
    are past bf16's largest number: NaN in their 32 elements, for those that see them."""
    need_gpu()
    say(f"[decode4 any bytes] {rows}")
    n_q, n_kv, d, n_new = rows
    keys = 200 + n_new
    q, cache = base.make(n_q, n_kv, d, keys, keys, n_new, seed=5)
    k, v = base.held(cache, keys)
    clean = oracle.decode4_ref(q, k, v, causal=1, bound=True)
    at = keys - n_new // 2  # tokens j >= n_new - n_new // 2 see it
    sees = np.arange(n_new) >= n_new - n_new // 2
    kept = {n: t.clone() for n, t in cache.items()}
    for which in ("v", "k", "kv"):
        for b in (0, 1, 6, 7, 127, 251, 252, 253, 254, 255):
            for n in which:
                cache[n + "_scales"][:, at] = kept[n + "_scales"][:, at]
                cache[n + "_scales"][:, at, 1] = b
                cache[n + "_codes"][:, at] = 0xF7  # 6 and -6
            o, lse = base.run(q, cache, n_kv, keys, keys, 1)
            check(f"{which} {b} {rows}", (o[:, ~sees], lse[:, ~sees]),
                  [x[:, ~sees] for x in clean], keys, d, 1e-6)
            if which == "v":
                bad = np.isnan(o[:, sees])
                assert bad[..., 32:64].all() if b > 252 else not bad.any()
                assert not bad[..., :32].any() and not bad[..., 64:].any()
        for n, t in kept.items():
            cache[n].copy_(t)


@pytest.mark.parametrize("shape", [(4, 1, 64, 140, 1, 32), (8, 2, 64, 2000, 1, 128),
                                   (8, 2, 128, 2000, 9, 128), (14, 7, 64, 450, 100, 128),
                                   (7, 1, 128, 1800, 37, 128)])
def test_nan_among_keys_without_weight(shape):
    """The first keys overflow to logits of -inf for every row, 64 products of -2^129 and
    more: they have no weight, a whole split of them either, but a NaN group of their
    values is one of visible rows, and its 32 elements of o are NaN."""
    need_gpu()
    say(f"[decode4 no weight] {shape}")
    n_q, n_kv, d, keys, n_new, n = shape
    q, cache = base.make(n_q, n_kv, d, keys, keys, n_new, seed=9)
    q[:] = 0xC080  # -4
    cache["k_scales"][:, :n] = 252
    cache["k_codes"][:, :n] = 0x77
    k, v = (x[:, n:] for x in base.held(cache, keys))
    ref = oracle.decode4_ref(q, k, v, causal=0, bound=True)
    check(f"no weight {shape}", base.run(q, cache, n_kv, keys, keys, 0), ref, keys, d, 1e-5)
    cache["v_scales"][:, n // 2, 1] = 255
    o, lse = base.run(q, cache, n_kv, keys, keys, 0)
    nan = np.zeros(o.shape, bool)
    nan[..., 32:64] = True
    assert np.array_equal(np.isnan(o), nan)
    check(f"no weight, NaN {shape}", (np.where(nan, ref[0], o), lse), ref, keys, d, 1e-5)


@pytest.mark.parametrize("rows", [(4, 1, 64, 4), (8, 2, 128, 20), (8, 2, 128, 3)])
def test_the_rows_beside_one_that_overflows(rows):
    """A key of the largest numbers in one group of 32, where all queries but two are zero:
    32 products of 2^129 and more are a NaN for the first, a key without weight for the
    last, and a logit like another for the rows between."""
    need_gpu()
    say(f"[decode4 beside overflow] {rows}")
    n_q, n_kv, d, n_new = rows
    keys, at = 300, 77
    q, cache = base.make(n_q, n_kv, d, keys, keys, n_new, seed=15)
    q[:, :, :32] = 0
    q[0, 0, :32], q[-1, -1, :32] = 0x4080, 0xC080  # 4 and -4
    cache["k_scales"][:, at, 0] = 252
    cache["k_codes"][:, at, :16] = 0x77
    o, lse = base.run(q, cache, n_kv, keys, keys, 0)
    assert np.isnan(o[0, 0]).all() and np.isnan(lse[0, 0])
    k, v = base.held(cache, keys)
    q[0, 0, :32] = q[-1, -1, :32] = 0
    ref = oracle.decode4_ref(q, k, v, causal=0, bound=True)
    between = np.ones((n_q, n_new), bool)
    between[0, 0] = between[-1, -1] = False
    check(f"beside {rows}", (o[between], lse[between]), [x[between] for x in ref], keys, d, 1e-6)
    # the last without the key (its other logits carry the -4)
    q[-1, -1, :32] = 0xC080
    ref = oracle.decode4_ref(q, *(np.delete(x, at, axis=1) for x in (k, v)), causal=0, bound=True)
    check(f"without the key {rows}", (o[-1:, -1:], lse[-1:, -1:]), [x[-1:, -1:] for x in ref], keys,
          d, 1e-5)
