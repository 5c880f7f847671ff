"""GPU parity of decoding-stage attention over a KV cache in 4 bits against the
fp64 oracle on the cache's exact values.

Bound of an element of o, by its arithmetic.  A logit is an fp32 sum of d products
(each exact: a bf16 query times a value of two significant bits): in whatever order,
off by at most (d + 8) 2^-24 of sum |q_i k_i| (8: the scale, the base-2 exponent
and its subtraction of the maximum), doubled for what a matrix instruction's own
additions may round beside.  A probability carries that as a relative error, and so
does the sum that divides it: twice; the exponential is good to 2^-22.  A probability
enters the value product as the sum of three bf16 numbers, which hold its 24 bits, or
of two fp16 ones, each rounded to nearest: the first leaves 2^-12 of it, the second
2^-12 of that, 2^-24 together where both are normal.  Else the second is off by half the
2^-24 that fp16 numbers are apart, and the largest probability of a row then stands at
2^6 at least: 2^-25 / 2^6 = 2^-31 of the largest, which is 1 at most, times max |v| for
each key.  The value product and the sum add in fp32: blocks of 32 keys one after another
in a part, then the parts: (keys / 32 + 64) 2^-24, doubled as above.  All of it is
relative to sum p |v|, which the oracle gives.  The LSE has the logits' error once,
its sum's and its own rounding.

These are worst cases.  Where logits are of ordinary size the errors of the keys are
of independent signs, and the norm of o's error is held too: under 2^-24 sqrt(d) times
a logit of 5 (1e-6 to 3e-6) of each probability, and 1e-6 of its exponential, parts and
sum, are together within 1e-5 of o's norm.
"""
import numpy as np
import pytest

import oracle
from paper_2502_12085_amd import inputs
from gpu_util import dev_bf16, host_bf16_to_f64, need_gpu, say
from test_gpu_cache4 import bf16_rows, new_cache

pytestmark = pytest.mark.gpu


V_MAX = 64.0  # no value of these tests' finite rows is larger


def bounds(keys, d, lse_ref, pv, qk):
    logit = 2 * (d + 8) * 2.0 ** -24 * qk
    add = 2 * (keys / 32 + 64) * 2.0 ** -24
    o = pv * (2 * logit + 2.0 ** -21 + 2.0 ** -24 + 2 * add)[..., None]
    o = o + keys * 2.0 ** -31 * V_MAX
    lse = logit + 2.0 ** -22 + add + 2.0 ** -23 * np.abs(np.where(np.isfinite(lse_ref), lse_ref, 0))
    return o, lse


def make(n_q, n_kv, d, cap, keys, n_new, seed, past=0xFF):
    """q, and a cache whose first ``keys`` rows hold quantised N(0, 1) rows and whose
    other bytes are all ``past`` (0xFF: scales of NaN)."""
    import torch
    from paper_2502_12085_amd import apb
    q = bf16_rows(n_q, n_new, d, seed, wide=False)
    k, v = (bf16_rows(n_kv, max(keys, 1), d, seed + s, wide=False) for s in (1, 2))
    cache = new_cache(n_kv, cap, d, fill=past)
    apb.cache4_write(apb.Cache4Problem(n_kv, d, cap, 0, keys, max(keys, 1), 0), dev_bf16(k),
                     dev_bf16(v), cache)
    torch.cuda.synchronize()
    return q, cache


def held(cache, keys):
    c = {n: t[:, :keys].cpu().numpy() for n, t in cache.items()}
    return (oracle.values4_ref(c["k_codes"], c["k_scales"]),
            oracle.values4_ref(c["v_codes"], c["v_scales"]))


def run(q, cache, n_kv, cap, keys, causal, scale=0.0, stream=None):
    import torch
    from paper_2502_12085_amd import apb
    n_q, n_new, d = q.shape
    p = apb.Decode4Problem(n_q, n_kv, d, cap, keys, n_new, causal)
    # a guard row behind each output and bytes behind the workspace's
    o = torch.full((n_q * n_new + 1, d), float("nan"), dtype=torch.float32, device="cuda")
    lse = torch.full((n_q * n_new + 1,), float("nan"), dtype=torch.float32, device="cuda")
    need = apb.decode4_workspace_size(p)
    ws = torch.full((need + 64,), FILL, dtype=torch.uint8, device="cuda")
    apb.decode4_attention(p, dev_bf16(q), cache, o[:-1].view(n_q, n_new, d),
                          lse[:-1].view(n_q, n_new), ws[:need], scale, stream)
    torch.cuda.synchronize()
    assert torch.isnan(o[-1]).all() and torch.isnan(lse[-1]) and (ws[need:] == FILL).all()
    return (o[:-1].view(n_q, n_new, d).cpu().numpy().astype(np.float64),
            lse[:-1].view(n_q, n_new).cpu().numpy().astype(np.float64))


FILL = 0x5A


def check(what, got, ref, keys, d, norm_bound=None):
    (o, lse), (ro, rl, pv, qk) = got, ref
    bo, bl = bounds(keys, d, rl, pv, qk)
    empty = np.isneginf(rl)
    assert np.array_equal(np.isneginf(lse), empty), what
    assert np.isfinite(o).all() and np.isfinite(lse[~empty]).all(), what
    eo, el = np.abs(o - ro), np.abs(np.where(empty, 0, lse) - np.where(empty, 0, rl))
    norm = np.linalg.norm(ro)
    say(f"  {what}: o {np.linalg.norm(o - ro) / norm if norm else 0:.2e} of its norm, worst "
        f"{(eo / np.maximum(bo, 1e-300)).max():.3f} of its bound, lse {el.max():.2e} = "
        f"{(el / bl).max():.3f}")
    assert norm_bound is None or np.linalg.norm(o - ro) <= norm_bound * norm, what
    for name, e, b in (("o", eo, bo), ("lse", el, bl)):
        over = np.argwhere(e > b)
        first = tuple(over[0]) if len(over) else None
        assert first is None, f"{what}: {name} at {first}: off by {e[first]}, bound {b[first]}"


@pytest.mark.parametrize("shape", [
    # n_q, n_kv, d, capacity, cache_len, n_new, causal
    (4, 1, 64, 1021, 515, 3, 1),      # the tiny step
    (1, 1, 64, 1, 1, 1, 1),           # one key, the token's own
    (1, 1, 128, 2, 1, 1, 0),
    (4, 2, 128, 40, 33, 1, 1),        # just past 32 keys
    (4, 2, 128, 40, 31, 2, 0),
    (8, 2, 64, 64, 64, 5, 1),
    (8, 2, 128, 128, 127, 1, 1),
    (8, 2, 128, 1000, 129, 4, 1),
    (8, 8, 128, 1000, 1000, 1, 1),    # no shared heads
    (7, 1, 64, 3100, 3000, 1, 0),     # a group of 7
    (16, 1, 128, 700, 600, 1, 1),     # 16 rows of one KV head
    (17, 1, 128, 700, 600, 1, 1),     # and 17
    (32, 8, 128, 4500, 4097, 1, 1),
    (56, 8, 128, 4200, 4100, 2, 1),   # 14 rows
    (12, 2, 128, 800, 777, 5, 1),     # 30 rows
    (8, 2, 64, 300, 288, 9, 0),       # 36 rows
    (40, 8, 128, 9301, 9300, 17, 0),  # 85 rows
    (6, 2, 64, 513, 511, 21, 1),      # 63 rows
    (6, 2, 64, 513, 512, 22, 1),      # 66
    (4, 4, 128, 643, 643, 130, 1),    # no shared heads, 130 rows
    (8, 2, 64, 1100, 1040, 40, 1),    # 160
    (32, 8, 128, 2200, 2112, 64, 1),  # 256
    (5, 1, 128, 400, 391, 77, 0),     # 385
    (1, 1, 64, 1400, 1391, 391, 1),
    (2, 2, 128, 300, 300, 300, 1),    # all rows new: token 0 sees one key
    (4, 1, 64, 700, 65, 65, 1),
])
def test_matches_oracle(shape):
    need_gpu()
    say(f"[decode4] {shape}")
    n_q, n_kv, d, cap, keys, n_new, causal = shape
    q, cache = make(n_q, n_kv, d, cap, keys, n_new, seed=keys)
    k, v = held(cache, keys)
    got = run(q, cache, n_kv, cap, keys, causal)
    check(f"decode4 {shape}", got, oracle.decode4_ref(q, k, v, causal=causal, bound=True), keys, d,
          norm_bound=1e-5)


@pytest.mark.parametrize("shape", [
    (32, 8, 128, 16390, 16385, 1, 1),
    (4, 1, 64, 70000, 65537, 2, 0),
    (8, 2, 128, 33000, 32801, 24, 1),
    (16, 4, 64, 12000, 11111, 64, 1),
])
def test_long_caches(shape):
    need_gpu()
    say(f"[decode4 long] {shape}")
    n_q, n_kv, d, cap, keys, n_new, causal = shape
    q, cache = make(n_q, n_kv, d, cap, keys, n_new, seed=7)
    k, v = held(cache, keys)
    got = run(q, cache, n_kv, cap, keys, causal)
    check(f"decode4 {shape}", got, oracle.decode4_ref(q, k, v, causal=causal, bound=True), keys, d,
          norm_bound=1e-5)


@pytest.mark.parametrize("shape", [
    # the forms that the shapes above leave out: one launch, one split of many rows, so
    # many heads that a split of each fills the GPU, splits of several rounds
    (4, 1, 64, 130, 128, 4, 1),       # 16 rows, four blocks
    (8, 2, 128, 120, 100, 3, 1),
    (4, 1, 64, 300, 300, 5, 1),       # 20 rows, ten blocks: one launch
    (8, 1, 128, 300, 290, 4, 0),
    (4, 1, 64, 100, 97, 7, 1),        # 28 rows, four blocks
    (8, 1, 128, 100, 90, 3, 1),
    (4, 1, 64, 2000, 1999, 7, 1),     # 28 rows, splits
    (8, 1, 128, 2000, 1777, 4, 0),
    (8, 2, 64, 100, 77, 15, 1),       # 60 rows, one split
    (8, 2, 128, 128, 128, 11, 0),
    (8, 2, 64, 120, 120, 40, 1),      # 160 rows, one split
    (8, 2, 128, 100, 93, 33, 0),
    (8, 2, 64, 1500, 1450, 15, 1),    # 60 rows, splits
    (8, 2, 128, 1500, 1450, 15, 1),
    (8, 2, 64, 30000, 29000, 1, 1),   # splits of eight waves
    (8, 1, 64, 50000, 49000, 5, 1),
    (8, 1, 128, 50000, 49000, 5, 0),
    (16, 8, 64, 8000, 7777, 66, 1),
    (16, 8, 128, 8000, 7777, 66, 1),
    (300, 300, 64, 200, 199, 1, 1),   # one split each of more heads than CUs
    (600, 300, 128, 200, 160, 9, 0),
    (300, 300, 64, 200, 150, 35, 1),
    (260, 260, 64, 140, 131, 70, 1),
    (270, 90, 64, 400, 400, 30, 1),   # 90 heads: 270 row blocks
    (3, 3, 128, 900, 900, 300, 1),    # ten row blocks, of heads and splits off 8
    (200, 100, 64, 1700, 1650, 17, 1),  # 200 row blocks: splits of more than one round
    (128, 128, 128, 700, 650, 40, 1),
    (16, 16, 128, 900, 850, 200, 0),
    (14, 7, 64, 500, 450, 100, 0),
    (7, 1, 128, 1810, 1800, 37, 1),     # 259 rows, 9 to 16 splits
    (7, 1, 64, 1810, 1800, 37, 0),
])
def test_forms(shape):
    need_gpu()
    say(f"[decode4 forms] {shape}")
    n_q, n_kv, d, cap, keys, n_new, causal = shape
    q, cache = make(n_q, n_kv, d, cap, keys, n_new, seed=n_q + keys)
    k, v = held(cache, keys)
    got = run(q, cache, n_kv, cap, keys, causal)
    check(f"decode4 {shape}", got, oracle.decode4_ref(q, k, v, causal=causal, bound=True), keys, d,
          norm_bound=1e-5)


def _random_shapes():
    rng = np.random.default_rng(77)
    out = []
    for _ in range(40):
        n_kv, g = int(rng.choice([1, 2, 3, 8])), int(rng.integers(1, 9))
        d, causal = int(rng.choice([64, 128])), int(rng.integers(0, 2))
        n_new = int(2 ** rng.uniform(0, 6.6))
        keys = max(int(2 ** rng.uniform(0, 12)), n_new if causal else 1)
        out.append((n_kv * g, n_kv, d, keys + int(rng.integers(0, 70)), keys, n_new, causal))
    return out


@pytest.mark.parametrize("shape", _random_shapes())
def test_random_shapes(shape):
    need_gpu()
    say(f"[decode4 random] {shape}")
    n_q, n_kv, d, cap, keys, n_new, causal = shape
    q, cache = make(n_q, n_kv, d, cap, keys, n_new, seed=keys + n_new)
    k, v = held(cache, keys)
    got = run(q, cache, n_kv, cap, keys, causal)
    check(f"decode4 {shape}", got, oracle.decode4_ref(q, k, v, causal=causal, bound=True), keys, d,
          norm_bound=1e-5)


# one or a few row blocks, many rows; each with a late key that dwarfs the others
ROWS = [(4, 1, 64, 1), (8, 2, 128, 3), (8, 2, 128, 20), (4, 2, 64, 70), (4, 2, 128, 70)]


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("scale", [0.0, 1.0])
def test_a_maximum_that_comes_late(rows, scale):
    """Keys of 8 times the size towards the end, and with a scale of 1.0 logits
    that differ by hundreds: the running maximum rises many times."""
    torch = need_gpu()
    from paper_2502_12085_amd import apb
    say(f"[decode4 late maximum] {rows} {scale}")
    n_q, n_kv, d, n_new = rows
    keys = 1500
    q, cache = make(n_q, n_kv, d, keys, keys, n_new, seed=31)
    k = bf16_rows(n_kv, keys, d, 3, wide=False)
    k = inputs.f32_to_bf16_bits(
        (inputs.bf16_bits_to_f32(k) * np.linspace(0.1, 8, keys)[None, :, None]).astype(np.float32))
    apb.cache4_write(apb.Cache4Problem(n_kv, d, keys, 0, keys, keys, 0), dev_bf16(k), dev_bf16(k),
                     cache)
    torch.cuda.synchronize()
    kv, vv = held(cache, keys)
    got = run(q, cache, n_kv, keys, keys, 1, scale)
    ref = oracle.decode4_ref(q, kv, vv, causal=1, scale=scale or None, bound=True)
    check(f"late {rows} {scale}", got, ref, keys, d)


@pytest.mark.parametrize("rows", ROWS)
def test_every_logit_far_below_zero(rows):
    # logits near -3000: the maximum has to be found, not assumed near zero
    torch = need_gpu()
    from paper_2502_12085_amd import apb
    n_q, n_kv, d, n_new = rows
    keys = 700
    q = inputs.f32_to_bf16_bits(
        (4 + np.random.default_rng(1).standard_normal((n_q, n_new, d)) / 8).astype(np.float32))
    k = inputs.f32_to_bf16_bits(
        (-8 + np.random.default_rng(2).standard_normal((n_kv, keys, d)) / 4).astype(np.float32))
    v = bf16_rows(n_kv, keys, d, 3, wide=False)
    cache = new_cache(n_kv, keys, d)
    apb.cache4_write(apb.Cache4Problem(n_kv, d, keys, 0, keys, keys, 0), dev_bf16(k), dev_bf16(v),
                     cache)
    torch.cuda.synchronize()
    kv, vv = held(cache, keys)
    got = run(q, cache, n_kv, keys, keys, 1, 1.0)
    ref = oracle.decode4_ref(q, kv, vv, causal=1, scale=1.0, bound=True)
    assert ref[1].max() < -1000
    check(f"far {rows}", got, ref, keys, d)


@pytest.mark.parametrize("shape", [(8, 2, 64, 100, 0, 3, 0), (32, 1, 128, 5, 0, 64, 0)])
def test_no_keys(shape):
    torch = need_gpu()
    from paper_2502_12085_amd import apb
    n_q, n_kv, d, cap, keys, n_new, causal = shape
    q = bf16_rows(n_q, n_new, d, 1, wide=False)
    o, lse = run(q, None, n_kv, cap, 0, 0)
    assert not o.any() and np.all(lse == -np.inf)
    o, lse = run(q, new_cache(n_kv, cap, d, fill=0xFF), n_kv, cap, 0, 0)
    assert not o.any() and np.all(lse == -np.inf)


@pytest.mark.parametrize("rows", [(4, 1, 64, 6), (8, 2, 128, 20), (4, 2, 128, 70), (2, 2, 64, 150)])
def test_what_a_row_does_not_see(rows):
    """Rows of NaN and of the largest numbers among the new tokens' own: the tokens
    before them are as if they were not there, those that see a NaN key are NaN, and a
    NaN group of values is seen in its 32 elements alone."""
    torch = need_gpu()
    from paper_2502_12085_amd import apb
    say(f"[decode4 unseen] {rows}")
    n_q, n_kv, d, n_new = rows
    keys = 200 + n_new
    q, cache = make(n_q, n_kv, d, keys, keys, n_new, seed=5)
    k, v = held(cache, keys)
    clean = oracle.decode4_ref(q, k, v, causal=1, bound=True)
    at = keys - n_new // 2  # row of a token in the middle: tokens j >= n_new - n_new // 2 see it
    sees = np.arange(n_new) >= n_new - n_new // 2
    vs = cache["v_scales"].clone()
    cache["v_scales"][:, at, 1] = 255
    o, lse = run(q, cache, n_kv, keys, keys, 1)
    nan = np.zeros((n_q, n_new, d), bool)
    nan[:, sees, 32:64] = True
    assert np.array_equal(np.isnan(o), nan)
    check(f"values {rows}", (np.where(nan, clean[0], o), lse), clean, keys, d)
    cache["v_scales"].copy_(vs)
    cache["k_scales"][:, at, 0] = 255
    o, lse = run(q, cache, n_kv, keys, keys, 1)
    nan = np.broadcast_to(sees[None, :], lse.shape)
    assert np.array_equal(np.isnan(lse), nan)
    assert np.array_equal(np.isnan(o).all(-1), nan) and np.array_equal(np.isnan(o).any(-1), nan)
    check(f"keys {rows}", (np.where(nan[..., None], clean[0], o), np.where(nan, clean[1], lse)),
          clean, keys, d)
    # the largest numbers, seen by some: their rows follow the oracle, the others stay
    cache["k_scales"][:, at] = 252
    cache["k_codes"][:, at] = 0x77
    o, lse = run(q, cache, n_kv, keys, keys, 1)
    check(f"before {rows}", (o[:, ~sees], lse[:, ~sees]), [x[:, ~sees] for x in clean], keys, d)


@pytest.mark.parametrize("rows", [(4, 1, 64, 6), (8, 2, 128, 3), (8, 2, 128, 20), (4, 2, 64, 70)])
def test_values_of_every_size(rows):
    """Groups of dims whose values are times a power of two, to the ends of what goes into
    the products as fp16 (scale bytes 108 to 134) and past them: the output is times
    that power.  Then
    blocks with a group of zeros under the least scale among the others, in runs and
    in turn: only the zeros show."""
    need_gpu()
    say(f"[decode4 sizes] {rows}")
    n_q, n_kv, d, n_new = rows
    keys = 1100
    groups = d // 32
    odd = np.repeat(np.random.default_rng(3).integers(0, 2, 35), 32)[:keys].astype(bool)
    for sizes in ([104, 140, 127, 118], [108, 134, 127, 118], [107, 135, 7, 199],
                  [108, 20, 134, 190]):
        q, cache = make(n_q, n_kv, d, keys, keys, n_new, seed=18)
        cache["v_scales"].fill_(127)
        k, v = held(cache, keys)
        scale = np.repeat([2.0 ** (b - 127) for b in sizes[:groups]], 32)
        for g in range(groups):
            cache["v_scales"][:, :, g] = sizes[g]
        o, lse = run(q, cache, n_kv, keys, keys, 1)
        check(f"sizes {sizes} {rows}", (o / scale, lse),
              oracle.decode4_ref(q, k, v, causal=1, bound=True), keys, d, norm_bound=1e-5)
        cache["v_codes"][:, odd, :16] = 0
        cache["v_scales"][:, odd, 0] = 7
        v[:, odd, :32] = 0
        o, lse = run(q, cache, n_kv, keys, keys, 1)
        check(f"mixed {sizes} {rows}", (o / scale, lse),
              oracle.decode4_ref(q, k, v, causal=1, bound=True), keys, d, norm_bound=1e-5)


def test_a_query_that_is_not_a_number():
    need_gpu()
    n_q, n_kv, d, keys, n_new = 8, 2, 128, 300, 9
    q, cache = make(n_q, n_kv, d, keys, keys, n_new, seed=12)
    k, v = held(cache, keys)
    clean = oracle.decode4_ref(q, k, v, causal=1, bound=True)
    q[3, 4, 77] = 0x7FC0
    o, lse = run(q, cache, n_kv, keys, keys, 1)
    nan = np.zeros((n_q, n_new), bool)
    nan[3, 4] = True
    assert np.array_equal(np.isnan(lse), nan) and np.array_equal(np.isnan(o).all(-1), nan)
    check("query", (np.where(nan[..., None], clean[0], o), np.where(nan, clean[1], lse)), clean,
          keys, d)


@pytest.mark.parametrize("rows", [(4, 1, 64, 4), (8, 2, 128, 20)])
def test_logits_that_overflow(rows):
    """A key of the largest numbers against queries of 4 and of -4: 64 products of 2^129
    and more pass fp32's largest number in any order.  NaN for the first, a key without
    weight for the second, and the other rows as they were."""
    need_gpu()
    say(f"[decode4 overflow] {rows}")
    n_q, n_kv, d, n_new = rows
    keys = 300
    q, cache = make(n_q, n_kv, d, keys, keys, n_new, seed=15)
    q[0, 0], q[n_q - 1, n_new - 1] = 0x4080, 0xC080
    at = 77
    cache["k_scales"][:, at] = 252
    cache["k_codes"][:, at] = 0x77
    o, lse = run(q, cache, n_kv, keys, keys, 0)
    assert np.isnan(o[0, 0]).all() and np.isnan(lse[0, 0])
    k, v = held(cache, keys)
    k, v = (np.delete(x, at, axis=1) for x in (k, v))
    ref = oracle.decode4_ref(q, k, v, causal=0, bound=True)
    last = (slice(n_q - 1, None), slice(n_new - 1, None))
    check(f"overflow {rows}", (o[last], lse[last]), [x[last] for x in ref], keys, d)


@pytest.mark.parametrize("rows", [(4, 1, 64, 4, 90), (8, 2, 128, 3, 3000), (8, 2, 128, 20, 900)])
def test_logits_of_millions(rows):
    """Logits of 2^22 times N(0, 1): the largest takes all, by far more than an fp32 sum
    of d products is off, and o is its key's value: a probability over itself, in
    products and sums of relative error 2^-24 each, a few of them."""
    need_gpu()
    say(f"[decode4 millions] {rows}")
    n_q, n_kv, d, n_new, keys = rows
    q, cache = make(n_q, n_kv, d, keys, keys, n_new, seed=16)
    q = (q + (11 << 7)).astype(np.uint16)  # times 2^11
    cache["k_scales"] += 11
    k, v = held(cache, keys)
    s = np.einsum("htd,hkd->htk", oracle.bf16_to_f64(q), np.repeat(k, n_q // n_kv, 0)) / d ** 0.5
    top = np.sort(s, -1)
    clear = top[..., -1] - top[..., -2] > 1000
    assert np.abs(s).max() < 2 ** 26 / 1.4427 and clear.mean() > 0.9
    o, lse = run(q, cache, n_kv, keys, keys, 0)
    assert np.isfinite(o).all() and np.isfinite(lse).all()
    want = np.stack([np.repeat(v, n_q // n_kv, 0)[h][s[h].argmax(-1)] for h in range(n_q)])
    assert np.all(np.abs(o - want)[clear] <= 2.0 ** -21 * np.abs(want)[clear])
    # the LSE: a sum of d products and a few roundings of its own
    qk = np.einsum("htd,hkd->htk", np.abs(oracle.bf16_to_f64(q)), np.abs(np.repeat(k, n_q // n_kv, 0)))
    assert np.all(np.abs(lse - top[..., -1]) <= 2 * (d + 8) * 2.0 ** -24 * qk.max(-1) / d ** 0.5)


@pytest.mark.parametrize("shape", [(8, 2, 64, 401, 400, 2), (8, 2, 128, 700, 699, 9)])
def test_scales_at_any_address(shape):
    """Scale bytes from an odd address on, written, read and attended over: bit for bit
    what they are at an aligned one."""
    torch = need_gpu()
    from paper_2502_12085_amd import apb
    say(f"[decode4 addresses] {shape}")
    n_q, n_kv, d, cap, keys, n_new = shape
    q, cache = make(n_q, n_kv, d, cap, keys, n_new, seed=31)
    want = run(q, cache, n_kv, cap, keys, 1)
    n = n_kv * cap * (d // 32)
    moved = dict(cache)
    for name, at in (("k_scales", 1), ("v_scales", 3)):
        raw = torch.full((n + 8,), FILL, dtype=torch.uint8, device="cuda")
        moved[name] = raw[at:at + n].view(n_kv, cap, d // 32)
        moved[name].copy_(cache[name])
        assert moved[name].data_ptr() % 4 == at
    rows = apb.Cache4Problem(n_kv, d, cap, 3, 50, 50, 0)
    out = [torch.zeros(n_kv, 50, d, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    apb.cache4_read(rows, cache, out[0], out[1])
    apb.cache4_read(rows, moved, out[2], out[3])
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3])
    for name in ("k_scales", "v_scales"):
        moved[name][:, 3:53] = FILL
    k, v = (dev_bf16(bf16_rows(n_kv, keys, d, 31 + s, wide=False))[:, 3:53].contiguous()
            for s in (1, 2))
    apb.cache4_write(rows, k, v, moved)
    for name in ("k_scales", "v_scales"):
        assert torch.equal(moved[name], cache[name])
    got = run(q, moved, n_kv, cap, keys, 1)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


@pytest.mark.parametrize("n_new", [1, 5])
def test_offsets_past_32_bits(n_new):
    """2^26 + 5 keys of two heads: the second head's codes start 4.3 GB into the tensor, and
    so do the last keys' of the first.  Queries of 8 against positive keys in the last
    300 rows: logits of 50 and more there, so that the others, zeros, weigh less than
    7e7 e^-50 = 2e-14 together."""
    torch = need_gpu()
    from paper_2502_12085_amd import apb
    say(f"[decode4 long offsets] {n_new} tokens")
    n_q, n_kv, d, tail = 8, 2, 128, 300
    keys = (1 << 26) + 5
    cap = keys + 3
    cache = new_cache(n_kv, cap, d, fill=0)
    k = bf16_rows(n_kv, tail, d, 41, wide=False) & 0x7FFF
    v = bf16_rows(n_kv, tail, d, 42, wide=False)
    apb.cache4_write(apb.Cache4Problem(n_kv, d, cap, keys - tail, tail, tail, 0), dev_bf16(k),
                     dev_bf16(v), cache)
    cache["k_scales"][:, keys:] = 255
    cache["v_scales"][:, keys:] = 255
    q = np.full((n_q, n_new, d), 0x4100, np.uint16)
    q[:, :, ::2] = 0x4110  # 9
    hk, hv = (oracle.values4_ref(*oracle.quantise4_ref(x)) for x in (k, v))
    assert (hk.sum(-1) * 8 / d ** 0.5).min() > 50
    ref = oracle.decode4_ref(q, hk, hv, causal=1, bound=True)
    check(f"long offsets, {n_new} tokens", run(q, cache, n_kv, cap, keys, 1), ref, tail, d)


@pytest.mark.parametrize("shape", [(32, 8, 128, 5000, 4999, 1), (8, 2, 64, 2000, 1999, 90)])
def test_the_same_every_time_and_on_any_stream(shape):
    torch = need_gpu()
    n_q, n_kv, d, cap, keys, n_new = shape
    q, cache = make(n_q, n_kv, d, cap, keys, n_new, seed=2)
    first = run(q, cache, n_kv, cap, keys, 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (None, side):
        again = run(q, cache, n_kv, cap, keys, 1, stream=stream)
        assert np.array_equal(first[0], again[0]) and np.array_equal(first[1], again[1])


def test_two_calls_at_once():
    torch = need_gpu()
    from paper_2502_12085_amd import apb
    jobs = []
    for i, (n_q, n_kv, d, keys, n_new) in enumerate([(32, 8, 128, 9000, 1), (16, 4, 64, 3000, 50)]):
        q, cache = make(n_q, n_kv, d, keys, keys, n_new, seed=20 + i)
        want = run(q, cache, n_kv, keys, keys, 1)
        p = apb.Decode4Problem(n_q, n_kv, d, keys, keys, n_new, 1)
        ws = torch.empty(apb.decode4_workspace_size(p), dtype=torch.uint8, device="cuda")
        o = torch.zeros(n_q, n_new, d, device="cuda")
        lse = torch.zeros(n_q, n_new, device="cuda")
        jobs.append((p, dev_bf16(q), cache, o, lse, ws, torch.cuda.Stream(), want))
    torch.cuda.synchronize()
    for _ in range(20):
        for p, q, cache, o, lse, ws, stream, _ in jobs:
            apb.decode4_attention(p, q, cache, o, lse, ws, stream=stream)
    torch.cuda.synchronize()
    for *_, o, lse, _, _, want in jobs:
        assert np.array_equal(o.cpu().numpy(), want[0].astype(np.float32))
        assert np.array_equal(lse.cpu().numpy(), want[1].astype(np.float32))


@pytest.mark.parametrize("shape", [(32, 8, 128, 3000, 1), (8, 2, 64, 1500, 40)])
def test_captured_step(shape):
    """Write, attend and read of a decoding step in a graph, replayed over other
    inputs with eager work between."""
    torch = need_gpu()
    from paper_2502_12085_amd import apb
    say(f"[decode4 graph] {shape}")
    n_q, n_kv, d, keys, n_new = shape
    q0, cache = make(n_q, n_kv, d, keys, keys, n_new, seed=40)
    q, k = dev_bf16(q0), dev_bf16(bf16_rows(n_kv, n_new, d, 1, wide=False))
    v, k_out = k.clone(), torch.zeros_like(k)
    v_out = torch.zeros_like(k)
    p = apb.Decode4Problem(n_q, n_kv, d, keys, keys, n_new, 1)
    rows = apb.Cache4Problem(n_kv, d, keys, keys - n_new, n_new, n_new, 0)
    ws = torch.empty(apb.decode4_workspace_size(p), dtype=torch.uint8, device="cuda")
    o = torch.zeros(n_q, n_new, d, device="cuda")
    lse = torch.zeros(n_q, n_new, device="cuda")

    def step():
        apb.cache4_write(rows, k, v, cache)
        apb.decode4_attention(p, q, cache, o, lse, ws)
        apb.cache4_read(rows, cache, k_out, v_out)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(4):
        q.copy_(dev_bf16(bf16_rows(n_q, n_new, d, 50 + seed, wide=False)))
        k.copy_(dev_bf16(bf16_rows(n_kv, n_new, d, 60 + seed, wide=False)))
        v.copy_(dev_bf16(bf16_rows(n_kv, n_new, d, 70 + seed, wide=False)))
        o.fill_(7)
        ws.fill_(seed)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (o, lse, k_out, v_out)]
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (o, lse, k_out, v_out)):
            assert torch.equal(a, b)


def test_two_graphs_share_a_workspace():
    """Two captured steps of other shapes over one workspace, replayed in turn: nothing of
    one is left for the other."""
    torch = need_gpu()
    from paper_2502_12085_amd import apb
    say("[decode4 two graphs]")
    jobs, ws = [], torch.empty(8 << 20, dtype=torch.uint8, device="cuda")
    for i, (n_q, n_kv, d, keys, n_new) in enumerate([(32, 8, 128, 6000, 1), (8, 2, 64, 2500, 30)]):
        q, cache = make(n_q, n_kv, d, keys, keys, n_new, seed=80 + i)
        want = run(q, cache, n_kv, keys, keys, 1)
        p = apb.Decode4Problem(n_q, n_kv, d, keys, keys, n_new, 1)
        assert 16 < apb.decode4_workspace_size(p) <= ws.numel()
        qd, o = dev_bf16(q), torch.zeros(n_q, n_new, d, device="cuda")
        lse = torch.zeros(n_q, n_new, device="cuda")
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            apb.decode4_attention(p, qd, cache, o, lse, ws)
        jobs.append((graph, qd, cache, o, lse, want))
    for turn in range(3):
        for graph, _, _, o, lse, want in jobs:
            o.fill_(turn)
            graph.replay()
            torch.cuda.synchronize()
            assert np.array_equal(o.cpu().numpy(), want[0].astype(np.float32))
            assert np.array_equal(lse.cpu().numpy(), want[1].astype(np.float32))


def test_a_decoding_step_over_three_hosts():
    """As they are used: each host writes its local block (out of K/V with the anchor
    rows before it), the last one its new tokens' rows after it, every host attends,
    and the partials are merged; against the fp64 attention over all the rows."""
    torch = need_gpu()
    from paper_2502_12085_amd import apb
    say("[decode4 hosts]")
    n_q, n_kv, d, anchor, n_new = 8, 2, 128, 37, 5
    blocks = [700, 513, 611]
    q = bf16_rows(n_q, n_new, d, 1, wide=False)
    qd = dev_bf16(q)
    parts_o = torch.empty(3, n_q, n_new, d, device="cuda")
    parts_lse = torch.empty(3, n_q, n_new, device="cuda")
    ks, vs = [], []
    for h, n in enumerate(blocks):
        last = h == 2
        k, v = (dev_bf16(bf16_rows(n_kv, anchor + n, d, 10 * h + s, wide=False)) for s in (1, 2))
        cap = n + 64
        cache = new_cache(n_kv, cap, d, fill=0xFF)
        apb.cache4_write(apb.Cache4Problem(n_kv, d, cap, 0, n, anchor + n, anchor), k, v, cache)
        if last:
            kn, vn = (dev_bf16(bf16_rows(n_kv, n_new, d, s, wide=False)) for s in (91, 92))
            apb.cache4_write(apb.Cache4Problem(n_kv, d, cap, n, n_new, n_new, 0), kn, vn, cache)
        keys = n + (n_new if last else 0)
        p = apb.Decode4Problem(n_q, n_kv, d, cap, keys, n_new, int(last))
        ws = torch.empty(apb.decode4_workspace_size(p), dtype=torch.uint8, device="cuda")
        apb.decode4_attention(p, qd, cache, parts_o[h], parts_lse[h], ws)
        hk, hv = held(cache, keys)
        ks.append(hk)
        vs.append(hv)
    o = torch.empty(n_q * n_new, d, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(n_q * n_new, device="cuda")
    apb.merge_partials(parts_o.view(3, n_q * n_new, d), parts_lse.view(3, -1), o, lse)
    torch.cuda.synchronize()
    ro, rl, pv, qk = oracle.decode4_ref(q, np.concatenate(ks, 1), np.concatenate(vs, 1), causal=1,
                                        bound=True)
    bo, bl = bounds(sum(blocks) + n_new, d, rl, pv, qk)
    got = host_bf16_to_f64(o).reshape(n_q, n_new, d)
    # the merge's own arithmetic, 2^-20, and its rounding to bf16
    assert np.all(np.abs(got - ro) <= bo + pv * 2.0 ** -20 + np.abs(ro) * 2.0 ** -8)
    assert np.all(np.abs(lse.cpu().numpy().reshape(n_q, n_new) - rl) <= bl + 2.0 ** -20)
