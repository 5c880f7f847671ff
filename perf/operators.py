"""Performance cases of the key/value cache held in 4 bits: writing it, reading
it back, and decoding-stage attention over it, each through its public entry
point (``paper_2502_12085_amd.apb``) where ``own`` is true, and in plain torch
operations where it is not.

The cache holds K and V of a host in groups of 32 elements along the head size:
an element is sign, two bits of exponent and one of mantissa (magnitudes 0, 0.5,
1, 1.5, 2, 3, 4, 6), two to a byte, the even element in the low half; a group has
one byte b that scales it by 2^(b - 127), and b = 255 makes it NaN.  A group with
largest magnitude a is written with the smallest e for which a <= 7 * 2^e, held
to -120 .. 125, b = e + 127, and elements x * 2^-e rounded to the nearest, ties
to the even code, magnitudes past 6 to 6.

A case is a plain dict whose ``"path"`` is one of

- ``store``   ``cache4_write`` of some rows, read back by ``cache4_read``: the
  values that the cache then holds;
- ``load``    ``cache4_read`` of some rows of a written cache;
- ``attend``  ``decode4_attention`` of the new tokens over a written cache;
- ``step``    all three as a decoding step has them: the new tokens' rows are
  written, attended with the rest of the cache, and read back (for a host that
  keeps them in bf16 too).
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"

# Query heads, KV heads and head size of the models that the workloads are shaped
# like (Llama-3.1-8B, Qwen-2.5-14B, Yi-34B), and two small ones with d = 64.
GEOMETRIES = ((32, 8, 128), (40, 8, 128), (56, 8, 128), (8, 2, 64), (4, 1, 64))
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _heads(g):
    return dict(n_q=g[0], n_kv=g[1], d=g[2])


LLAMA, QWEN, YI = _heads(GEOMETRIES[0]), _heads(GEOMETRIES[1]), _heads(GEOMETRIES[2])
SMALL, TINY = _heads(GEOMETRIES[3]), _heads(GEOMETRIES[4])


# ------------------------------------------------------------------- cases
def listed():
    return [
        # One generated token's K and V into a small cache, at an odd row: the
        # smallest call, launches and the host path.
        dict(name="store_token", path="store", **TINY, capacity=1021, first=515, rows=1,
             src_rows=1, src_first=0),
        # The local block of the 128K share, out of the layer's own K/V (its
        # anchor rows before it), into a cache with room for 4096 tokens more.
        dict(name="store_128k", path="store", **LLAMA, capacity=20480, first=0, rows=16384,
             src_rows=20480, src_first=4096),
        # The local block of a 1024K document over 8 hosts.
        dict(name="store_1024k", path="store", **LLAMA, capacity=131072, first=0, rows=131072,
             src_rows=131072, src_first=0),
        # A ragged piece of a 32K share's cache, to be sent on in bf16.
        dict(name="load_32k_ragged", path="load", **SMALL, capacity=8192, first=1001, rows=2777,
             src_rows=2777, src_first=0),
        # The whole cache of a 256K share back in bf16.
        dict(name="load_256k", path="load", **QWEN, capacity=33000, first=0, rows=32768,
             src_rows=32768, src_first=0),
        # A three-token step of the tiny shape: latency.
        dict(name="attend_tiny", path="attend", **TINY, capacity=1021, cache=515, new=3,
             causal=True),
        # Every generated token after a 128K prefill over 8 hosts, last host.
        dict(name="attend_128k_token", path="attend", **LLAMA, capacity=20480, cache=16385,
             new=1, causal=True),
        # The first decoding step of the same document: 64 question tokens.
        dict(name="attend_128k_question", path="attend", **LLAMA, capacity=20480, cache=16448,
             new=64, causal=True),
        # A short question over an uneven split of a 256K document, on a host
        # that is not the last.
        dict(name="attend_256k_ragged", path="attend", **QWEN, capacity=30001, cache=30001,
             new=17, causal=False),
        # A generated token over a 512K document that one GPU holds whole, which
        # 4 bits make room for.
        dict(name="attend_512k_token", path="attend", **YI, capacity=524800, cache=524289,
             new=1, causal=True),
        # A generated token of the last host of a 1024K document, from its new
        # row to the attention.
        dict(name="step_1024k", path="step", **LLAMA, capacity=135168, cache=131073, new=1,
             causal=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    path = rng.choice(("store", "load", "attend", "attend", "attend", "step"))
    g = _heads(rng.choice(GEOMETRIES))
    if path in ("store", "load"):
        rows = _log_int(rng, 1, 131072)
        first = rng.choice((0, rng.randint(0, 5000)))
        src_first = rng.choice((0, rng.randint(0, 4096)))
        return dict(path=path, **g, capacity=first + rows + rng.randint(0, 4096), first=first,
                    rows=rows, src_rows=src_first + rows + rng.randint(0, 64),
                    src_first=src_first)
    new = 1 if rng.random() < 0.5 else _log_int(rng, 2, 256)
    cache = new + _log_int(rng, 1, 524288)
    return dict(path=path, **g, capacity=cache + rng.randint(0, 4096), cache=cache, new=new,
                causal=path == "step" or rng.random() < 0.5)


def draw(rng):
    """One more case of the same ranges, no costlier than the largest listed."""
    most_bytes = max(work(c)["bytes"] for c in listed())
    most_flops = max(work(c)["flops"] for c in listed())
    while True:
        c = _draw_once(rng)
        w = work(c)
        if w["bytes"] <= most_bytes and w["flops"] <= most_flops:
            return c


def work(case):
    """Bytes and operations that one pass cannot do without: every bf16 row, code
    and scale that a call takes or gives once, and 4 d operations for each query
    row and visible key."""
    d, n_kv = case["d"], case["n_kv"]
    packed = d // 2 + d // 32  # bytes of a row in the cache
    if case["path"] in ("store", "load"):
        moves = 2 if case["path"] == "store" else 1
        return {"bytes": moves * 2 * n_kv * case["rows"] * (2 * d + packed), "flops": 0}
    n_q, new, keys = case["n_q"], case["new"], case["cache"]
    pairs = new * keys - (new * (new - 1) // 2 if case["causal"] else 0)
    moved = n_q * new * (2 * d + 4 * d + 4) + 2 * n_kv * keys * packed
    if case["path"] == "step":
        moved += 2 * 2 * n_kv * new * (2 * d + packed)
    return {"bytes": moved, "flops": 4 * d * n_q * pairs}


# ------------------------------------------------------------------- inputs
def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32)


def _rows(case, gen, rows):
    """K and V rows in bf16 as a layer leaves them: N(0, 1), and in K 2% of the
    channels of each head 8 times that."""
    n_kv, d = case["n_kv"], case["d"]
    k, v = _normal(gen, n_kv, rows, d), _normal(gen, n_kv, rows, d)
    pick = torch.rand(n_kv, d, generator=gen, device=DEV).argsort(1)[:, :math.ceil(0.02 * d)]
    wide = torch.ones(n_kv, d, device=DEV).scatter_(1, pick, 8.0)
    return (k * wide[:, None]).bfloat16(), v.bfloat16()


def _cache_like(case):
    n_kv, cap, d = case["n_kv"], case["capacity"], case["d"]
    new = lambda n: torch.zeros(n_kv, cap, n, dtype=torch.uint8, device=DEV)  # noqa: E731
    return dict(k_codes=new(d // 2), k_scales=new(d // 32),
                v_codes=new(d // 2), v_scales=new(d // 32))


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    st = dict(case=case, cache=_cache_like(case))
    n_q, n_kv, d = case["n_q"], case["n_kv"], case["d"]
    if case["path"] in ("store", "load"):
        k, v = _rows(case, gen, case["src_rows"])
        if case["path"] == "load":
            cut = slice(case["src_first"], case["src_first"] + case["rows"])
            _write(st["cache"], case["first"], k[:, cut], v[:, cut])
        st.update(k=k, v=v)
        rows = case["rows"]
    else:
        k, v = _rows(case, gen, case["cache"])
        new = case["new"] if case["path"] == "step" else 0
        done = case["cache"] - new
        _write(st["cache"], 0, k[:, :done], v[:, :done])
        st["q"] = _normal(gen, n_q, case["new"], d).bfloat16()
        if new:
            st.update(k=k[:, done:].contiguous(), v=v[:, done:].contiguous())
        rows = new
    # what the framework's calls write to
    st["k_out"] = torch.empty(n_kv, rows, d, dtype=torch.bfloat16, device=DEV)
    st["v_out"] = torch.empty_like(st["k_out"])
    if "q" in st:
        st["o"] = torch.empty(n_q, case["new"], d, dtype=torch.float32, device=DEV)
        st["lse"] = torch.empty(n_q, case["new"], dtype=torch.float32, device=DEV)
        if own:
            from paper_2502_12085_amd import apb
            st["p"] = apb.Decode4Problem(n_q, n_kv, d, case["capacity"], case["cache"],
                                         case["new"], int(case["causal"]))
            st["ws"] = torch.empty(apb.decode4_workspace_size(st["p"]), dtype=torch.uint8,
                                   device=DEV)
    return st


# --------------------------------------------------------------- plain forms
def _pow2(e):
    """2^e in float32, from its bits (-126 <= e <= 127)."""
    return ((e + 127) << 23).view(torch.float32)


def _quantise(x):
    """Codes 0 .. 15 [.., d] and scale bytes [.., d / 32] of bf16 rows."""
    g = x.float().unflatten(-1, (-1, 32))
    top = g.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)
    e = torch.where(top == 0, -120, e - 3 + (m > 0.875).int()).clamp(-120, 125).int()
    bad = ~torch.isfinite(g).all(-1, keepdim=True)
    y = (g * _pow2(-e)).abs()
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5)
            + (y >= 3.5) + (y > 5.0))
    code = torch.where(bad, 0, code + 8 * torch.signbit(g).to(torch.uint8))
    scale = torch.where(bad, 255, e + 127)
    return code.flatten(-2).to(torch.uint8), scale.squeeze(-1).to(torch.uint8)


def _values(code, scale):
    """What codes and scale bytes stand for, in float32."""
    level = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device=code.device)
    by = torch.where(scale == 255, math.nan, (scale.int() << 23).view(torch.float32))
    return (level[code.int()].unflatten(-1, (-1, 32)) * by[..., None]).flatten(-2)


def _unpack(codes):
    return torch.stack((codes & 15, codes >> 4), -1).flatten(-2)


def _write(cache, first, k, v):
    at = slice(first, first + k.shape[1])
    for x, codes, scales in ((k, "k_codes", "k_scales"), (v, "v_codes", "v_scales")):
        code, scale = _quantise(x)
        cache[codes][:, at] = code[..., 0::2] | (code[..., 1::2] << 4)
        cache[scales][:, at] = scale


def _read(cache, first, rows):
    at = slice(first, first + rows)
    return (_values(_unpack(cache["k_codes"][:, at]), cache["k_scales"][:, at]),
            _values(_unpack(cache["v_codes"][:, at]), cache["v_scales"][:, at]))


def _attend(case, q, k, v):
    n_q, n_kv, d, new, keys = (case[x] for x in ("n_q", "n_kv", "d", "new", "cache"))
    s = q.float().reshape(n_kv, -1, d) @ k.transpose(1, 2) * d ** -0.5
    if case["causal"]:
        last = torch.arange(keys - new, keys, device=DEV).repeat(n_q // n_kv)
        s.masked_fill_(torch.arange(keys, device=DEV) > last[:, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - m)
    total = p.sum(-1, keepdim=True)
    o = p @ v / total
    return o.view(n_q, new, d), (m + total.log()).view(n_q, new)


def _plain(st):
    case, cache = st["case"], st["cache"]
    if case["path"] == "store":
        cut = slice(case["src_first"], case["src_first"] + case["rows"])
        _write(cache, case["first"], st["k"][:, cut], st["v"][:, cut])
    if case["path"] in ("store", "load"):
        k, v = _read(cache, case["first"], case["rows"])
        return {"k": k.bfloat16(), "v": v.bfloat16()}
    new, keys = case["new"], case["cache"]
    if case["path"] == "step":
        _write(cache, keys - new, st["k"], st["v"])
    k, v = _read(cache, 0, keys)
    o, lse = _attend(case, st["q"], k, v)
    out = {"o": o, "lse": lse}
    if case["path"] == "step":
        out.update(k=k[:, keys - new:].bfloat16(), v=v[:, keys - new:].bfloat16())
    return out


# ---------------------------------------------------------- the framework's
def _rows_problem(case, rows, first, src_rows, src_first):
    from paper_2502_12085_amd import apb
    return apb.Cache4Problem(case["n_kv"], case["d"], case["capacity"], first, rows, src_rows,
                             src_first)


def _own(st):
    from paper_2502_12085_amd import apb
    case, cache = st["case"], st["cache"]
    out = {}
    if case["path"] in ("store", "load"):
        first, rows = case["first"], case["rows"]
    else:
        first, rows = case["cache"] - case["new"], case["new"]
    if case["path"] == "store":
        apb.cache4_write(_rows_problem(case, rows, first, case["src_rows"], case["src_first"]),
                         st["k"], st["v"], cache)
    if case["path"] == "step":
        apb.cache4_write(_rows_problem(case, rows, first, rows, 0), st["k"], st["v"], cache)
    if case["path"] in ("attend", "step"):
        apb.decode4_attention(st["p"], st["q"], cache, st["o"], st["lse"], st["ws"])
        out.update(o=st["o"], lse=st["lse"])
    if case["path"] != "attend":
        apb.cache4_read(_rows_problem(case, rows, first, rows, 0), cache, st["k_out"],
                        st["v_out"])
        out.update(k=st["k_out"], v=st["v_out"])
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------- exact
def _held(x):
    """What the cache holds of bf16 rows, in 64 bits: the nearest level of each
    element by its distance to all eight."""
    g = x.double().unflatten(-1, (-1, 32))
    top = g.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top / 7)).clamp(-120, 125)
    by = torch.pow(torch.tensor(2.0, dtype=torch.float64, device=x.device), e)
    y = g.abs() / by
    best, held = torch.full_like(y, math.inf), torch.zeros_like(y)
    for code in (0, 2, 4, 6, 1, 3, 5, 7):  # an even code keeps a tie
        far = (y - LEVELS[code]).abs()
        held = torch.where(far < best, LEVELS[code], held)
        best = torch.minimum(best, far)
    return (held * by * torch.sign(g)).flatten(-2)


def exact(case, seed):
    st = prepare(case, seed)
    n_q, n_kv, d = case["n_q"], case["n_kv"], case["d"]
    gen = torch.Generator(device=DEV).manual_seed(seed)
    if case["path"] in ("store", "load"):
        cut = slice(case["src_first"], case["src_first"] + case["rows"])
        return {x: torch.cat([_held(st[x][h:h + 1, cut]) for h in range(n_kv)]) for x in "kv"}
    k, v = _rows(case, gen, case["cache"])
    new, keys = case["new"], case["cache"]
    g, o, lse, tail = n_q // n_kv, [], [], {"k": [], "v": []}
    for h in range(n_kv):
        kh, vh = _held(k[h]), _held(v[h])
        tail["k"].append(kh[keys - new:])
        tail["v"].append(vh[keys - new:])
        for i in range(h * g, (h + 1) * g):
            s = torch.mv(kh, st["q"][i, 0].double())[None] if new == 1 else \
                st["q"][i].double() @ kh.T.contiguous()
            s = s / math.sqrt(d)
            if case["causal"]:
                s = s + torch.full((new, keys), -math.inf, device=DEV,
                                   dtype=torch.float64).triu(keys - new + 1)
            lse.append(torch.logsumexp(s, -1))
            o.append(torch.exp(s - lse[-1][:, None]) @ vh)
    out = {"o": torch.stack(o), "lse": torch.stack(lse)}
    if case["path"] == "step":
        out.update(k=torch.stack(tail["k"]), v=torch.stack(tail["v"]))
    return out
