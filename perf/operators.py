"""Performance cases of two groups of operators of the paged-KV attention library: rotary positions
(queries rotated at their positions, keys rotated on their way into the cache) and a KV cache held in
4 bits (append, one-time transfer, batched decode, extend and prefill attention over it).

``listed()`` / ``draw(rng)`` give cases, ``prepare(case, seed)`` the state a program has in hand
before the call, ``run(state)`` one pass, ``work(case)`` what it has to do, ``exact(case, seed)`` its
outputs in 64 bits. With ``own`` false ``run`` is the plain form: elementary torch operations in fp32.

The 4-bit cache holds e2m1 values (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) times powers of
two: for K one for every 32 dims of a token and kv head, for V one for every token and kv head. With
the largest magnitude a of such a group the power is 2^(floor(log2 a) - 2), at least 2^-126; values
round to the nearest, ties to the even code, and at most to 6.
"""
from __future__ import annotations

import math
import random

import torch

own = False

# (query heads, kv heads, head dim)
SHAPES = [(32, 8, 128), (16, 8, 128), (64, 8, 128), (8, 8, 128), (32, 8, 64), (16, 2, 64), (4, 2, 64)]


def listed():
    return [
        # The smallest: the two-conversation trace decodes, and its queries are rotated. Launch latency.
        dict(name="rope q tiny d64", kind="rope_q", hq=4, hkv=2, d=64, layers=1, convs=2, lo=272, hi=368, new_lo=1, new_hi=1,
             rotary=64, interleaved=False, scaling="none", mix=1),
        # A layer's queries of several long prompts; half of the head turns, in pairs, scaled for long contexts.
        dict(name="rope q prompts", kind="rope_q", hq=32, hkv=8, d=128, layers=1, convs=3, lo=3000, hi=20000, new_lo=3000, new_hi=20000,
             rotary=64, interleaved=True, scaling="parts", mix=2),
        # First prompts enter a prefiller of 16-bit pages: keys and queries of all layers are rotated.
        dict(name="rope append prompts", kind="append", hq=32, hkv=8, d=128, layers=32, convs=3, lo=700, hi=4000,
             fmt="bf16", rotary=128, interleaved=False, scaling="none", mix=3),
        # Short replies enter a small pool of 4-bit pages: a few tokens each.
        dict(name="fp4 append replies d64", kind="append", hq=16, hkv=2, d=64, layers=4, convs=5, lo=1, hi=60,
             fmt="fp4", rotary=0, interleaved=False, scaling="none", mix=4),
        # Whole prompts enter a decoder of 4-bit pages, all layers.
        dict(name="fp4 append prompts", kind="append", hq=32, hkv=8, d=128, layers=32, convs=3, lo=900, hi=9000,
             fmt="fp4", rotary=0, interleaved=False, scaling="none", mix=5),
        # The one-time transfer from a prefiller of 16-bit pages to a decoder of 4-bit pages.
        dict(name="fp4 transfer", kind="transfer", hq=32, hkv=8, d=128, layers=32, convs=3, lo=900, hi=9000, mix=6),
        # Decode over 4-bit pages: the smallest batch, one user's long conversation, a full decoder.
        dict(name="fp4 decode tiny d64", kind="decode", hq=4, hkv=2, d=64, convs=2, lo=272, hi=368, noalloc=False, mix=7),
        dict(name="fp4 decode one 24k", kind="decode", hq=32, hkv=8, d=128, convs=1, lo=24571, hi=24571, noalloc=True, mix=8),
        dict(name="fp4 decode 64 8k-32k", kind="decode", hq=32, hkv=8, d=128, convs=64, lo=8192, hi=32768, noalloc=False, mix=9),
        # A tool's reply against a long cached context; several replies in one launch.
        dict(name="fp4 extend one reply", kind="extend", hq=32, hkv=8, d=128, convs=1, lo=41000, hi=41000, new_lo=301, new_hi=301, mix=10),
        dict(name="fp4 extend 8 batch", kind="extend", hq=32, hkv=8, d=128, convs=8, lo=8192, hi=40000, new_lo=128, new_hi=2048, mix=11),
        # First prompts of ragged lengths: rotated, appended in 4 bits and attended, a layer at a time.
        dict(name="fp4 rope prefill d64", kind="prefill", hq=32, hkv=8, d=64, layers=2, convs=6, lo=300, hi=5000,
             rotary=64, interleaved=False, scaling="linear", mix=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_rope(rng, d):
    return dict(rotary=rng.choice([r for r in (16, 32, 48, 64, 96, 128) if r <= d]), interleaved=rng.random() < 0.5,
                scaling=rng.choice(["none", "linear", "ntk", "parts"]))


def draw(rng):
    """One more case of the same ranges, no larger than the listed ones of its kind."""
    kind = rng.choice(["rope_q", "append", "append", "transfer", "decode", "decode", "extend", "prefill"])
    hq, hkv, d = rng.choice(SHAPES)
    case = dict(kind=kind, hq=hq, hkv=hkv, d=d, mix=rng.randrange(1 << 30))
    if kind == "rope_q":
        hi = _log_int(rng, 20, 100000)
        convs = _log_int(rng, 1, 64)
        new_hi = min(_log_int(rng, 1, 20000), hi, max(1, 4 * 10 ** 7 // (convs * hq * d)))
        case.update(layers=rng.choice([1, 1, 2]), convs=convs, lo=max(1, hi // rng.choice([1, 3])), hi=hi, new_lo=max(1, new_hi // rng.choice([1, 8])),
                    new_hi=new_hi, **_draw_rope(rng, d))
    elif kind == "append":
        hi = _log_int(rng, 10, 8000)
        fmt = rng.choice(["bf16", "fp4"])
        rope = _draw_rope(rng, d) if fmt == "bf16" else dict(rotary=0, interleaved=False, scaling="none")
        layers = rng.choice([1, 8, 32])
        hi = min(hi, 5 * 10 ** 8 // (layers * (hq + 2 * hkv) * d))
        convs = max(1, min(rng.randint(1, 12), 5 * 10 ** 8 // (hi * layers * (hq + 2 * hkv) * d)))
        case.update(layers=layers, convs=convs, lo=max(1, hi // rng.choice([1, 10])), hi=hi, fmt=fmt, **rope)
    elif kind == "transfer":
        hi = _log_int(rng, 50, 9000)
        case.update(layers=rng.choice([1, 8, 32]), convs=rng.randint(1, 3), lo=max(1, hi // rng.choice([1, 10])), hi=hi)
    elif kind == "decode":
        hi = _log_int(rng, 200, 32768)
        convs = _log_int(rng, 1, 64)
        case.update(convs=convs, lo=max(1, hi // rng.choice([1, 3, 10])), hi=hi, noalloc=convs <= 8 and rng.random() < 0.3)
    elif kind == "extend":
        hi = _log_int(rng, 100, 40000)
        convs = _log_int(rng, 1, 8)
        new_hi = max(1, min(_log_int(rng, 2, 2048), int(3e12 / (4 * d * hq * convs * (hi + 2048)))))
        case.update(convs=convs, lo=max(1, hi // rng.choice([1, 3])), hi=hi, new_lo=max(1, new_hi // rng.choice([1, 2, 8])), new_hi=new_hi)
    else:
        convs = _log_int(rng, 1, 6)
        hi = min(_log_int(rng, 60, 8000), int(math.sqrt(1e12 / (2 * d * hq * convs))))
        case.update(layers=rng.choice([1, 2]), convs=convs, lo=max(1, hi // rng.choice([1, 4, 10])), hi=hi, **_draw_rope(rng, d))
    return case


# ------------------------------------------------------------------------------------------------
# sizes and inputs
# ------------------------------------------------------------------------------------------------
def _spread(rng, n, lo, hi):
    """n lengths over [lo, hi], evenly in the logarithm with a jitter, in random order."""
    if n == 1:
        return [hi]
    a, b = math.log(lo), math.log(hi)
    xs = [int(round(math.exp(a + (b - a) * min(1.0, (i + rng.random()) / n)))) for i in range(n)]
    rng.shuffle(xs)
    return [min(hi, max(lo, x)) for x in xs]


def _lens(case):
    """(tokens of each conversation when its queries attend, its query tokens)."""
    rng = random.Random(case["mix"])
    n = case["convs"]
    total = _spread(rng, n, case["lo"], case["hi"])
    if case["kind"] == "decode":
        return total, [1] * n
    if case["kind"] == "rope_q":
        return total, [min(t, x) for t, x in zip(total, _spread(rng, n, case["new_lo"], case["new_hi"]))]
    if case["kind"] == "extend":
        new = _spread(rng, n, case["new_lo"], case["new_hi"])
        return [t + x for t, x in zip(total, new)], new
    return total, list(total)


def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _normal(shape, key, scale=None):
    """bf16 normal values of a stream of their own; `scale`: one factor for each head (axis -2)."""
    g = torch.Generator(device=_device())
    g.manual_seed(key)
    x = torch.randn(shape, generator=g, device=_device(), dtype=torch.float32)
    return (x if scale is None else x * scale[:, None]).to(torch.bfloat16)


def _inputs(case, seed):
    """K, V [layers][tokens][kv heads][d] and Q [layers][rows][query heads][d], conversations one after
    the other. K and V magnitudes differ by head, as in trained models: factors of 0.5 to 2."""
    total, new = _lens(case)
    r = random.Random(seed * 7919 + 1)
    layers, key = case.get("layers", 1), (seed * 1000003) % (1 << 60)
    scales = [torch.tensor([r.uniform(0.5, 2.0) for _ in range(case["hkv"])], device=_device()) for _ in range(2)]
    kind = case["kind"]
    k = v = q = None
    if kind != "rope_q":
        k, v = (_normal((layers, sum(total), case["hkv"], case["d"]), key + i, scales[i]) for i in (0, 1))
    if kind not in ("append", "transfer") or case.get("rotary"):
        q = _normal((layers, sum(new), case["hq"], case["d"]), key + 2)
    return k, v, q


def _pages(n):
    return (n + 15) // 16


BASE, FACTOR, ORIGINAL = 500000.0, 4.0, 8192.0   # of the rotations


def _frequencies(case):
    """Radians per position of each pair of dims, and the factor on what is rotated."""
    r = case["rotary"]
    i = torch.arange(r // 2, dtype=torch.float64, device=_device())
    if case["scaling"] == "ntk":
        return (BASE * FACTOR ** (r / (r - 2.0))) ** (-2 * i / r), 1.0
    f = BASE ** (-2 * i / r)
    if case["scaling"] == "linear":
        return f / FACTOR, 1.0
    if case["scaling"] == "parts":
        # pairs that turn less than once over the original context are slowed down, those that turn over 32
        # times are not
        keep = ((ORIGINAL * f / (2 * math.pi) - 1) / 31).clamp(0, 1)
        return f * (keep + (1 - keep) / FACTOR), 0.1 * math.log(FACTOR) + 1
    return f, 1.0


def _positions(case):
    """Position of every query row."""
    total, new = _lens(case)
    return torch.cat([torch.arange(t - n, t, device=_device()) for t, n in zip(total, new)])


# ------------------------------------------------------------------------------------------------
# state and passes
# ------------------------------------------------------------------------------------------------
def prepare(case, seed):
    """Attention over a cache: the filled cache (of the library: a pool and its conversations; in plain
    form: packed codes and scales) and the queries. Else: the new keys, values and queries, and the
    library's pools."""
    k, v, q = _inputs(case, seed)
    total, new = _lens(case)
    kind = case["kind"]
    state = dict(case=case, total=total, new=new, q=q)
    if kind in ("rope_q", "append", "prefill") and case["rotary"]:
        state["freq"] = _frequencies(case)
    if kind in ("append", "prefill", "transfer"):
        state.update(k=k, v=v)
    if own:
        state.update(_own_state(case, seed, k, v, total))
    elif kind in ("decode", "extend"):
        state["cache"] = _quantise(k[0], case["d"] // 32) + _quantise(v[0], 1)
    return state


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"rope_q": _own_rope_q, "append": _own_append, "transfer": _own_transfer, "decode": _own_decode,
                "extend": _own_extend, "prefill": _own_prefill}[kind](state)
    return {"rope_q": _plain_rope_q, "append": _plain_append, "transfer": _plain_transfer, "decode": _plain_decode,
            "extend": _plain_extend, "prefill": _plain_prefill}[kind](state)


# ---- the library's calls -------------------------------------------------------------------------
def _own_pool(case, total, fmt, placement):
    from paper_2606_01839_amd import KVPool
    return KVPool(case.get("layers", 1), case["hq"], case["hkv"], case["d"], n_pages=sum(_pages(t) for t in total) + 16,
                  max_convs=len(total) + 2, max_pages_per_conv=_pages(max(total)) + 1, placement_seed=placement, kv_format=fmt)


def _own_state(case, seed, k, v, total):
    from paper_2606_01839_amd import Rope
    kind = case["kind"]
    fmt = case.get("fmt", "fp4")
    out = {}
    if case.get("rotary"):
        out["rope"] = Rope(case["rotary"], base=BASE, interleaved=case["interleaved"], scaling=case["scaling"], factor=FACTOR,
                           original_len=ORIGINAL)
    if kind == "transfer":
        src, dst = _own_pool(case, total, "bf16", 1 + seed % 1000), _own_pool(case, total, "fp4", 2 + seed % 1000)
        convs = [src.conv_create() for _ in total]
        src.kv_append_batch(convs, total, k, v)
        return dict(src=src, pool=dst, convs=convs, wires=[torch.empty(src.kv_pack_fp4_size(c), dtype=torch.uint8, device=_device())
                                                           for c in convs])
    out["pool"] = pool = _own_pool(case, total, fmt, seed % 1000)
    if kind in ("append", "prefill"):
        return out
    out["convs"] = [pool.conv_create() for _ in total]
    if kind == "rope_q":     # only the conversations' lengths matter here
        z = torch.zeros((case.get("layers", 1), sum(total), case["hkv"], case["d"]), dtype=torch.bfloat16, device=_device())
        pool.kv_append_batch(out["convs"], total, z, z)
    else:
        pool.kv_append_batch(out["convs"], total, k, v)
    if case.get("noalloc"):
        out["out"] = torch.empty((len(total), case["hq"], case["d"]), dtype=torch.bfloat16, device=_device())
    return out


def _own_rope_q(s):
    return s["pool"].rope_q(s["convs"], s["new"], s["q"], s["rope"])


def _own_append(s):
    """The prompts' conversations begin, their tokens are appended and read back, and they end."""
    pool, lens = s["pool"], s["total"]
    convs = [pool.conv_create() for _ in lens]
    if s["case"]["rotary"]:
        q = pool.kv_append_rope(convs, lens, s["k"], s["v"], s["rope"], q=s["q"])
    else:
        q = None
        pool.kv_append_batch(convs, lens, s["k"], s["v"])
    k, v = pool.kv_read(convs, [0] * len(lens), lens)
    for c in convs:
        pool.conv_destroy(c)
    return {"k": k, "v": v, "q": q}


def _own_transfer(s):
    src, pool, lens = s["src"], s["pool"], s["total"]
    convs = []
    for c, n, wire in zip(s["convs"], lens, s["wires"]):
        src.kv_pack_fp4(c, wire)
        convs.append(pool.kv_unpack(wire, n))
    k, v = pool.kv_read(convs, [0] * len(lens), lens)
    for c in convs:
        pool.conv_destroy(c)
    return {"k": k, "v": v}


def _own_decode(s):
    if s["case"]["noalloc"]:
        return s["pool"].attn_decode_batch_noalloc(s["convs"], 0, s["q"][0], s["out"])
    return s["pool"].attn_decode_batch(s["convs"], 0, s["q"][0])


def _own_extend(s):
    return s["pool"].attn_extend(s["convs"], s["new"], 0, s["q"][0])


def _own_prefill(s):
    pool, lens = s["pool"], s["total"]
    convs = [pool.conv_create() for _ in lens]
    q = pool.kv_append_rope(convs, lens, s["k"], s["v"], s["rope"], q=s["q"])
    out = [pool.attn_prefill_turn1(convs, lens, layer, q[layer]) for layer in range(s["case"]["layers"])]
    for c in convs:
        pool.conv_destroy(c)
    return out


# ---- the plain forms -----------------------------------------------------------------------------
def _rotate(x, pos, freq, interleaved):
    """Rotated fp32 values of x [..][row][head][d]: pairs of the first 2 len(frequencies) dims turn by
    position x frequency; the others stay."""
    f, amplitude = freq
    r = 2 * f.numel()
    angle = pos.to(torch.float64)[:, None] * f
    c, s = ((amplitude * t).to(torch.float32)[:, None, :] for t in (torch.cos(angle), torch.sin(angle)))
    x = x.to(torch.float32)
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    a, b = a * c - b * s, a * s + b * c
    turned = torch.stack([a, b], dim=-1).flatten(-2) if interleaved else torch.cat([a, b], dim=-1)
    return torch.cat([turned, x[..., r:]], dim=-1)


def _codes(x, groups):
    """e2m1 codes (0 to 15) of x [..][d] with one power of two for each of `groups` parts of d, and the
    powers' exponents + 127."""
    x = x.to(torch.float32).unflatten(-1, (groups, x.shape[-1] // groups))
    e = torch.frexp(x.abs().amax(-1, keepdim=True)).exponent - 3
    e = e.clamp(min=-126)
    y = torch.ldexp(x.abs(), -e)
    c = (y > 0.25).to(torch.uint8)
    c += y >= 0.75
    c += y > 1.25
    c += y >= 1.75
    c += y > 2.5
    c += y >= 3.5
    c += y > 5
    c += 8 * (x < 0)
    return c.flatten(-2), (e.squeeze(-1) + 127).to(torch.uint8)


def _values(codes, exponents):
    """fp32 values of codes [..][d] with exponents [..][groups]."""
    lut = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    x = lut[codes.to(torch.int32)].unflatten(-1, (exponents.shape[-1], -1))
    return torch.ldexp(x, exponents.to(torch.int32).unsqueeze(-1) - 127).flatten(-2)


def _quantise(x, groups):
    """The plain form's cache: two codes a byte, and the exponents."""
    c, e = _codes(x, groups)
    return c[..., 0::2] + 16 * c[..., 1::2], e


def _cached(packed, exponents, rows):
    """fp32 values of the cache's rows."""
    p = packed[rows]
    return _values(torch.stack([p & 15, p >> 4], dim=-1).flatten(-2), exponents[rows])


def _plain_rope_q(s):
    return _rotate(s["q"], _positions(s["case"]), s["freq"], s["case"]["interleaved"]).to(torch.bfloat16)


def _stored(case, s):
    """K and V as the cache holds them, in fp32, and the rotated queries."""
    k, v, q = s["k"], s["v"], s["q"]
    if case["kind"] != "transfer" and case["rotary"]:
        pos = _positions(case)
        k, q = (_rotate(x, pos, s["freq"], case["interleaved"]) for x in (k, q))
        q = q.to(torch.bfloat16)
    if case.get("fmt", "fp4") == "fp4":
        return _values(*_codes(k, case["d"] // 32)), _values(*_codes(v, 1)), q
    return k, v, q


def _plain_append(s):
    k, v, q = _stored(s["case"], s)
    return {"k": k.to(torch.bfloat16), "v": v.to(torch.bfloat16), "q": q}


def _plain_transfer(s):
    k, v, _ = _stored(s["case"], s)
    return {"k": k.to(torch.bfloat16), "v": v.to(torch.bfloat16)}


def _plain_decode(s):
    """All conversations at once, padded to the longest."""
    case, dev = s["case"], s["q"].device
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    lens = torch.tensor(s["total"], device=dev)
    at = torch.arange(max(s["total"]), device=dev)
    rows = (lens.cumsum(0) - lens)[:, None] + torch.minimum(at, lens[:, None] - 1)
    kc, ke, vc, ve = s["cache"]
    q = s["q"][0].to(torch.float32).view(-1, hkv, hq // hkv, d)
    score = torch.matmul(q, _cached(kc, ke, rows).permute(0, 2, 3, 1)) / math.sqrt(d)
    score = score.masked_fill((at >= lens[:, None])[:, None, None], -math.inf)
    w = torch.exp(score - score.amax(-1, keepdim=True))
    w /= w.sum(-1, keepdim=True)
    return torch.matmul(w, _cached(vc, ve, rows).transpose(1, 2)).reshape(-1, hq, d).to(torch.bfloat16)


def _attend(q, k, v):
    """Causal attention of the last rows: q [n][hq][d], k, v [L][hkv][d] in fp32."""
    n, hq, d = q.shape
    length, hkv = k.shape[:2]
    q = q.to(torch.float32).view(n, hkv, hq // hkv, d).permute(1, 2, 0, 3).reshape(hkv, -1, d)
    score = torch.matmul(q, k.permute(1, 2, 0)).view(hkv, hq // hkv, n, length)
    score /= math.sqrt(d)
    at = torch.arange(length, device=q.device)
    score.masked_fill_(at > at[length - n:, None], -math.inf)
    score -= score.amax(-1, keepdim=True)
    score.exp_()
    score /= score.sum(-1, keepdim=True)
    o = torch.matmul(score.view(hkv, -1, length), v.transpose(0, 1))
    return o.view(hkv, hq // hkv, n, d).permute(2, 0, 1, 3).reshape(n, hq, d).to(torch.bfloat16)


def _plain_extend(s):
    """A conversation at a time: their scores are of different shapes."""
    kc, ke, vc, ve = s["cache"]
    out, t0, r0 = [], 0, 0
    for t, n in zip(s["total"], s["new"]):
        rows = slice(t0, t0 + t)
        out.append(_attend(s["q"][0, r0:r0 + n], _cached(kc, ke, rows), _cached(vc, ve, rows)))
        t0, r0 = t0 + t, r0 + n
    return torch.cat(out)


def _plain_prefill(s):
    k, v, q = _stored(s["case"], s)
    split = [list(zip(*(x[layer].split(s["total"]) for x in (q, k, v)))) for layer in range(s["case"]["layers"])]
    return [torch.cat([_attend(*x) for x in convs]) for convs in split]


# ------------------------------------------------------------------------------------------------
# what a pass has to do and to give
# ------------------------------------------------------------------------------------------------
def work(case):
    total, new = _lens(case)
    hq, hkv, d, layers, kind = case["hq"], case["hkv"], case["d"], case.get("layers", 1), case["kind"]
    kv, q = 4 * hkv * d, 2 * hq * d            # bytes of a token's K and V, of a query row, in 16 bits; one layer
    small = hkv * (d + d // 32 + 1)            # a token's K and V in 4 bits, and their exponents
    if kind == "rope_q":
        return {"bytes": 2 * layers * sum(new) * q, "flops": 3 * layers * sum(new) * hq * case["rotary"]}
    if kind == "append":                       # read, stored in the cache, given back from it
        held = small if case["fmt"] == "fp4" else kv
        turned = q if case["rotary"] else 0
        return {"bytes": layers * sum(total) * (2 * kv + 2 * held + 2 * turned), "flops": 3 * layers * sum(total) * (hq + hkv) * case["rotary"]}
    if kind == "transfer":                     # the 16-bit pages read, the wire and the 4-bit pages written and read, given back
        return {"bytes": layers * sum(total) * (2 * kv + 4 * small), "flops": 0}
    pairs = sum(n * (t - n) + n * (n + 1) // 2 for t, n in zip(total, new))
    bytes_ = layers * (sum(total) * small + 2 * sum(new) * q)
    if kind == "prefill":
        bytes_ += layers * sum(total) * (kv + q + small)
    return {"bytes": bytes_, "flops": 4 * d * hq * pairs * layers}


def _exact_rotate(x, pos, freq, interleaved):
    """Pairs of dims as complex numbers, turned by e^(i position frequency)."""
    f, amplitude = freq
    r = 2 * f.numel()
    x = x.double().clone()
    even, odd = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    turn = torch.polar(torch.full((pos.numel(), f.numel()), amplitude, dtype=torch.float64, device=x.device),
                       pos.double()[:, None] * f)
    z = torch.complex(x[..., even], x[..., odd]) * turn[:, None, :]
    x[..., even], x[..., odd] = z.real, z.imag
    return x


def _exact_held(x, groups):
    """The values a 4-bit cache holds of x, by the nearest entry of the table of e2m1 values."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    y = x.double().reshape(*x.shape[:-1], groups, -1)
    top = y.abs().max(-1, keepdim=True).values
    step = torch.exp2(torch.log2(top.clamp(min=2.0 ** -120)).floor() - 2)
    # log2 rounds: its floor may be one too high just below a power of two
    step = torch.where(step * 4 > top, step / 2, step).clamp(min=2.0 ** -126)
    y = y / step
    lower = (torch.bucketize(y.abs(), table, right=True) - 1).clamp(max=6)
    a, b = table[lower], table[lower + 1]
    up = (y.abs() - a > b - y.abs()) | ((y.abs() - a == b - y.abs()) & (lower % 2 == 1))
    return (torch.where(up, b, a) * torch.sign(y) * step).reshape(x.shape)


def _exact_attend(q, k, v):
    n, hq, d = q.shape
    length, hkv = k.shape[0], k.shape[1]
    out = torch.empty((n, hq, d), dtype=torch.float64, device=q.device)
    for h in range(hq):
        kh, vh = k[:, h // (hq // hkv)].t().contiguous(), v[:, h // (hq // hkv)]
        for r0 in range(0, n, 2048):
            r1 = min(n, r0 + 2048)
            seen = length - n + r1
            s = torch.matmul(q[r0:r1, h], kh[:, :seen]) / math.sqrt(d)
            s.masked_fill_(torch.arange(seen, device=q.device) > torch.arange(length - n + r0, seen, device=q.device)[:, None], -math.inf)
            out[r0:r1, h] = torch.matmul(torch.softmax(s, dim=1), vh[:seen])
    return out


def exact(case, seed):
    k, v, q = _inputs(case, seed)
    total, new = _lens(case)
    kind, d, layers = case["kind"], case["d"], case.get("layers", 1)
    if kind in ("append", "transfer") and layers * sum(total) * case["hkv"] * d > 1 << 30:
        return None
    if case.get("rotary"):
        turn = [_positions(case), _frequencies(case), case["interleaved"]]
        k, q = (None if x is None else _exact_rotate(x, *turn) for x in (k, q))
    if kind == "rope_q":
        return q
    if case.get("fmt", "fp4") == "fp4":
        k, v = _exact_held(k, d // 32), _exact_held(v, 1)
    if kind in ("append", "transfer"):
        out = {"k": k.double(), "v": v.double()}
        return out if kind == "transfer" else {**out, "q": q}
    if case.get("rotary"):
        q = q.to(torch.bfloat16)               # the rotated queries are a 16-bit tensor
    out = []
    for layer in range(layers):
        t0 = r0 = 0
        rows = []
        for t, n in zip(total, new):
            rows.append(_exact_attend(q[layer, r0:r0 + n].double(), k[layer, t0:t0 + t], v[layer, t0:t0 + t]))
            t0, r0 = t0 + t, r0 + n
        out.append(torch.cat(rows))
    return out if kind == "prefill" else out[0]
