"""Performance cases of the paged-KV library's operators for drafted tokens and encoder states: attention of a
tree of drafted tokens over a cache, the append that rotates them at their positions in the tree, the step
that keeps the accepted ones, and attention to an encoder's states of another length.

``listed()`` / ``draw(rng)`` give cases, ``prepare(case, seed)`` the state a program has in hand before the
call, ``run(state)`` one pass, ``work(case)`` what it has to do, ``exact(case, seed)`` its outputs in 64
bits. With ``own`` false ``run`` is the plain form: elementary torch operations in fp32.

A tree of n drafted tokens follows the P cached ones: token i has a parent among those before it, or -1 for
the last cached token. It sees the cached tokens, its ancestors and itself, and its position is P plus its
depth (0 for a parent of -1). A 4-bit cache holds e2m1 values times powers of two: for K one for every 32
dims of a token and kv head, for V one for every token and kv head; with the largest magnitude a of such a
group the power is 2^(floor(log2 a) - 2), at least 2^-126, and values round to the nearest, ties to even.
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
        # The smallest verification: the two-conversation trace with a few guesses each. Launch latency.
        dict(name="tree tiny d64", kind="tree", hq=4, hkv=2, d=64, convs=2, lo=272, hi=368, new_lo=5, new_hi=7, fmt="bf16", mix=1),
        # One user's long conversation, a tree of sixteen guesses.
        dict(name="tree one 24k", kind="tree", hq=32, hkv=8, d=128, convs=1, lo=24571, hi=24571, new_lo=16, new_hi=16, fmt="bf16", mix=2),
        # A full decoder verifies a few guesses of every conversation: bound by the cache's bytes.
        dict(name="tree 64 8k-32k", kind="tree", hq=32, hkv=8, d=128, convs=64, lo=8192, hi=32768, new_lo=4, new_hi=11, fmt="bf16", mix=3),
        # Wider trees over a cache in 4 bits.
        dict(name="tree fp4 16 1k-9k", kind="tree", hq=16, hkv=8, d=128, convs=16, lo=1000, hi=9000, new_lo=17, new_hi=100, fmt="fp4", mix=4),
        # Very wide trees on long contexts: bound by the matrix cores.
        dict(name="tree wide 8k-40k", kind="tree", hq=32, hkv=8, d=128, convs=8, lo=8192, hi=40000, new_lo=130, new_hi=250, fmt="bf16", mix=5),
        # A decoder's single tokens look at short encoder states (a caption, a small image).
        dict(name="cross tiny d64", kind="cross", hq=4, hkv=2, d=64, convs=2, lo=50, hi=77, new_lo=1, new_hi=1, fmt="bf16", mix=6),
        # A batch of decoders with up to five hypotheses each, on some 1500 states (half a minute of sound).
        dict(name="cross decode 48", kind="cross", hq=16, hkv=8, d=128, convs=48, lo=700, hi=1500, new_lo=1, new_hi=5, fmt="bf16", mix=7),
        # Whole texts look at documents of other, ragged lengths.
        dict(name="cross texts", kind="cross", hq=32, hkv=8, d=128, convs=6, lo=600, hi=9000, new_lo=100, new_hi=3500, fmt="bf16", mix=8),
        # A draft enters a small pool: keys and queries turn at their positions in the tree.
        dict(name="append tree one", kind="append", hq=16, hkv=8, d=128, layers=4, convs=1, lo=300, hi=300, new_lo=26, new_hi=26, fmt="bf16",
             rotary=128, interleaved=False, mix=9),
        # Every conversation of a decoder gets one, all layers; half of the head turns, in pairs.
        dict(name="append tree 48", kind="append", hq=32, hkv=8, d=128, layers=32, convs=48, lo=20, hi=200, new_lo=20, new_hi=64, fmt="bf16",
             rotary=64, interleaved=True, mix=10),
        # A draft is appended and the accepted tokens of it stay: one conversation, a few layers.
        dict(name="keep one d64", kind="keep", hq=16, hkv=2, d=64, layers=4, convs=1, lo=300, hi=300, new_lo=26, new_hi=26, fmt="bf16", mix=11),
        # The same for a whole decoder, all layers.
        dict(name="keep 64", kind="keep", hq=32, hkv=8, d=128, layers=32, convs=64, lo=17, hi=200, new_lo=8, new_hi=32, fmt="bf16", mix=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, no larger than the listed ones of its kind."""
    kind = rng.choice(["tree", "tree", "tree", "cross", "cross", "append", "keep"])
    hq, hkv, d = rng.choice(SHAPES)
    case = dict(kind=kind, hq=hq, hkv=hkv, d=d, fmt=rng.choice(["bf16", "bf16", "fp4"]), mix=rng.randrange(1 << 30))
    if kind == "tree":
        hi = _log_int(rng, 30, 32768)
        convs = _log_int(rng, 1, 64)
        most = max(1, min(hi, int(5e11 / (4 * d * hq * convs * hi)), int(3e9 / (hq * convs * hi))))
        new_hi = min(_log_int(rng, 1, 250), most)
        case.update(convs=convs, lo=max(new_hi, hi // rng.choice([1, 3, 10])), hi=hi, new_lo=max(1, new_hi // rng.choice([1, 2, 8])), new_hi=new_hi)
    elif kind == "cross":
        hi = _log_int(rng, 1, 9000)
        convs = _log_int(rng, 1, 64)
        most = max(1, min(int(5e11 / (4 * d * hq * convs * hi)), int(2e9 / (hq * convs * hi)), 4 * 10 ** 7 // (convs * hq * d)))
        new_hi = min(_log_int(rng, 1, 3500), most)
        case.update(convs=convs, lo=max(1, hi // rng.choice([1, 3, 10])), hi=hi, new_lo=max(1, new_hi // rng.choice([1, 2, 8])), new_hi=new_hi)
    else:
        layers = rng.choice([1, 4, 32])
        convs = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, 200)
        new_hi = min(_log_int(rng, 1, 64), max(1, int(2.5e8 / (convs * layers * (hq + 2 * hkv) * d))))
        case.update(layers=layers, convs=convs, lo=max(1, hi // rng.choice([1, 10])), hi=hi, new_lo=max(1, new_hi // rng.choice([1, 3])), new_hi=new_hi)
        if kind == "append":   # (into 16-bit pages: values turned in fp32 and in fp64 round to different 4-bit neighbours now and then)
            case.update(fmt="bf16", rotary=rng.choice([r for r in (16, 32, 48, 64, 96, 128) if r <= d]), interleaved=rng.random() < 0.5)
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
    """Of each conversation: the tokens in its cache when the pass attends (tree, cross) or before it (append,
    keep), its drafted tokens or rows of queries, and (keep) how many of the drafted ones stay."""
    rng = random.Random(case["mix"])
    total = _spread(rng, case["convs"], case["lo"], case["hi"])
    new = _spread(rng, case["convs"], case["new_lo"], case["new_hi"])
    if case["kind"] == "tree":
        total = [max(t, n) for t, n in zip(total, new)]
    return total, new, [rng.randint(1, min(n, 8)) for n in new]


def _parents(case, seed):
    """The trees' parents, one list for each conversation: chains and branches, as a draft model makes them."""
    r = random.Random(seed * 104729 + case["mix"])
    return [[-1 if i == 0 or r.random() < 0.05 else i - 1 if r.random() < 0.3 else r.randrange(i) for i in range(n)] for n in _lens(case)[1]]


def _kept(case, seed):
    """Which of its drafted tokens each conversation keeps."""
    r = random.Random(seed * 15485863 + case["mix"])
    _, new, stay = _lens(case)
    return [sorted(r.sample(range(n), m)) for n, m in zip(new, stay)]


def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _normal(shape, key, scale=None):
    """bf16 normal values of a stream of their own; `scale`: one factor for each head (axis -2)."""
    g = torch.Generator(device=_device())
    g.manual_seed(key)
    x = torch.randn(shape, generator=g, device=_device(), dtype=torch.float32)
    return (x if scale is None else x * scale[:, None]).to(torch.bfloat16)


def _inputs(case, seed):
    """K, V of the cache and of the drafted tokens [layers][tokens][kv heads][d], and Q
    [layers][rows][query heads][d], conversations one after the other. Magnitudes differ by head, as in
    trained models: factors of 0.5 to 2."""
    total, new, _ = _lens(case)
    r = random.Random(seed * 7919 + 1)
    layers, key = case.get("layers", 1), (seed * 1000003) % (1 << 60)
    scales = [torch.tensor([r.uniform(0.5, 2.0) for _ in range(case["hkv"])], device=_device()) for _ in range(2)]
    cache = [_normal((layers, sum(total), case["hkv"], case["d"]), key + i, scales[i]) for i in (0, 1)]
    q = k = v = None
    if case["kind"] in ("append", "keep"):
        k, v = (_normal((layers, sum(new), case["hkv"], case["d"]), key + 2 + i, scales[i]) for i in (0, 1))
    if case["kind"] != "keep":
        q = _normal((layers, sum(new), case["hq"], case["d"]), key + 4)
    return cache, k, v, q


def _pages(n):
    return (n + 15) // 16


BASE = 500000.0   # of the rotations
BACK = 16         # cached tokens in front of the kept ones that a pass reads back with them


def _index(xs, dtype=torch.int64):
    return torch.tensor(xs, dtype=dtype, device=_device())


# ------------------------------------------------------------------------------------------------
# state and passes
# ------------------------------------------------------------------------------------------------
def prepare(case, seed):
    """The filled cache (of the library: a pool and its conversations; in plain form: the values, or packed
    codes and powers), the queries, drafted tokens and the trees."""
    cache, k, v, q = _inputs(case, seed)
    total, new, _ = _lens(case)
    state = dict(case=case, total=total, new=new, k=k, v=v, q=q)
    if case["kind"] in ("tree", "append"):
        state["parents"] = _parents(case, seed)
    if case["kind"] == "keep":
        state["kept"] = _kept(case, seed)
    if own:
        state.update(_own_state(case, seed, cache, total, new))
    elif case["kind"] in ("tree", "cross"):
        state["cache"] = _quantise(cache[0][0], case["d"] // 32) + _quantise(cache[1][0], 1) if case["fmt"] == "fp4" else [x[0] for x in cache]
    elif case["kind"] == "keep":
        state["cache"] = cache
    return state


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"tree": _own_tree, "cross": _own_cross, "append": _own_append, "keep": _own_keep}[kind](state)
    return {"tree": _plain_attend, "cross": _plain_attend, "append": _plain_append, "keep": _plain_keep}[kind](state)


# ---- the library's calls -------------------------------------------------------------------------
def _own_state(case, seed, cache, total, new):
    from paper_2606_01839_amd import KVPool, Rope
    more = new if case["kind"] in ("append", "keep") else [0] * len(new)
    pool = KVPool(case.get("layers", 1), case["hq"], case["hkv"], case["d"], n_pages=sum(_pages(t + n) for t, n in zip(total, more)) + 16,
                  max_convs=len(total) + 2, max_pages_per_conv=_pages(max(total) + max(more)) + 1, placement_seed=seed % 1000, kv_format=case["fmt"])
    convs = [pool.conv_create() for _ in total]
    pool.kv_append_batch(convs, total, *cache)
    out = dict(pool=pool, convs=convs)
    if case["kind"] == "append":
        out["rope"] = Rope(case["rotary"], base=BASE, interleaved=case["interleaved"])
    return out


def _own_tree(s):
    return s["pool"].attn_tree(s["convs"], s["new"], s["parents"], 0, s["q"][0])


def _own_cross(s):
    return s["pool"].attn_cross(s["convs"], s["new"], 0, s["q"][0])


def _own_append(s):
    """The drafts enter the cache, are read back, and are dropped again."""
    pool, convs, new = s["pool"], s["convs"], s["new"]
    q = pool.kv_append_tree(convs, new, s["parents"], s["k"], s["v"], s["rope"], q=s["q"])
    k, v = pool.kv_read(convs, s["total"], new)
    pool.kv_keep(convs, new, [[] for _ in convs])
    return {"k": k, "v": v, "q": q}


def _own_keep(s):
    """The drafts enter the cache, the accepted tokens stay and are read back with some tokens in front of
    them, and are dropped again."""
    pool, convs = s["pool"], s["convs"]
    pool.kv_append_batch(convs, s["new"], s["k"], s["v"])
    pool.kv_keep(convs, s["new"], s["kept"])
    stay = [len(x) for x in s["kept"]]
    back = [min(t, BACK) for t in s["total"]]
    k, v = pool.kv_read(convs, [t - b for t, b in zip(s["total"], back)], [b + m for b, m in zip(back, stay)])
    pool.kv_keep(convs, stay, [[] for _ in convs])
    return {"k": k, "v": v}


# ---- the plain forms -----------------------------------------------------------------------------
def _codes(x, groups):
    """e2m1 codes (0 to 15) of x [..][d] with one power of two for each of `groups` parts of d, and the
    powers' exponents + 127."""
    x = x.to(torch.float32).unflatten(-1, (groups, x.shape[-1] // groups))
    e = (torch.frexp(x.abs().amax(-1, keepdim=True)).exponent - 3).clamp(min=-126)
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
    """The plain form's 4-bit cache: two codes a byte, and the exponents."""
    c, e = _codes(x, groups)
    return [c[..., 0::2] + 16 * c[..., 1::2], e]


def _cached(cache, which, rows):
    """fp32 K (which = 0) or V (1) of the cache's rows."""
    if len(cache) == 2:
        return cache[which][rows].to(torch.float32)
    p, e = cache[2 * which][rows], cache[2 * which + 1][rows]
    return _values(torch.stack([p & 15, p >> 4], dim=-1).flatten(-2), e)


def _depths(parents):
    """Depth of every drafted token, one conversation after the other."""
    out = []
    for tree in parents:
        d = []
        for p in tree:
            d.append(0 if p < 0 else d[p] + 1)
        out += d
    return out


def _ancestors(parents, n):
    """[trees][n][n]: whether token j is token i or an ancestor of it; the first power of two of the tree's
    steps that reaches every depth."""
    up = _index([t + [-1] * (n - len(t)) for t in parents])
    see = torch.nn.functional.one_hot(up + 1, n + 1)[..., 1:].to(torch.float32) + torch.eye(n, device=up.device)
    for _ in range(max(1, n - 1).bit_length()):
        see = (torch.matmul(see, see) > 0).to(torch.float32)
    return see > 0


def _plain_attend(s):
    """All conversations at once, tokens and rows padded to the longest."""
    case, total, new = s["case"], _index(s["total"]), _index(s["new"])
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    b, n = len(s["new"]), max(s["new"])
    at, row = torch.arange(max(s["total"]), device=total.device), torch.arange(n, device=total.device)
    there = row < new[:, None]
    tokens = (total.cumsum(0) - total)[:, None] + torch.minimum(at, total[:, None] - 1)
    rows = (new.cumsum(0) - new)[:, None] + torch.minimum(row, new[:, None] - 1)
    q = s["q"][0][rows].to(torch.float32).view(b, n, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, -1, d)
    score = torch.matmul(q, _cached(s["cache"], 0, tokens).permute(0, 2, 3, 1).contiguous()).view(b, hkv, hq // hkv, n, -1)
    score /= math.sqrt(d)
    hidden = (at >= total[:, None])[:, None].expand(b, n, -1)
    if case["kind"] == "tree":
        # token `at` as the draft's token j, where it is one
        j = at - (total - new)[:, None]
        drafted = torch.gather(_ancestors(s["parents"], n), 2, j.clamp(0, n - 1)[:, None].expand(b, n, -1))
        hidden = hidden | ((j >= 0)[:, None] & ~drafted)
    score.masked_fill_(hidden[:, None, None], -math.inf)
    score -= score.amax(-1, keepdim=True)
    score.exp_()
    score /= score.sum(-1, keepdim=True)
    o = torch.matmul(score.flatten(2, 3), _cached(s["cache"], 1, tokens).transpose(1, 2).contiguous())
    return o.view(b, hkv, hq // hkv, n, d).permute(0, 3, 1, 2, 4).reshape(b, n, hq, d)[there].to(torch.bfloat16)


def _positions(case, parents):
    """Position of every drafted token."""
    total, new, _ = _lens(case)
    return torch.repeat_interleave(_index(total), _index(new)) + _index(_depths(parents))


def _rotate(x, pos, r, interleaved):
    """Rotated fp32 values of x [..][row][head][d]: pairs of the first r dims turn by position x frequency."""
    f = BASE ** (-2 * torch.arange(r // 2, dtype=torch.float64, device=x.device) / r)
    angle = pos.to(torch.float64)[:, None] * f
    c, s = (t.to(torch.float32)[:, None, :] for t in (torch.cos(angle), torch.sin(angle)))
    x = x.to(torch.float32)
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    a, b = a * c - b * s, a * s + b * c
    turned = torch.stack([a, b], dim=-1).flatten(-2) if interleaved else torch.cat([a, b], dim=-1)
    return torch.cat([turned, x[..., r:]], dim=-1)


def _stored(case, k, v):
    """K and V as they come back from the cache."""
    if case["fmt"] == "fp4":
        k, v = _values(*_codes(k, case["d"] // 32)), _values(*_codes(v, 1))
    return {"k": k.to(torch.bfloat16), "v": v.to(torch.bfloat16)}


def _plain_append(s):
    case = s["case"]
    turn = _positions(case, s["parents"]), case["rotary"], case["interleaved"]
    return {**_stored(case, _rotate(s["k"], *turn), s["v"]), "q": _rotate(s["q"], *turn).to(torch.bfloat16)}


def _window(s):
    """Rows of (cache, drafted tokens) that a pass gives back, the drafted ones behind all of the cache."""
    rows, t0, n0, behind = [], 0, 0, sum(s["total"])
    for t, n, kept in zip(s["total"], s["new"], s["kept"]):
        rows += list(range(t0 + t - min(t, BACK), t0 + t)) + [behind + n0 + i for i in kept]
        t0, n0 = t0 + t, n0 + n
    return _index(rows)


def _plain_keep(s):
    rows, held = _window(s), s["cache"][0].shape[1]
    from_cache = (rows < held)[:, None, None]
    k, v = (torch.where(from_cache, c[:, rows.clamp(max=held - 1)], x[:, (rows - held).clamp(min=0)]) for c, x in zip(s["cache"], (s["k"], s["v"])))
    return _stored(s["case"], k, v)


# ------------------------------------------------------------------------------------------------
# what a pass has to do and to give
# ------------------------------------------------------------------------------------------------
def work(case):
    total, new, stay = _lens(case)
    hq, hkv, d, layers, kind = case["hq"], case["hkv"], case["d"], case.get("layers", 1), case["kind"]
    kv, q = 4 * hkv * d, 2 * hq * d            # bytes of a token's K and V, of a query row, in 16 bits; one layer
    held = hkv * (d + d // 32 + 1) if case["fmt"] == "fp4" else kv
    if kind == "append":                       # read, stored in the cache, given back from it; queries read and written
        return {"bytes": layers * sum(new) * (2 * kv + 2 * held + 2 * q), "flops": 3 * layers * sum(new) * (hq + hkv) * case["rotary"]}
    if kind == "keep":                         # the drafts stored; the kept ones moved; those and the tokens in front given back
        back = sum(min(t, BACK) for t in total)
        return {"bytes": layers * (sum(new) * (kv + held) + 2 * sum(stay) * held + (back + sum(stay)) * (kv + held)), "flops": 0}
    pairs = sum(n * t if kind == "cross" else n * (t - n) + n for t, n in zip(total, new))   # (a tree's ancestors aside)
    return {"bytes": sum(total) * held + 2 * sum(new) * q, "flops": 4 * d * hq * pairs}


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


def _exact_rotate(x, pos, r, interleaved):
    """Pairs of dims as complex numbers, turned by e^(i position frequency)."""
    f = BASE ** (-2 * torch.arange(r // 2, dtype=torch.float64, device=x.device) / r)
    x = x.double().clone()
    even, odd = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    angle = pos.double()[:, None] * f
    z = torch.complex(x[..., even], x[..., odd]) * torch.polar(torch.ones_like(angle), angle)[:, None, :]
    x[..., even], x[..., odd] = z.real, z.imag
    return x


def _exact_sees(tree, length):
    """[n][length]: the tokens that each drafted token sees, found by climbing the tree."""
    n = len(tree)
    see = torch.zeros((n, length), dtype=torch.bool)
    see[:, :length - n] = True
    for i in range(n):
        j = i
        while j >= 0:
            see[i, length - n + j] = True
            j = tree[j]
    return see.to(_device())


def exact(case, seed):
    cache, k, v, q = _inputs(case, seed)
    total, new, _ = _lens(case)
    kind, d, hq, hkv = case["kind"], case["d"], case["hq"], case["hkv"]
    if kind in ("append", "keep"):
        if kind == "append":
            turn = _positions(case, _parents(case, seed)), case["rotary"], case["interleaved"]
            out = {"k": _exact_rotate(k, *turn), "v": v.double(), "q": _exact_rotate(q, *turn)}
        else:
            held = [list(zip(c.double().split(total, 1), x.double().split(new, 1), _kept(case, seed))) for c, x in zip(cache, (k, v))]
            out = {n: torch.cat([torch.cat([c[:, -BACK:], x[:, kept]], 1) for c, x, kept in h], 1) for n, h in zip("kv", held)}
        if case["fmt"] == "fp4":
            out["k"], out["v"] = _exact_held(out["k"], d // 32), _exact_held(out["v"], 1)
        return out
    trees = _parents(case, seed) if kind == "tree" else [None] * len(new)
    outs = []
    for kc, vc, qc, tree in zip(cache[0][0].split(total), cache[1][0].split(total), q[0].split(new), trees):
        if case["fmt"] == "fp4":
            kc, vc = _exact_held(kc, d // 32), _exact_held(vc, 1)
        see = None if tree is None else _exact_sees(tree, kc.shape[0])
        o = torch.empty((qc.shape[0], hq, d), dtype=torch.float64, device=qc.device)
        for h in range(hq):
            s = torch.matmul(qc[:, h].double(), kc[:, h // (hq // hkv)].double().t()) / math.sqrt(d)
            if see is not None:
                s = torch.where(see, s, -math.inf)
            o[:, h] = torch.matmul(torch.softmax(s, 1), vc[:, h // (hq // hkv)].double())
        outs.append(o)
    return torch.cat(outs)
