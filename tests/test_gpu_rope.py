"""GPU: rotary positions against the float64 oracle. The bound of a rotated value: half a bf16 step,
2^-8 of it; and before that rounding the error of fp32 arithmetic on a cos and sin that are within 2^-22
(v_sin_f32, v_cos_f32 on an angle exact to 2^-34 turns): 2^-21 of amplitude (|a| + |b|), which
covers four roundings of 2^-24 each and the two functions'."""
import numpy as np
import pytest
import torch

from oracle import fp4 as o4
from oracle import rope as orope
from oracle.attention import attend_last
from tests.helpers import assert_close, f64, kv_tokens, q_tokens

pytestmark = pytest.mark.gpu

SEED = 707
BASE = 500000.0


def _pool(nl, hq, hkv, d, n_pages, fmt="bf16", max_pages=512, max_convs=8):
    from paper_2606_01839_amd import KVPool
    return KVPool(nl, hq, hkv, d, n_pages=n_pages, max_convs=max_convs, max_pages_per_conv=max_pages, placement_seed=3,
                  device="cuda", kv_format=fmt)


def _turn(x, pos, rope):
    return orope.rotate(f64(x), pos, rope.inv_freq, rope.amplitude, rope.interleaved)


def _assert_turned(got, x, pos, rope, what=""):
    want = _turn(x, pos, rope)
    size = np.abs(_partner_sum(f64(x), rope)) * abs(rope.amplitude)
    tol = 2.0 ** -8 * np.maximum(np.abs(want), np.abs(f64(got))) + 2.0 ** -21 * size
    r = rope.rotary_dim
    tol[..., r:] = 0
    err = np.abs(f64(got) - want)
    worst = np.unravel_index(np.argmax(err - tol), err.shape)
    assert (err <= tol).all(), f"{what} at {worst}: {f64(got)[worst]} {want[worst]}"


def _partner_sum(x, rope):
    """|a| + |b| of each dim's pair"""
    a = np.abs(x)
    r = rope.rotary_dim
    out = a.copy()
    if rope.interleaved:
        s = a[..., 0:r:2] + a[..., 1:r:2]
        out[..., 0:r:2] = out[..., 1:r:2] = s
    else:
        s = a[..., :r // 2] + a[..., r // 2:r]
        out[..., :r // 2] = out[..., r // 2:r] = s
    return out


ROPES = [(64, 64, False, "none"), (64, 16, True, "none"), (64, 48, False, "linear"), (128, 128, False, "none"),
         (128, 128, True, "parts"), (128, 64, False, "ntk"), (128, 96, True, "none"), (128, 16, False, "parts")]


def _rope(r, inter, scaling):
    from paper_2606_01839_amd import Rope
    return Rope(r, base=BASE, interleaved=inter, scaling=scaling, factor=8.0, original_len=8192)


@pytest.mark.parametrize("d,r,inter,scaling", ROPES)
def test_queries(d, r, inter, scaling):
    """Ragged batches, in place and not, one layer and several; rows beside them stay as they were."""
    hq, hkv = 24, 3      # (24 query heads: two groups of the kernel, the second not full)
    rope = _rope(r, inter, scaling)
    pool = _pool(1, hq, hkv, d, 400, max_pages=400)
    lens, q_lens = [1, 40, 333, 17, 3000], [1, 40, 70, 0, 1]
    convs = [pool.conv_create() for _ in lens]
    z = torch.zeros(1, sum(lens), hkv, d, dtype=torch.bfloat16, device="cuda")
    pool.kv_append_batch(convs, lens, z, z)
    rows = sum(q_lens)
    pos = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, q_lens)])
    for layers in (None, 1, 3):
        shape = (rows, hq, d) if layers is None else (layers, rows, hq, d)
        q = torch.randn(shape, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
        buf = torch.full((q.numel() + 2 * hq * d,), 7.0, dtype=torch.bfloat16, device="cuda")
        mine = buf[hq * d:-hq * d].view(shape)
        qc = q.cuda()
        out = pool.rope_q(convs, q_lens, qc, rope, out=mine)
        torch.cuda.synchronize()
        assert torch.equal(qc.cpu(), q) and (buf[:hq * d] == 7).all() and (buf[-hq * d:] == 7).all()
        _assert_turned(out.cpu(), q, pos, rope)
        assert torch.equal(out, pool.rope_q(convs, q_lens, qc, rope))
        assert torch.equal(pool.rope_q(convs, q_lens, qc, rope, out=qc), out) and torch.equal(qc, out)
    empty = pool.rope_q(convs, [0] * 5, torch.zeros(0, hq, d, dtype=torch.bfloat16, device="cuda"), rope)
    assert empty.shape == (0, hq, d)
    assert pool.rope_q([], [], empty, rope).shape == (0, hq, d)
    pool.close()


def test_far_positions():
    """A million tokens on: the angles are exact, where fp32 products would be off by 0.06 radians."""
    from paper_2606_01839_amd import Rope
    n, d, hq = 1_000_003, 64, 2
    pool = _pool(1, hq, 1, d, (n + 15) // 16 + 2, fmt="fp4", max_pages=(n + 15) // 16 + 1)
    c = pool.conv_create()
    z = torch.zeros(1, n, 1, d, dtype=torch.bfloat16, device="cuda")
    pool.kv_append(c, z, z)
    q = q_tokens(SEED, 0, 0, 0, 50, hq, d)
    for rope in (Rope(64), Rope(64, base=1e6, interleaved=True)):
        out = pool.rope_q([c], [50], q.cuda(), rope)
        torch.cuda.synchronize()
        _assert_turned(out.cpu(), q, np.arange(n - 50, n), rope)
    # frequencies of the caller's own, negative and over a turn a token
    rope = Rope(16)
    rope.inv_freq = [-0.3, 7.0, 1e-7, 3.0, -12.5, 0.0, 2.5, 1.0]
    out = pool.rope_q([c], [50], q.cuda(), rope)
    torch.cuda.synchronize()
    # (the double product of the oracle is itself off by 1e-16 x 1.25e7 radians)
    _assert_turned(out.cpu(), q, np.arange(n - 50, n), rope)
    pool.close()


@pytest.mark.parametrize("d,r,inter,scaling", ROPES)
@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_appends(d, r, inter, scaling, fmt):
    """Ragged appends, page by page and token by token, with their queries; V stays as it is."""
    nl, hq, hkv = 2, 6, 3
    rope = _rope(r, inter, scaling)
    pool = _pool(nl, hq, hkv, d, 64, fmt)
    pool.kv.fill_(0xFF)
    a, b = pool.conv_create(), pool.conv_create()
    pos = {a: 0, b: 0}
    ks, vs = {a: [], b: []}, {a: [], b: []}
    for na, nb in [(1, 0), (15, 3), (16, 40), (17, 1), (1, 1), (100, 33)]:
        kv = [kv_tokens(SEED, c, nl, pos[c], n, hkv, d) for c, n in ((a, na), (b, nb))]
        k, v = (torch.cat([x[j] for x in kv], 1) for j in (0, 1))
        q = torch.stack([torch.cat([q_tokens(SEED, c, l, pos[c], n, hq, d) for c, n in ((a, na), (b, nb))]) for l in range(nl)])
        qc = q.cuda()
        out = pool.kv_append_rope([a, b], [na, nb], k.cuda(), v.cuda(), rope, q=qc)
        at = np.r_[pos[a]:pos[a] + na, pos[b]:pos[b] + nb]
        torch.cuda.synchronize()
        assert torch.equal(qc.cpu(), q)
        _assert_turned(out.cpu(), q, at, rope, "q")
        for c, n, x in ((a, na, kv[0]), (b, nb, kv[1])):
            ks[c].append(x[0])
            vs[c].append(x[1])
            pos[c] += n
            assert pool.conv_len(c) == pos[c]
        # the same rotation as rope_q's, bit for bit
        assert torch.equal(out, pool.rope_q([a, b], [na, nb], qc, rope))
    for c in (a, b):
        k, v = torch.cat(ks[c], 1), torch.cat(vs[c], 1)
        gk, gv = pool.kv_read([c], [0], [pos[c]])
        torch.cuda.synchronize()
        at = np.arange(pos[c])
        if fmt == "bf16":
            _assert_turned(gk.cpu(), k, at, rope, "k")
            assert torch.equal(gv.cpu(), v)
        else:
            want = _turn(k, at, rope)
            assert np.array_equal(f64(gv.cpu()), o4.held(f64(v), f64(v))[1])
            # K: the code of the turned value or, within the fp32 error of a border between two, its neighbour
            eps = 2.0 ** -21 * _partner_sum(f64(k), rope) * rope.amplitude
            below, above = _held_range(want, eps)
            got = f64(gk.cpu())
            assert ((got >= below) & (got <= above)).all()
            assert (got == o4.held(want, want)[0]).mean() > 0.999
    pool.close()


def _held_range(x, eps):
    """Bounds of what the cache may hold of x within eps: the group's power may change where its largest
    value is within eps of a power of two."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    e = eps.reshape(g.shape)
    top, slack = np.abs(g).max(-1, keepdims=True), e.max(-1, keepdims=True)
    lo, hi = [], []
    for t in (top - slack, top + slack):
        step = 2.0 ** np.maximum(np.frexp(np.maximum(t, 2.0 ** -120))[1] - 3.0, -126)
        for y in (g - e, g + e):
            m = np.abs(y) / step
            dist = np.abs(m[..., None] - o4.VALUES)
            c = np.arange(8)
            near = np.where(dist == dist.min(-1, keepdims=True), c + 8 * (c % 2), 99).min(-1) % 8
            v = np.sign(y) * o4.VALUES[near] * step
            lo.append(v)
            hi.append(v)
    return np.min(lo, 0).reshape(x.shape), np.max(hi, 0).reshape(x.shape)


def test_append_in_place_and_without_queries():
    rope = _rope(64, False, "none")
    k, v = kv_tokens(SEED, 0, 1, 0, 50, 2, 64)
    q = q_tokens(SEED, 0, 0, 0, 50, 8, 64)[None]
    outs = []
    for mode in range(3):
        pool = _pool(1, 8, 2, 64, 16)
        c = pool.conv_create()
        qc = q.cuda()
        out = pool.kv_append_rope([c], [50], k.cuda(), v.cuda(), rope, **({} if mode == 0 else dict(q=qc, q_out=qc if mode == 1 else None)))
        assert (out is None) == (mode == 0) and (mode != 1 or out is qc)
        outs.append((pool.kv_read([c], [0], [50])[0], out))
        torch.cuda.synchronize()
        pool.close()
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[1][0], outs[2][0]) and torch.equal(outs[1][1], outs[2][1])


def test_large_appends_are_uploaded_in_parts():
    """More page chunks than an upload of the ring holds, and than a launch's own arguments."""
    from paper_2606_01839_amd import Rope
    rope, n = Rope(64, interleaved=True), 16 * 66000 + 3
    pool = _pool(1, 1, 1, 64, 66010, fmt="fp4", max_pages=66005)
    c = pool.conv_create()
    g = torch.Generator(device="cuda").manual_seed(2)
    k, v, q = (torch.randn((1, n, 1, 64), generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    out = pool.kv_append_rope([c], [n], k, v, rope, q=q)
    at = np.r_[0:40, 524250:524300, n - 40:n]
    torch.cuda.synchronize()
    _assert_turned(out[:, at].cpu(), q[:, at].cpu(), at, rope)
    assert torch.equal(out[0], pool.rope_q([c], [n], q[0], rope))
    pool.close()


@pytest.mark.parametrize("n,nl", [(7, 2), (64, 20)])
def test_single_tokens_of_many_conversations(n, nl):
    """One token each, its queries in the append's launch (few) or in one of their own (many): the bits of rope_q, in
    place too, and the oracle's."""
    rope = _rope(48, True, "linear")
    pool = _pool(nl, 32, 4, 64, 600, max_convs=n)
    lens = [3 * i for i in range(n)]
    convs = [pool.conv_create() for _ in range(n)]
    k, v = (x.cuda() for x in kv_tokens(SEED, 0, nl, 0, sum(lens) + 2 * n, 4, 64))
    pool.kv_append_rope(convs, lens, k[:, :sum(lens)].contiguous(), v[:, :sum(lens)].contiguous(), rope)
    for step in range(2):
        at = slice(sum(lens) + step * n, sum(lens) + (step + 1) * n)
        x = torch.stack([q_tokens(SEED + step, 0, l, 0, n, 32, 64) for l in range(nl)])
        q = x.cuda()
        out = pool.kv_append_rope(convs, [1] * n, k[:, at].contiguous(), v[:, at].contiguous(), rope, q=q, q_out=q if step else None)
        again = pool.rope_q(convs, [1] * n, x.cuda(), rope)
        gk, gv = pool.kv_read(convs, [m + step for m in lens], [1] * n)
        torch.cuda.synchronize()
        assert torch.equal(out, again) and torch.equal(gv, v[:, at])
        _assert_turned(out.cpu(), x, np.array(lens) + step, rope)
        _assert_turned(gk.cpu(), k[:, at].cpu(), np.array(lens) + step, rope)
    pool.close()


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("hq,hkv,d,r", [(32, 8, 128, 128), (4, 2, 64, 32)])
def test_a_served_conversation(fmt, hq, hkv, d, r):
    """All of it together, as a program uses it: a prompt enters a prefiller with rotated keys and is
    attended, its cache moves to the decoder, a tool's reply is appended there, then single tokens."""
    nl = 2
    rope = _rope(r, False, "none")
    pre, dec = _pool(nl, hq, hkv, d, 64), _pool(nl, hq, hkv, d, 64, fmt)
    n, total = 210, 210 + 33 + 4
    k, v = kv_tokens(SEED, 0, nl, 0, total, hkv, d)
    q = torch.stack([q_tokens(SEED, 0, l, 0, total, hq, d) for l in range(nl)])
    cut = lambda x, i, j: x[:, i:j].contiguous().cuda()
    held = [_turn(k, np.arange(total), rope), f64(v)]
    c = pre.conv_create()
    qr = pre.kv_append_rope([c], [n], cut(k, 0, n), cut(v, 0, n), rope, q=cut(q, 0, n))
    k16 = torch.from_numpy(held[0]).to(torch.bfloat16)
    for l in range(nl):
        out = pre.attn_prefill_turn1([c], [n], l, qr[l])
        torch.cuda.synchronize()
        # tolerance of the attention alone on queries and keys that may differ by a bf16 rounding: the scores move by
        # 2^-8 of them (rel-L2 2 x 3e-3 and as much again in the largest)
        ref = attend_last(f64(qr[l].cpu()), f64(k16[l, :n]), f64(v[l, :n]))
        got = f64(out.cpu())
        assert np.sqrt(((got - ref) ** 2).sum() / (ref ** 2).sum()) <= 6e-3 and np.abs(got - ref).max() <= 3e-2
    wire = pre.kv_pack_fp4(c) if fmt == "fp4" else pre.kv_pack(c)
    c = dec.kv_unpack(wire, n)
    pos = n
    for m in (33, 1, 1, 1, 1):
        qr = dec.kv_append_rope([c], [m], cut(k, pos, pos + m), cut(v, pos, pos + m), rope, q=cut(q, pos, pos + m))
        pos += m
        gk, gv = dec.kv_read([c], [0], [pos])
        torch.cuda.synchronize()
        for l in range(nl):
            out = dec.attn_extend([c], [m], l, qr[l]) if m > 1 else dec.attn_decode_batch([c], l, qr[l])
            torch.cuda.synchronize()
            # on exactly what the cache holds and the queries that were given
            assert_close(out, attend_last(f64(qr[l].cpu()), f64(gk[l].cpu()), f64(gv[l].cpu())), f"{pos} layer {l}")
    # and the cache holds the rotated keys, as bf16 or 4 bits hold them
    err = np.linalg.norm(f64(gk.cpu()) - held[0]) / np.linalg.norm(held[0])
    assert err <= (2.0 ** -8 if fmt == "bf16" else 0.25), err   # 4 bits: half of the largest step, 2 of 8
    pre.close()
    dec.close()


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("hq,hkv,d,r,inter", [(32, 8, 128, 128, False), (4, 2, 64, 32, True), (8, 8, 128, 64, False)])
@pytest.mark.parametrize("ordered", [False, True])
def test_mixed_step(fmt, hq, hkv, d, r, inter, ordered):
    """A step with rotated keys and queries, its outputs apart from its queries or in their place: the same bits as
    an append of rotated keys and queries and the separate calls on a second pool."""
    nl = 2
    rope = _rope(r, inter, "none")
    lens, new = [300, 1, 1500, 64, 900, 9], [40, 1, 1, 130, 1, 17]
    ext, dec = [0, 3, 5], [1, 2, 4]
    kv = [kv_tokens(SEED, i, nl, 0, n + m, hkv, d) for i, (n, m) in enumerate(zip(lens, new))]
    cat = lambda idx, j, new_part: torch.cat([kv[i][j][:, lens[i]:] if new_part else kv[i][j][:, :lens[i]] for i in idx], 1).contiguous().cuda()
    q = [torch.stack([q_tokens(SEED, i, l, lens[i], new[i], hq, d) for l in range(nl)]) for i in range(6)]
    qe, qd = (torch.cat([q[i] for i in g], 1).contiguous().cuda() for g in (ext, dec))
    outs = []
    for mode in range(3):
        pool = _pool(nl, hq, hkv, d, 400, fmt)
        convs = [pool.conv_create() for _ in lens]
        pool.kv_append_rope(convs, lens, cat(range(6), 0, False), cat(range(6), 1, False), rope)
        k, v = cat(ext + dec, 0, True), cat(ext + dec, 1, True)
        e, x = [convs[i] for i in ext], [convs[i] for i in dec]
        if mode < 2:
            a, b = qe.clone(), qd.clone()
            oe, od = pool.mixed_step(e, [new[i] for i in ext], x, k, v, a, b, layer_ordered=ordered, rope=rope,
                                     **(dict(out_ext=a, out_dec=b) if mode else {}))
            torch.cuda.synchronize()
            assert mode or (torch.equal(a, qe) and torch.equal(b, qd))
        else:
            qr = pool.kv_append_rope(e + x, [new[i] for i in ext + dec], k, v, rope, q=torch.cat([qe, qd], 1).contiguous())
            ne = qe.shape[1]
            oe = torch.stack([pool.attn_extend(e, [new[i] for i in ext], l, qr[l, :ne].contiguous()) for l in range(nl)])
            od = torch.stack([pool.attn_decode_batch(x, l, qr[l, ne:].contiguous()) for l in range(nl)])
        held = pool.kv_read(convs, [0] * 6, [n + m for n, m in zip(lens, new)])
        torch.cuda.synchronize()
        outs.append((oe, od) + held)
        pool.close()
    for other in outs[1:]:
        assert all(torch.equal(x, y) for x, y in zip(outs[0], other))
    # and against the oracle, on what the cache holds
    k, v = (f64(x.cpu()) for x in outs[0][2:])
    starts = np.cumsum([0] + [n + m for n, m in zip(lens, new)])
    row = 0
    for i in ext:
        turned = torch.from_numpy(_turn(q[i], np.arange(lens[i], lens[i] + new[i]), rope)).to(torch.bfloat16)
        part = slice(starts[i], starts[i + 1])
        got = outs[0][0][1, row:row + new[i]]
        ref = attend_last(f64(turned[1]), k[1, part], v[1, part])
        # (a query may differ from the oracle's by a bf16 step of single dims: twice the attention's tolerance)
        assert np.sqrt(((f64(got.cpu()) - ref) ** 2).sum() / (ref ** 2).sum()) <= 6e-3
        row += new[i]


def test_scores_depend_on_distance_only():
    """What rotary positions are for: the same query and keys at another place give the same weights."""
    from paper_2606_01839_amd import Rope
    rope, d, L = Rope(128), 128, 64
    outs = []
    k, v = kv_tokens(SEED, 0, 1, 0, L, 1, d)
    q = q_tokens(SEED, 0, 0, 0, 1, 4, d)
    for shift in (0, 16 * 500):
        pool = _pool(1, 4, 1, d, 600, max_pages=600)
        c = pool.conv_create()
        if shift:   # tokens before, of keys that no weight falls on
            far = torch.zeros(1, shift, 1, d, dtype=torch.bfloat16, device="cuda")
            pool.kv_append(c, far, far)
        qr = pool.kv_append_rope([c], [L], k.cuda(), v.cuda(), rope, q=q[None].expand(1, L, 4, d).contiguous().cuda())
        gk, _ = pool.kv_read([c], [shift], [L])
        torch.cuda.synchronize()
        s = f64(qr[0, -1].cpu()) @ f64(gk[0, :, 0].cpu()).T
        outs.append(s)
        pool.close()
    # both sides are rounded to bf16: sums of d products each off by 2^-8 relative twice
    bound = 2 * 2.0 ** -8 * 2 * np.linalg.norm(f64(q[0]), axis=-1)[:, None] * np.linalg.norm(f64(k[0, :, 0]), axis=-1)[None]
    assert (np.abs(outs[0] - outs[1]) <= bound).all() and np.abs(outs[0]).max() > 5


def test_failed_launch_changes_nothing_and_streams():
    from paper_2606_01839_amd import CS_EHIP, ConserveError
    rope = _rope(64, True, "none")
    pool = _pool(1, 8, 2, 64, 16)
    k, v = kv_tokens(SEED, 0, 1, 0, 40, 2, 64)
    c = pool.conv_create()
    s = torch.cuda.Stream()
    kc, vc = k.cuda(), v.cuda()
    qc = q_tokens(SEED, 0, 0, 0, 40, 8, 64)[None].cuda()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        pool.kv_append_rope([c], [20], kc[:, :20].contiguous(), vc[:, :20].contiguous(), rope)
    pool.debug_fail_launches(0)
    with pytest.raises(ConserveError) as e:
        pool.kv_append_rope([c], [20], kc[:, 20:].contiguous(), vc[:, 20:].contiguous(), rope)
    assert e.value.code == CS_EHIP and pool.conv_len(c) == 20
    with pytest.raises(ConserveError) as e:
        pool.rope_q([c], [20], qc[0, :20].contiguous(), rope)
    assert e.value.code == CS_EHIP
    pool.debug_fail_launches(-1)
    out = pool.kv_append_rope([c], [20], kc[:, 20:].contiguous(), vc[:, 20:].contiguous(), rope, q=qc[:, 20:].contiguous())
    gk, gv = pool.kv_read([c], [0], [40])
    torch.cuda.synchronize()
    _assert_turned(gk.cpu(), k, np.arange(40), rope)
    _assert_turned(out.cpu(), qc[:, 20:].cpu(), np.arange(20, 40), rope)
    assert torch.equal(gv.cpu(), v)
    pool.close()


def test_a_refused_step_leaves_queries_in_place():
    """A step that the pool has no pages for, its outputs its queries: refused before a query turns."""
    from paper_2606_01839_amd import CS_ENOMEM, ConserveError
    rope = _rope(64, False, "none")
    pool = _pool(1, 8, 2, 64, 4)
    k, v = (x.cuda() for x in kv_tokens(SEED, 0, 1, 0, 64, 2, 64))
    c, d = pool.conv_create(), pool.conv_create()
    pool.kv_append_rope([c, d], [32, 16], k[:, :48].contiguous(), v[:, :48].contiguous(), rope)
    qe = q_tokens(SEED, 0, 0, 32, 17, 8, 64)[None].cuda()
    qd = q_tokens(SEED, 1, 0, 16, 1, 8, 64)[None].cuda()
    a, b = qe.clone(), qd.clone()
    for _ in range(2):
        with pytest.raises(ConserveError) as e:
            pool.mixed_step([c], [17], [d], k[:, :18].contiguous(), v[:, :18].contiguous(), a, b, out_ext=a, out_dec=b, rope=rope)
        assert e.value.code == CS_ENOMEM
    torch.cuda.synchronize()
    assert torch.equal(a, qe) and torch.equal(b, qd) and pool.conv_len(c) == 32 and pool.conv_len(d) == 16
    pool.close()


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_captured_queries_and_decode_replay(fmt):
    """Queries rotated and attended in a captured graph, the rotated ones in place of a buffer of the graph's: every
    replay gives the eager calls' bits, with eager work between replays."""
    rope = _rope(96, True, "parts")
    lens = [450, 1, 2100]
    pool = _pool(1, 32, 8, 128, 200, fmt)
    convs = [pool.conv_create() for _ in lens]
    kv = [kv_tokens(SEED, i, 1, 0, n, 8, 128) for i, n in enumerate(lens)]
    s = torch.cuda.Stream()
    q = torch.zeros(3, 32, 128, dtype=torch.bfloat16, device="cuda")
    turned, out = torch.empty_like(q), torch.empty_like(q)
    k, v = (torch.cat([x[j] for x in kv], 1).cuda() for j in (0, 1))
    torch.cuda.synchronize()
    with torch.cuda.stream(s):   # the pool's work moves to this stream before the capture
        pool.kv_append_rope(convs, lens, k, v, rope)
        pool.rope_q(convs, [1, 1, 1], q, rope, turned)
        pool.attn_decode_batch_noalloc(convs, 0, turned, out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        pool.rope_q(convs, [1, 1, 1], q, rope, turned)
        pool.attn_decode_batch_noalloc(convs, 0, turned, out)
    for turn in range(4):
        x = torch.cat([q_tokens(SEED + turn, i, 0, n - 1, 1, 32, 128) for i, n in enumerate(lens)]).cuda()
        q.copy_(x)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            want_q = pool.rope_q(convs, [1, 1, 1], x, rope)
            want = pool.attn_decode_batch(convs, 0, want_q)
        torch.cuda.synchronize()
        assert torch.equal(turned, want_q) and torch.equal(out, want), turn
    pool.close()
