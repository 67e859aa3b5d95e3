"""CPU: the oracles of the 4-bit cache and of rotary positions on values worked out by hand; the
library's host side of both (sizes, frequencies, refusals before anything touches a device)."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import fp4 as o4
from oracle import rope as orope


# ---- oracles -------------------------------------------------------------------------------------
def test_encode_by_hand():
    x = np.zeros(32)
    # largest magnitude 6 -> power 2^(2-2) = 1: the table, ties to the even code, saturation at 6
    x[:16] = [6, 5, 5.01, 3.5, 3.49, 2.5, 2.51, 1.75, 1.25, 0.75, 0.25, 0.26, -0.25, -5, -3.5, 0]
    c, e = o4.encode(x, 32)
    assert e.tolist() == [0]
    assert c[:16].tolist() == [7, 6, 7, 6, 5, 4, 5, 4, 2, 2, 0, 1, 8, 14, 14, 0]
    # 7.9 lies in [4, 8): power 1, saturates at 6; 8 doubles the power
    assert o4.decode(*o4.encode(np.r_[7.9, np.zeros(31)], 32))[0] == 6.0
    c, e = o4.encode(np.r_[8.0, 1.0, np.zeros(30)], 32)
    assert e[0] == 1 and c[0] == 6 and o4.decode(c, e)[1] == 1.0
    # each group has its own power; zeros and values below the least power
    c, e = o4.encode(np.r_[np.full(32, 3e-3), np.full(32, 100.0)], 32)
    assert e.tolist() == [math.floor(math.log2(3e-3)) - 2, 4]
    c, e = o4.encode(np.r_[2.0 ** -130, np.zeros(31)], 32)
    assert e[0] == -126 and c[0] == 0
    assert (o4.decode(*o4.encode(np.zeros(64), 64)) == 0).all()


def test_serialize_by_hand():
    d = 64
    k, v = np.zeros((1, 2, 1, d)), np.zeros((1, 2, 1, d))
    k[0, 1, 0, 49] = 4.0      # token 1, group 1 (dims 32 .. 63), its code 17: the second of byte 8
    v[0, 1, 0, 35] = -0.5     # dim 35 = 16 * 2 + 3: tile 2, row 3, token 1 of part 0
    w = o4.serialize(k, v)
    assert w.size == 17 * d
    want = np.zeros(17 * d, dtype=np.uint8)
    want[(1 * 16 + 1) * 16 + 8] = 6 << 4                  # 4.0 with power 1
    want[8 * d + (0 * 16 + 3) * 8 + 2 * 2] = 0xE << 4     # -0.5 = -4 x 2^-3
    ks = 16 * d
    want[[ks, ks + 1, ks + 2]] = 1                        # groups of zeros: 2^-126
    want[ks + 3] = 127
    want[ks + 32], want[ks + 33] = 1, 127 - 3
    assert w.tolist() == want.tolist()


def test_rotate_by_hand():
    f = np.array([math.pi / 2, math.pi])
    x = np.arange(1.0, 7.0).reshape(1, 1, 6)
    y = orope.rotate(x, [1], f)          # pairs (1, 3), (2, 4): quarter turn, half turn; 5, 6 stay
    assert np.allclose(y.ravel(), [-3, -2, 1, -4, 5, 6])
    y = orope.rotate(x, [1], f, 2.0, True)   # pairs (1, 2), (3, 4), doubled
    assert np.allclose(y.ravel(), [-4, 2, -6, -8, 5, 6])
    assert np.allclose(orope.rotate(x, [0], f), x)


def test_a_query_is_the_sum_of_three_e3m2_numbers():
    """The arithmetic of the score product over 4-bit pages: with the largest magnitude of a block scaled to
    [8, 16), rounding to e3m2 (values to 28, 3 significant bits, subnormal step 1/16) three times, each time
    what is left times 16, gives a bf16 value exactly down to 2^-8 of the largest and within 2^-16 of it."""
    grid = np.array(sorted({m / 16 for m in range(4)} | {(4 + m) / 4 * 2.0 ** e for m in range(4) for e in range(-2, 5)}))

    def e3m2(x):
        d = np.abs(np.abs(x)[:, None] - grid)
        near = np.where(d == d.min(1, keepdims=True), np.arange(32) + 32 * (np.arange(32) % 2), 99).min(1) % 32
        return np.sign(x) * grid[near]

    x = np.array([(128 + m) * 2.0 ** e for m in range(128) for e in range(-30, -3)])   # every bf16 value below 16
    left, total = x.copy(), np.zeros_like(x)
    for k in range(3):
        part = e3m2(left * 16.0 ** k)
        assert np.abs(left * 16.0 ** k).max() <= 16
        total += part / 16.0 ** k
        left = x - total
    assert (left[x >= 8 * 2.0 ** -8] == 0).all() and np.abs(left).max() <= 8 * 2.0 ** -16


# ---- host side of the library ----------------------------------------------------------------------
@pytest.mark.parametrize("r", [16, 48, 64, 128])
@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "parts"])
def test_frequencies(r, scaling):
    from paper_2606_01839_amd import Rope
    rope = Rope(r, base=500000.0, interleaved=True, scaling=scaling, factor=8.0, original_len=8192, low_turns=1, high_turns=4)
    f, amp = orope.frequencies(r, 500000.0, scaling, 8.0, 8192, 1, 4)
    assert rope.rotary_dim == r and rope.interleaved and rope.inv_freq.shape == (r // 2,)
    # a power, a quotient and a sum in double: a few roundings
    assert np.allclose(rope.inv_freq, f, rtol=1e-13, atol=0) and abs(rope.amplitude - amp) < 1e-15
    rope.amplitude, rope.inv_freq = 0.5, f * 2
    assert rope.amplitude == 0.5 and np.array_equal(rope.inv_freq, f * 2)
    with pytest.raises(ValueError):
        rope.inv_freq = [1.0]


def test_rope_refusals():
    from paper_2606_01839_amd import CS_EINVAL, ConserveError, Rope
    nan = float("nan")
    for bad in [dict(rotary_dim=0), dict(rotary_dim=24), dict(rotary_dim=144), dict(rotary_dim=-16), dict(rotary_dim=64, base=1.0),
                dict(rotary_dim=64, base=nan), dict(rotary_dim=64, scaling="linear", factor=0.5),
                dict(rotary_dim=64, scaling="ntk", factor=nan), dict(rotary_dim=64, scaling="parts", factor=4.0),
                dict(rotary_dim=64, scaling="parts", factor=4.0, original_len=8192, low_turns=4, high_turns=4)]:
        with pytest.raises(ConserveError) as e:
            Rope(**bad)
        assert e.value.code == CS_EINVAL
    with pytest.raises(ValueError):
        Rope(64, scaling="dynamic")
    from paper_2606_01839_amd.conserve import RopeDesc, load_library
    lib, d = load_library(), RopeDesc()
    assert lib.cs_rope_init(None, 64, 0, 1e4, 0, 1.0, 0.0, 0.0, 0.0) == CS_EINVAL
    assert lib.cs_rope_init(ctypes.byref(d), 64, 2, 1e4, 0, 1.0, 0.0, 0.0, 0.0) == CS_EINVAL
    assert lib.cs_rope_init(ctypes.byref(d), 64, 0, 1e4, 4, 1.0, 0.0, 0.0, 0.0) == CS_EINVAL


def _pool(**kw):
    from paper_2606_01839_amd import KVPool
    args = dict(n_layers=1, n_q_heads=4, n_kv_heads=2, head_dim=64, n_pages=32, max_convs=3, max_pages_per_conv=8,
                placement_seed=1, device="cpu", kv_format="fp4")
    args.update(kw)
    return KVPool(**args)


def test_pool_formats():
    from paper_2606_01839_amd import CS_EINVAL
    from paper_2606_01839_amd.conserve import PoolDesc, load_library
    lib, d = load_library(), PoolDesc(32, 32, 8, 128, 256, 8192, 1000)
    b16 = lib.cs_pool_kv_bytes(ctypes.byref(d))
    assert lib.cs_pool_kv_bytes_as(ctypes.byref(d), 0) == b16
    assert lib.cs_pool_kv_bytes_as(ctypes.byref(d), 1) == 32 * 1000 * 8 * 17 * 128 == b16 * 17 // 64
    assert lib.cs_pool_kv_bytes_as(ctypes.byref(d), 2) == lib.cs_pool_kv_bytes_as(ctypes.byref(d), -1) == 0
    assert lib.cs_pool_kv_bytes_as(None, 1) == 0
    h = ctypes.c_void_p()
    buf = torch.zeros(4096, dtype=torch.uint8)
    assert lib.cs_pool_create_as(ctypes.byref(d), 2, buf.data_ptr(), 4096, buf.data_ptr(), 4096, 0, ctypes.byref(h)) == CS_EINVAL
    with pytest.raises(ValueError):
        _pool(kv_format="int4")
    with _pool() as p:
        assert p.kv.numel() == 32 * 2 * 17 * 64 and tuple(p.kv_view().shape) == (1, 32, 2, 17 * 64)
        assert p.page_block_bytes == 17 * 64
        a = p.conv_create()
        assert p.kv_pack_size(a) == p.kv_pack_fp4_size(a) == 0


def test_refusals_change_nothing():
    """Everything that validation refuses, before a device is touched."""
    from paper_2606_01839_amd import CS_EINVAL, CS_ENOENT, CS_ENOMEM, CS_ERANGE, CS_ESTATE, ConserveError, Rope
    from paper_2606_01839_amd.conserve import RopeDesc
    rope = Rope(64)
    for fmt in ("fp4", "bf16"):
        p = _pool(kv_format=fmt)
        a, b = p.conv_create(), p.conv_create()
        z = lambda n, h=2: torch.zeros(1, n, h, 64, dtype=torch.bfloat16)

        def refused(code, fn, *args, **kw):
            with pytest.raises(ConserveError) as e:
                fn(*args, **kw)
            assert e.value.code == code, e.value

        refused(CS_EINVAL, p.kv_append_rope, [a, a], [1, 1], z(2), z(2), rope)
        refused(CS_ENOENT, p.kv_append_rope, [a, 77], [1, 1], z(2), z(2), rope)
        refused(CS_ERANGE, p.kv_append_rope, [a], [129], z(129), z(129), rope)
        wide = Rope(128)
        refused(CS_EINVAL, p.kv_append_rope, [a], [1], z(1), z(1), wide)
        refused(CS_EINVAL, p.rope_q, [a], [0], z(0, 4)[0], wide)
        for field, value in [("rotary_dim", 24), ("rotary_dim", 0), ("interleaved", 2), ("amplitude", float("inf")),
                             ("amplitude", 1e300)]:
            bad = Rope(64)
            setattr(bad.desc, field, value)
            refused(CS_EINVAL, p.kv_append_rope, [a], [1], z(1), z(1), bad)
            refused(CS_EINVAL, p.rope_q, [a], [0], z(0, 4)[0], bad)
        bad = Rope(64)
        bad.desc.inv_freq[31] = float("nan")
        refused(CS_EINVAL, p.kv_append_rope, [a], [1], z(1), z(1), bad)
        bad = Rope(32)
        bad.desc.inv_freq[16] = float("nan")     # not in use
        p.rope_q([a], [0], z(0, 4)[0], bad)
        refused(CS_ESTATE, p.rope_q, [a], [1], z(1, 4)[0], rope)
        refused(CS_EINVAL, p.rope_q, [a, a], [0, 0], z(0, 4)[0], rope)
        refused(CS_ENOENT, p.rope_q, [123], [0], z(0, 4)[0], rope)
        refused(CS_ERANGE, p.kv_read, [a], [0], [1])
        refused(CS_ERANGE, p.kv_read, [a], [1], [0])
        refused(CS_EINVAL, p.kv_read, [a], [-1], [0])
        refused(CS_EINVAL, p.kv_read, [a, b, a], [0, 0, 0], [0, 0, 0])
        refused(CS_ENOENT, p.kv_read, [99], [0], [0])
        k, v = p.kv_read([a, b], [0, 0], [0, 0])
        assert k.shape == v.shape == (1, 0, 2, 64)
        # shapes, dtypes and overlaps are the binding's
        with pytest.raises(ValueError):
            p.kv_append_rope([a], [1], z(1), z(1), rope, q=z(1, 2))
        with pytest.raises(ValueError):
            p.kv_append_rope([a], [1], z(1), z(1), rope, q_out=z(1, 4))
        with pytest.raises(ValueError):
            p.kv_append_rope([a], [1, 1], z(1), z(1), rope)
        with pytest.raises(ValueError):
            p.rope_q([a], [0], z(0, 4)[0].float(), rope)
        with pytest.raises(ValueError):
            p.kv_read([a], [0, 0], [0])
        buf = torch.zeros(1 + 3 * 256, dtype=torch.bfloat16)
        q, shifted = buf[:512].view(1, 2, 4, 64), buf[256:768].view(1, 2, 4, 64)
        with pytest.raises(ValueError, match="overlaps"):
            p.kv_append_rope([a], [2], z(2), z(2), rope, q=q, q_out=shifted)
        # raw calls: null pointers
        lib, P = p.lib, ctypes.byref(rope.desc)
        from paper_2606_01839_amd.conserve import _i32_array
        ca, cp = _i32_array([a])
        na, npp = _i32_array([1])
        x = z(1, 4).data_ptr()
        assert lib.cs_kv_append_rope(None, P, 1, cp, npp, x, x, None, None, None) == CS_EINVAL
        assert lib.cs_kv_append_rope(p._handle, None, 1, cp, npp, x, x, None, None, None) == CS_EINVAL
        assert lib.cs_kv_append_rope(p._handle, P, 1, cp, npp, x, x, x, None, None) == CS_EINVAL
        assert lib.cs_kv_append_rope(p._handle, P, 1, cp, npp, None, x, None, None, None) == CS_EINVAL
        assert lib.cs_kv_append_rope(p._handle, P, 1, cp, None, x, x, None, None, None) == CS_EINVAL
        neg, negp = _i32_array([-1])
        assert lib.cs_kv_append_rope(p._handle, P, 1, cp, negp, x, x, None, None, None) == CS_EINVAL
        assert lib.cs_rope_q(p._handle, P, 1, cp, negp, 1, x, x, None) == CS_EINVAL
        assert lib.cs_rope_q(p._handle, P, 1, cp, npp, -1, x, x, None) == CS_EINVAL
        assert lib.cs_rope_q(p._handle, P, 1, cp, None, 1, x, x, None) == CS_EINVAL
        assert lib.cs_rope_q(None, P, 1, cp, npp, 1, x, x, None) == CS_EINVAL
        assert lib.cs_kv_read(None, 1, cp, x, npp, x, x, None) == CS_EINVAL
        assert lib.cs_kv_read(p._handle, 1, cp, None, npp, x, x, None) == CS_EINVAL
        refused(CS_EINVAL, p.mixed_step, [a], [1], [], z(1), z(1), z(1, 4), rope=wide)
        refused(CS_EINVAL, p.mixed_step, [a], [1], [a], z(2), z(2), z(1, 4), z(1, 4), rope=rope)
        refused(CS_ERANGE, p.mixed_step, [a], [129], [], z(129), z(129), z(129, 4), rope=rope)
        assert lib.cs_mixed_step_rope(p._handle, None, 1, cp, npp, 0, None, x, x, x, x, None, None, 0, None) == CS_EINVAL
        assert lib.cs_mixed_step_rope(p._handle, P, 1, cp, npp, 0, None, x, x, x, x, None, None, 2, None) == CS_EINVAL
        assert lib.cs_mixed_step_rope(None, P, 1, cp, npp, 0, None, x, x, x, x, None, None, 0, None) == CS_EINVAL
        with pytest.raises(ValueError, match="overlaps"):
            p.mixed_step([a], [2], [], z(2), z(2), q, out_ext=shifted, rope=rope)
        n = ctypes.c_size_t()
        assert lib.cs_kv_pack_fp4_size(p._handle, 99, ctypes.byref(n)) == CS_ENOENT
        assert lib.cs_kv_pack_fp4_size(None, a, ctypes.byref(n)) == CS_EINVAL
        assert lib.cs_kv_pack_fp4(p._handle, a, x, 16, None) == CS_EINVAL
        assert lib.cs_kv_pack_fp4(None, a, x, 0, None) == CS_EINVAL
        assert lib.cs_kv_pack(None, a, x, 0, None) == CS_EINVAL
        refused(CS_EINVAL, p.kv_unpack, torch.zeros(2 * 64 * 64 if fmt == "fp4" else 2 * 17 * 64, dtype=torch.uint8), 3)
        assert p.conv_len(a) == p.conv_len(b) == 0 and p.occupancy() == (0, 32)
        small = _pool(kv_format=fmt, n_pages=2)
        c = small.conv_create()
        refused(CS_ENOMEM, small.kv_append_rope, [c], [40], z(40), z(40), rope)
        assert small.conv_len(c) == 0 and small.occupancy() == (0, 2)
        small.close()
        p.close()


@pytest.mark.skipif(torch.cuda.is_available(), reason="has a GPU")
def test_device_calls_fail_cleanly_without_gpu():
    from paper_2606_01839_amd import CS_EHIP, ConserveError, Rope
    for fmt in ("fp4", "bf16"):
        p = _pool(kv_format=fmt)
        a = p.conv_create()
        k = torch.zeros(1, 5, 2, 64, dtype=torch.bfloat16)
        with pytest.raises(ConserveError) as e:
            p.kv_append_rope([a], [5], k, k, Rope(64))
        assert e.value.code == CS_EHIP and p.conv_len(a) == 0 and p.occupancy() == (0, 32)
        p.close()


def test_wire_version_matches_the_header():
    import os
    import re
    from paper_2606_01839_amd import conserve
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = open(os.path.join(root, "include", "conserve_attn.h")).read()
    m = re.search(r"#define\s+CS_WIRE_FP4_VERSION\s+(\d+)", src)
    assert m and int(m.group(1)) == conserve.WIRE_FP4_VERSION == 1
