"""CPU: refusals of the calls for drafted tokens and encoder states, the oracle's own pins, and the host's words of a tree."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import seen as so
from tests.seen_helpers import tree

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_01839_amd", "csrc", "host")


def test_oracle_by_hand():
    #      0   1   2: 0 -> 1, 0 -> 2; 3 is a second root
    p = [-1, 0, 0, -1]
    assert so.ancestors(p).astype(int).tolist() == [[1, 0, 0, 0], [1, 1, 0, 0], [1, 0, 1, 0], [0, 0, 0, 1]]
    assert so.depths(p).tolist() == [0, 1, 1, 0]
    # equal scores: the mean of what is seen
    q, k = np.zeros((4, 1, 2)), np.ones((6, 1, 2))
    v = np.arange(12.0).reshape(6, 1, 2)
    out = so.attend(q, k, v, so.tree_sees(p, 6))
    assert np.allclose(out[2, 0], v[[0, 1, 2, 4], 0].mean(0)) and np.allclose(out[3, 0], v[[0, 1, 5], 0].mean(0))
    assert np.allclose(so.attend(q, k, v)[0, 0], v[:, 0].mean(0)) and (so.attend(q, k[:0], v[:0]) == 0).all()
    v[3] = np.nan
    assert np.isfinite(so.attend(q, k, v, so.tree_sees(p, 6))[[0, 2, 3]]).all()
    assert so.keep(np.arange(10), 6, [0, 2, 5]).tolist() == [0, 1, 2, 3, 4, 6, 9]


def test_oracle_chain_is_causal():
    from oracle.attention import attend_last
    r = np.random.default_rng(0)
    q, k, v = r.standard_normal((5, 4, 8)), r.standard_normal((11, 2, 8)), r.standard_normal((11, 2, 8))
    assert np.allclose(so.attend(q, k, v, so.tree_sees(tree(5, 0, "chain"), 11)), attend_last(q, k, v))


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    d = tmp_path_factory.mktemp("seen")
    shim = d / "shim.cpp"
    shim.write_text('''#include "seen.hpp"
extern "C" int words(const int* p, int n, long prefix, unsigned* out) {
  std::vector<unsigned> v(3, 7u);   // appended behind what is there
  int w = cs::tree_words(p, n, prefix, v);
  for (size_t i = 3; i < v.size(); ++i) out[i - 3] = v[i];
  return w;
}
extern "C" int split(const long* p, int n, int heads) { return cs::rows_split(std::vector<int64_t>(p, p + n), heads, cs::kCus); }
extern "C" int ok(const int* p, int n) { return cs::tree_ok(p, n); }
extern "C" void depths(const int* p, int n, int* out) { cs::tree_depths(p, n, out); }
''')
    so_path = d / "seen.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-I", CSRC, str(shim), os.path.join(CSRC, "seen.cpp"), "-o", str(so_path)],
                   check=True)
    return ctypes.CDLL(str(so_path))


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 100, 1024])
@pytest.mark.parametrize("prefix", [0, 1, 31, 32, 47, 64, 1000])
def test_words_of_a_tree(host, n, prefix):
    p = np.array(tree(n, n + prefix), dtype=np.int32)
    out = np.zeros(n * (n // 32 + 2), dtype=np.uint32)
    w = host.words(p.ctypes.data_as(ctypes.c_void_p), n, ctypes.c_long(prefix), out.ctypes.data_as(ctypes.c_void_p))
    assert w == (prefix + n - 1) // 32 - prefix // 32 + 1
    bits = np.unpackbits(out[:n * w].view(np.uint8), bitorder="little").reshape(n, 32 * w)
    want = np.zeros((n, 32 * w), dtype=bool)
    want[:, :prefix % 32 + n] = so.tree_sees(p, prefix + n)[:, prefix - prefix % 32:]
    assert (bits == want).all()
    d = np.zeros(n, dtype=np.int32)
    host.depths(p.ctypes.data_as(ctypes.c_void_p), n, d.ctypes.data_as(ctypes.c_void_p))
    assert (d == so.depths(p)).all()


def test_trees_refused(host):
    for p in ([0], [-1, 1], [-1, -2], [-1, 5]):
        a = np.array(p, dtype=np.int32)
        assert not host.ok(a.ctypes.data_as(ctypes.c_void_p), len(p))


def _pool(**kw):
    from paper_2606_01839_amd import KVPool
    return KVPool(1, 4, 2, 64, n_pages=32, max_convs=3, max_pages_per_conv=8, device="cpu", **kw)


def _code(fn):
    from paper_2606_01839_amd import ConserveError
    with pytest.raises(ConserveError) as e:
        fn()
    return e.value.code


def test_calls_refused():
    from paper_2606_01839_amd import CS_EINVAL, CS_ENOENT, CS_ERANGE, CS_ESTATE, Rope
    p = _pool()
    a, b = p.conv_create(), p.conv_create()
    z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    q1, q2 = z(1, 4, 64), z(2, 4, 64)
    rope = Rope(64)
    # trees
    assert _code(lambda: p.attn_tree([a], [1], [[-1]], 0, q1)) == CS_ESTATE          # longer than the conversation
    assert _code(lambda: p.attn_tree([a], [1], [[0]], 0, q1)) == CS_EINVAL           # its own parent
    assert _code(lambda: p.attn_tree([a], [2], [[-1, 1]], 0, q2)) == CS_EINVAL
    assert _code(lambda: p.attn_tree([a], [2], [[-1, -2]], 0, q2)) == CS_EINVAL
    assert _code(lambda: p.attn_tree([a], [1025], [[-1] * 1025], 0, z(1025, 4, 64))) == CS_ERANGE
    assert _code(lambda: p.attn_tree([a, a], [0, 0], [[], []], 0, z(0, 4, 64))) == CS_EINVAL
    assert _code(lambda: p.attn_tree([a], [0], [[]], 1, z(0, 4, 64))) == CS_ERANGE
    assert _code(lambda: p.attn_tree([12345], [0], [[]], 0, z(0, 4, 64))) == CS_ENOENT
    for bad in ([[-1]], [[-1], [-1]], [[-1, 0], []]):
        with pytest.raises(ValueError):
            p.attn_tree([a], [2], bad, 0, q2)
    with pytest.raises(ValueError):
        p.attn_tree([a], [2], [[-1, 0]], 0, q1)
    p.attn_tree([a, b], [0, 0], [[], []], 0, z(0, 4, 64))                              # nothing to do
    # cross attention
    assert _code(lambda: p.attn_cross([a], [1], 1, q1)) == CS_ERANGE
    assert _code(lambda: p.attn_cross([12345], [1], 0, q1)) == CS_ENOENT
    assert _code(lambda: p.attn_cross([a, b], [2, -1], 0, q1)) == CS_EINVAL
    with pytest.raises(ValueError):
        p.attn_cross([a], [1, 1], 0, q2)
    p.attn_cross([a, a], [0, 0], 0, z(0, 4, 64))
    # append at tree positions
    k1, k2 = z(1, 1, 2, 64), z(1, 2, 2, 64)
    assert _code(lambda: p.kv_append_tree([a], [1], [[0]], k1, k1, rope)) == CS_EINVAL
    assert _code(lambda: p.kv_append_tree([a, a], [1, 1], [[-1], [-1]], k2, k2, rope)) == CS_EINVAL
    assert _code(lambda: p.kv_append_tree([a], [200], [list(range(-1, 199))], z(1, 200, 2, 64), z(1, 200, 2, 64), rope)) == CS_ERANGE
    assert _code(lambda: p.kv_append_tree([a], [1025], [[-1] * 1025], z(1, 1025, 2, 64), z(1, 1025, 2, 64), rope)) == CS_ERANGE
    assert _code(lambda: p.kv_append_tree([a], [1], [[-1]], k1, k1, Rope(128))) == CS_EINVAL   # over the head
    with pytest.raises(ValueError):
        p.kv_append_tree([a], [1], [[-1]], k1, k1, rope, q_out=z(1, 1, 4, 64))
    big = z(3, 4, 64)
    with pytest.raises(ValueError):   # overlaps without being the same
        p.kv_append_tree([a], [2], [[-1, 0]], k2, k2, rope, q=big[None, :2], q_out=big[None, 1:])
    # keep
    assert _code(lambda: p.kv_keep([a], [1], [[]])) == CS_ESTATE
    assert _code(lambda: p.kv_keep([a], [0], [[0]])) == CS_EINVAL
    assert _code(lambda: p.kv_keep([a], [-1], [[]])) == CS_EINVAL
    assert _code(lambda: p.kv_keep([a, a], [0, 0], [[], []])) == CS_EINVAL
    assert _code(lambda: p.kv_keep([12345], [0], [[]])) == CS_ENOENT
    with pytest.raises(ValueError):
        p.kv_keep([a], [0, 0], [[]])
    p.kv_keep([a, b], [0, 0], [[], []])
    lib, h = p.lib, p._handle
    one = (ctypes.c_int32 * 1)(1)
    zero = (ctypes.c_int32 * 1)(a)
    for rc in (lib.cs_attn_tree(None, 1, zero, one, one, 0, None, None, None), lib.cs_attn_cross(None, 1, zero, one, 0, None, None, None),
               lib.cs_kv_keep(None, 1, zero, one, one, one, None), lib.cs_attn_cross(h, 1, zero, one, 0, None, None, None),
               lib.cs_attn_tree(h, 1, zero, None, one, 0, None, None, None), lib.cs_attn_tree(h, 1, zero, one, None, 0, None, None, None),
               lib.cs_kv_keep(h, 1, zero, None, one, one, None), lib.cs_kv_append_tree(h, None, 1, zero, one, one, None, None, None, None, None)):
        assert rc == CS_EINVAL
    assert p.conv_len(a) == 0 and p.occupancy() == (0, 32)
    p.close()


CALLS = {
    "attn_tree": "_, h = pool(64); print(lib.cs_attn_tree(h, N, 4096, 4096, 4096, 0, 4096, 4096, None), None)",
    "attn_cross": "_, h = pool(64); print(lib.cs_attn_cross(h, N, 4096, 4096, 0, 4096, 4096, None), None)",
    "kv_keep": "_, h = pool(64); print(lib.cs_kv_keep(h, N, 4096, 4096, 4096, 4096, None), None)",
    "kv_append_tree": """
_, h = pool(64); r = RopeDesc(); lib.cs_rope_init(ctypes.byref(r), 64, 0, 1e4, 0, 1., 0., 0., 0.)
print(lib.cs_kv_append_tree(h, ctypes.byref(r), N, 4096, 4096, 4096, 4096, 4096, None, None, None), None)""",
}


@pytest.mark.parametrize("name", CALLS)
def test_out_of_host_memory(name):
    """No exception leaves the C ABI, as in test_no_throw_cpu."""
    import sys

    from tests.test_no_throw_cpu import PRELUDE
    r = subprocess.run([sys.executable, "-c", PRELUDE + CALLS[name]], capture_output=True, text=True, timeout=120, cwd=ROOT)
    assert r.returncode == 0, r.stderr[-2000:]
    assert r.stdout.split() == ["-2", "None"], r.stdout


@pytest.mark.parametrize("lens,heads,want", [([300, 512], 8, 64), ([24571], 8, 96), ([1000] * 300, 8, 1024), ([9000, 300], 2, 32), ([1], 1, 64)])
def test_items_of_few_rows(host, lens, heads, want):
    """Keys per wave: one round of the 256 CUs where there is one."""
    a = (ctypes.c_int64 * len(lens))(*lens)
    split = host.split(a, len(lens), heads)
    assert split == want, split
    assert split % 32 == 0 and 32 <= split <= 1024
