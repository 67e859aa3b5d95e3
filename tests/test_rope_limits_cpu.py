"""CPU: the largest batches of a query rotation, refused before anything touches a device (without one, a batch that
passes validation fails with CS_EHIP)."""
import array
import ctypes

import pytest
import torch


@pytest.fixture
def pool():
    """Makes pools of 1 layer, 1 head of 64 whose device memory is a made-up address (validation does not read it)."""
    from paper_2606_01839_amd import CS_OK
    from paper_2606_01839_amd.conserve import PoolDesc, load_library
    lib, made = load_library(), []

    def make(max_convs, max_pages, n_pages):
        d, h = PoolDesc(1, 1, 1, 64, max_convs, max_pages, n_pages), ctypes.c_void_p()
        size = lib.cs_pool_kv_bytes_as(ctypes.byref(d), 1)
        assert lib.cs_pool_create_as(ctypes.byref(d), 1, 4096, size, 4096, 1 << 50, 0, ctypes.byref(h)) == CS_OK
        made.append(h)
        return lib, h

    yield make
    for h in made:
        lib.cs_pool_destroy(h)


def _append(lib, h, convs, n_new, q):
    from paper_2606_01839_amd import Rope
    ca, na = array.array("i", convs), array.array("i", n_new)
    return lib.cs_kv_append_rope(h, ctypes.byref(Rope(64).desc), len(ca), ca.buffer_info()[0], na.buffer_info()[0], 4096, 4096, q, q,
                                 None)


def _convs(lib, h, n):
    out, c = [], ctypes.c_int32()
    for _ in range(n):
        assert lib.cs_conv_create(h, ctypes.byref(c)) == 0
        out.append(c.value)
    return out


def _state(lib, h, c):
    n, used, free = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
    assert lib.cs_conv_len(h, c, ctypes.byref(n)) == 0 and lib.cs_pool_occupancy(h, ctypes.byref(used), ctypes.byref(free)) == 0
    return n.value, used.value


@pytest.mark.skipif(torch.cuda.is_available(), reason="the accepted batches would run")
def test_appends_with_more_query_rows_than_a_grid_takes(pool):
    from paper_2606_01839_amd import CS_EHIP, CS_EINVAL
    rows = (1 << 28) - 16
    lib, h = pool(2, 1 << 24, 1 << 24)
    a, b = _convs(lib, h, 2)
    assert _append(lib, h, [a], [rows + 1], 4096) == CS_EINVAL
    assert _append(lib, h, [a, b], [rows - 40, 41], 4096) == CS_EINVAL
    assert _append(lib, h, [a], [rows], 4096) == CS_EHIP           # as many as it takes
    assert _append(lib, h, [a], [rows + 1], None) == CS_EHIP       # no queries: no limit of theirs
    assert _state(lib, h, a) == _state(lib, h, b) == (0, 0)


@pytest.mark.skipif(torch.cuda.is_available(), reason="the accepted batches would run")
def test_appends_with_queries_of_more_conversations_than_an_upload_holds(pool):
    from paper_2606_01839_amd import CS_EHIP, CS_ENOMEM
    n = (1 << 18) + 1
    lib, h = pool(n, 1, n)
    convs = _convs(lib, h, n)
    assert _append(lib, h, convs, [1] * n, 4096) == CS_ENOMEM
    assert _append(lib, h, convs, [1] * (n - 1) + [0], 4096) == CS_EHIP   # one without rows
    assert _append(lib, h, convs, [1] * n, None) == CS_EHIP
    assert _state(lib, h, convs[0]) == (0, 0)
