"""CPU: waits of the tiles of trees and cross attention over bf16 pages, read from the built library's own gfx950 code, by the scan of
test_lds_ring_waits: at a step's barrier only the K reads of the next tile may be in flight."""
import os
import re

import pytest

from tests.test_lds_ring_waits import OBJDUMP, _kernels, _pending


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="llvm-objdump not available")
def test_no_read_of_a_retired_buffer_crosses_a_barrier(tmp_path):
    checked = 0
    for name, body in _kernels(str(tmp_path)).items():
        m = re.search(r"seen_tile_kernelILi(\d+)ELi\d+ELb0E", name)
        if not m:
            continue
        checked += 1
        d = int(m[1])
        assert any(op == "ds_read_b128" for _, op, _, _ in body)
        for pend in _pending(body):
            assert "w" not in pend, f"{name}: {pend}"
            regs = {r for r, _ in pend}
            offs = sorted({o for _, o in pend})
            assert len(pend) <= d // 8 and len(offs) <= 2 and len(regs) >= len(pend) / 2, f"{name}: {pend}"
            assert len(offs) < 2 or offs[1] - offs[0] == 64 * d, f"{name}: {pend}"
    assert checked == 8, checked   # 4 groups at each head dim
