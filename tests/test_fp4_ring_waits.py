"""CPU: the attention kernels over 4-bit pages, read from the built library's own gfx950 code as in
test_lds_ring_waits.py. Here the ring is written by the waves themselves: at a step's barrier none of a
wave's LDS writes may be in flight (behind it the other waves read them), and no read of the buffers that
a later step overwrites but those of the next tile's K; nor may a conversion instruction of several
passes write a register that it still reads."""
import os
import re

import pytest

from tests.test_lds_ring_waits import OBJDUMP, _kernels, _pending


def _regs(text):
    m = re.match(r"v\[(\d+):(\d+)\]", text)
    return set(range(int(m[1]), int(m[2]) + 1)) if m else {int(text[1:])} if re.match(r"v\d+$", text) else set()


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="llvm-objdump not available")
def test_fp4_kernels(tmp_path):
    kernels = _kernels(str(tmp_path))
    rings = conversions = 0
    for name, body in kernels.items():
        for _, op, args, _ in body:
            if re.match(r"v_cvt_scalef32_(2xpk16|pk32)", op):
                parts = re.findall(r"v\[\d+:\d+\]|v\d+", args)
                conversions += 1
                assert not any(_regs(parts[0]) & _regs(p) for p in parts[1:]), f"{name}: {op} {args}"
        m = re.search(r"attn_fp4_kernelILi(\d+)ELi\d+ELb([01])ELb[01]E", name) or re.search(r"mixed_fp4_kernelILi(\d+)ELi", name)
        if not m:
            continue
        rings += 1
        d, ahead = int(m[1]), "mixed" in name or m[2] == "1"
        for pend in _pending(body):
            assert ahead, f"{name}: {pend} in flight at a barrier"
            assert "w" not in pend, f"{name}: {pend} (a write, or a read that is not of 16 bytes)"
            assert len(pend) <= 2 * d // 64, f"{name}: {pend}"   # the next tile's K: two key halves, d / 64 steps
    assert rings == 40, rings   # 4 groups x (attn_fp4: 2 forms at d 128, 4 at d 64; mixed_fp4: 2 at each)
    assert conversions > 0
