"""The compiled code of the wide-tile kernel on operands in 8 bits and by group: what test_kernel_code asks of the others."""
import re

import pytest

from paper_2401_16677_amd import build as hip_build
from test_kernel_code import _blocks, _compile, _touched_in_flight

UNITS = [u for u in hip_build.UNITS if u[0] == "t3_wide_products_launch.hip"]


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    return _compile(tmp_path_factory.mktemp("asm"), UNITS, "wide_tile_kernel")


@pytest.mark.parametrize("unit", [u[1] for u in UNITS])
def test_hand_ordered_loop_is_as_written(code, unit):
    """No register an inline-assembly read is on its way to is touched; nothing is spilled to memory; the compiler waits for no memory access
    where products are; behind the barrier of a slab the first product follows at once; no load to a register in inline assembly."""
    assert len(code[unit]) == (5 if unit.endswith(("fused_i8.o", "overlap_i8.o", "gemm_i8.o")) else 6)      # (by group: quarters as well)
    for kernel, lines in code[unit].items():
        faults, reads = _touched_in_flight(lines)
        assert reads >= 24 and not faults, (kernel, sorted(faults)[:5])
        halves = 0
        for block, _ in _blocks(lines):
            assert not any(t.startswith("scratch_") for t, _ in block), kernel
            assert not any(asm and re.match(r"(global|buffer|flat)_(load|atomic)", t) and not re.search(r"\blds\b", t) for t, asm in block), kernel
            products = [i for i, (t, _) in enumerate(block) if t.startswith("v_mfma")]
            if len(products) < 8:
                continue
            assert all(("_i8 " in block[i][0]) == ("i8" in unit) for i in products), kernel
            assert not any(t.startswith("s_waitcnt") and "vmcnt" in t for t, asm in block if not asm), kernel
            if any(re.search(r"\blds\b", t) for t, _ in block):
                halves += 1
                assert products[0] <= 4, (kernel, block[:products[0]])
        assert halves == 1, kernel
