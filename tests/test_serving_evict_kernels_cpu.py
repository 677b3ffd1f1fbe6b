"""The kernels of evict as they are built, from the library's own gfx950 code objects (no GPU needed)."""
import re

from test_kernel_registers_cpu import kernels  # noqa: F401  (a fixture)


def test_ranks_stay_in_registers(kernels):  # noqa: F811
    """Up to 64 ranks a thread of workgroups of 1024, which have 128 registers each: none is spilled."""
    mine = {k: v for k, v in kernels.items() if re.search(r"3bkv\d+evict_(select|count|list|gather)_kernel", k)}
    assert len(mine) == 16 and any("evict_select_kernelILi64E" in k for k in mine)
    for name, (registers, spilled) in mine.items():
        assert spilled == 0 and registers <= 128, (name, registers, spilled)
