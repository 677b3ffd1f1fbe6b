"""The kernels of attend_prefix, attend_mass and evict as they are built, from the library's own gfx950 code objects (no GPU needed)."""
import os
import re
import subprocess

import pytest

from test_kernel_registers_cpu import LLVM, _code_objects, kernels  # noqa: F401  (a fixture)


def test_nothing_spilled(kernels):  # noqa: F811
    mine = {k: v for k, v in kernels.items() if re.search(r"3bkv\d+(tile_kernel|tile_merge|mass_kernel|attend_mass)", k) or
            re.search(r"attend_kernelI\w+ELi[12]EEEvNS_10AttendArgsE", k)}
    assert len(mine) > 20
    for name, (registers, spilled) in mine.items():
        assert spilled == 0, (name, registers, spilled)


def test_m0_is_only_where_loads_to_lds_go(tmp_path):
    """The statement that loads to LDS sets m0 by itself, which the compiler is not told: nothing else in these kernels may use it."""
    if not os.path.exists(os.path.join(LLVM, "llvm-objdump")):
        pytest.skip("no llvm-objdump")
    from paper_2502_07861_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2502_07861_amd.build import build
        build()
    seen = set()
    for i, obj in enumerate(_code_objects(binding.LIB_PATH)):
        if b"tile_kernel" not in obj and b"mass_kernel" not in obj:
            continue
        path = tmp_path / ("%d.elf" % i)
        path.write_bytes(obj)
        text = subprocess.run([os.path.join(LLVM, "llvm-objdump"), "-d", "--no-show-raw-insn", str(path)], capture_output=True, text=True, check=True).stdout
        for part in re.split(r"\n(?=[0-9a-f]{16} <)", text):
            name = re.match(r"[0-9a-f]{16} <(\S+)>:", part)
            if not name or not re.search(r"3bkv\d+(tile_kernel|mass_kernel)I", name.group(1)):
                continue
            lines = [line.split("//")[0].strip() for line in part.splitlines()[1:] if line.strip()]
            loads = [k for k, line in enumerate(lines) if line.startswith("global_load_lds_dwordx4")]
            assert loads, name.group(1)
            for k in loads:
                assert re.match(r"s_mov_b32 m0, s\d+$", lines[k - 2]) and lines[k - 1].startswith("s_nop"), (name.group(1), lines[k - 2:k + 1])
            others = [line for k, line in enumerate(lines) if re.search(r"\bm0\b", line) and k + 2 not in loads]
            assert not others, (name.group(1), others[:3])
            seen.add(name.group(1))
    assert len(seen) == 8
