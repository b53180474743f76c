"""The device code of the attention over packed sequences, read back as assembly: its loads into LDS are written in assembly,
where the compiler keeps no wait states."""
import subprocess

from test_kernel_code import TOOLS
from test_kernel_code_parts import address_hazards, parts


def test_addresses_of_loads_into_lds_have_settled(tmp_path):
    kernels, total = set(), 0
    for code in parts(tmp_path):
        lines, name = [], ""
        proc = subprocess.Popen([TOOLS["llvm-objdump"], "-d", code], stdout=subprocess.PIPE, text=True)
        for line in list(proc.stdout) + ["end>:\n"]:
            if line.endswith(">:\n"):
                if "prompt_tile_kernel" in name:
                    loads, found = address_hazards(lines)
                    assert not found, (name, found[:3])
                    kernels.add(name)
                    total += loads
                name, lines = line, []
            elif "prompt_tile_kernel" in name:
                lines.append(line)
        assert proc.wait() == 0
    # both types, five paddings of the head (one of them in one height, the others in two), whole heads and others
    assert len(kernels) == 2 * (4 * 2 + 1) * 2 and total >= 100
