"""The device code of every translation unit in the built library: no kernel keeps anything in scratch memory, and none has the
packed single-precision instructions that the build switches off."""
import re
import subprocess

import paper_2604_17709_amd as dn
from test_kernel_code import TOOLS

MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def parts(tmp_path):
    """Paths of the code objects: the library's bundles lie one after the other in one section."""
    run = lambda *a: subprocess.run(a, check=True, capture_output=True, text=True).stdout
    lib = tmp_path / "lib.so"
    lib.write_bytes(open(dn.LIB_PATH, "rb").read())
    run(TOOLS["llvm-objcopy"], "--dump-section=.hip_fatbin=%s" % (tmp_path / "fatbin"), str(lib))
    fat = (tmp_path / "fatbin").read_bytes()
    at = [m.start() for m in re.finditer(re.escape(MAGIC), fat)]
    for i, (a, b) in enumerate(zip(at, at[1:] + [len(fat)])):
        one, code = tmp_path / ("bundle%d" % i), tmp_path / ("code%d" % i)
        one.write_bytes(fat[a:b])
        run(TOOLS["clang-offload-bundler"], "--unbundle", "--type=o", "--input=%s" % one, "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", "--output=%s" % code)
        yield str(code)


def test_every_part(tmp_path):
    names = []
    for code in parts(tmp_path):
        notes = subprocess.run([TOOLS["llvm-readobj"], "--notes", code], check=True, capture_output=True, text=True).stdout
        for k in re.split(r"\n\s+- \.agpr_count:", notes)[1:]:
            names.append(re.search(r"\.name:\s+(_Z\S+)", k)[1])
            for field in (r"\.private_segment_fixed_size", r"\.vgpr_spill_count"):
                assert int(re.search(field + r":\s+(\d+)", k)[1]) == 0, (names[-1], field)
        listing = subprocess.Popen([TOOLS["llvm-objdump"], "-d", "--no-show-raw-insn", code], stdout=subprocess.PIPE, text=True)
        packed = [line for line in listing.stdout if re.search(r"\sv_pk_(add|mul|fma)_f32", line)]
        assert listing.wait() == 0 and not packed, packed[:3]
    for kernel in ("kv_step_kernel", "kv_plan_kernel", "tree_mask_kernel", "rope_store_kernel", "tree_attention_kernel", "tree_attention_tile_kernel", "tree_attention_join_kernel", "prefill"):
        assert any(kernel in n for n in names), kernel
