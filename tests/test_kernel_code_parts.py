"""The device code of every translation unit in the built library: no kernel keeps anything in scratch memory, and none has the
packed single-precision instructions that the build switches off."""
import re
import subprocess

import paper_2604_17709_amd as dn
from test_kernel_code import TOOLS, parse, paths_back, wait_states

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


ADDRESS_WAIT = 5      # wait states between a vector instruction that writes a scalar register and a load with that register as address


def scalars(text):
    m = re.match(r"^s(?:(\d+)|\[(\d+):(\d+)\])$", text.strip())
    if not m:
        return set()
    return set(range(int(m[1] or m[2]), int(m[1] or m[3]) + 1))


def address_hazards(lines):
    """Loads into LDS whose scalar address a vector instruction wrote less than ADDRESS_WAIT wait states before: (loads, texts)."""
    code = parse(lines)
    before, found, loads = paths_back(code) if code else [], [], 0
    for i, (at, op, operands, _) in enumerate(code):
        if not op.startswith("global_load_lds") or len(operands) < 2:
            continue
        address = scalars(operands[1].split()[0])
        if not address:
            continue
        loads += 1
        todo, seen = [(j, 0) for j in before[i]], {}
        while todo:
            j, states = todo.pop()
            if states >= ADDRESS_WAIT or seen.get(j, ADDRESS_WAIT) <= states:
                continue
            seen[j] = states
            if code[j][1].startswith("v_") and scalars(code[j][2][0]) & address:
                found.append("%x: %s after %x: %s" % (at, op, code[j][0], code[j][1]))
            todo += [(k, states + wait_states(code[j][1], code[j][2])) for k in before[j]]
    return loads, found


def test_addresses_of_loads_into_lds_have_settled(tmp_path):
    """The attention's loads into LDS are written in assembly, where the compiler keeps no wait states."""
    total = 0
    for code in parts(tmp_path):
        lines, name = [], ""
        proc = subprocess.Popen([TOOLS["llvm-objdump"], "-d", code], stdout=subprocess.PIPE, text=True)
        for line in list(proc.stdout) + ["end>:\n"]:
            if line.endswith(">:\n"):
                if "tree_attention_tile" in name:
                    loads, found = address_hazards(lines)
                    assert not found, (name, found[:3])
                    total += loads
                name, lines = line, []
            elif "tree_attention_tile" in name:
                lines.append(line)
        assert proc.wait() == 0
    assert total >= 100


def test_the_address_check_finds_planted_hazards():
    listing = lambda *code: ["\t%s // %012X: 00000000" % (c, 4 * i) for i, c in enumerate(code)]
    write, load = "v_readlane_b32 s5, v1, 3", "global_load_lds_dwordx4 v2, s[4:5]"
    assert address_hazards(listing(write, "s_mov_b32 m0, s9", "s_nop 0", load)) [1]
    assert not address_hazards(listing(write, "s_nop 4", "s_mov_b32 m0, s9", "s_nop 0", load))[1]
    assert not address_hazards(listing("v_readlane_b32 s6, v1, 3", load))[1]
    assert not address_hazards(listing("s_mov_b32 s5, s7", load))[1]
