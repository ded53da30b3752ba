"""What the compiler made of the layers' matrix kernels: registers and spills from the notes of the built library's code objects, and the
distances around matrix instructions that are written in assembly, which the compiler does not know about, from its listing."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LLVM = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin")
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def tool(name, *args):
    return subprocess.run([os.path.join(LLVM, name), *args], check=True, capture_output=True, text=True).stdout


@pytest.fixture(scope="module")
def objects(tmp_path_factory):
    """The code objects of the library's sources."""
    at = tmp_path_factory.mktemp("code")
    tool("llvm-objcopy", f"--dump-section=.hip_fatbin={at}/bundles", os.path.join(ROOT, "paper_2106_16064_amd", "libdgsp_layers.so"), f"{at}/copy")
    out = []
    for i, part in enumerate(open(f"{at}/bundles", "rb").read().split(MAGIC)[1:]):
        (at / f"bundle{i}").write_bytes(MAGIC + part)
        tool("clang-offload-bundler", "--unbundle", "--type=o", f"--input={at}/bundle{i}", f"--output={at}/code{i}",
             "--targets=hipv4-amdgcn-amd-amdhsa--gfx950")
        out.append(f"{at}/code{i}")
    return out


def test_tile_kernels_spill_nothing(objects):
    """The accumulators alone take half of the registers; a spilled one costs ten times the product."""
    found, name = {}, None
    for code in objects:
        for line in tool("llvm-readelf", "--notes", code).splitlines():
            m = re.match(r"    \.(name|vgpr_spill_count|sgpr_spill_count): +(\S+)", line)
            if m and m[1] == "name":
                name = m[2]
                found[name] = {}
            elif m:
                found[name][m[1]] = int(m[2])
    tiles = {name: r for name, r in found.items() if re.search(r"\d(float_)?tile_kernelI", name)}
    assert len(tiles) >= 30
    for name, r in tiles.items():
        assert r == {"vgpr_spill_count": 0, "sgpr_spill_count": 0}, name


def registers(text):
    out = set()
    for m in re.finditer(r"\bv\[(\d+):(\d+)\]|\bv(\d+)\b", text):
        out |= {int(m[3])} if m[3] else set(range(int(m[1]), int(m[2]) + 1))
    return out


def early_uses(lines):
    """Of one kernel's listing: instructions other than matrix ones that touch a matrix instruction's result, and matrix instructions that
    read a register another vector instruction has written, before the hardware's wait states (11 and 2) are over; counted along the code
    as it stands, an instruction as one state."""
    now, results, written, found = 0, {}, {}, []
    for line in lines:
        op, _, rest = line.partition(" ")
        now += 1
        if op == "s_nop":
            now += int(rest, 0)
        elif op.startswith("v_mfma"):
            into, *sources = rest.split(", ")
            for source in sources:
                if any(now - written.get(r, -9) <= 2 for r in registers(source)):
                    found.append(line)
            if any(now - results.get(r, -99) <= 11 for r in registers(sources[0]) | registers(sources[1])):
                found.append(line)
            results.update((r, now) for r in registers(into))
        elif op.startswith(("v_", "ds_", "buffer_", "global_")):
            if any(now - results.get(r, -99) <= 11 for r in registers(rest)):
                found.append(line)
            if op.startswith("v_"):
                written.update((r, now) for r in registers(rest.split(", ")[0]))
        elif op in ("s_branch", "s_endpgm"):
            results, written = {}, {}            # what follows is reached from elsewhere
    return found


def test_the_scan_finds_what_it_looks_for():
    product = "v_mfma_f32_16x16x32_bf16 v[0:3], v[4:7], v[8:11], v[0:3]"
    assert early_uses([product, product, "s_nop 15", "v_mov_b32_e32 v9, v1"]) == []
    assert early_uses([product, "s_nop 9", "v_mov_b32_e32 v9, v1"]) == ["v_mov_b32_e32 v9, v1"]
    assert early_uses(["v_mov_b32_e32 v2, v20", product]) == [product]
    assert early_uses(["v_mov_b32_e32 v2, v20", "s_nop 1", product]) == []


def test_matrix_results_and_operands_have_their_wait_states(objects):
    kernels = {}
    for code in objects:
        for line in tool("llvm-objdump", "-d", "--no-show-raw-insn", code).splitlines():
            m = re.match(r"[0-9a-f]+ <(\S+)>:", line)
            if m:
                lines = kernels.setdefault(m[1], [])
            elif line.startswith("\t"):
                lines.append(re.sub(r"\s+", " ", line.split("//")[0]).strip())
    tiles = {name: lines for name, lines in kernels.items() if re.search(r"\d+tile_kernelI", name)}
    assert len(tiles) >= 24
    for name, lines in tiles.items():
        assert sum(line.startswith("v_mfma") for line in lines) >= 16, name
        assert early_uses(lines) == [], name


def test_assembly_names_what_it_writes():
    """The compiler keeps values of its own in m0, the scalar flags and the like, and sees of an assembly statement what it names."""
    found = 0
    for source in sorted(os.listdir(os.path.join(ROOT, "paper_2106_16064_amd", "csrc_layers"))):
        text = open(os.path.join(ROOT, "paper_2106_16064_amd", "csrc_layers", source)).read()
        for statement in re.findall(r"\basm volatile\((.*?)\);", text, re.S):
            code, *operands = re.split(r'(?<!\\)"\s*:', statement, maxsplit=1)
            named = operands[0] if operands else ""
            for register in ("m0", "vcc", "exec", "scc"):
                if re.search(rf"\b(?:s|v)_\w+ {register}\b", code):
                    found += 1
                    assert f'"{register}"' in named, (source, statement)
    assert found >= 1
