"""What the compiler made of the kernels of the 8-bit product: distances around matrix instructions that are written in assembly, which it does not
know about, and registers."""
import os
import re

import pytest

from paper_2106_16064_amd import layers
from test_layers_resources import objects, registers, tool  # noqa: F401


def early_uses(lines, results_after, operands_after):
    """Instructions of one kernel's listing, other than matrix ones, that touch a matrix instruction's result, matrix instructions that read such a result as an
    operand, and those that read what another vector instruction wrote, before the wait states are over; counted along the code as it stands."""
    now, results, written, found = 0, {}, {}, []
    for line in lines:
        op, _, rest = line.partition(" ")
        now += 1
        if op == "s_nop":
            now += int(rest, 0)
        elif op.startswith("v_mfma"):
            into, a, b, _, *scales = rest.split(" op_sel")[0].split(", ")
            sources = registers(a) | registers(b) | set().union(*(registers(s) for s in scales))
            if any(now - written.get(r, -99) <= operands_after for r in sources) or any(now - results.get(r, -99) <= results_after for r in sources):
                found.append(line)
            results.update((r, now) for r in registers(into))
        elif op.startswith(("v_", "ds_", "buffer_", "global_", "scratch_")):
            if any(now - results.get(r, -99) <= results_after for r in registers(rest)):
                found.append(line)
            if op.startswith("v_"):
                written.update((r, now) for r in registers(rest.split(", ")[0]))
        elif op in ("s_branch", "s_endpgm"):
            results, written = {}, {}
    return found


def test_the_scan_finds_what_it_looks_for():
    product = "v_mfma_scale_f32_16x16x128_f8f6f4 v[0:3], v[4:11], v[12:19], v[0:3], v20, v21 op_sel_hi:[0,0,0]"
    scan = lambda lines: early_uses(lines, 19, 2)  # noqa: E731
    assert scan([product, product, "s_nop 15", "s_nop 15", "v_mov_b32_e32 v9, v1"]) == []
    assert scan([product, "s_nop 9", "v_mov_b32_e32 v9, v1"]) == ["v_mov_b32_e32 v9, v1"]
    assert scan(["v_mov_b32_e32 v20, v30", product]) == [product]
    assert scan(["v_mov_b32_e32 v20, v30", "s_nop 1", product]) == []


def test_wait_states_and_spills_of_the_8bit_product(objects):  # noqa: F811
    kernels, spills, name = {}, {}, None
    for code in objects:
        lines = []
        for line in tool("llvm-objdump", "-d", "--no-show-raw-insn", code).splitlines():
            m = re.match(r"[0-9a-f]+ <(\S+)>:", line)
            if m:
                lines = kernels.setdefault(m[1], [])
            elif line.startswith("\t"):
                lines.append(re.sub(r"\s+", " ", line.split("//")[0]).strip())
        for line in tool("llvm-readelf", "--notes", code).splitlines():
            m = re.match(r"    \.(name|vgpr_spill_count): +(\S+)", line)
            if m and m[1] == "name":
                name = m[2]
            elif m:
                spills[name] = int(m[2])
    found = {name: lines for name, lines in kernels.items() if "product_8bit_kernel" in name}
    assert len(found) == 9                                           # three tiles, three types
    for name, lines in found.items():
        assert sum(line.startswith("v_mfma_scale") for line in lines) >= 4 * 3, name
        assert early_uses(lines, 19, 2) == [], name
        assert spills[name] == 0, name


@pytest.mark.parametrize("kernel", ["narrow_linear_kernel", "narrow_linear_backward_kernel", "rms_norm_kernel", "rms_norm_backward_kernel", "linear_slope_kernel", "quantise_kernel"])
def test_vector_registers_are_not_spilled(objects, kernel):  # noqa: F811
    name, count = None, 0
    for code in objects:
        for line in tool("llvm-readelf", "--notes", code).splitlines():
            m = re.match(r"    \.(name|vgpr_spill_count): +(\S+)", line)
            if m and m[1] == "name":
                name = m[2]
            elif m and re.search(rf"\d{kernel}I", name):
                assert int(m[2]) == 0, name
                count += 1
    assert count >= 2, os.listdir(os.path.dirname(objects[0]))


def notes(objects):  # noqa: F811
    """Of each kernel what its notes say."""
    found = {}
    for code in objects:
        for entry in re.split(r"\n  - ", tool("llvm-readelf", "--notes", code)):
            name = re.search(r"^ +\.name: +(_Z\S+)", entry, re.M)
            if name:
                found[name[1]] = {key: int(value) for key, value in re.findall(r"^ *\.(\w+): +(\d+)$", entry, re.M)}
    return found


def test_as_many_workgroups_of_the_narrow_gradient_as_a_cu_holds(objects):  # noqa: F811
    """Registers and LDS of each kernel against what the workspace is for: a workgroup too few leaves room that nothing uses, one too many waits for its turn.
    Types of 16 bits and forms of x and z share a number."""
    L = layers.lib()
    fits = {}
    for name, note in notes(objects).items():
        m = re.search(r"29narrow_linear_backward_kernelI(f|DF16b|DF16_)Li(\d+)ELi(\d+)ELb(\d)ELb(\d)E", name)
        if not m:
            continue
        wide, width, out, x8, whole = m[1] == "f", int(m[2]), int(m[3]), int(m[4]), int(m[5])
        waves = note["max_flat_workgroup_size"] // 64
        room = min(163840 // note["group_segment_fixed_size"], 512 // (-(-note["vgpr_count"] // 8) * 8) * 4 // waves, 2)
        key = (wide, width, out, x8 if wide else None, whole)
        fits[key] = min(fits.get(key, 2), room)
    assert len(fits) == 8 * 4 + 9 * 2                                # 128 x 128 floats take tiles
    for (wide, width, out, x8, whole), most in fits.items():
        w, o = (width, out) if whole else (width - 1, out - 1)
        for keep in (layers.KEEP_WHOLE, layers.KEEP_8BIT) if x8 is None else (layers.KEEP_8BIT,) if x8 else (layers.KEEP_WHOLE,):
            for number in (layers.F32,) if wide else (layers.BF16, layers.F16):
                size = L.dgsp_linear_backward_workspace_bytes(1 << 24, w, o, number, layers.GELU, keep)
                found = [groups for groups in (256, 512) for parts in (1, 2, 4) if size == groups * (parts * o * w + o) * 4]
                assert found == [256 * most], (wide, width, out, x8, whole)


# Where a row's ends are looked at one by one, or a row is read twice, comparisons and addresses are more than the scalar registers hold: so many at most go to
# lanes of vector registers.
SCALARS = {"rms_norm_kernel": 26, "rms_norm_backward_kernel": 23, "rms_norm_long_kernel": 51, "rms_norm_backward_long_kernel": 19, "narrow_linear_kernel": 62,
           "narrow_linear_backward_kernel": 132}
NONE = ["few_rows_kernel", "few_rows_8bit_kernel", "linear_join_kernel", "join_kernel", "join_deep_kernel", "linear_slope_kernel", "quantise_kernel", "dequantise_kernel",
        "column_sums_kernel", "product_8bit_kernel", "tile_kernel", "float_tile_kernel", "rms_norm_long_params_kernel", "lay_out_kernel"]


@pytest.mark.parametrize("kernel", [*SCALARS, *NONE])
def test_nothing_is_spilled_to_memory(objects, kernel):  # noqa: F811
    found = {name: note for name, note in notes(objects).items() if re.search(rf"\d{kernel}I", name)}
    assert len(found) >= 2
    for name, note in found.items():
        assert note["vgpr_spill_count"] == 0 and note["private_segment_fixed_size"] == 0, name
        whole = re.search(r"Li(32|64|128)ELi(32|64|128)ELb[01]ELb1E", name) if "narrow" in kernel else None
        assert note["sgpr_spill_count"] <= (0 if whole else SCALARS.get(kernel, 0)), name
