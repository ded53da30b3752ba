"""The layers' library without a GPU: its symbols, its sizes, the generator behind dropout and what is refused before any launch."""
import os
import re
import subprocess
import sys

import pytest

import layer_reference as ref
from paper_2106_16064_amd import binding as dg
from paper_2106_16064_amd import layers

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "dgsp_layers.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    declared = set(re.findall(r"^(?:int|int64_t)\s+(dgsp_\w+)\s*\(", text, re.M))
    assert declared == set(layers.EXPORTS)
    for name in declared:
        getattr(layers.lib(), name)


def test_every_source_counts_for_a_stale_build():
    from paper_2106_16064_amd import build
    known = {f.resolve() for f in (*build.LAYERS_SOURCES, *build.LAYERS_HEADERS, build.LAYERS_TORCH_SOURCE)}
    assert {f.resolve() for f in build.LAYERS_CSRC.iterdir()} <= known and (build.HERE.parent / "include" / "dgsp_layers.h").resolve() in known


def test_header_compiles_as_c(tmp_path):
    source = tmp_path / "c.c"
    source.write_text('#include "dgsp_layers.h"\nint main(void) { dgsp_dropout_t d = {0.5, 1, 2, 0}; return (int)d.offset - 2; }\n')
    exe = tmp_path / "c"
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(source)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0


# Known answers that the generator's authors publish with it: counter, key, result.
KNOWN = [
    ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
    ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
    ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1)),
]


@pytest.mark.parametrize("counter,key,result", KNOWN)
def test_the_oracles_generator_gives_the_published_numbers(counter, key, result):
    assert tuple(ref.philox(counter, key)) == result


def test_the_librarys_generator_is_the_oracles(tmp_path):
    """Its header, compiled for the host, on the published counters and on the numbers of a few elements."""
    source = tmp_path / "check.cpp"
    source.write_text('#include <cstdio>\n#include <cstdlib>\n#include "%s/paper_2106_16064_amd/csrc_layers/drop_mask.hpp"\n'
                      'int main(int n, char** a) {\n'
                      '    uint32_t v[6];\n'
                      '    for (int i = 0; i < 6; ++i) v[i] = (uint32_t)strtoul(a[1 + i], nullptr, 0);\n'
                      '    const dgsp::PhiloxWords r = dgsp::philox4x32(v[0], v[1], v[2], v[3], v[4], v[5]);\n'
                      '    dgsp::DropMask d{};\n'
                      '    d.dropped = 20000;\n    d.key0 = v[4];\n    d.key1 = v[5];\n'
                      '    printf("%%u %%u %%u %%u %%u\\n", r.w[0], r.w[1], r.w[2], r.w[3],\n'
                      '           dgsp::keep_bits(d, (uint64_t)v[3] << 32 | v[2], v[1], v[0]));\n}\n' % ROOT)
    exe = tmp_path / "check"
    subprocess.run(["g++", "-std=c++17", "-O1", "-o", str(exe), str(source)], check=True)
    for counter, key, result in KNOWN + [((3, 5, 7, 9), (11, 13), tuple(ref.philox((3, 5, 7, 9), (11, 13))))]:
        *words, bits = map(int, subprocess.run([str(exe), *map(str, counter + key)], check=True, capture_output=True, text=True).stdout.split())
        assert tuple(words) == result
        numbers = [h for w in result for h in (w & 0xFFFF, w >> 16)]
        assert bits == sum((h >= 20000) << j for j, h in enumerate(numbers))
    seed, offset = 11 | 13 << 32, 7 | 9 << 32
    assert list(ref.halves(6, 32, seed, offset)[5, 24:32]) == [h for w in ref.philox((3, 5, 7, 9), (11, 13)) for h in (w & 0xFFFF, w >> 16)]


def test_sizes_of_workspaces():
    L = layers.lib()
    assert L.dgsp_layer_norm_backward_workspace_bytes(0, 8) >= 0 and L.dgsp_layer_norm_backward_workspace_bytes(100, 0) == 0
    assert L.dgsp_gated_ff_saved_bytes(100, 8, 0, 8, 0) == 0 and L.dgsp_gated_ff_workspace_bytes(100, 8, 16, 8, 7) == 0
    big = L.dgsp_gated_ff_saved_bytes(1 << 24, 64, 4096, 64, layers.F32)
    assert big % 16 == 0 and big >= 0


def test_tensors_on_the_host_are_refused():
    import torch
    x = torch.randn((4, 8))
    for call in (lambda: layers.layer_norm(x), lambda: layers.dropout(x, 0.5, 1), lambda: layers.add_layer_norm(x, x),
                 lambda: layers.gated_ff(x, x, x, x)):
        with pytest.raises(dg.DgspError, match="GPU"):
            call()
    with pytest.raises(dg.DgspError, match="silu, gelu, relu"):
        layers.gated_ff(x, x, x, x, activation=3)


def test_sizes_of_a_block_without_rows():
    """Deep enough for products to be split along the depth, where nothing is left to split.  In a process of its own: a division by
    zero ends it."""
    script = ("from paper_2106_16064_amd import layers\n"
              "L = layers.lib()\n"
              "for t in (layers.F32, layers.BF16, layers.F16):\n"
              "    for block in ((4096, 64, 64), (64, 1024, 64), (40, 4096, 64), (512, 1024, 512), (64, 64, 4096), (4096, 16384, 4096), (1, 1, 1)):\n"
              "        for size in (L.dgsp_gated_ff_saved_bytes, L.dgsp_gated_ff_workspace_bytes, L.dgsp_gated_ff_backward_workspace_bytes):\n"
              "            assert 0 <= size(0, *block, t) <= size(1, *block, t), (block, t)\n")
    run = subprocess.run([sys.executable, "-c", script], cwd=ROOT, capture_output=True, text=True)
    assert run.returncode == 0, (run.returncode, run.stderr)


def test_sizes_of_extents_that_are_refused_are_zero():
    L = layers.lib()
    most = (1 << 31) - 1 - 4096
    assert L.dgsp_layer_norm_backward_workspace_bytes(most, 64) > 0 and L.dgsp_layer_norm_backward_workspace_bytes(1, most) > 0
    for rows, width in ((-1, 8), (8, 0), (8, -1), (most + 1, 64), (1, most + 1), (1 << 62, 8), (8, 1 << 62), (8, (1 << 63) - 1)):
        assert L.dgsp_layer_norm_backward_workspace_bytes(rows, width) == 0, (rows, width)
    for size in (L.dgsp_gated_ff_saved_bytes, L.dgsp_gated_ff_workspace_bytes, L.dgsp_gated_ff_backward_workspace_bytes):
        for extents in ((most + 1, 8, 8, 8), (-1, 8, 8, 8), (8, 1 << 22, 8, 8), (8, 8, 1 << 62, 8), (8, 8, 8, 0)):
            assert size(*extents, layers.F32) == 0, extents


def test_a_block_of_more_tiles_than_a_launch_has_is_refused():
    """Before anything is enqueued: the pointers are not looked at."""
    L = layers.lib()
    rows, p, most = 1 << 30, 1 << 20, (1 << 63) - 1
    matrices = [p, 8] * 4
    assert L.dgsp_gated_ff(rows, 8, 8, 8, layers.F32, layers.SILU, *matrices, p, 8, None, p, most, None) == dg.ERR_UNSUPPORTED
    assert L.dgsp_gated_ff_backward(rows, 8, 8, 8, layers.F32, layers.SILU, *matrices, p, 8, p, p, p, p, p, p, most, None) == dg.ERR_UNSUPPORTED
