"""Shifts of 64 bits by an amount of a lane's own, in the assembly of the library as built.  Such a shift gave wrong results, in one wave of some ten thousand, where its amount
lay in the last register of the wave's allocation."""
import os
import re
import subprocess

import pytest

from paper_2511_18871_amd import build

LLVM = "/opt/rocm/llvm/bin/"
SHIFT = re.compile(r"\tv_(?:lshrrev_b64|lshlrev_b64|ashrrev_i64) v\[\d+:\d+\], v(\d+),")
GRANULE = 8               # registers are given to a wave by eights


def tool(name, *args):
    return subprocess.run([LLVM + name, *args], check=True, capture_output=True, text=True).stdout


def kernels(source, folder):
    """[(name, assembly, registers, accumulation registers among them)] of a source's device code."""
    obj, fat, elf = os.path.join(build.OBJ, source.replace(".hip", ".o")), os.path.join(folder, "fat"), os.path.join(folder, "elf")
    tool("llvm-objcopy", "--dump-section", f".hip_fatbin={fat}", obj, os.path.join(folder, "copy"))
    tool("clang-offload-bundler", "--unbundle", "--type=o", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", f"--input={fat}", f"--output={elf}")
    bodies = re.split(r"^[0-9a-f]+ <(.+)>:$", tool("llvm-objdump", "-d", elf), flags=re.M)
    body = dict(zip(bodies[1::2], bodies[2::2]))
    found = []
    for note in re.split(r"^ *- (?=\.agpr_count:)", tool("llvm-readelf", "--notes", elf), flags=re.M)[1:]:
        value = lambda key: re.search(rf"^ *{re.escape(key)}: +(\S+)$", "  " + note, flags=re.M).group(1)
        found.append((value(".name"), body[value(".name")], int(value(".vgpr_count")), int(value(".agpr_count"))))
    return found


@pytest.mark.skipif(not os.path.exists(LLVM + "llvm-objdump"), reason="no disassembler")
@pytest.mark.parametrize("source", [s for s in build.SOURCES if s != "sp_api.hip"])          # (which has no kernels)
def test_amounts_of_64_bit_shifts(source, tmp_path):
    if not os.path.exists(os.path.join(build.OBJ, source.replace(".hip", ".o"))):
        pytest.skip("not built")
    found = kernels(source, str(tmp_path))
    assert found and all("s_endpgm" in text for _, text, _, _ in found)
    for name, text, registers, accumulators in found:
        amounts = {int(x) for x in SHIFT.findall(text)}
        last = {-(-n // GRANULE) * GRANULE - 1 for n in (registers, registers - accumulators)} | {registers - 1, registers - accumulators - 1}
        assert not amounts & last, f"{name}: v{amounts & last} of {registers}"
        if source in ("sp_pages.hip", "sp_tree.hip"):                    # where it was seen, and the code beside it: none at all
            assert not amounts, f"{name}: {sorted(amounts)}"
