"""The scans of test_generated_code.py over the sources that the ring and the paged cache share: the matrix
absorption (k_attend.hip), the cache writes, the layer kernels. They take minutes to compile, so that the objects
that the library was linked from are disassembled, where these are not older than the sources."""
import glob
import os
import re
import shutil
import subprocess

import pytest

from tests import test_generated_code
from tests._build_once import _builder, ensure_built
from tests.test_generated_code import early_work, unsettled_m0

# loads into LDS that the scan has to find, at least
SOURCES = {"k_attend.hip": 150, "k_cache_write.hip": 800, "k_layer.hip": 90, "k_pages_copy.hip": 0}
OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


def functions(source, tmp_path):
    """The disassembled functions of a source's device code, with labels as the compiler writes them."""
    build = _builder()
    if not os.path.exists(OBJDUMP):
        pytest.skip("llvm-objdump not found")
    ensure_built()
    obj = os.path.join(build.BUILD, source + ".o")
    inputs = [os.path.join(build.CSRC, source), *glob.glob(os.path.join(build.CSRC, "*.h"))]
    if not os.path.exists(obj) or os.path.getmtime(obj) < max(map(os.path.getmtime, inputs)):
        obj = build._compile(inputs[0], [], str(tmp_path))
    shutil.copy(obj, tmp_path / "own.o")
    subprocess.run([OBJDUMP, "--offloading", "own.o"], cwd=tmp_path, check=True, capture_output=True)
    (code,) = glob.glob(str(tmp_path / f"own.o.*{build.ARCH}"))
    text = subprocess.run([OBJDUMP, "-d", "--symbolize-operands", code], check=True, capture_output=True, text=True).stdout
    text = re.sub(r"^<(L\d+)>:", r"\1:", text, flags=re.M)
    return re.split(r"^[0-9a-f]+ <.*>:\n", text, flags=re.M)[1:]


@pytest.mark.parametrize("source", SOURCES)
def test_masks_are_restored_first_and_m0_is_settled(source, tmp_path):
    loads, found = 0, []
    parts = functions(source, tmp_path)
    assert parts
    for text in parts:  # (labels are a function's own)
        n, bad = unsettled_m0(text)
        loads += n
        found += bad + early_work(text)
    assert loads >= SOURCES[source] and not found, (loads, found[:3])


def test_the_disassembly_shows_a_planted_mistake():
    """The form that the scans read, as the disassembler writes it."""
    head = "\ts_cbranch_execz L3     // 000000037F44: BF8802E3\n\tv_mov_b32_e32 v1, 0    // 00: 7E\n<L3>:\n"
    text = head + "\tv_accvgpr_write_b32 a1, v7   // 00: D3\n\ts_or_b64 exec, exec, s[2:3]  // 00: 87\n"
    assert early_work(re.sub(r"^<(L\d+)>:", r"\1:", text, flags=re.M)) == ["v_accvgpr_write_b32 a1, v7"]
    load = "\ts_mov_b32 m0, s4   // 00: BE\n\tglobal_load_lds_dwordx4 v[0:1], off   // 00: DD\n"
    assert unsettled_m0(load)[1]


def test_every_source_is_scanned():
    """(videomla_noalloc.hip has no kernel.)"""
    names = {os.path.basename(p) for p in glob.glob(os.path.join(_builder().CSRC, "*.hip"))}
    assert names == set(SOURCES) | set(test_generated_code.SOURCES) | {"videomla_noalloc.hip"}
