"""Host checks of the generated code of the kernels, compiled for gfx950 as build.py does.

Rejoined lanes: where a branch that lanes take differently ends, the block that they rejoin in restores the
execution mask first. In kernels that fill the register file the compiler has moved a value to another
register before that, for the lanes in the branch only; the other lanes then read what the register held.

m0: an instruction that loads into LDS by m0 needs one wait state behind the scalar write of m0, which the
compiler does not put into inline assembly."""
import functools
import os
import re
import shutil
import subprocess

import pytest

from tests._build_once import _builder
from tests.test_direct_loads import WAIT_STATES, parse, scalar_registers, writers

WORK = ("v_", "ds_", "global_", "buffer_", "scratch_", "flat_")
RESTORES = re.compile(r"s_or_b64 exec, exec|s_(or|andn2)_saveexec|s_xor_b64 exec, exec")
LEAVES = re.compile(r"s_c?branch|s_setpc|s_endpgm|s_and_saveexec|s_(mov|and|andn2)_b64 exec|s_barrier")


def instructions(text):
    for line in text.splitlines():
        t = re.split(r";|//", line)[0].strip()
        if t and not (t.startswith(".") and not t.endswith(":")):
            yield t


def early_work(text):
    """Vector instructions at the head of a block that lanes rejoin in, before the mask is restored."""
    code = list(instructions(text))
    joins = {t.split()[-1] for t in code if t.startswith("s_cbranch_execz")}
    bad, head = [], None
    for t in code:
        if t.endswith(":"):
            head = [] if t[:-1] in joins else None
        elif head is not None:
            if RESTORES.match(t):
                bad += head
                head = None
            elif LEAVES.match(t):
                head = None
            elif t.startswith(WORK) and not t.startswith(("v_readlane", "v_readfirstlane")):
                head.append(t)
    return bad


def unsettled_m0(text):
    """(loads into LDS, those right behind a write of m0)."""
    loads, bad, before = 0, [], ""
    for t in instructions(text):
        if re.match(r"(global_load_lds|buffer_load\S* .*\blds\b)", t):
            loads += 1
            if re.match(r"s_\S+ m0,", before):
                bad.append((before, t))
        before = t
    return loads, bad


@functools.lru_cache(maxsize=None)
def assembly(source):
    build = _builder()
    if shutil.which(build.HIPCC) is None:
        pytest.skip("hipcc not found")
    r = subprocess.run([build.HIPCC, *build.COMMON, "-x", "hip", "--cuda-device-only", "-S",
                        os.path.join(build.CSRC, source), "-o", "-"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    return r.stdout


def test_scans_find_planted_mistakes():
    head = "s_and_saveexec_b64 s[2:3], vcc\n s_cbranch_execz .LBB0_2\n v_mov_b32 v1, 0\n.LBB0_2: ; join\n"
    assert early_work(head + " v_accvgpr_write_b32 a1, v7\n s_or_b64 exec, exec, s[2:3]\n") == ["v_accvgpr_write_b32 a1, v7"]
    assert early_work(head + " s_or_b64 exec, exec, s[2:3]\n v_accvgpr_write_b32 a1, v7\n") == []
    load = "global_load_lds_dwordx4 v1, s[4:5]"
    assert unsettled_m0("s_mov_b32 m0, s1\n " + load)[1] and not unsettled_m0("s_mov_b32 m0, s1\n s_nop 0\n " + load)[1]


SOURCES = {"k_paged.hip": 100, "k_paged_wide.hip": 10, "k_paged_wide512.hip": 25, "k_paged_absorb.hip": 0,
           "k_attend_wide.hip": 20, "k_dense.hip": 4}


@pytest.mark.parametrize("source", SOURCES)
def test_masks_are_restored_first_and_m0_is_settled(source):
    text = assembly(source)
    assert early_work(text) == []
    loads, bad = unsettled_m0(text)
    assert loads >= SOURCES[source] and not bad, (loads, bad[:3])


@pytest.mark.parametrize("source,least", [("k_paged.hip", 64), ("k_paged_wide512.hip", 24)])
def test_scalar_bases_of_the_paged_loads_are_settled(source, least):
    """No VALU write of a load's scalar base in the wait states before it (see test_direct_loads)."""
    code, sources = parse(assembly(source))
    loads = [(i, scalar_registers(args[1])) for i, (op, args) in enumerate(code)
             if op == "global_load_lds_dwordx4" and len(args) > 1 and scalar_registers(args[1])]
    assert len(loads) >= least
    for i, base in loads:
        assert not writers(code, sources, i, base, WAIT_STATES), (source, i)
