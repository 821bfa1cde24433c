"""The written-out loads into LDS (mma_tile.h, load_to_lds): the compiler does not keep
the wait states that such a load needs after a vector instruction has written one of
its scalar operands (5), so the sources must, and this reads the gfx950 assembly to see
that none is short. No kernel that uses them spills to scratch."""

import os
import re
import subprocess

import pytest

from paper_1904_00962_amd import build

SOURCES = [s for s in build.SOURCES
           if s.endswith(".hip") and '#include "mma_tile.h"' in open(s).read()]
WAIT_STATES = 5


@pytest.fixture(scope="module", params=SOURCES, ids=[os.path.basename(s) for s in SOURCES])
def assembly(request, tmp_path_factory):
    out = tmp_path_factory.mktemp("isa") / "k.s"
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    r = subprocess.run([build.hipcc(), *flags, "-I", build.INCLUDE, "-I", build.CSRC,
                        "--cuda-device-only", "-S", request.param, "-o", str(out)],
                       capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stderr[-2000:]
    return out.read_text()


def scalars(token):
    m = re.match(r"s\[(\d+):(\d+)\]$", token)
    if m:
        return set(range(int(m.group(1)), int(m.group(2)) + 1))
    m = re.match(r"s(\d+)$", token)
    return {int(m.group(1))} if m else {token} if token in ("m0", "vcc") else set()


def short_waits(text):
    """[(vector instruction, load)] with too few wait states between, and the loads."""
    lines = [line.strip() for line in text.splitlines()]
    code = [line for line in lines if line and line[0] not in ";." and not line.endswith(":")]
    found, loads = [], 0
    for k, line in enumerate(code):
        if not re.match(r"buffer_load_\w+ .* lds$", line):
            continue
        loads += 1
        need = scalars(re.search(r"s\[\d+:\d+\]", line).group(0)) | {"m0"}
        waits = 0
        for before in reversed(code[max(0, k - WAIT_STATES):k]):
            if waits >= WAIT_STATES:
                break
            if before.startswith("v_") and scalars(before.split(None, 1)[1].split(",")[0]) & need:
                found.append((before, line))
            m = re.match(r"s_nop (\d+)", before)
            waits += int(m.group(1)) + 1 if m else 1
    return found, loads


def test_the_reader_sees_a_short_wait():
    bad = "v_readfirstlane_b32 s36, v8\ns_nop 0\nbuffer_load_dwordx4 v13, s[36:39], 0 offen lds\n"
    good = bad.replace("s_nop 0", "s_nop 4")
    assert len(short_waits(bad)[0]) == 1 and short_waits(good) == ([], 1)


def test_loads_wait_for_their_scalars(assembly):
    found, loads = short_waits(assembly)
    assert loads > 0 and not found, found[:5]


def test_no_spills(assembly):
    sizes = re.findall(r"\.amdhsa_private_segment_fixed_size\s+(\d+)", assembly)
    assert sizes and not any(int(s) for s in sizes)
