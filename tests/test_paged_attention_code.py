"""What the compiler makes of the paged attention's assembly (compiled for gfx950 here, nothing is run)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2602_08387_amd import build as b

HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
SOURCE = os.path.join(b.CSRC, "paged_attention.hip")


def _compiled(folder, *args):
    out = folder / "out"
    r = subprocess.run([HIPCC, *b.FLAGS, "--offload-device-only", "-S", *args, SOURCE, "-o", str(out)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    return out.read_text()


@pytest.fixture(scope="module")
def ir(tmp_path_factory):
    return _compiled(tmp_path_factory.mktemp("ir"), "-emit-llvm")


def test_loads_to_lds_say_that_they_write_m0(ir):
    """The assembly sets m0; where that is not declared, the compiler may keep a value of its own in it across the block."""
    blocks = re.findall(r'asm sideeffect "([^"]*)", "([^"]*)"', ir)
    setting = [(text, constraints) for text, constraints in blocks if "m0" in text]
    assert len(setting) > 100 and all(" lds" in text or "_lds_" in text for text, _ in setting)
    assert all("~{m0}" in constraints.split(",") for _, constraints in setting), setting[0]


def _blocks(code):
    """Instructions of each assembly block."""
    return [[line.strip() for line in text.splitlines() if line.strip()] for text in re.findall(r";;?#ASMSTART\n(.*?);;?#ASMEND", code, re.S)]


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    return _compiled(tmp_path_factory.mktemp("code"))


def test_loads_to_lds_keep_their_distance_from_who_wrote_their_descriptor(code):
    """A buffer load reads its descriptor's scalar registers right only five wait states behind a vector instruction that wrote them, such as the one that
    brings a spilled register back.  The compiler counts none in front of an instruction that it does not see: the block holds them itself."""
    loads = [block for block in _blocks(code) if block and block[-1].startswith("buffer_load")]
    assert len(loads) > 100
    for block in loads:
        states = sum(int(op.split()[1], 0) + 1 if op.startswith("s_nop") else 1 for op in block[:-1])
        assert states >= 5, block


def test_a_wave_is_done_with_a_stage_before_it_loads_into_it(code):
    """rows_kernel's waves load a stage that they read from a round before, without a barrier between: what they read has to be waited for in the source, and not where the
    compiler happens to use it."""
    kernels = re.findall(r"^(_ZN2dl11rows_kernel\w+):", code, re.M)
    assert len(kernels) == 12, kernels
    for name in kernels:
        blocks = [b for b in _blocks(code[code.index(f"\n{name}:"):].split(".Lfunc_end")[0]) if b]
        waits = [i for i, b in enumerate(blocks) if b[0].startswith("s_waitcnt")]
        assert waits and all("vmcnt(0)" in blocks[i][0] and "lgkmcnt(0)" in blocks[i][0] for i in waits), (name, [blocks[i] for i in waits])
        assert any("_load" in b[-1] for b in blocks[waits[-1]:]), name
