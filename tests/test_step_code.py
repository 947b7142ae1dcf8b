"""Wait states in the code built here for gfx950.

The compiler leaves the instructions of inline assembly as they are, so what the hardware does not wait for by itself is
counted in the built kernels: a load into LDS takes its address from M0, which a scalar instruction must have written at
least one wait state before, and the scalar registers of a load's address must not have been written by a vector
instruction in the five wait states before it.
"""

import re
import subprocess

import pytest

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """The instructions of every kernel of libgrid.so that loads into LDS, by name."""
    from paper_2607_11951_amd import build
    if not build.OUT.exists():
        build.build()
    at = tmp_path_factory.mktemp("code")
    (at / "lib.so").write_bytes(build.OUT.read_bytes())
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=at, check=True, capture_output=True)
    found = {}
    for code in at.glob("*gfx950"):
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", code], check=True,
                              capture_output=True, text=True).stdout
        for part in re.split(r"^<", text, flags=re.M)[1:]:
            name, _, body = part.partition(">:")
            lines = [l.split("//")[0].strip() for l in body.split("\n")]
            if "global_load_lds" in body:
                found[name] = [l for l in lines if l]
    assert found
    return found


def loads(lines):
    """(load into LDS, the instructions before it, nearest first, with the wait states between)"""
    for i, line in enumerate(lines):
        if line.startswith("global_load_lds"):
            before, waits = [], 0
            for x in reversed(lines[max(0, i - 16):i]):
                before.append((waits, x))
                waits += int(x.split()[1], 0) + 1 if x.startswith("s_nop") else 1
            yield line, before


def test_m0_is_written_a_wait_state_before_a_load_into_lds(kernels):
    for name, lines in kernels.items():
        for line, before in loads(lines):
            waits = next((w for w, x in before if re.match(r"s_\w+ m0,", x)), 16)
            assert waits >= 1, (name, line, [x for _, x in before[:3]])


def test_scalar_addresses_are_not_fresh_from_a_vector_instruction(kernels):
    for name, lines in kernels.items():
        for line, before in loads(lines):
            m = re.search(r"s\[(\d+):(\d+)\]", line)
            if not m:
                continue
            mine = range(int(m.group(1)), int(m.group(2)) + 1)
            for waits, x in before:
                w = re.match(r"v_read\w+ s(\d+)", x)
                assert not w or int(w.group(1)) not in mine or waits >= 5, (name, line, x)
