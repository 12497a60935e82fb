"""Instructions of the library's kernels that need wait states between them have them, those written out in the source too, between
which the compiler puts none."""

import os
import re
import subprocess
import tempfile

import pytest

import paper_2411_15100_amd as xgm
from paper_2411_15100_amd import build as lib_build
from test_host_registers import code_objects

ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
MEMORY = ("global_", "buffer_", "scratch_", "flat_")
ENDS = ("s_branch", "s_endpgm", "s_setpc", "s_swappc")
CARRIES = ("v_add_co", "v_sub_co", "v_subrev_co", "v_addc_co", "v_subb_co", "v_subbrev_co", "v_mad_u64", "v_mad_i64", "v_div_scale")


def scalars(operand):
    """The scalar registers of an operand."""
    if m := re.fullmatch(r"s(\d+)", operand):
        return {int(m[1])}
    if m := re.fullmatch(r"s\[(\d+):(\d+)\]", operand):
        return set(range(int(m[1]), int(m[2]) + 1))
    return {operand} if operand in ("vcc", "m0") else set()


def written(name, operands):
    """The scalar registers that a vector instruction writes."""
    if not name.startswith("v_"):
        return set()
    return scalars(operands[1] if name.startswith(CARRIES) else operands[0]) if len(operands) > 1 else set()


@pytest.fixture(scope="module")
def listing():
    """[kernel, [name, operands] of each instruction] of the library."""
    objdump = os.path.join(ROCM, "llvm", "bin", "llvm-objdump")
    if not os.path.exists(objdump):
        pytest.skip("no llvm-objdump")
    xgm.load_library()  # (built if it is not)
    kernels = []
    for code in code_objects(open(lib_build.LIB, "rb").read()):
        with tempfile.NamedTemporaryFile(suffix=".co") as f:
            f.write(code)
            f.flush()
            text = subprocess.run([objdump, "-d", "--no-show-raw-insn", f.name], capture_output=True, text=True, check=True).stdout
        for line in text.splitlines():
            if m := re.match(r"[0-9a-f]+ <(.+)>:", line):
                kernels.append((m[1], []))
            elif m := re.match(r"\s+([a-z]\w+)\s*(.*?)\s*(//.*)?$", line):
                operands = [o for part in m[2].split(",") for o in part.split()[:1]]
                kernels[-1][1].append((m[1], operands))
    assert len(kernels) > 100
    return kernels


def states(name, operands):
    """Wait states that an instruction counts for."""
    return int(operands[0], 0) + 1 if name == "s_nop" else 1


def missing(code, reads, writes, needed):
    """Places where `needed` wait states do not lie between an instruction that writes what another one reads: reads(name, operands), writes(...) give registers."""
    found = []
    for at, one in enumerate(code):
        wanted, passed = reads(*one), 0
        if not wanted:
            continue
        for before in reversed(code[max(0, at - needed):at]):
            if passed >= needed or before[0].startswith(ENDS):
                break
            if wanted & writes(*before):
                found.append((at, passed, before, one))
            passed += states(*before)
    return found


def test_loads_to_lds_come_a_wait_state_behind_their_m0(listing):
    into_lds = lambda name, operands: {"m0"} if name.startswith(MEMORY) and "_load_lds" in name else set()    # noqa: E731
    sets = lambda name, operands: {"m0"} & set(operands[:1]) if name.startswith("s_") else set()              # noqa: E731
    loads = sum(bool(into_lds(*one)) for _, code in listing for one in code)
    assert loads > 100
    found = {kernel: len(m) for kernel, code in listing if (m := missing(code, into_lds, sets, 1))}
    assert not found, (sum(found.values()), loads, found)


def test_loads_with_a_scalar_address_come_five_wait_states_behind_a_vector_instruction_that_writes_it(listing):
    def address(name, operands):
        return set().union(*map(scalars, operands), {"m0"} if "_load_lds" in name else ()) if name.startswith(MEMORY) else set()

    loads = sum(bool(address(*one)) for _, code in listing for one in code)
    assert loads > 1000
    found = {kernel: m[:2] for kernel, code in listing if (m := missing(code, address, written, 5))}
    assert not found, (loads, found)


def test_texts_leave_m0_to_the_compiler():
    """Loads to LDS take it as an operand; set in a text, it would change behind the compiler's back."""
    found = 0
    for name in os.listdir(lib_build.CSRC):
        for text in re.findall(r"\basm\b[^;]*;", open(os.path.join(lib_build.CSRC, name)).read()):
            assert not re.search(r"\bm0,", text), (name, text)
            if "_load_lds" in text:
                found += 1
                assert '"{m0}"' in text, (name, text)
    assert found
