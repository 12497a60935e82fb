"""No kernel for 8-bit matrices or beams keeps vector registers in memory: a reload waits for every load that is on its way to LDS."""

import os
import re
import struct
import subprocess
import tempfile

import pytest

import paper_2411_15100_amd as xgm
from paper_2411_15100_amd import build as lib_build

NAMES = ("f8_quantize_kernel", "f8_few_kernel", "f8_many_kernel", "f8_turn_scales_kernel", "embed_kernel", "beam_slices_kernel", "beam_join_kernel", "reorder_kernel")


def code_objects(data):
    """The gfx950 code of every source file: each has a bundle of its own."""
    at = data.find(b"__CLANG_OFFLOAD_BUNDLE__")
    while at >= 0:
        entry = at + 32
        for _ in range(struct.unpack_from("<Q", data, at + 24)[0]):
            offset, size, length = struct.unpack_from("<QQQ", data, entry)
            if data[entry + 24:entry + 24 + length].endswith(b"gfx950"):
                yield data[at + offset:at + offset + size]
            entry += 24 + length
        at = data.find(b"__CLANG_OFFLOAD_BUNDLE__", at + 1)


def test_kernels_keep_their_registers():
    readelf = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-readelf")
    if not os.path.exists(readelf):
        pytest.skip("no llvm-readelf")
    xgm.load_library()  # (built if it is not)
    found = {name: [] for name in NAMES}
    for code in code_objects(open(lib_build.LIB, "rb").read()):
        with tempfile.NamedTemporaryFile(suffix=".co") as f:
            f.write(code)
            f.flush()
            notes = subprocess.run([readelf, "--notes", f.name], capture_output=True, text=True, check=True).stdout
        for kernel, scratch, vgpr in re.findall(r"\.name: +(\S+).*?\.private_segment_fixed_size: (\d+).*?\.vgpr_spill_count: (\d+)", notes, re.S):
            for name in NAMES:
                if name in kernel:
                    found[name].append((int(scratch), int(vgpr)))
    assert all(found.values()), found
    assert all(k == (0, 0) for kernels in found.values() for k in kernels), found
