"""The kernels of the iteration operators keep everything in registers. A vector register that is spilled costs memory traffic in an inner
loop, and more: the compiler has been seen to place such a store where lanes were switched off, which then read something else back."""
import os
import re
import struct
import subprocess

import pytest

from paper_2602_02987_amd import build

READELF = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build.HIPCC))), "llvm", "bin", "llvm-readelf")
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def device_code(path):
    """The gfx950 code objects in a library: bundles of a magic word, a count, and (offset, size, name) of each entry."""
    data = open(path, "rb").read()
    at = data.find(MAGIC)
    while at >= 0:
        n, = struct.unpack_from("<Q", data, at + len(MAGIC))
        pos = at + len(MAGIC) + 8
        for _ in range(n):
            offset, size, length = struct.unpack_from("<QQQ", data, pos)
            name = data[pos + 24:pos + 24 + length].decode()
            pos += 24 + length
            if "gfx950" in name and size:
                yield data[at + offset:at + offset + size]
        at = data.find(MAGIC, at + 1)


def test_no_kernel_spills(tmp_path):
    if not os.path.exists(READELF):
        pytest.skip("llvm-readelf is not installed")
    seen = {}
    for i, code in enumerate(device_code(build.lib_path())):
        f = tmp_path / f"{i}.co"
        f.write_bytes(code)
        notes = subprocess.run([READELF, "--notes", str(f)], capture_output=True, text=True, check=True).stdout
        for part in re.split(r"\n\s+- \.agpr_count:", notes)[1:]:
            name = re.search(r"\.name:\s+(\S+)", part.split(".args:")[-1]).group(1) if ".args:" in part else ""
            name = re.findall(r"\.symbol:\s+(\S+)", part)[0] if re.findall(r"\.symbol:\s+(\S+)", part) else name
            seen[name] = (int(re.search(r"\.vgpr_spill_count:\s+(\d+)", part).group(1)), int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", part).group(1)))
    ours = {n: v for n, v in seen.items() if re.search("gnr_(attention|kv|adapters)", n)}
    assert len(ours) > 20
    assert {n: v for n, v in ours.items() if v != (0, 0)} == {}
