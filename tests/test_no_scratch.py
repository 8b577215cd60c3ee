"""The kernels of new tokens' attention hold what they work on in registers: none spills to scratch memory (told by the built library's own metadata)."""
import os
import re
import shutil
import struct
import subprocess

import pytest

from paper_2412_20105_amd import binding as st3

READELF = shutil.which("llvm-readelf") or "/opt/rocm/llvm/bin/llvm-readelf"


def code_objects(path):
    """The gfx950 code objects that hipcc bundled into the library."""
    data, magic, at = open(path, "rb").read(), b"__CLANG_OFFLOAD_BUNDLE__", -1
    while (at := data.find(magic, at + 1)) >= 0:
        n, = struct.unpack_from("<Q", data, at + len(magic))
        entry = at + len(magic) + 8
        for _ in range(n):
            offset, size, name = struct.unpack_from("<QQQ", data, entry)
            if b"gfx950" in data[entry + 24:entry + 24 + name] and size:
                yield data[at + offset:at + offset + size]
            entry += 24 + name


def kernels(path, tmp_path):
    """{name: (bytes of scratch a lane, vector registers spilled)}"""
    found = {}
    for i, image in enumerate(code_objects(path)):
        f = tmp_path / f"{i}.elf"
        f.write_bytes(image)
        notes = subprocess.run([READELF, "--notes", str(f)], check=True, capture_output=True, text=True).stdout
        for kernel in re.split(r"\n\s+- \.agpr_count:", notes)[1:]:
            get = lambda key: re.search(rf"\.{key}:\s+(\S+)", kernel).group(1)  # noqa: E731
            found[get("symbol")] = int(get("private_segment_fixed_size")), int(get("vgpr_spill_count"))
    return found


def test_attention_of_new_tokens_spills_nothing(tmp_path):
    if not os.path.exists(READELF):
        pytest.skip("no llvm-readelf")
    st3.lib()
    used = {name: x for name, x in kernels(st3.LIB_PATH, tmp_path).items() if "chunk_" in name}
    assert len(used) == 54                  # (36 for few rows, 8 for tiles, 8 for scores, 2 that join)
    assert not {name: x for name, x in used.items() if x != (0, 0)}
