"""What the compiler kept of the built kernels in scratch memory, read from the code objects in the library: kernels whose loops
are measured without it have to stay so."""
import re
import struct

import pytest

from paper_2604_09731_amd import binding as B

msgpack = pytest.importorskip("msgpack")


def _kernels():
    """name -> metadata of every gfx950 kernel in the library's bundles."""
    data, found, at = open(B.LIB_PATH, "rb").read(), {}, 0
    magic = b"__CLANG_OFFLOAD_BUNDLE__"
    while (at := data.find(magic, at)) >= 0:
        entries, = struct.unpack_from("<Q", data, at + len(magic))
        p = at + len(magic) + 8
        for _ in range(entries if entries < 16 else 0):         # (the compiler's own string has no entries behind it)
            offset, size, length = struct.unpack_from("<QQQ", data, p)
            target, p = data[p + 24:p + 24 + length], p + 24 + length
            if b"gfx950" in target and size:
                found.update(_notes(data[at + offset:at + offset + size]))
        at += len(magic)
    return found


def _notes(elf):
    sections, = struct.unpack_from("<Q", elf, 40)
    size, count = struct.unpack_from("<HH", elf, 58)
    for i in range(count):
        kind, = struct.unpack_from("<I", elf, sections + i * size + 4)
        offset, length = struct.unpack_from("<QQ", elf, sections + i * size + 24)
        if kind == 7:                                           # a note: name size, description size, type; both padded to 4
            name, desc, _ = struct.unpack_from("<III", elf, offset)
            start = offset + 12 + (name + 3) // 4 * 4
            meta = msgpack.unpackb(elf[start:start + desc])
            return {k[".name"]: k for k in meta["amdhsa.kernels"]}
    return {}


def test_prompt_kernels_without_a_window_keep_nothing_in_scratch():
    """The exception: 256 rows of head dim 64 with log-sum-exp, 64 rows a wavefront."""
    prompts = {n: k for n, k in _kernels().items() if re.search(r"prompt_bf16_kernel.*ELb0EE|prompt_f32_kernel.*ELb0EE", n)}
    assert len(prompts) == 14
    spilled = {n for n, k in prompts.items() if k[".private_segment_fixed_size"] or k[".vgpr_spill_count"]}
    assert all("ILi64ELi4ELi4ELb1E" in n for n in spilled), spilled
