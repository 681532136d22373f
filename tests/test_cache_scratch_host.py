"""CPU-only: no kernel of the 4-bit cache keeps anything in scratch memory: their registers are counted out to the last one, and a spill
would cost them more than what brought it.  Read from the kernel descriptors of the library that is built."""
import re
import struct

import pytest

import paper_2605_02568_amd as P

MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"
KERNELS = {
    "quantize_rows_kernel": 3, "dequantize_rows_kernel": 3, "quantized_attention_kernel": 8, "quantized_attention_few_kernel": 8,
    "accumulate_weights_kernel": 4, "gather_weights_kernel": 8, "clear_sums_kernel": 1, "add_sums_kernel": 1,
    "evict_select_kernel": 1, "evict_clear_kernel": 1, "evict_digits_kernel": 1, "evict_count_kernel": 1, "evict_move_kernel": 1,
    "evict_few_kernel": 1,
}


def _code_objects(blob):
    """The gfx950 code objects of every offload bundle in a file."""
    at = blob.find(MAGIC)
    while at >= 0:
        n, = struct.unpack_from("<Q", blob, at + len(MAGIC))
        entry = at + len(MAGIC) + 8
        for _ in range(n):
            offset, size, length = struct.unpack_from("<QQQ", blob, entry)
            target = blob[entry + 24:entry + 24 + length]
            entry += 24 + length
            if b"gfx950" in target:
                yield blob[at + offset:at + offset + size]
        at = blob.find(MAGIC, at + 1)


def _descriptors(elf):
    """Name and 64-byte descriptor of every kernel of a code object."""
    sections_at, = struct.unpack_from("<Q", elf, 40)
    n_sections, = struct.unpack_from("<H", elf, 60)
    sections = [struct.unpack_from("<IIQQQQIIQQ", elf, sections_at + 64 * i) for i in range(n_sections)]
    for kind, offset, size, link in ((s[1], s[4], s[5], s[6]) for s in sections):
        if kind != 2:  # the symbol table
            continue
        names = sections[link][4]
        for at in range(offset, offset + size, 24):
            name_at, _, _, index, value, _ = struct.unpack_from("<IBBHQQ", elf, at)
            name = elf[names + name_at:elf.index(b"\0", names + name_at)].decode()
            if name.endswith(".kd"):
                _, _, _, address, start = sections[index][:5]
                yield name[:-3], elf[start + value - address:start + value - address + 64]


@pytest.fixture(scope="module")
def scratch_bytes():
    """Scratch bytes a lane of each kernel of the library, by its mangled name."""
    with open(P.LIB_PATH, "rb") as f:
        blob = f.read()
    return {name: struct.unpack_from("<I", kd, 4)[0] for elf in _code_objects(blob) for name, kd in _descriptors(elf)}


@pytest.mark.parametrize("kernel,forms", KERNELS.items())
def test_no_kernel_of_the_cache_uses_scratch(scratch_bytes, kernel, forms):
    found = {n: b for n, b in scratch_bytes.items() if re.search(rf"\d{kernel}[IE]", n)}
    assert len(found) == forms, sorted(found)
    assert all(b == 0 for b in found.values()), found
