"""What the compiler says of the kernels in the built library: the metadata of its code objects, a MessagePack note in each."""
import struct

BUNDLE = b"__CLANG_OFFLOAD_BUNDLE__"


def code_objects(data):
    """The gfx950 code objects of a library: one bundle for each source file."""
    at = data.find(BUNDLE)
    while at >= 0:
        count, = struct.unpack_from("<Q", data, at + len(BUNDLE))
        p = at + len(BUNDLE) + 8
        for _ in range(count):
            offset, size, length = struct.unpack_from("<QQQ", data, p)
            name = data[p + 24:p + 24 + length]
            p += 24 + length
            if b"gfx950" in name and size:
                yield data[at + offset:at + offset + size]
        at = data.find(BUNDLE, at + 1)


def notes(elf):
    """Descriptions of the AMDGPU metadata notes of a code object."""
    table, = struct.unpack_from("<Q", elf, 0x20)
    size, count = struct.unpack_from("<HH", elf, 0x36)
    for i in range(count):
        kind, _, offset, _, _, length = struct.unpack_from("<IIQQQQ", elf, table + i * size)
        if kind != 4:                                                 # PT_NOTE
            continue
        p = offset
        while p < offset + length:
            name, desc, what = struct.unpack_from("<III", elf, p)
            p += 12 + (name + 3) // 4 * 4
            if what == 32:                                            # NT_AMDGPU_METADATA
                yield elf[p:p + desc]
            p += (desc + 3) // 4 * 4


def kernels(path):
    """{mangled name: metadata} of all kernels."""
    import msgpack
    with open(path, "rb") as f:
        data = f.read()
    found = {}
    for obj in code_objects(data):
        for note in notes(obj):
            for k in msgpack.unpackb(note, strict_map_key=False)["amdhsa.kernels"]:
                found[k[".name"]] = k
    return found
