"""What a built library says about its kernels."""

import struct

import pytest


def kernels(path):
    """The metadata of a library's kernels: the message-pack notes of its device code objects."""
    msgpack = pytest.importorskip("msgpack")
    data, found = open(path, "rb").read(), []
    name = b"AMDGPU\0\0"
    at = data.find(name)
    while at >= 0:
        name_size, size, kind = struct.unpack("<III", data[at - 12:at])
        if name_size == 7 and kind == 32:
            found += msgpack.unpackb(data[at + 8:at + 8 + size])["amdhsa.kernels"]
        at = data.find(name, at + 1)
    return found
