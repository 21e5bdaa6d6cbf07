"""What the built append kernels hold, from the metadata of their code objects in the library."""

import os
import re
import struct

import pytest

from paper_2609_33269_amd import qwam as Q

NOTE = re.compile(struct.pack("<I", 7) + b"(....)" + struct.pack("<I", 32) + b"AMDGPU\0\0", re.S)


def _kernels():
    """The metadata of every kernel of the library, by name."""
    msgpack = pytest.importorskip("msgpack")
    if not os.path.exists(Q.LIB_PATH):
        from paper_2609_33269_amd import build
        build.build()
    with open(Q.LIB_PATH, "rb") as f:
        data = f.read()
    out = {}
    for m in NOTE.finditer(data):
        size, = struct.unpack("<I", m[1])
        for k in msgpack.unpackb(data[m.end():m.end() + size])["amdhsa.kernels"]:
            out[k[".name"]] = k
    return out


def test_append_keeps_its_vectors_in_registers():
    """The keys' and the values' vector of a thread are two registers each, not an array that goes through LDS or scratch."""
    found = [k for n, k in _kernels().items() if "kv_append_kernel" in n]
    assert len(found) == 2
    for k in found:
        assert k[".group_segment_fixed_size"] == 0 and k[".private_segment_fixed_size"] == 0, k[".name"]
