"""Registers and scratch memory of the kernels with an epilogue and of those around the products, as the compiler wrote them beside the
code (in every part of the library that holds code for the GPU)."""
import re
import struct

import msgpack
import pytest

from paper_2507_12205_amd import build


def kernels():
    """{mangled name: (VGPRs, scratch bytes per lane)} of every kernel in the library."""
    data, found, base = open(build.LIB, "rb").read(), {}, -1
    while True:
        base = data.find(b"__CLANG_OFFLOAD_BUNDLE__", base + 1)
        if base < 0:
            return found
        (count,), pos = struct.unpack_from("<Q", data, base + 24), base + 32
        for _ in range(count if count < 16 else 0):
            offset, size, length = struct.unpack_from("<QQQ", data, pos)
            name = data[pos + 24:pos + 24 + length]
            pos += 24 + length
            elf = data[base + offset:base + offset + size]
            if b"gfx950" not in name or elf[:4] != b"\x7fELF":
                continue
            (shoff,) = struct.unpack_from("<Q", elf, 40)
            shentsize, shnum = struct.unpack_from("<HH", elf, 58)
            for i in range(shnum):
                kind, _, _, at, length = struct.unpack_from("<IQQQQ", elf, shoff + i * shentsize + 4)
                if kind != 7 or struct.unpack_from("<III", elf, at)[2] != 32:
                    continue
                namesz, descsz = struct.unpack_from("<II", elf, at)
                start = at + 12 + (namesz + 3) // 4 * 4
                for k in msgpack.unpackb(elf[start:start + descsz], strict_map_key=False)["amdhsa.kernels"]:
                    found[k[".name"]] = (k[".vgpr_count"], k[".private_segment_fixed_size"])


@pytest.fixture(scope="module")
def table():
    return kernels()


def test_epilogues(table):
    """As without one: no scratch memory but with FP32 values in 8- or 16-grained sets, and 64 registers where two workgroups of 1024
    threads are to share a compute unit."""
    found = {}
    for name, figures in table.items():
        args = re.search(r"ecspmv_kernelI((?:Li\d+E){6})E", name)
        if args:
            key = tuple(int(v) for v in re.findall(r"Li(\d+)E", args.group(1)))
            if key[3] >= 8:
                found[key] = figures
    assert len(found) > 200 and {k[4] for k in found} == {1, 2, 4, 8} and not [k for k in found if k[2] in (1, 2)]
    assert not {k: v for k, v in found.items() if v[1] and not (k[5] == 4 and k[0] >= 7)}
    assert not {k: v for k, v in found.items() if k[5] == 2 and k[2] != 3 and v[0] > 64 and k[0] <= {1: 3, 2: 3, 4: 3, 8: 1}[k[4]]}


def test_around_the_products(table):
    found = {n: v for n, v in table.items() if re.search(r"attention_|kv_write|kv_read|verify", n)}
    assert len(found) > 20 and not {n: v for n, v in found.items() if v[1]}
