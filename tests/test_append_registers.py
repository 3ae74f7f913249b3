"""Registers and arguments of the kernels that append to the 8-bit cache, as the compiler states them in the library that was built here."""
import os
import struct

import pytest

msgpack = pytest.importorskip("msgpack")


def _kernels(path):
    """Metadata of every kernel in the shared object: its GPU code objects lie in bundles, each an ELF file with a note of messagepack."""
    data, at, found = open(path, "rb").read(), 0, {}
    while (at := data.find(b"__CLANG_OFFLOAD_BUNDLE__", at)) >= 0:
        count, p = struct.unpack_from("<Q", data, at + 24)[0], at + 32
        if count > 16:                                            # (the bytes of another program's string)
            at += 24
            continue
        for _ in range(count):
            offset, size, n = struct.unpack_from("<QQQ", data, p)
            target, p = data[p + 24:p + 24 + n], p + 24 + n
            if b"gfx950" in target and size:
                found.update(_notes(data[at + offset:at + offset + size]))
        at += 24
    return found


def _notes(elf):
    assert elf[:4] == b"\x7fELF"
    start, = struct.unpack_from("<Q", elf, 40)
    each, count = struct.unpack_from("<HH", elf, 58)
    for i in range(count):
        kind, = struct.unpack_from("<I", elf, start + i * each + 4)
        if kind != 7:                                             # SHT_NOTE
            continue
        offset, size = struct.unpack_from("<QQ", elf, start + i * each + 24)
        end = offset + size
        while offset < end:
            n, d, t = struct.unpack_from("<III", elf, offset)
            body = offset + 12 + (n + 3) // 4 * 4
            if t == 32:                                           # NT_AMDGPU_METADATA
                for k in msgpack.unpackb(elf[body:body + d])["amdhsa.kernels"]:
                    yield k[".name"], k
            offset = body + (d + 3) // 4 * 4


@pytest.fixture(scope="module")
def appends():
    from paper_2301_12017_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    found = {name: k for name, k in _kernels(binding.LIB_PATH).items() if "kv8_append_kernel" in name}
    assert len(found) == 24                                       # two types, four sizes of heads; without positions, with them, with queries too
    return found


def _of(appends, D, positions):
    return [k for name, k in appends.items() if f"ELi{D}ELNS0_9PositionsE{positions}E" in name]


@pytest.mark.parametrize("D,waves", [(64, 5), (96, 5), (128, 4), (256, 3)])
def test_waves_of_the_append_without_positions(appends, D, waves):
    """A SIMD has 512 vector registers a lane, which its waves get by eights; none of theirs lies in memory."""
    kernels = _of(appends, D, 0)
    assert len(kernels) == 2
    for k in kernels:
        assert 512 // (-(-k[".vgpr_count"] // 8) * 8) >= waves and k[".vgpr_spill_count"] == 0, k


@pytest.mark.parametrize("positions", [1, 2])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
def test_waves_of_the_append_with_positions(appends, D, positions):
    kernels = _of(appends, D, positions)
    assert len(kernels) == 2
    for k in kernels:
        assert k[".vgpr_count"] <= 168 and k[".vgpr_spill_count"] <= (13 if D == 256 else 0), k


def test_arguments_of_the_append_without_positions(appends):
    """What the host copies for each call: nothing of positions, angles and queries."""
    for D in (64, 96, 128, 256):
        for k in _of(appends, D, 0):
            assert sum(a[".size"] for a in k[".args"] if a[".value_kind"] == "by_value") == 96
