"""What the compiler gave the kernels of the built library, from the notes of its code objects."""
import re
import struct

import pytest

from paper_2609_35099_amd import e3mi

msgpack = pytest.importorskip("msgpack")


@pytest.fixture(scope="module")
def kernels():
    """{mangled name: its metadata and "objects", where its code objects lie in the library} of every kernel."""
    e3mi.lib()
    data = open(e3mi.LIB_PATH, "rb").read()
    out, at = {}, 0
    while (at := data.find(b"\x7fELF", at)) >= 0:
        if struct.unpack_from("<H", data, at + 18)[0] == 224:                     # an AMD GPU's code object
            phoff, = struct.unpack_from("<Q", data, at + 32)
            size, count = struct.unpack_from("<HH", data, at + 54)
            for i in range(count):
                kind, _, off, _, _, length = struct.unpack_from("<IIQQQQ", data, at + phoff + size * i)
                if kind != 4:                                                     # notes
                    continue
                p, end = at + off, at + off + length
                while p < end:
                    n, d, note = struct.unpack_from("<III", data, p)
                    name = p + 12 + (n + 3) // 4 * 4
                    if note == 32:
                        meta = msgpack.unpackb(data[name:name + d], strict_map_key=False)
                        for k in meta["amdhsa.kernels"]:
                            out.setdefault(k[".name"], {**k, "objects": set()})["objects"].add(at)
                    p = name + (d + 3) // 4 * 4
        at += 4
    return out


def test_the_notes_are_read(kernels):
    for part in ("k_dense_direct", "k_gated_direct", "k_dense_two", "k_res_bwd", "k_gated_bwd", "k_dropout"):
        assert any(part in n for n in kernels), part


def test_the_largest_dense_tiles_keep_their_registers(kernels):
    """dW's tiles of 256 x 256 with an operand that is formed on the way to LDS are at the registers' end: the few
    that they spill lie outside the loop; 136 in it cost them two thirds of their rate."""
    tiles = {n: k for n, k in kernels.items() if re.search(r"\d+k_dense(_direct)?I", n) and ("Li256E" in n or "direct" in n)}
    assert len(tiles) >= 8
    spills = {n: k[".vgpr_spill_count"] for n, k in tiles.items() if k[".vgpr_spill_count"]}
    assert all(v <= 28 for v in spills.values()), spills


def test_the_direct_tiles_lie_apart(kernels):
    """In front of the register kernels their code moved those to where they took up to an eighth longer."""
    direct, others = set(), set()
    for n, k in kernels.items():
        direct |= k["objects"] if "k_dense_direct" in n else set()
        others |= k["objects"] if "k_dense_two" in n or "k_dense_panel" in n else set()
    assert len(direct) == 1 and len(others) >= 3 and not direct & others


@pytest.mark.parametrize("name", ["k_gated_direct", "k_gated_walk", "k_gated_few", "k_gated_panel", "k_gated_join",
                                  "k_gated_bwd", "k_gated_dz", "k_res_", "k_dropout"])
def test_a_kernel_is_compiled_where_it_is_launched(kernels, name):
    """Once, by the unit that launches it, and not by every one that reads its header."""
    copies = {n: len(k["objects"]) for n, k in kernels.items() if name in n}
    assert copies and all(v == 1 for v in copies.values()), copies
