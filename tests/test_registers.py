"""What the kernels of attention over a cache take of a CU's registers, as the built library says it of itself: so many workgroups are held side by side."""
import re
import struct
import subprocess

import pytest

from paper_2605_13473_amd import binding as ob
from paper_2605_13473_amd import build as hb

MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def code_objects(blob):
    at = blob.find(MAGIC)
    while at >= 0:
        n, = struct.unpack_from("<Q", blob, at + len(MAGIC))
        p = at + len(MAGIC) + 8
        for _ in range(n):
            offset, size, name = struct.unpack_from("<QQQ", blob, p)
            p += 24 + name
            if b"gfx950" in blob[p - name:p]:
                yield blob[at + offset:at + offset + size]
        at = blob.find(MAGIC, at + 1)


def kernels_of(elf, path):
    path.write_bytes(elf)
    notes = subprocess.run(["/opt/rocm/llvm/bin/llvm-readelf", "--notes", str(path)], capture_output=True, text=True, check=True).stdout
    for k in re.findall(r"- \.agpr_count:.*?\.vgpr_count: +\d+", notes, re.S):
        number = lambda name: int(re.search(rf"\.{name}: +(\d+)", k)[1])
        yield re.search(r"\.symbol: +'?(\w+)\.kd", k)[1], number("agpr_count") + number("vgpr_count"), number("private_segment_fixed_size")


@pytest.fixture(scope="module")
def decode_kernels(tmp_path_factory):
    """(rows' format, element, K, chosen pages, R, shares) of every instance of decode_kernel: (registers, scratch)."""
    ob.lib()
    found, path = {}, tmp_path_factory.mktemp("code") / "code.elf"
    with open(hb.LIB, "rb") as f:
        for elf in code_objects(f.read()):
            for name, registers, scratch in kernels_of(elf, path):
                m = re.match(r"_ZN4osdn13decode_kernelINS_7(RowTile|Fp4Tile)I(f|DF16b)Li(\d+)ELb([01])E(?:Lb([01])ELb[01]E)?EELi([124])ELb([01])E", name)
                if m:
                    tile, io, K, first, second, R, shared = m.groups()
                    found[tile, io, int(K), (second if tile == "Fp4Tile" else first) == "1", int(R), shared == "1", name] = (registers, scratch)
    assert len([k for k in found if k[0] == "RowTile"]) == 2 * 3 * 2 * 3 * 2 and len(found) > 144
    return found


def test_nothing_is_kept_in_memory(decode_kernels):
    assert not {k: v for k, v in decode_kernels.items() if v[1]}


def test_three_workgroups_a_cu_where_a_workgroup_takes_a_row_of_128(decode_kernels):
    """512 registers a lane of a SIMD, in eights: 168 for three wavefronts."""
    rows = {k: v[0] for k, v in decode_kernels.items() if k[0] == "RowTile" and k[2] == 128 and not k[5]}
    assert len(rows) == 12 and all(n <= 168 for n in rows.values()), rows
