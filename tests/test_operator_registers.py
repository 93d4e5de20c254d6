"""Registers of the kernels of rotation, page tables, packed caches and log probabilities, as the built library's own notes give them (no GPU)."""
import os
import re
import struct
import subprocess

import pytest

from paper_2307_05740_amd import _build


@pytest.fixture(scope="module")
def notes(tmp_path_factory):
    """(vector registers, bytes of a lane in memory) of every kernel of the library, by its mangled name."""
    with open(_build.ARROW_LIB, "rb") as f:
        lib = f.read()
    readelf = os.path.join(os.path.dirname(os.path.dirname(_build._hipcc())), "llvm", "bin", "llvm-readelf")
    found = {}
    for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", lib):
        at = m.end() + 8
        for _ in range(struct.unpack_from("<Q", lib, m.end())[0]):
            offset, size, name = struct.unpack_from("<QQQ", lib, at)
            target = lib[at + 24:at + 24 + name]
            at += 24 + name
            if b"gfx950" not in target or size == 0:
                continue
            path = tmp_path_factory.mktemp("code") / "gfx950.o"
            path.write_bytes(lib[m.start() + offset:m.start() + offset + size])
            text = subprocess.run([readelf, "--notes", str(path)], stdout=subprocess.PIPE, text=True, check=True).stdout
            for kernel in re.split(r"\n  - ", text):
                values = [re.search(p, kernel) for p in (r"\.name: +(_Z\S+)", r"\.vgpr_count: +(\d+)", r"\.private_segment_fixed_size: +(\d+)")]
                if all(values):
                    found[values[0].group(1)] = int(values[1].group(1)), int(values[2].group(1))
    return found


@pytest.mark.parametrize("part,least", [("rotation_", 20), ("pages_", 6), ("packed_", 36), ("score_", 60)])
def test_nothing_spills(notes, part, least):
    kernels = {name: n for name, n in notes.items() if re.search(r"arrow12_GLOBAL__N_1\d+" + part, name)}
    assert len(kernels) >= least, sorted(kernels)
    assert not {name: n for name, n in kernels.items() if n[1]}


# 512 registers of a SIMD's lane, given out eight at a time
@pytest.mark.parametrize("kernel,waves", [(r"rotation_grad_kernelIDF16b", 4), (r"packed_decode_kernelIDF16bLi128ELi4E", 4), (r"packed_decode_kernelIDF16_Li64ELi8E", 4),
                                          (r"score_sums_kernelIDF16b", 6), (r"score_kernelIDF16bLi16E", 4), (r"score_kernelIDF16bLi32E", 2)])
def test_wavefronts_per_simd(notes, kernel, waves):
    """What the launches count on: workgroups of a gradient that stay on the chip, four to a compute unit; tiles of a cache on their way; rows that are held."""
    counts = [n[0] for name, n in notes.items() if re.search(kernel, name)]
    assert counts and all(512 // (-(-n // 8) * 8) >= waves for n in counts), counts
