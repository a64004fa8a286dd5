"""What launch rules take for granted of kernels, from the metadata that the compiler leaves in the built library."""
import re

import pytest

from paper_2502_13542_amd import build


def kernels():
    """name: (registers of a lane, vector and accumulation together; bytes of scratch) of every kernel of the library."""
    msgpack = pytest.importorskip("msgpack")
    data = open(build.LIB, "rb").read()
    found, at = {}, -1
    while (at := data.find(b"\xaeamdhsa.kernels", at + 1)) >= 0:       # the first key of a code object's map, a byte behind the map's head
        unpacker = msgpack.Unpacker(strict_map_key=False)
        unpacker.feed(data[at - 1: at + (4 << 20)])
        for k in unpacker.unpack()["amdhsa.kernels"]:
            found[k[".name"]] = k[".vgpr_count"], k[".private_segment_fixed_size"]
    return found


@pytest.mark.parametrize("name", ["paged8_step_kernel", "paged_selected_kernel"])
def test_two_workgroups_of_four_wavefronts_share_a_compute_unit(name):
    """A SIMD's 512 registers hold two wavefronts of 256: the rules that choose four wavefronts a workgroup count on it."""
    four = {k: v for k, v in kernels().items() if re.search(name + r"I[ft]Li\d+ELi4E", k)}
    assert len(four) == 16                         # two types, two head sizes, four score forms
    assert all(registers <= 256 for registers, _ in four.values()), {k: v for k, v in four.items() if v[0] > 256}


def test_scratch_of_steps_over_8_bits():
    """Of fp32 with 128 channels up to 8 registers a lane are in scratch, of the others none."""
    for k, (_, scratch) in kernels().items():
        if "paged8_step_kernel" in k or "paged_selected_kernel" in k:
            assert scratch <= (40 if "paged8_step_kernelIfLi128" in k else 0), (k, scratch)
