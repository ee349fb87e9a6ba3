"""Copies into LDS take their place from register m0.  A copy that is written out tells the compiler
of it, so that one made by a builtin behind it, to the place of an earlier one, sets the register
again.  Read from the assembly of a kernel compiled here, with the library's flags."""
import os
import re
import subprocess

from paper_2608_11919_amd import build

SOURCE = """
#include "tiles.h"
__global__ void copies(const uint8_t* a, uint8_t* out)
{
    __shared__ __align__(1024) uint8_t lds[4096];
    const uint32_t at = threadIdx.x * 16;
    tiles::copy_to_lds<false>(a, at, lds + 1024);
    tiles::copy_to_lds<true>(tiles::uniform(a + 1024), at, lds + 2048);
    tiles::copy_to_lds<false>(a + 2048, at, lds + 1024);
    tiles::wait_loads<0>();
    out[threadIdx.x] = lds[threadIdx.x * 7];
}
"""


def test_each_copy_s_place_is_set(tmp_path):
    source, listing = tmp_path / "copies.hip", tmp_path / "copies.s"
    source.write_text(SOURCE)
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-fPIC", "-shared")]
    subprocess.run([build.hipcc(), *flags, "--offload-device-only", "-S",
                    "-I", os.path.join(build.ROOT, "include"),
                    "-I", os.path.join(build.HERE, "csrc"), "-o", str(listing), str(source)],
                   check=True, capture_output=True)
    lines = [l.strip() for l in listing.read_text().splitlines()]
    copies = [i for i, l in enumerate(lines) if l.startswith("global_load_lds_dwordx4")]
    assert len(copies) == 3
    for before, copy in zip([0] + copies, copies):
        assert any(re.match(r"s_\w+ m0,", l) for l in lines[before:copy]), lines[before:copy]
