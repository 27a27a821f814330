"""The attention kernels with direct loads into LDS as they are built: those loads are inline assembly, so the listings are looked through as
those of the tile products are, and no register of theirs may spill."""
import os
import re
import subprocess

import pytest

from paper_2405_16283_amd import build
from test_asm_hazards import _kernels, _scalars_read_too_early


@pytest.mark.parametrize("source", ["attn_rule", "attn_rule_f32"])
def test_direct_loads_keep_their_distance(source, tmp_path):
    out = str(tmp_path / "listing.s")
    subprocess.run([build.HIPCC] + build.COMMON + build.DEVICE + ["-w", "--cuda-device-only", "-S", os.path.join(build.CSRC, source + ".hip"), "-o", out],
                   check=True, capture_output=True)
    text = open(out).read()
    assert not any(int(n) for n in re.findall(r"\.private_segment_fixed_size:\s+(\d+)", text))
    kernels = _kernels(out)
    assert kernels
    for name, blocks in kernels.items():
        loads = sum(inside and "lds" in line for b in blocks for _, _, inside, line in b["code"])
        assert loads > 0 and not _scalars_read_too_early(blocks), name
