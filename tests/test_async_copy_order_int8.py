"""The 8-bit linear's asynchronous copies in its machine code, checked as the
packed linear's are: no vector instruction writes a scalar register that a copy
reads less than five wait states later; and in the ring kernels no LDS read is
outstanding where a copy is issued (the tiled kernel issues its copies between
reads of its other buffers, a barrier after the last read of the one they fill)."""
import os
import subprocess

import pytest

from paper_2308_13137_amd import build
from tests.test_async_copy_order import findings, kernels


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="needs hipcc")
def test_copies_of_the_8_bit_linear(tmp_path):
    asm = tmp_path / "int8.s"
    subprocess.run([build.HIPCC, *build.FLAGS, "-Wno-everything", "--cuda-device-only", "-S",
                    os.path.join(build.CSRC, "int8_linear.hip"), "-o", str(asm)], check=True, timeout=600)
    found = {k: findings(v) for k, v in kernels(asm.read_text()).items()
             if "i8_ring_kernel" in k or "i8_tile_kernel" in k}
    assert len(found) == 14                         # six rings and the tile, fp32 and bf16 outputs
    for name, (copies, unordered, hazards) in found.items():
        assert copies > 0, name
        assert not hazards, (name, hazards[:3])
        if "ring" in name:
            assert not unordered, (name, unordered[:3], len(unordered))
