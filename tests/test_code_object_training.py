"""The code objects of the operators around the module (each source of the library brings one of its own; no GPU needed)."""
import os
import re
import struct
import subprocess

import pytest

from paper_2401_06197_amd import binding as dcn

READELF = "/opt/rocm/llvm/bin/llvm-readelf"
pytestmark = pytest.mark.skipif(not os.path.exists(READELF), reason="no llvm-readelf")


def test_kernels_keep_no_registers_in_scratch_memory(tmp_path):
    blob, found, at = open(dcn.LIB_PATH, "rb").read(), {}, -1
    while (at := blob.find(b"__CLANG_OFFLOAD_BUNDLE__", at + 1)) >= 0:
        pos = at + 32
        for _ in range(struct.unpack_from("<Q", blob, at + 24)[0]):
            offset, size, length = struct.unpack_from("<3Q", blob, pos)
            if b"gfx950" in blob[pos + 24:pos + 24 + length]:
                obj = tmp_path / "gfx950.o"
                obj.write_bytes(blob[at + offset:at + offset + size])
                notes = subprocess.run([READELF, "--notes", str(obj)], capture_output=True, text=True, check=True).stdout
                for entry in notes.split("- .agpr_count:")[1:]:
                    name = re.search(r"\.name:\s+(\S+)", entry).group(1)
                    found[name] = {k: int(v) for k, v in re.findall(r"\.(\w+):\s+(\d+)\s*$", entry, flags=re.M)}
            pos += 24 + length
    mine = {n: k for n, k in found.items() if re.search("dcnv4_(norm|dropout|loss)", n)}
    for part in ("dcnv4_norm_kernel", "dcnv4_norm_backward_kernel", "dcnv4_dropout_kernel", "dcnv4_loss_kernel", "dcnv4_loss_delta_kernel",
                 "dcnv4_loss_product_kernel"):
        assert any(part in n for n in mine), part
    for name, k in mine.items():
        assert k["private_segment_fixed_size"] == 0, (name, k["private_segment_fixed_size"])
        assert k["group_segment_fixed_size"] <= 160 * 1024, name
