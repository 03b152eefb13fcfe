"""No kernel of the block norms, the integer FFN and the layer for a few tokens keeps anything in scratch memory (CPU only; the search for open LDS accesses and for FLAT
instructions, in test_kernel_code.py, is over every kernel of the library)."""
import re
import shutil
import subprocess

from paper_2410_17043_amd import _lib
from tests.test_kernel_code import OBJDUMP

READELF = OBJDUMP.replace("objdump", "readelf")
FAMILIES = {"block_norm_kernel": 8, "quantize_int8_kernel": 8, "gemm_int8_stream_kernel": 24, "gemm_int8_kernel": 9, "gemm_int8_sum_kernel": 1, "few_gate_kernel": 18, "few_up_kernel": 12,
            "few_down_kernel": 4, "few_small_kernel": 6}


def test_no_scratch(tmp_path):
    shutil.copy(_lib.LIB_PATH, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    found = {}
    for f in sorted(tmp_path.glob("lib.so.*gfx950")):
        notes = subprocess.run([READELF, "--notes", str(f)], check=True, capture_output=True, text=True).stdout
        for size, name in re.findall(r"\.private_segment_fixed_size:\s*(\d+).*?\.symbol:\s*(\S+)\.kd", notes, re.S):
            for family in FAMILIES:
                if family in name:
                    found.setdefault(family, []).append((name, int(size)))
    for family, least in FAMILIES.items():
        assert len(found.get(family, [])) >= least, (family, len(found.get(family, [])))
        assert all(size == 0 for _, size in found[family]), [n for n, size in found[family] if size]
