"""No kernel of the built library touches a register whose LDS read may still be in flight, the products from 4 bits, whose scales are read by inline
asm too, and the gated FFN's among them."""
import shutil
import subprocess

import pytest

from paper_2407_00599_amd import api
from test_lds_reads_cpu import OBJDUMP, hazards, parse


@pytest.mark.skipif(shutil.which(OBJDUMP) is None, reason="needs the ROCm disassembler")
def test_no_register_of_any_kernel_is_touched_before_its_lds_read(tmp_path):
    api.lib()
    shutil.copy(api.LIB_PATH, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    seen, found = [], []
    for obj in sorted(tmp_path.glob("lib.so.*gfx950")):
        out = subprocess.run([OBJDUMP, "-d", obj.name], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
        for name, code in parse(out).items():
            seen.append(name)
            found += [(name, hex(a), op, args, r) for a, op, args, r in hazards(code)]
    for kind, least in (("mx4_gemm", 4), ("glu_gemm_dma", 18), ("glu_bwd_quad", 5)):
        assert sum(kind in name for name in seen) >= least, kind
    assert not found, (len(found), found[:20])
