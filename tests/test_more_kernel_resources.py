"""Compile-time guard (no GPU): RMS norm, rotary positions and AdamW keep what they hold in registers, and enough waves fit
on a compute unit to keep memory busy."""
import os
import re
import subprocess

import pytest

from paper_2307_02031_amd import build as b


def _kernels(source, folder):
    """mangled kernel name -> (scratch bytes per lane, waves per SIMD)"""
    flags = [f for f in b.FLAGS if f not in ("-shared", "-fPIC")]
    cmd = [b.HIPCC, *flags, "--cuda-device-only", "-c", "-Rpass-analysis=kernel-resource-usage", os.path.join(b.CSRC, source),
           "-o", str(folder / "k.o")]
    out = subprocess.run(cmd, check=True, capture_output=True, text=True).stderr
    found = {}
    for blk in re.split(r"remark: Function Name: ", out)[1:]:
        num = lambda what: int(re.search(what + r"[^:]*: (\d+)", blk).group(1))
        found[blk.split()[0]] = (num("ScratchSize"), num("Occupancy"))
    return found


@pytest.mark.parametrize("source,name,kernels,least", [("gbmw_rotary.hip", "k_rotary", 50, 7), ("gbmw_adamw.hip", "k_adamw", 2, 6)])
def test_short_kernels(source, name, kernels, least, tmp_path):
    found = {k: v for k, v in _kernels(source, tmp_path).items() if name in k}
    assert len(found) == kernels
    for k, (scratch, waves) in found.items():
        assert scratch == 0 and waves >= least, (k, scratch, waves)


def test_norms(tmp_path):
    found = _kernels("gbmw_rms.hip", tmp_path)
    seen = 0
    for k, (scratch, waves) in found.items():
        m = re.search(r"k_rms_(fwd|bwd)I(f|DF16_|DF16b)Li(\d+)ELi(\d)E", k)
        if not m:
            continue
        seen += 1
        threads, pieces, wide = int(m.group(3)), int(m.group(4)), m.group(2) == "f"
        # rows of up to 16384 columns of 16 bits, 8192 of 32, stay in registers; longer ones may spill
        if threads < 1024 or pieces <= 2:
            assert scratch == 0, (k, scratch)
            # two workgroups of 512 threads where a thread has up to two pieces, else one and a half
            assert waves >= (4 if pieces <= 2 else 3), (k, waves)
    # fifteen shapes (one more in 32 bits, and one backward in 16), each of whole pieces, past the cache, and of any length
    assert seen == ((3 * 15 + 1) * 2 + 2) * 3
