"""Compile-time guard (no GPU): the attention kernels keep a row's sums and operands in registers, so a spill in their
loops costs a large factor, and their speed is that of several workgroups on a compute unit at a time."""
import os
import re
import subprocess

import pytest

from paper_2307_02031_amd import build as b


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """(kernel, head pieces, direct loads) -> (scratch bytes per lane, waves per SIMD, LDS bytes), the worst of the two types."""
    src = os.path.join(b.CSRC, "gbmw_attention.hip")
    flags = [f for f in b.FLAGS if f not in ("-shared", "-fPIC")]
    cmd = [b.HIPCC, *flags, "--cuda-device-only", "-c", "-Rpass-analysis=kernel-resource-usage", src,
           "-o", str(tmp_path_factory.mktemp("resources") / "k.o")]
    out = subprocess.run(cmd, check=True, capture_output=True, text=True).stderr
    found = {}
    for blk in re.split(r"remark: Function Name: ", out)[1:]:
        m = re.search(r"k_attn_(fwd|few|dq|dkv)I(DF16b?_?)Li(\d)ELb([01])E", blk.split()[0])
        if m:
            num = lambda what: int(re.search(what + r"[^:]*: (\d+)", blk).group(1))
            new = (num("ScratchSize"), num("Occupancy"), num("LDS Size"))
            key = (m.group(1), int(m.group(3)), m.group(4) == "1")
            old = found.get(key, new)
            found[key] = (max(old[0], new[0]), min(old[1], new[1]), new[2])
    return found


def test_every_kernel_is_there(kernels):
    want = {(k, p, True) for k in ("fwd", "few", "dq", "dkv") for p in (2, 3, 4, 5, 6, 8)}
    want |= {(k, p, False) for k in ("fwd", "few", "dq", "dkv") for p in (4, 8)}
    assert set(kernels) == want


def test_kernels_with_direct_loads_do_not_spill(kernels):
    for (kernel, pieces, direct), (scratch, _, _) in kernels.items():
        if direct:
            # dk and dv: a few registers outside the loop with heads of 128, and where three workgroups share the registers
            assert scratch <= (64 if kernel == "dkv" else 0), (kernel, pieces, scratch)


def test_workgroups_on_a_compute_unit(kernels):
    for (kernel, pieces, direct), (_, waves, lds) in kernels.items():
        together = min(waves, 160 * 1024 // lds)     # a workgroup is one wave on each SIMD
        least = dict(few=1, fwd=4 if pieces <= 4 else 3 if pieces <= 6 else 2, dq=3 if pieces <= 4 else 2,
                     dkv=3 if pieces <= 4 else 2)[kernel]
        assert together >= least - (not direct and pieces <= 4), (kernel, pieces, direct, waves, lds)


def test_scratch_memory_without_direct_loads(kernels):
    """Rows that come through registers leave the backward kernels too few; forward has enough."""
    for (kernel, pieces, direct), (scratch, _, _) in kernels.items():
        if not direct:
            most = {"dq": {4: 0, 8: 128}, "dkv": {4: 128, 8: 224}}.get(kernel, {}).get(pieces, 0)
            assert scratch <= most, (kernel, pieces, scratch)
