"""Registers, scratch and occupancy of the kernels around the attention in a layer, from the compiler's own report (no GPU needed)."""
import os
import re
import subprocess

import pytest

from paper_2505_09326_amd._build import CSRC, HIPCC_FLAGS


@pytest.fixture(scope="module")
def usage(tmp_path_factory):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    flags = [f for f in HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    out = tmp_path_factory.mktemp("res") / "dev.s"
    res = subprocess.run([hipcc, *flags, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-S", "-o", str(out),
                          os.path.join(CSRC, "sphattn_layer.hip")], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    kernels, cur = {}, None
    for line in res.stderr.splitlines():
        m = re.search(r"remark:\s+(.*?) \[-Rpass", line)
        if not m:
            continue
        t = m.group(1).strip()
        if t.startswith("Function Name:"):
            cur = kernels.setdefault(t.split("Function Name:")[1].strip(), {})
        elif cur is not None and ":" in t:
            k, v = t.split(":", 1)
            cur[k.strip()] = v.strip()
    return kernels


def test_no_kernel_has_scratch(usage):
    for kernel, n in (("heads_fwd", 12), ("heads_bwd", 12), ("ffn_gate", 12), ("ffn_rows", 18), ("ffn_dx", 6), ("ffn_dw", 6)):
        assert sum(kernel in name for name in usage) >= n, kernel
    for name, v in usage.items():
        assert int(v["ScratchSize [bytes/lane]"]) == 0, name


def test_tiles_run_as_many_waves_as_they_are_cut_for(usage):
    for tile in ("ILi256ELi256E", "ILi128ELi128E"):
        kernels = {n: v for n, v in usage.items() if tile in n}
        assert len(kernels) >= 12, (tile, len(kernels))
        for name, v in kernels.items():
            assert int(v["Occupancy [waves/SIMD]"]) >= 2, name
            assert int(v["VGPRs"]) + int(v["AGPRs"]) <= 256, name


def test_heads_have_waves_enough_for_memory(usage):
    for name, v in usage.items():
        if "heads_fwd" in name or "heads_bwd" in name:
            assert int(v["Occupancy [waves/SIMD]"]) >= 3, name
