"""Registers, scratch and occupancy of the embedding's, the vocabulary loss's and the clipping's kernels, from the compiler's own report (no GPU needed), and the
LDS layout of operands that are stored across against the bank model of test_lds_layout.py.

The 256 x 256 tiles are eight waves of 128 x 64, two per SIMD: 256 registers each, of which 128 hold the sums.  A loop around their loop over the sum once
made 228 bytes of scratch per lane, with nothing failing."""
import os
import re
import subprocess

import pytest

from paper_2505_09326_amd._build import CSRC, HIPCC_FLAGS
from test_lds_layout import conflict_degree, passes_tr64


@pytest.fixture(scope="module")
def usage(tmp_path_factory):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    flags = [f for f in HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    out = tmp_path_factory.mktemp("res") / "dev.s"
    res = subprocess.run([hipcc, *flags, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-S", "-o", str(out),
                          os.path.join(CSRC, "sphattn_train.hip")], capture_output=True, text=True)
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
    for kernel, n in (("embed_", 10), ("vocab_", 40), ("clip_", 2)):
        assert sum(kernel in name for name in usage) >= n, kernel
    for name, v in usage.items():
        assert int(v["ScratchSize [bytes/lane]"]) == 0, name


def test_tiles_run_as_many_waves_as_they_are_cut_for(usage):
    # Tile<BP, BQ, ..>: two waves per SIMD for 256 x 256, two workgroups of four waves per CU for 128 x 128 and for fewer rows
    for tile, count in (("ILi256ELi256E", 12), ("ILi128ELi128E", 12), ("ILi128ELi64E", 6), ("ILi128ELi16E", 6)):
        kernels = {n: v for n, v in usage.items() if tile in n}
        assert len(kernels) >= count, (tile, len(kernels))
        for name, v in kernels.items():
            assert int(v["Occupancy [waves/SIMD]"]) >= 2, name
            assert int(v["VGPRs"]) + int(v["AGPRs"]) <= 256, name


def across_slot(k, c):
    return c ^ (2 * ((k & 3) | (k >> 1 & 4)))


@pytest.mark.parametrize("size", [128, 256])
def test_operands_stored_across(size):
    """32 rows of `size` 16-bit values in LDS: copies put every 16-byte piece where its reader looks for it, and no transposing read has a conflict."""
    slots, place = size // 8, {}
    for block in range(size // 16):
        for lane in range(64):
            at = block * 64 + lane
            k, c = at // slots, at % slots
            place[at * 16] = (k, across_slot(k, c))           # LDS byte -> (row, piece of its columns)
    assert len(set(place.values())) == 32 * slots
    for i in range(size // 16):
        for half in (0, 4):
            def read(lane):
                n16, g = lane & 15, lane >> 4
                k = 8 * g + (n16 >> 2)
                return k * size * 2 + across_slot(k, 2 * i + ((lane >> 1) & 1)) * 16 + (lane & 1) * 8 + half * size * 2
            for lane in range(64):
                n16, g = lane & 15, lane >> 4
                row, piece = place[read(lane) // 16 * 16]
                assert (row, piece * 8 + read(lane) % 16 // 2) == (8 * g + (n16 >> 2) + half, 16 * i + 4 * (n16 & 3))
            assert conflict_degree(read, 8, passes_tr64()) == 1
