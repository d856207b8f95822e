"""Register budget of the decoding operators' kernels, read from the device
compiler's resource report (no GPU needed).

None of them may spill: every one runs its loop with all registers it has, and
scratch memory there costs a load and a store a tile.  The attention of more
than 32 rows and the 8-wave products need two waves a SIMD, the 16-wave
products four.
"""
import os
import re
import subprocess

import pytest

from paper_2006_12645_amd import build as B

from test_kernel_resources_cpu import _have_hipcc

pytestmark = pytest.mark.skipif(not _have_hipcc(), reason="hipcc not available")
FIELD = re.compile(r"remark:.*?(VGPRs Spill|ScratchSize \[bytes/lane\]|Occupancy \[waves/SIMD\]): (\d+)")


def kernels(name, tmp_path):
    """{(kernel, its number and truth arguments): resources} of one unit."""
    src, flags, obj = next(u for u in B.UNITS if u[0].endswith(f"gba_{name}.hip"))
    r = subprocess.run([B._hipcc()] + B.HIPCC_FLAGS + flags + ["-Rpass-analysis=kernel-resource-usage", "--cuda-device-only", "-c",
                                                               os.path.join(B.CSRC, src), "-o", str(tmp_path / obj)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    found, now = {}, None
    for line in r.stderr.splitlines():
        m = re.search(r"Function Name: (\S+)", line)
        if m:
            kernel = re.search(r"N_1\d+([a-z]\w*?_kernel)(I\S*)?", m.group(1))
            args = tuple(int(v) for v in re.findall(r"L[ib](\d+)E", kernel.group(2) or ""))
            now = found.setdefault((kernel.group(1), "BF16" in m.group(1), args), {})
        m = FIELD.search(line)
        if m:
            now[m.group(1).split()[0] + ("Spill" if "Spill" in m.group(1) else "")] = int(m.group(2))
    return found


def test_attention_kernels(tmp_path):
    seen = 0
    for (kernel, _, args), res in kernels("tree_attention", tmp_path).items():
        assert res["ScratchSize"] == 0 and res["VGPRsSpill"] == 0, (kernel, args, res)
        if kernel == "attention_kernel":
            seen += 1
            assert res["Occupancy"] >= (2 if args[2] > 1 else 1), (args, res)
    assert seen == 2 * (2 * 7 + 3)


def test_product_kernels(tmp_path):
    few = rows = 0
    for (kernel, _, args), res in kernels("q4", tmp_path).items():
        assert res["ScratchSize"] == 0 and res["VGPRsSpill"] == 0, (kernel, args, res)
        if kernel == "q4_kernel":  # column blocks, steps of a group, zeros, waves, chunks ahead
            few += 1
            assert res["Occupancy"] >= args[3] // 4, (args, res)
        if kernel == "q4_rows_kernel":
            rows += 1
            assert res["Occupancy"] >= 2, (args, res)
    assert few == 2 * 2 * (3 * 3 + 3 + 2) and rows == 2 * 2 * (3 * 3 + 2 + 3 * 2), (few, rows)


@pytest.mark.parametrize("name", ["tables", "cache"])
def test_other_kernels(name, tmp_path):
    for key, res in kernels(name, tmp_path).items():
        assert res["ScratchSize"] == 0 and res["VGPRsSpill"] == 0, (key, res)
