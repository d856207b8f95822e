"""The order, in the code that is built, of what joins a request's runs: where
sums are written through, a wave's stores have arrived before the barrier after
which its workgroup is counted, by a wait that the compiler moves no store past,
and the last workgroup reads the others' sums after the count, past its own L2."""
import os
import re
import subprocess

import pytest

from paper_2006_12645_amd import build as B

from test_kernel_resources_cpu import _have_hipcc

pytestmark = pytest.mark.skipif(not _have_hipcc(), reason="hipcc not available")


def bodies(name, tmp_path):
    """{symbol: the lines of its code} of the kernels of a unit."""
    src, flags, _ = next(u for u in B.UNITS if u[0].endswith(f"gba_{name}.hip"))
    out = tmp_path / f"{name}.s"
    r = subprocess.run([B._hipcc()] + B.HIPCC_FLAGS + flags + ["--cuda-device-only", "-S", os.path.join(B.CSRC, src), "-o", str(out)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    found = re.findall(r"^(_Z\S*attention_kernel\S*):[^\n]*\n(.*?)\n\ts_endpgm", out.read_text(), re.S | re.M)
    return {symbol: [line.strip() for line in body.splitlines()] for symbol, body in found}


# kernels whose runs are joined through stores that write through: all over 4
# bits, and with a window those of one wave or two of rows
@pytest.mark.parametrize("name,count", [("q4_attention", 2 * 8), ("window_attention", 2 * (2 * 5 + 3))])
def test_sums_arrive_before_the_count(name, count, tmp_path):
    seen = 0
    for symbol, lines in bodies(name, tmp_path).items():
        counts = [i for i, line in enumerate(lines) if re.match(r"global_atomic_(add|inc)", line)]
        if not counts:
            continue
        seen += 1
        assert len(counts) == 1, symbol
        at = counts[0]
        barrier = max(i for i in range(at) if lines[i].startswith("s_barrier"))
        assert not any("store" in line for line in lines[barrier:at]), symbol
        stores = [i for i in range(barrier) if re.match(r"global_store\S* .*\bsc1\b", lines[i])]
        waits = [i for i in range(barrier) if lines[i].startswith("s_waitcnt vmcnt(0)") and "#ASMSTART" in lines[i - 1]]
        assert stores and waits and stores[-1] < waits[-1], symbol
        assert not any("store" in line for line in lines[waits[-1]:barrier] if not line.startswith("ds_")), symbol
        after = [line for line in lines[at:] if line.startswith("global_load")]
        assert after and all(re.search(r"\bsc1\b", line) for line in after), symbol
    assert seen == count
