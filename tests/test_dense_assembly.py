"""CPU: what the compiler makes of the large tiles' products, which are written as instructions of their own (csrc/dense_large.hpp).  It does not know
that a result comes some cycles later, so nothing between the last product and the wait behind the loop may touch the result of one of the last
eight: a product takes 8 passes of 4 cycles, and a read of its result 11 wait states more."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1710_06952_amd", "csrc")


def registers(text):
    """The accumulation registers that an instruction names."""
    of = set()
    for one, first, last in re.findall(r"\ba(?:(\d+)|\[(\d+):(\d+)\])", text):
        of.update([int(one)] if one else range(int(first), int(last) + 1))
    return of


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_no_result_is_touched_before_it_is_there(tmp_path, dtype):
    from paper_1710_06952_amd import build
    out = str(tmp_path / "dense.s")
    subprocess.run([build.hipcc(), *build.FLAGS, "--offload-device-only", "-S", "-x", "hip", os.path.join(CSRC, "kernels_dense_%s.hip" % dtype), "-o", out], check=True,
                   stderr=subprocess.DEVNULL)
    kernels, lines = {}, None
    with open(out) as f:
        for line in f:
            name = re.match(r"^(_Z\S+):", line)
            if name:
                lines = kernels.setdefault(name[1], [])
            elif lines is not None and re.match(r"^\s+[a-z]", line):
                lines.append(line.split(";")[0].strip())
    large = {k: v for k, v in kernels.items() if "dense_large_kernel" in k}
    assert len(large) == 6
    for name, lines in large.items():
        last = max(i for i, s in enumerate(lines) if s.startswith("v_mfma"))
        wait = lines.index("s_nop 15", last)
        written = [registers(s.split(",")[0]) for s in lines[:last + 1] if s.startswith("v_mfma")][-8:]
        early = [s for s in lines[last + 1:wait] if any(registers(s) & w for w in written)]
        assert len(set().union(*written)) == 32 and not early and lines[wait + 1] == "s_nop 15", (name, early)
