"""CPU: what the kernels of dense layers need from a device is asked of every device of a process (csrc/per_device.hpp, per_device_check.cpp)."""
import os
import re
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_1710_06952_amd", "csrc")


def test_every_device_is_asked(tmp_path):
    exe = str(tmp_path / "check")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, os.path.join(HERE, "per_device_check.cpp"), "-o", exe])
    out = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0 and out.stdout == "ok\n"


def test_no_answer_is_kept_for_the_process():
    """No function-local static of one device's answer: hipFuncSetAttribute speaks for the device that is current."""
    for name in os.listdir(CSRC):
        if name.endswith((".hpp", ".hip", ".cpp")):
            with open(os.path.join(CSRC, name)) as f:
                assert not re.search(r"static const hipError_t", f.read()), name
