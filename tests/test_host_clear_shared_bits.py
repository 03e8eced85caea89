"""Which calls with shared prefixes take their weights as two numbers (csrc/clear_attend_shape.cpp, compiled for the host)."""
import os
import subprocess

import test_host_client as H


def test_no_fewer_bits_than_attention_over_one_row(tmp_path):
    from paper_1906_00148_amd import build as B
    exe = str(tmp_path / "shared_bits")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-w", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(B.HIPCC))), "include"),
                           "-I", B.CSRC, os.path.join(B.CSRC, "clear_attend_shape.cpp"), os.path.join(H.CHECKS, "shared_bits.cpp"), "-o", exe])
    ran = subprocess.run([exe], capture_output=True, text=True)
    assert ran.returncode == 0, ran.stdout
