"""What a token attends to behind a shared prefix (csrc/clear_reach.h, compiled for the host)."""
import os
import subprocess

import test_host_client as H


def test_places_near_the_end_of_32_bits(tmp_path):
    from paper_1906_00148_amd import build as B
    exe = str(tmp_path / "reach_check")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-w", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(B.HIPCC))), "include"),
                           "-I", B.CSRC, os.path.join(H.CHECKS, "reach_check.cpp"), "-o", exe])
    ran = subprocess.run([exe], capture_output=True, text=True)
    assert ran.returncode == 0, ran.stdout
