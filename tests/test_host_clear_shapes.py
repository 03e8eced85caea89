"""What the host decides for an attention call (csrc/clear_attend_shape.cpp, compiled for the host): the kernel, its pieces, the scratch."""
import os
import subprocess

import pytest

import test_gpu_clear_attend_tile as A
import test_host_client as H


@pytest.fixture(scope="module")
def shapes(tmp_path_factory):
    """calls -> for each (kernel, tiles, places of a piece, pieces, bytes of scratch)"""
    from paper_1906_00148_amd import build as B
    exe = str(tmp_path_factory.mktemp("shape") / "attend_shape")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-w", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(B.HIPCC))), "include"),
                           "-I", B.CSRC, os.path.join(B.CSRC, "clear_attend_shape.cpp"), os.path.join(H.CHECKS, "attend_shape.cpp"), "-o", exe])

    def ask(calls):
        text = "".join(" ".join(map(str, c)) + "\n" for c in calls)
        lines = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(lines) == len(calls)
        return [(k, *map(int, rest)) for k, *rest in (line.split() for line in lines)]
    return ask


def test_the_calls_of_the_tile_kernel_s_tests_are_that_kernel_s(shapes):
    calls = A.calls()
    got = shapes(calls)
    assert [c for c, s in zip(calls, got) if s[0] != "tile"] == []
    # whole tiles and cut ones, and every padded size of a head, with a window and without
    assert {(s[3] > 1, c[5] > 0, 64 if c[4] <= 64 else 128 if c[4] <= 128 else 256) for c, s in zip(calls, got)} == \
        {(cut, window, head) for cut in (False, True) for window in (False, True) for head in (64, 128, 256)}
