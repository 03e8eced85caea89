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


def test_scratch_follows_the_rows_and_not_the_table(shapes):
    """Single tokens of 8 key heads of 128 and four rows each: pieces of the rows that there are, and not as many as a wide table has
    room for."""
    tokens, widths = (1, 16, 64, 256, 1024, 5000), (1 << 10, 1 << 14, 1 << 17, 1 << 22)
    for T in tokens:
        got = shapes([(T, T, 32, 8, 128, 0, w // 16, 16) for w in widths])
        for w, (kernel, tiles, chunk, pieces, scratch) in zip(widths, got):
            assert kernel == "few" and scratch == (T * 32 * pieces * (128 + 2) * 4 if pieces > 1 else 0), (T, w)
            assert pieces <= max(8, 32 * 512 // (tiles * 8) + 1)
            # pieces of a full table end on time: no fewer of them than the table's places in pieces of 2048, up to eight
            assert pieces >= min(8, w // 2048)
        # tables of up to 16384 places are cut as finely as places that are looked up together allow
        assert all(g[3] * g[2] >= w for w, g in zip(widths[:2], got))
