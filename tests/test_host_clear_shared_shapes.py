"""What the host decides for a call with shared prefixes (csrc/clear_attend_shape.cpp, compiled for the host): the walks, their pieces, the scratch."""
import os
import subprocess

import pytest

import test_gpu_clear_shared_walks as W
import test_host_client as H


@pytest.fixture(scope="module")
def shapes(tmp_path_factory):
    """calls -> for each (prefix walk, own walk, pieces of either, bytes of scratch)"""
    from paper_1906_00148_amd import build as B
    exe = str(tmp_path_factory.mktemp("shape") / "shared_shape")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-w", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(B.HIPCC))), "include"),
                           "-I", B.CSRC, os.path.join(B.CSRC, "clear_attend_shape.cpp"), os.path.join(H.CHECKS, "shared_shape.cpp"), "-o", exe])

    def ask(calls):
        text = "".join(" ".join(map(str, c)) + "\n" for c in calls)
        lines = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(lines) == len(calls)
        return [(p, b, *map(int, rest)) for p, b, *rest in (line.split() for line in lines)]
    return ask


def test_the_calls_of_the_walks_tests_go_their_ways(shapes):
    calls = W.shapes()
    got = {name: (p, b, own > 1) for name, (p, b, _, own, _) in zip(calls, shapes(list(calls.values())))}
    assert got == {name: c[0] for name, c in W.CALLS.items()}
    padded = {name: 64 if c[1][2] <= 64 else 128 if c[1][2] <= 128 else 256 for name, c in W.CALLS.items()}
    ways = {(*got[name][:2], padded[name]) for name in calls}
    # heads of more than 128 have no tiles of many rows behind a prefix's: they go as one walk
    assert ways >= {(p, b, d) for p, b in (("few", "few"), ("tile", "few")) for d in (64, 128, 256)} | {("tile", "tile", 64), ("tile", "tile", 128)} | \
        {("whole", b, d) for b in ("few", "tile") for d in (64, 128, 256)}


def test_scratch_follows_the_rows(shapes):
    """Wide tables that few requests fill do not make pieces without end; a call of many tokens has few of them."""
    for tokens, requests in ((1, 1), (64, 64), (1000, 1000), (4000, 8), (20000, 20)):
        for prefix in (10, 1 << 12, 1 << 16, 1 << 20):
            for own in (1, 100, 1 << 13, 1 << 20):
                (p, b, of_prefix, of_own, scratch), = shapes([(tokens, requests, 32, 8, 128, 0, 1, prefix // 16 + 1, own // 16 + 1, 16)])
                pieces = of_own if p == "whole" else of_prefix + of_own
                assert scratch == (0 if pieces == 1 else tokens * 32 * pieces * 130 * 4)
                assert of_prefix <= 64 and scratch <= 1 << 32, (tokens, prefix, own, p, b, of_prefix, of_own)
