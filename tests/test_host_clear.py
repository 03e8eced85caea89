"""The clear side's calls of the C ABI without a GPU: their refusals on a fake device, and the structs of the binding."""
import ctypes as C
import os
import subprocess

import test_host_client as H


def test_refusals_and_scratch_on_the_fake_device(tmp_path, monkeypatch):
    monkeypatch.setattr(H, "HOST_SOURCES", H.HOST_SOURCES + ["she_clear.cpp"])
    H.run_on_fake_device("clear_check.cpp", tmp_path)


def test_structs_are_the_header_s(tmp_path):
    """Sizes and the offset of every field."""
    from paper_1906_00148_amd import clear
    structs = [clear._Adapters, clear._AdaptersGrad, clear._QkRotate, clear._QkRotateGrad, clear._AttendPages]
    lines = [f'printf("%zu\\n", sizeof({s.__name__}));' for s in structs]
    lines += [f'printf("%zu\\n", offsetof({s.__name__}, {f}));' for s in structs for f, _ in s._fields_]
    source = tmp_path / "offsets.c"
    source.write_text("#include <stddef.h>\n#include <stdio.h>\n#include \"she_clear.h\"\nint main(void) {" + "\n".join(lines) + "return 0; }")
    exe = str(tmp_path / "offsets")
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(H.ROOT, "include"), str(source), "-o", exe])
    got = [int(v) for v in subprocess.check_output([exe]).split()]
    assert got == [C.sizeof(s) for s in structs] + [getattr(s, f).offset for s in structs for f, _ in s._fields_]
