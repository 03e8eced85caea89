"""The clear side's calls of the C ABI without a GPU: their refusals on a fake device, and the structs of the binding."""
import os
import subprocess

import test_host_client as H


def test_refusals_and_scratch_on_the_fake_device(tmp_path, monkeypatch):
    monkeypatch.setattr(H, "HOST_SOURCES", H.HOST_SOURCES + ["she_clear.cpp"])
    H.run_on_fake_device("clear_check.cpp", tmp_path)


def test_structs_are_the_header_s(tmp_path):
    """Sizes and the offset of every field."""
    from paper_1906_00148_amd import clear
    lines = [f'printf("%zu\\n", sizeof({s.name}));' for s in clear.LAYOUTS]
    lines += [f'printf("%zu\\n", offsetof({s.name}, {f}));' for s in clear.LAYOUTS for f, _ in s.fields]
    source = tmp_path / "offsets.c"
    source.write_text("#include <stddef.h>\n#include <stdio.h>\n#include \"she_clear.h\"\nint main(void) {" + "\n".join(lines) + "return 0; }")
    exe = str(tmp_path / "offsets")
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(H.ROOT, "include"), str(source), "-o", exe])
    got = [int(v) for v in subprocess.check_output([exe]).split()]
    assert got == [s.size for s in clear.LAYOUTS] + [s.offsets()[f] for s in clear.LAYOUTS for f, _ in s.fields]
