"""How the library is built (build.py), with a compiler that only writes down what it is called with."""
import json
import os
import sys

from paper_1906_00148_amd import build as B


def test_flags_of_the_caller_reach_every_compilation_and_the_link(tmp_path, monkeypatch):
    log, compiler = tmp_path / "calls", tmp_path / "compiler"
    compiler.write_text(f"#!{sys.executable}\nimport json, sys\nopen(sys.argv[sys.argv.index('-o') + 1], 'w').close()\n"
                        f"open({str(log)!r}, 'a').write(json.dumps(sys.argv[1:]) + '\\n')\n")
    os.chmod(compiler, 0o755)
    monkeypatch.setattr(B, "HIPCC", str(compiler))
    extra = ["-DANYTHING=1", "--coverage", "-L/some/where"]
    out = str(tmp_path / "lib.so")
    assert B.build(extra=extra, out=out) == out and os.path.exists(out)
    calls = [json.loads(line) for line in log.read_text().splitlines()]
    links = [c for c in calls if "-c" not in c]
    assert len(calls) == len(B.SOURCES) + 1 and len(links) == 1
    for c in calls:
        assert all(f in c for f in extra), c
        assert ("-shared" in c) == (c in links) and all(f in c for f in B.FLAGS if f != "-shared")
