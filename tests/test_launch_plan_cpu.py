"""The host arithmetic behind launches (csrc/launch_plan.h), compiled for the host."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def run(tmp_path, body, includes=""):
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text('#include <cstdio>\n%s#include "launch_plan.h"\nint main() {\n%s\nreturn 0;\n}\n' % (includes, body))
    subprocess.run(["g++", "-std=c++17", "-O1", "-pthread", "-I", os.path.join(ROOT, "paper_2609_32415_gb300", "csrc"),
                    str(src), "-o", str(exe)], check=True)
    return subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()


def test_few_pieces_of_any_number_of_samples(tmp_path):
    """The product of samples and segments passes 31 bits: 2^30 rows are allowed, in up to three segments."""
    cases = [(b, s) for s in (1, 2, 3) for b in (1, 2, 4, 5, 6, 7, 12, 13, 32, 715827882, 715827883, (1 << 30) - 1, 1 << 30)]
    got = run(tmp_path, "\n".join('printf("%%d\\n", int(ra::few_pieces(%d, %d)));' % c for c in cases))
    assert [int(v) for v in got] == [int(1 < b * s <= 12) for b, s in cases]
