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


def test_resident_clusters_are_those_of_the_device_and_kernel(tmp_path):
    """Each (device, kernel, shared memory) has its own counts, asked once; a failed query is not kept."""
    got = run(tmp_path, r"""
      static ra::ClusterTable table;
      static int asked;
      const int kernels[2] = {0, 0};
      auto count = [&](int device, int kernel, int smem, int c, bool fails = false) {
        return table.get(device, kernels + kernel, smem, [&](int size) {
          ++asked;
          return fails ? -(size == 5) : 10000 * device + 1000 * kernel + 100 * (smem > 1000) + size;
        }).of[c];
      };
      printf("%d %d ", count(1, 0, 500, 4, true), count(1, 0, 500, 5, true));  // failed: not kept
      for (int again = 0; again < 2; ++again) {
        printf("%d %d %d %d ", count(1, 0, 500, 4), count(1, 1, 500, 4), count(2, 0, 500, 8), count(1, 0, 2000, 1));
        printf("%d ", asked);
      }
      for (int device = 3; device < 300; ++device)  // past the end of the table
        if (count(device, 1, 500, 2) != 10000 * device + 1002) return 1;
      printf("%d\n", count(1, 0, 500, 4));
    """)
    assert [int(v) for v in got] == [0, 1, 10004, 11004, 20008, 10101, 48, 10004, 11004, 20008, 10101, 48, 10004]


def test_overlap_of_rows_is_seen_where_it_is_certain(tmp_path):
    """Against the sets of bytes: never said of tensors apart, always of one address and of dense ranges."""
    import itertools
    spans = [(0, 0, 64, 1, 4, 64), (64, 0, 64, 1, 4, 64), (192, 0, 64, 1, 1, 64), (256, 256, 64, 2, 4, 64),
             (0, 0, 128, 1, 4, 64), (64, 0, 128, 1, 4, 64), (0, 512, 128, 2, 4, 64), (0, 64, 128, 2, 4, 64),
             (240, 0, 0, 1, 1, 16), (256, 0, 0, 1, 1, 0), (0, 64, 0, 4, 1, 64), (64, 0, 64, 1, 0, 64)]
    body = "const char* base = reinterpret_cast<const char*>(1 << 20);\nconst ra::RowSpan t[] = {%s};\n" % ", ".join(
        "{base + %d, %d, %d, %d, %d, %d}" % s for s in spans)
    body += 'for (auto& a : t) for (auto& b : t) printf("%d\\n", int(ra::surely_overlap(a, b)));\n'
    body += 'ra::RowSpan gone = t[0]; gone.ptr = nullptr; printf("%d\\n", int(ra::surely_overlap(gone, gone)));'
    got = [bool(int(v)) for v in run(tmp_path, body)]

    def bytes_of(at, ss, sr, B, n, size):
        return {at + s * ss + r * sr + i for s in range(B) for r in range(n) for i in range(size)}

    def dense(at, ss, sr, B, n, size):
        return len(bytes_of(at, ss, sr, B, n, size)) == max(bytes_of(at, ss, sr, B, n, size), default=0) - at + 1 == B * n * size

    for (a, b), said in zip(itertools.product(spans, spans), got):
        shared = bool(bytes_of(*a) & bytes_of(*b))
        if said:
            assert shared, (a, b)
        elif shared:
            assert a[0] != b[0] and not (dense(*a) and dense(*b)), (a, b)
    assert got[-1] is False
