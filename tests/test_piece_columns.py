"""Where the adapters' first product reads 16 bytes of a row (opd_piece.h), compiled for the
host: for every width of a row up to four steps, every piece of a step and every type, the
read lies in the row rounded up to whole pieces, and a piece that has columns of the row
is read where it is."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_24143_amd", "csrc")

PROGRAM = r"""
#include "opd_piece.h"
#include <cstdio>

// pieces: 16-byte pieces of a step; steps: of the waves that take a row in turn
template <int EACH>
int check(int pieces, int steps) {
  int wrong = 0;
  for (int64_t end = 1; end <= 4 * EACH * pieces + 1; ++end) {
    const int64_t whole = (end + EACH - 1) / EACH * EACH;
    for (int s = 0; s < steps; ++s) {
      for (int p = 0; p < pieces; ++p) {
        const int64_t d = (int64_t)s * EACH * pieces, mine = d + (int64_t)p * EACH;
        const int64_t c = opd::piece_column<EACH>(d, p, end);
        if (c < 0 || c % EACH != 0 || c + EACH > whole || (mine < end && c != mine)) {
          if (++wrong <= 5)
            std::printf("%d columns a piece, width %lld, step %d, piece %d: column %lld\n", EACH,
                        (long long)end, s, p, (long long)c);
        }
      }
    }
  }
  return wrong;
}

int main() {
  // bf16 rows in steps of 64 columns, fp32 ones and bf16 ones beside them in steps of 32
  const int wrong = check<8>(8, 8) + check<4>(8, 8) + check<8>(4, 8);
  return wrong ? 1 : 0;
}
"""


def test_no_piece_lies_past_its_row(tmp_path):
    source, program = tmp_path / "piece.cpp", tmp_path / "piece"
    source.write_text(PROGRAM)
    build = subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined",
                            "-fno-sanitize-recover=all", "-I", CSRC, "-o", str(program),
                            str(source)], capture_output=True, text=True)
    assert build.returncode == 0, build.stderr
    run = subprocess.run([str(program)], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0, run.stdout + run.stderr

