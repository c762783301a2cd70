"""Rows of every alignment on their way to shared memory (csrc/row_copy.h): what is read lies inside the tensor, what arrives is the row."""
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_18719_gb300", "csrc")

PROGRAM = r"""
#include <stdio.h>
#include <string.h>
#include "row_copy.h"
int main() {
  alignas(64) static unsigned char memory[4096];
  long n_copies = 0;
  for (int i = 0; i < 4096; ++i) memory[i] = (unsigned char)(i * 37 + (i >> 8));
  for (int size = 2; size <= 4; size += 2)
    for (int off = 0; off < 32; off += size)
      for (int dim = 1; dim <= 40; ++dim)
        for (int gap = 0; gap <= 9; ++gap)
          for (int rows = 1; rows <= 5; ++rows)
            for (int r = 0; r < rows; ++r) {
              const unsigned n = dim * size;
              const uintptr_t origin = (uintptr_t)memory, lo = origin + 512 + off, ld = (dim + gap) * size;
              const uintptr_t hi = lo + (rows - 1) * ld + n, p = lo + r * ld;
              const vla::RowCopy c = vla::row_copy(p, n, lo, hi);
              unsigned char stage[512];
              const unsigned room = (n + 31u) & ~15u;
              memset(stage, 0, sizeof stage);
              if (c.head >= 16 || c.tail >= 16 || (c.head & 1) || (c.tail & 1) || c.head > n || c.tail > n) return 1;
              if ((c.from & 15) || (c.bytes & 15)) return 2;
              if (c.bytes) {
                const uintptr_t at = c.from - (p & ~(uintptr_t)15);
                if (c.from < lo || c.from + c.bytes > hi) return 3;          // reads inside the tensor
                if ((at & 15) || at + c.bytes > room) return 4;              // lands inside the stage
                memcpy(stage + at, (const void*)c.from, c.bytes);
              }
              for (unsigned i = 0; i < c.head; ++i) stage[(p & 15) + i] = *(const unsigned char*)(p + i);
              for (unsigned i = n - c.tail; i < n; ++i) stage[(p & 15) + i] = *(const unsigned char*)(p + i);
              if (memcmp(stage + (p & 15), (const void*)p, n)) return 5;      // the row, whole
              ++n_copies;
            }
  printf("%ld\n", n_copies);
  return 0;
}
"""


def test_rows_of_every_alignment(tmp_path):
    src, exe = tmp_path / "rows.cc", tmp_path / "rows"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and int(out.stdout) == 24 * 40 * 10 * 15, (out.returncode, out.stdout)


def test_the_norm_gradient_reads_by_it_at_the_ends():
    text = open(os.path.join(CSRC, "block_norm.cu")).read()
    request = text[text.index("auto request = "):text.index("auto add_ends = ")]
    at_ends = request[request.index("if (is_end(r)) {"):request.index("return;")]
    assert text.count("bulk_load(") == request.count("bulk_load(") == 2 and at_ends.count("bulk_load(") == 1
    assert "c.from), c.bytes" in at_ends and "copy_of(r, k)" in at_ends and "if (is_end(r)) add_ends(r, buf);" in text
    assert "row_copy(lo + static_cast<uintptr_t>(r * ld[k]), n, lo, lo + static_cast<uintptr_t>((a.f.rows - 1) * ld[k]) + n)" in text
    # rows that are not among `ends` have 16 bytes of their tensor before and behind them, of the narrowest type and without gaps
    assert "const int ends = V < 8 ? (8 + dim - 1) / dim : 0;" in text
    for dim in range(1, 40):
        assert (8 + dim - 1) // dim * dim * 2 >= 16


def test_every_lane_takes_part_in_the_shuffles():
    # a shuffle in one arm of a choice, or behind a lane's `continue`, reads lanes that are not there
    for path in sorted(os.listdir(CSRC)):
        for line in open(os.path.join(CSRC, path)):
            for call in ("__shfl_sync(", "__shfl_down_sync(", "__shfl_up_sync(", "__shfl_xor_sync("):
                before = line.split("//")[0].partition(call)[0]
                assert not re.search(r"(\blane\b|threadIdx)[^;]*\?[^;]*$", before), (path, line)
