"""How 16-bit rows at any address are stored: aligned 16-byte blocks shared by
neighbouring lanes, and what no block covers one by one. Each value of a row is
written once, and nothing beside the row. The rule is compiled for the host and
walked over every start, length and number of lanes."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include <stdio.h>
#include "nrq_ops.cuh"
int main() {
  static int hits[16 + 40 * 8 + 16];
  long cases = 0, singles = 0;
  for (int s = 0; s < 8; ++s)                 // values from an aligned address to the row's first
    for (int lanes = 1; lanes <= 32; lanes *= 2)
      for (int n = 1; n <= lanes * 8 + 3; ++n) {  // the last few: the row goes on in other lanes' hands
        for (int &h : hits) h = 0;
        int *row = hits + 8 + s;              // 8 values before the row's first aligned block
        for (int l = 0; l < lanes; ++l) {
          const Span16x8 w = span16x8(s, n - 8 * l, l > 0, l + 1 < lanes);
          if (w.block)
            for (int q = -s; q < 8 - s; ++q) ++row[8 * l + q];
          for (int q = w.from; q < w.to; ++q) ++row[8 * l + q], ++singles;
        }
        const int end = n < lanes * 8 ? n : lanes * 8;
        for (int i = 0; i < 16 + 40 * 8; ++i) {
          const int q = i - 8 - s, want = q >= 0 && q < end;
          if (hits[i] != want) {
            printf("start %d, %d lanes, %d values: value %d written %d times\n", s, lanes, n, q, hits[i]);
            return 1;
          }
        }
        ++cases;
      }
  printf("%ld rows, %ld values one by one\n", cases, singles);
  return 0;
}
"""


def test_every_value_is_written_once(tmp_path):
    src, exe = tmp_path / "spans.cu", str(tmp_path / "spans")
    src.write_text(SOURCE)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc, "-gencode", "arch=compute_103a,code=sm_103a", "-std=c++17", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2608_15438_gb300", "csrc"), "-o", exe, str(src)], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
