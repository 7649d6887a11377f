"""Host arithmetic of the layer operators that no test can reach on a GPU: built from their headers and run on the CPU."""
import os
import subprocess

from paper_2305_16588_amd import build


def run(tmp_path, text):
    src, exe = str(tmp_path / "main.hip"), str(tmp_path / "main")
    with open(src, "w") as f:
        f.write(text)
    r = subprocess.run([build.HIPCC, *build.FLAGS, "-o", exe, src], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr


def test_parts_of_a_document_are_all_of_it(tmp_path):
    """Up to as many keys as the entry points take: each part begins where the one before ends."""
    assert os.path.exists(os.path.join(build.CSRC, "attend.hpp"))
    run(tmp_path, r"""
#include "attend.hpp"
#include <cstdio>
int main() {
  for (int32_t keys : {0, 1, 31, 32, 33, 1000, 50001, 1 << 30, 2147450880, 2147450881, 2147483391})
    for (int32_t size : {32, 64})
      for (int32_t splits : {1, 2, 7, 255, 256, 1024}) {
        int64_t at = 0;
        for (int32_t s = 0; s < splits; ++s) {
          int32_t begin, end;
          lgp::layer::part_of(keys, size, s, splits, begin, end);
          if (begin != at || end < begin || end > keys || (begin % size && begin != keys)) return std::printf("%d keys by %d, part %d of %d: %d to %d\n", keys, size, s, splits, begin, end), 1;
          at = end;
        }
        if (at != keys) return std::printf("%d keys by %d in %d parts: %lld\n", keys, size, splits, (long long)at), 1;
      }
  return 0;
}
""")
