"""How the norm's gradient shares its blocks out (csrc/norm_grid.h), compiled for the host: over all
head counts no more blocks than its workspace has rows, and some for each kind of head (no GPU)."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_24063_gb300", "csrc")

PROGRAM = r"""
#include <initializer_list>
#include <stdio.h>
#include "norm_grid.h"
int main() {
  for (int64_t n_rows : {1, 16, 17, 160, 4848, 4849, 4864, 4865, 12544, 1 << 24})
    for (int Hq = 0; Hq <= 4096; ++Hq)
      for (int Hkv = Hq ? 0 : 1; Hkv <= 4096; Hkv += Hkv < 40 || Hkv > 2300 || Hq < 40 ? 1 : 37) {
        const vc::NormGradGrid g = vc::norm_grad_grid(n_rows, Hq, Hkv);
        const int64_t groups = (n_rows + vc::kGradRows - 1) / vc::kGradRows;
        if (g.nq + g.nk > vc::kNormGradBlocks || (Hq > 0) != (g.nq > 0) || (Hkv > 0) != (g.nk > 0) || g.nq > groups ||
            g.nk > groups) {
          printf("%lld rows, %d + %d heads: %d + %d blocks\n", (long long)n_rows, Hq, Hkv, g.nq, g.nk);
          return 1;
        }
      }
  return 0;
}
"""


def test_no_more_blocks_than_the_workspace_has_rows(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    (tmp_path / "grid.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", CSRC, str(tmp_path / "grid.cpp"), "-o", str(tmp_path / "grid")],
                   check=True)
    run = subprocess.run([str(tmp_path / "grid")], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0, run.stdout
