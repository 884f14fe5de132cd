"""Attention's tile arithmetic (csrc/attend_tile.hpp), the kernels' own code compiled for the host: no length, start, window or bound makes a
key that is none, or a look-up outside the table.  Under UndefinedBehaviorSanitizer, so that no sum of them passes 32 bits."""
import os
import shutil
import subprocess
from pathlib import Path

import pytest

from paper_2403_07221_amd import binding

ROOT = Path(__file__).resolve().parent.parent
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CLANG = "/opt/rocm/lib/llvm/bin/clang++"


@pytest.mark.skipif(not (shutil.which(HIPCC) and shutil.which(CLANG)), reason="hipcc / clang not found")
def test_tiles_of_any_lengths(tmp_path):
    obj, exe = tmp_path / "tile.o", tmp_path / "tile"
    build = [[HIPCC, "--cuda-host-only", "-x", "hip", "-O1", "-g", "-std=c++17", "-Wno-unused-command-line-argument",
              "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined",
              f"-I{ROOT / 'paper_2403_07221_amd' / 'csrc'}", "-c", "-o", str(obj), str(ROOT / "tests" / "sanitize" / "attend_tile_driver.cpp")],
             [CLANG, "-fsanitize=undefined", "-o", str(exe), str(obj)]]
    for cmd in build:
        p = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
        assert p.returncode == 0, p.stdout[-3000:]
    p = subprocess.run([str(exe)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert p.returncode == 0 and "ran clean" in p.stdout and "runtime error" not in p.stdout, p.stdout[-3000:]


def test_the_most_rows():
    """What the driver takes as the most rows is what attention refuses to go beyond (a type that is none tells what is looked at after)."""
    L, fake = binding.lib(), 1 << 20

    def attend(n, heads, kv):
        return L.lookupffn_attend(fake, fake, fake, fake, fake, fake, fake, fake, fake, n, 1, heads, kv, 64, 7, 16, 2, 2, None, n, 32, 1, 0, 3, None, 0, None)

    most = (1 << 31) - 256
    for heads in (2, 4, 8):
        assert attend(most // heads, heads, 2) == -4 and attend(most // heads + 1, heads, 2) == -2
    assert attend(1 << 30, 1, 1) == -4 and attend((1 << 30) + 1, 1, 1) == -2
