"""KV heads of an attention tile (csrc/chunk_kernels.h), on the CPU: a tile whose
waves share its stages is of one KV head, and no tile has more units (a KV head and a
row tile) than the workgroup has waves."""
import os
import subprocess

import pytest

import host_sanitizer

SOURCE = r"""
#include <cstdio>
#include "chunk_kernels.h"
using namespace spork;

// Every number of packed rows that a tile can have, every number of KV heads that a batch may let it take.
template <int NARROW>
int check() {
  for (int group = 1; group <= kChunkTileRows; ++group)
    for (int rows = 1; rows * group <= kChunkTileRows; ++rows)
      for (int most = 1; most <= kChunkWaves; most *= 2) {
        const int row_tiles = (rows * group + 31) / 32, heads = chunk_heads<NARROW>(most, row_tiles);
        const bool shared = row_tiles > NARROW;
        const bool good = heads >= 1 && heads <= most && heads * row_tiles <= kChunkWaves && (heads & (heads - 1)) == 0 &&
                          (!shared || heads == 1) && (shared || most * row_tiles > kChunkWaves || heads == most);
        if (!good) {
          std::printf("%d row tiles at most, %d x %d packed rows, %d heads at most: %d\n", NARROW, rows, group, most, heads);
          return 1;
        }
      }
  return 0;
}

int main() { return check<1>() || check<2>() || check<4>() || check<kChunkWaves>(); }
"""


def test_tiles_that_share_stages_are_of_one_head(tmp_path):
    src, exe = tmp_path / "heads.cpp", tmp_path / "heads"
    src.write_text(SOURCE)
    cmd = ["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-D__HIP_PLATFORM_AMD__",
           f"-I{os.path.join(host_sanitizer.ROCM, 'include')}", f"-I{host_sanitizer.CSRC}", str(src), "-o", str(exe)]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        pytest.fail(r.stdout)
    r = subprocess.run([str(exe)], stdout=subprocess.PIPE, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
