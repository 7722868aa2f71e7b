"""Counts of tiles near the largest capacity (the library's own header, compiled for the host)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_tiles_up_to_the_largest_capacity(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text("""
#include <cstdint>
#include <cstdio>
#include <initializer_list>
#include "kvc_internal.h"
int main() { for (int n : {0, 1, 64, 65, INT32_MAX - 63, INT32_MAX - 62, INT32_MAX}) std::printf("%d ", kvc::tile_count(n)); }
""")
    subprocess.check_call(["g++", "-std=c++17", "-O0", "-I", os.path.join(ROOT, "include"), "-I",
                           os.path.join(ROOT, "paper_2609_24298_amd", "csrc"), str(src), "-o", str(exe)])
    got = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    assert got == [0, 1, 1, 2, 2 ** 25 - 1, 2 ** 25, 2 ** 25]


def test_every_capacity_is_counted_by_it():
    csrc = os.path.join(ROOT, "paper_2609_24298_amd", "csrc")
    for name in sorted(os.listdir(csrc)):
        with open(os.path.join(csrc, name)) as f:
            assert "capacity + kTile" not in f.read(), name  # a sum of 32 bits overflows past 2^31 - 64
