"""The range-checked loads of the 4-bit product: csrc's own offsets, compiled for the
host, and the library's code as built (no GPU). What a load's check counts is the
lane's offset and the instruction's; an offset in a scalar register may be left out of
it, so none is used."""
import os
import re
import shutil
import subprocess

import pytest

from paper_1611_06172_amd import w2v

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LLVM = "/opt/rocm/llvm/bin"
# Every load of every wavefront's sets of tiles, the sets past the end among them: it
# lies outside the range, or inside and then within the matrix; and what the product
# uses is inside, each word and scale in its place.
SOURCE = r"""
#include <cstdio>
#include <cstdlib>
#include <set>
#include "linear_q4.h"
using namespace w2v;
static int bad = 0;
static void test(const char* what, int64_t base, int64_t at, int size, int64_t range, int64_t all) {
  if (at < 0 || at % size != 0 || (at < range && (at + size > range || base + at + size > all))) {
    if (bad++ < 10) printf("%s: base %ld at %ld size %d range %ld of %ld\n", what, (long)base,
                           (long)at, size, (long)range, (long)all);
  }
}
int main(int argc, char** argv) {
  const int N = atoi(argv[1]), K = atoi(argv[2]), group = atoi(argv[3]), NT = atoi(argv[4]);
  const bool dense = argc > 5;  // also what is found where
  const Q4Shape q = q4_shape(N, K, group);
  const int GB = group / 32;
  const int64_t words = q.tiles * q.blocks * 256, scales = q.tiles * q.groups * 32;
  std::set<int64_t> used_words, used_scales, used_bias;
  for (int64_t end = dense ? 0 : q.tiles; end <= q.tiles; end++)
    for (int64_t tile = 0; tile <= q.tiles + 3 * NT; tile += NT) {
      const Q4Range r = q4_range(q, tile, end, NT, true);
      if (q4_range(q, tile, end, NT, false).bias != 0) bad++;
      for (int block = 0; block < q.blocks; block += 4) {
        if (!dense && block >= 64 && block < q.blocks - 8) continue;
        for (int t = 0; t < NT; t++)
          for (int lane = 0; lane < 64; lane++) {
            const int row = lane & 15, rest = q.blocks - block, g0 = block / GB;
            const bool there = tile + t < end;
            const int64_t w = q4_words_at(q, t, block, lane);
            if (rest >= 4) {
              test("four words", tile * q.blocks * 256, w, 16, r.words, words);
            } else {
              for (int i = 0; i < 3; i++)
                test("word", tile * q.blocks * 256, w + 4 * i, 4, r.words, words);
            }
            for (int i = 0; i < (rest < 4 ? rest : 4); i++) {
              if (there && w + 4 * i + 4 > r.words) bad++;
              if (!there && w + 4 * i < r.words) bad++;
              if (dense && there) used_words.insert(tile * q.blocks * 256 + w + 4 * i);
            }
            const int64_t s = q4_scales_at(q, t, g0, row);
            if (GB == 1 && q.groups - (g0 & ~3) >= 4)
              test("four scales", tile * q.groups * 32, s, 8, r.scales, scales);
            for (int i = 0; i < 4; i++)
              test("scale", tile * q.groups * 32, s + 2 * i, 2, r.scales, scales);
            for (int g = g0; g < q.groups && (g - g0) * GB < 4; g++) {
              if (there && s + 2 * (g - g0) + 2 > r.scales) bad++;
              if (dense && there) used_scales.insert(tile * q.groups * 32 + s + 2 * (g - g0));
            }
            const int64_t b = q4_bias_at(t, row);
            test("bias", tile * 64, b, 4, r.bias, 4 * (int64_t)N);
            const int64_t n = (tile + t) * 16 + row;
            if (there && n < N && b + 4 > r.bias) bad++;
            if (there && n < N && dense) used_bias.insert(tile * 64 + b);
          }
      }
    }
  if (dense && ((int64_t)used_words.size() * 4 != words ||
                (int64_t)used_scales.size() * 2 != scales || (int64_t)used_bias.size() != N))
    bad++;
  printf("%d\n", bad);
}
"""


@pytest.fixture(scope="module")
def offsets(tmp_path_factory):
    if shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"):
        pytest.skip("needs g++ and HIP's headers")
    folder = tmp_path_factory.mktemp("q4")
    source, exe = folder / "loads.cpp", str(folder / "loads")
    source.write_text(SOURCE)
    r = subprocess.run(
        ["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
         "-I" + os.path.join(ROOT, "include"),
         "-I" + os.path.join(ROOT, "paper_1611_06172_amd", "csrc"), str(source), "-o", exe],
        capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    return exe


def run(exe, *args):
    r = subprocess.run([exe, *map(str, args)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout == "0\n", (args, r.stdout, r.stderr)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("K", [1, 33, 65, 97, 128, 130, 161, 300, 385, 640, 1000])
def test_loads_stay_within_the_matrix(offsets, K, group):
    for N in (1, 15, 16, 17, 32, 33, 50, 90):
        for tiles in (1, 2):
            run(offsets, N, K, group, tiles, "dense")


@pytest.mark.parametrize("group", [32, 64, 128])
def test_loads_of_the_longest_rows(offsets, group):
    """Offsets of 2^24 columns stay below 2^31."""
    for tiles in (1, 2):
        run(offsets, 33, 1 << 24, group, tiles)
        run(offsets, 33, (1 << 24) - 127, group, tiles)


LOAD = re.compile(r"\bbuffer_load_\w+ .*?s\[\d+:\d+\], (\S+)")


def test_the_search_finds_a_scalar_offset():
    assert LOAD.search("\tbuffer_load_dwordx4 v[2:5], v9, s[4:7], s11 offen nt")[1] == "s11"
    assert LOAD.search("\tbuffer_load_ushort v2, v9, s[4:7], 0 offen offset:4")[1] == "0"


@pytest.mark.skipif(not os.path.exists(os.path.join(LLVM, "llvm-objdump")),
                    reason="llvm-objdump not found")
def test_no_load_has_a_scalar_offset(tmp_path):
    path = str(tmp_path / "libw2v.so")
    shutil.copy(w2v.LIB_PATH, path)
    dump = os.path.join(LLVM, "llvm-objdump")
    subprocess.run([dump, "--offloading", path], check=True, capture_output=True, timeout=120)
    loads = 0
    for f in sorted(os.listdir(tmp_path)):
        if not f.endswith("gfx950"):
            continue
        out = subprocess.run([dump, "-d", str(tmp_path / f)], check=True, capture_output=True,
                             text=True, timeout=240).stdout
        inside = False
        for line in out.splitlines():
            head = re.match(r"^[0-9a-f]+ <(.+)>:$", line)
            if head:
                inside = "k_linear_q4" in head[1]
            load = LOAD.search(line.split("//")[0]) if inside else None
            if load:
                loads += 1
                assert load[1] == "0", line
    assert loads > 100
