"""How the library cuts calls over shared rows and chosen blocks, from the planning functions that the entry points use:
a C++ program linked with the library prints them (host code, no GPU)."""
import os
import shutil
import subprocess
import tempfile

from paper_2608_08878_amd import binding as B

CSRC = os.path.join(os.path.dirname(B.LIB_PATH), "csrc")

PROGRAM = r"""
#include <cstdio>
#include <cstring>
#include "dc_kernels.hpp"
int main() {
  char kind;
  int dtype, D, batch, hk, gshift, tokens, most, L, x, y, z;
  while (scanf(" %c %d %d %d %d %d %d %d %d %d %d %d", &kind, &dtype, &D, &batch, &hk, &gshift, &tokens, &most, &L, &x, &y,
               &z) == 12) {
    dc::SharedArgs s;
    dc::BlockArgs b;
    memset(&s, 0, sizeof s);
    memset(&b, 0, sizeof b);
    dc::AttendArgs& a = kind == 'S' ? (dc::AttendArgs&)s : (dc::AttendArgs&)b;
    a.tok.tokens = tokens;
    a.tok.max_tokens = most;
    a.batch = batch;
    a.n_layers = 1;
    a.hq = hk << gshift;
    a.hk = hk;
    a.gshift = gshift;
    bool ok;
    if (kind == 'S') {
      s.prefixes = x;
      s.max_members = y;
      s.plen = z;
      const long all = (long)y * most;
      s.group_tokens = (int)(all < tokens ? all : tokens);
      ok = dc::shared_plan(s, dtype, D, L, z > 0 ? z : 1);
    } else {
      b.count = x;
      b.bshift = y == 16 ? 4 : y == 32 ? 5 : y == 64 ? 6 : 7;
      b.share = z;
      b.groups = (most + z - 1) / z;
      ok = dc::block_plan(b, dtype, D, L);
    }
    printf("%d %d %d %d %d %d\n", (int)ok, a.bm, s.through, s.psplits, a.splits, a.once);
  }
}
"""


def can_ask():
    return os.path.exists(B.LIB_PATH) and shutil.which("g++") is not None


def ask(lines):
    """For every line (ok, rows of a tile, through, parts of the shared rows, parts, once)."""
    libdir = os.path.dirname(B.LIB_PATH)
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "plans.cpp"), os.path.join(d, "plans")
        with open(src, "w") as f:
            f.write(PROGRAM)
        subprocess.run(["g++", "-std=c++17", "-O0", "-I", CSRC, "-I", os.path.join(CSRC, "../../include"), src, "-o", exe,
                        "-L", libdir, "-ldistillcache", "-Wl,-rpath," + libdir], check=True, capture_output=True, text=True)
        r = subprocess.run([exe], input="\n".join(lines) + "\n", check=True, capture_output=True, text=True, timeout=300)
    return [tuple(int(x) for x in line.split()) for line in r.stdout.splitlines()]


def shared_line(dtype, D, hk, G, counts, members, plen, rows):
    return " ".join(map(str, ("S", int(dtype == "bf16"), D, len(counts), hk, G.bit_length() - 1, sum(counts), max(counts),
                              rows + max(counts), len(members), max(members), plen)))


def blocks_line(dtype, D, hk, G, counts, n, block, count, share):
    return " ".join(map(str, ("B", int(dtype == "bf16"), D, len(counts), hk, G.bit_length() - 1, sum(counts), max(counts),
                              n + max(counts), count, block, share)))
