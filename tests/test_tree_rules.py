"""Launch rules of a tree's attention (csrc/eq_attn_rules.h), compiled with the host
compiler: those of causal attention but for the chunks of batches that fill the card by
themselves, which the device sets from all lengths."""
import os
import subprocess

import pytest

from paper_2601_22787_amd import _build
from test_attn_rules import _rows

PROG = r"""
#include <cstdio>
#include "eq_attn_rules.h"
int main() {
  unsigned v[6];
  while (scanf("%u %u %u %u %u %u", v, v + 1, v + 2, v + 3, v + 4, v + 5) == 6) {
    for (int tree = 0; tree < 3; ++tree) {
      const eq_attn::Plan p = eq_attn::plan_attn(v[0], v[1], v[2], v[3], v[4], tree == 2 ? 0 : v[5], tree > 0);
      printf("%d %u %u %u %u %u ", p.prompt, p.cols, p.tile, p.q_tiles, p.chunks, p.chunk_tiles);
    }
    printf("%u\n", eq_attn::head_blocks(v[1]));
  }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    d = tmp_path_factory.mktemp("tree_rules")
    src, exe = os.path.join(d, "rules.cpp"), os.path.join(d, "rules")
    with open(src, "w") as f:
        f.write(PROG)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined",
                    "-fno-sanitize-recover=all", "-I", _build.CSRC, src, "-o", exe], check=True)

    def run(rows):
        text = "\n".join(" ".join(str(v) for v in r[:6]) for r in rows)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True)
        return [[int(v) for v in line.split()] for line in out.stdout.splitlines()]
    return run


def test_chunks_hold_every_token_and_a_window_needs_no_more(plans):
    rows = [(s, k, g, min(n, 256), t, w) for s, k, g, n, t, w, _ in _rows(20000, 9)]
    shared = 0
    for (seqs, kv, group, new, longest, window), got in zip(rows, plans(rows)):
        causal, tree, unbounded, run = got[:6], got[6:12], got[12:18], got[18]
        prompt, _, tile, q_tiles, chunks, length = tree
        work = seqs * kv * q_tiles
        seen = -(-longest // tile)
        if window:
            seen = min(seen, (window + new + tile - 2) // tile + 1)
        assert chunks * length >= seen and chunks <= unbounded[4]
        assert tree[:4] == causal[:4] and run == max(512 // kv, 1)
        if not (prompt and seqs <= 64 and 256 <= work <= 1024 and longest >= 8192):
            assert tree == causal
            continue
        assert causal[4] == 1 and work * (chunks - 1) < 2048 and unbounded[5] * tile >= 1024
        shared += chunks > 1
    assert shared > 100
