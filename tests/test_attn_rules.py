"""Launch rules of attention over the 4-bit cache (csrc/eq_attn_rules.h),
compiled with the host compiler: every token that a query sees is in a chunk,
a window never needs more workspace, and the Python copy that GPU tests use to
name their paths."""
import os
import random
import subprocess

import pytest

import attn_rules
from paper_2601_22787_amd import _build

PROG = r"""
#include <cstdio>
#include "eq_attn_rules.h"
int main() {
  unsigned v[7];
  while (scanf("%u %u %u %u %u %u %u", v, v + 1, v + 2, v + 3, v + 4, v + 5, v + 6) == 7) {
    const eq_attn::Plan p = eq_attn::plan_attn(v[0], v[1], v[2], v[3], v[4], v[5]);
    printf("%d %u %u %u %u %u %d %d\n", p.prompt, p.cols, p.tile, p.q_tiles, p.chunks, p.chunk_tiles,
           eq_attn::pair_columns(v[3], v[2]), STREAM);
  }
}
"""
STREAM = "eq_attn::stream_cache(p, v[0], v[1], v[6], v[3], v[4], v[5])"


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("attn_rules")
    src, exe = os.path.join(d, "rules.cpp"), os.path.join(d, "rules")
    with open(src, "w") as f:
        f.write(PROG.replace("STREAM", STREAM))
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined",
                    "-fno-sanitize-recover=all", "-I", _build.CSRC, src, "-o", exe], check=True)

    def run(rows):
        text = "\n".join(" ".join(str(v) for v in r) for r in rows)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True)
        return [attn_rules.Plan(*(int(v) for v in line.split())) for line in out.stdout.splitlines()]
    return run


def _log(r, lo, hi):
    return min(hi, max(lo, int(2 ** r.uniform(lo.bit_length() - 1, hi.bit_length()))))


def _rows(n, seed):
    """sequences, key/value heads, group, new tokens, longest length, window, channels"""
    r = random.Random(seed)
    return [(_log(r, 1, 512), _log(r, 1, 64), _log(r, 1, 64), _log(r, 1, 8192), _log(r, 1, 1 << 20),
             r.choice([0, 0, 1, _log(r, 1, 8192), _log(r, 1, 1 << 21), (1 << 32) - 1]),
             r.choice([64, 128])) for _ in range(n)]


def test_the_python_copy_is_the_rule(rules):
    rows = _rows(20000, 1)
    for row, got in zip(rows, rules(rows)):
        assert got == tuple(int(v) for v in attn_rules.plan(*row)), row


def test_every_seen_token_is_in_a_chunk(rules):
    rows = _rows(4000, 2)
    r = random.Random(3)
    whole = rules([row[:5] + (0, row[6]) for row in rows])
    for row, p, w in zip(rows, rules(rows), whole):
        _, _, group, max_new, max_len, window, _ = row
        assert (p.prompt, p.cols, p.q_tiles) == (w.prompt, w.cols, w.q_tiles), row
        assert 1 <= p.chunks <= w.chunks and p.chunk_tiles % 4 == 0, row
        count = min(r.randint(1, max_new), 4096)
        for kv_len in {max_len, r.randint(0, max_len), max_len + r.randint(0, 5000)}:
            at = attn_rules.spans(p, group, count, kv_len, max_len, window)
            assert len(at) <= p.q_tiles
            assert max(b - a for a, b in at) <= p.chunks * p.chunk_tiles, (row, count, kv_len)


def test_codes_that_a_window_leaves_out_are_not_counted(rules):
    """16 sequences of 8 heads of 128, bounded by 32768 tokens: 558 MB of codes,
    of which windows of 512 leave 9 MB and of 16384 279 MB."""
    got = rules([(16, 8, 8, 1, 32768, w, 128) for w in (0, 512, 1 << 14, 1 << 15, (1 << 32) - 1)])
    assert [p.stream for p in got] == [1, 0, 1, 1, 1]
