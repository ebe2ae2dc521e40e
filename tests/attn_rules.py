"""How attention over the 4-bit cache is launched, in Python (a helper module of
the tests, not a test file), so that a test can name the path its shape is meant
for.  tests/test_attn_rules.py holds it to the C++ of csrc/eq_attn_rules.h."""
from collections import namedtuple

Plan = namedtuple("Plan", "prompt cols tile q_tiles chunks chunk_tiles pair stream")


def _up(a, b):
    return -(-a // b)


def plan(n_seqs, kv_heads, group, max_new, max_len, window, dim):
    cols = max_new * group
    prompt = cols > 64 and (n_seqs * kv_heads * _up(cols, 128) >= 256 or max_len >= 8192)
    width, tile = (128, 64) if prompt else (16, 128)
    q_tiles = _up(cols, width)
    work, tiles = n_seqs * kv_heads * q_tiles, _up(max_len, tile)
    short = 32 if work >= 128 else 16
    whole = work >= 256 if prompt else tiles <= short
    want = 1 if whole else max(1, _up(512 if prompt else 256, work))

    def four(v):
        return max(4, _up(v, 4) * 4)

    ct = four(_up(tiles, want))
    if not whole and work < 2048:
        ct = min(ct, (2048 if prompt else 4096) // tile)
    chunks = max(1, _up(tiles, ct))
    ct = four(_up(tiles, chunks))
    seen = min(tiles, (window + max_new + tile - 2) // tile + 1) if window else tiles
    if seen < tiles:
        ct = four(_up(seen, chunks))
        if not prompt and seen <= short:
            ct = four(seen)
        chunks = max(1, _up(seen, ct))
    tokens = min(max_len, window + max_new - 1) if window else max_len
    read = n_seqs * tokens * kv_heads * (dim + dim // 32 + 1)
    return Plan(prompt, width, tile, q_tiles, chunks, ct, cols <= 8, q_tiles == 1 and read > 192 << 20)


def spans(p, group, count, kv_len, max_len, window):
    """(first, last) tile that each tile of query columns of a sequence sees, in
    the launch's order: `count` new tokens at the end of kv_len."""
    out = []
    length, base = min(kv_len, max_len), kv_len - count
    for col0 in range(0, count * group, p.cols):
        pos0 = base + col0 // group
        pos1 = base + (min(col0 + p.cols, count * group) - 1) // group
        start = pos0 + 1 - window if window and pos0 >= window else 0
        first = start // p.tile
        out.append((first, max(_up(max(min(pos1 + 1, length), 0), p.tile), first)))
    return out


def joined(p, group, count, kv_len, max_len, window):
    """Chunks of each of those that are joined."""
    return [min(_up(b - a, p.chunk_tiles), p.chunks)
            for a, b in spans(p, group, count, kv_len, max_len, window)]
