"""How the kernels over shared caches divide their work (decode_prefix.hip: plan_prefix, find_shared, find_work), in plain integers."""
import math


def up(a, b):
    return -(-a // b)


def plan(dtype, d, g, h, of, groups, own_kept, headroom):
    """plan_prefix: `dtype` "bf16", "fp16" or "fp32"; `own_kept`: rows that the own segments were built with."""
    wide = dtype == "fp32"
    rows_of = [g * sum(p == q for q in of) for p in range(groups)]
    most = max(rows_of)
    rb = 16 if wide and most <= 32 else 32 if not wide and d == 64 and most <= 32 else 64 if most <= 64 else 128
    blocks = [up(m, rb) for m in rows_of]
    n = sum(blocks) * h
    spare = max(256, n // 2 + 1)
    tile_us = 1.0 if not wide else (3.0 if d == 64 or rb == 128 else 6.0) * (0.25 if rb == 16 else 1.0)
    cost = min(most, rb) * (d + 2) * 8.0 / 5.0e6 / tile_us
    tile = 128 if d == 64 and not wide else 64
    own = len(of) * h
    own_cap = sum(own_kept) + own * headroom
    return dict(rb=rb, blocks=blocks, spare=spare, sums_cost=cost, shared_blocks=spare + n + sum(7 * b for b in blocks if b > 1) if n else 0,
                tile=32 if wide and d == 128 and rb == 128 else tile,       # (of the shared segments)
                own_tile=tile, own_split=up(max(up(own_cap, 512), tile), tile) * tile)


def shared_parts(p, h, lens):
    """find_shared: how often parts were made longer, a segment's tiles a part at most, and for every workgroup its (segment, first row, rows,
    block of query rows, where its sums go), or None."""
    blocks = p["blocks"]
    tiles = [up(n, p["tile"]) for n in lens]
    used = [t if blocks[s // h] else 0 for s, t in enumerate(tiles)]
    all_tiles = sum(t * blocks[s // h] for s, t in enumerate(used))
    split = max(max(1, up(all_tiles, p["spare"])), int(math.sqrt(all_tiles * p["sums_cost"]) + 0.5))
    count = lambda: [up(t, split) for t in used]
    turns = 0
    if len(lens) <= 64:
        while turns < 2:
            over = sum(c * blocks[s // h] for s, c in enumerate(count())) - p["spare"]
            if over <= 0:
                break
            split += max(1, int(split * over / p["spare"] + 0.999))
            turns += 1
    parts, found, base = count(), [], 0
    for cache, many in enumerate(blocks):
        mine = [(s, j) for s in range(cache * h, cache * h + h) for j in range(parts[s])]
        size = many * up(len(mine), 8) * 8 if many > 1 else len(mine) if many else 0
        for at in range(size):
            eights = at // 8 // many
            i, block = (eights * 8 + at % 8, at // 8 - eights * many) if many > 1 else (at, 0)
            if i >= len(mine):
                found.append(None)
                continue
            s, j = mine[i]
            rows = up(tiles[s], parts[s]) * p["tile"]
            found.append((s, j * rows, min(lens[s] - j * rows, rows), block, base + block * len(mine) + i))
        base += size
    return turns, split, found


def own_parts(p, lens):
    """find_work and what a workgroup makes of it: (segment, first row, rows)."""
    found = []
    for s, n in enumerate(lens):
        parts = up(n, p["own_split"])
        for j in range(parts):
            rows = min(p["own_split"], up(up(n, parts), p["own_tile"]) * p["own_tile"])
            found.append((s, j * rows, min(n - j * rows, rows)))
    return found
