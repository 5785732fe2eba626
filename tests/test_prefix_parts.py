"""The division of shared and own segments into parts, modelled on the host: every row once for every block of query rows, no part without rows, and room for all sums."""
import random

import pytest
from prefix_parts import own_parts, plan, shared_parts, up


def lengths(rng, n, most):
    return [rng.choice([0, 1, 63, 64, 65, 128, 129]) if rng.random() < 0.3 else int(most ** rng.random()) for _ in range(n)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
def test_every_row_once(dtype, d):
    rng = random.Random(d)
    turned = set()
    for turn in range(120):
        g, h, groups, batch = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 7, 8, 8, 20]), rng.choice([1, 1, 2, 3, 9, 64]), rng.choice([1, 2, 9, 33, 64])
        if turn < 10:                           # made longer twice
            g, h, groups, batch = 8, 32, 1, 64
        of = [rng.randrange(-1, groups) for _ in range(batch)] if rng.random() < 0.5 else [0] * batch
        lens = lengths(rng, groups * h, rng.choice([100, 3000, 40000])) if turn >= 10 else [int(rng.expovariate(1 / 2500)) for _ in range(h)]
        own, headroom = lengths(rng, batch * h, rng.choice([30, 3000])), rng.choice([0, 5, 700])
        p = plan(dtype, d, g, h, of, groups, [max(1, n) for n in own], headroom)
        turns, split, found = shared_parts(p, h, lens)
        turned.add(turns)
        assert len(found) <= p["shared_blocks"]
        work = [w for w in found if w]
        assert len({w[4] for w in work}) == len(work) and all(0 <= w[4] < len(found) for w in work)
        rows = {}
        for s, first, n, block, _ in work:
            assert 0 < n <= split * p["tile"] and first % p["tile"] == 0
            rows.setdefault((s, block), []).append((first, n))
        want = {(s, block): n for s, n in enumerate(lens) if n for block in range(p["blocks"][s // h])}
        assert set(rows) == set(want)
        for key, pieces in rows.items():
            at = 0
            for first, n in sorted(pieces):
                assert first == at
                at += n
            assert at == want[key]
        pieces = own_parts(p, own)
        assert all(0 < n <= p["own_split"] for _, _, n in pieces)
        assert [sum(n for t, _, n in pieces if t == s) for s in range(len(own))] == own
        assert len(pieces) <= up(sum(max(1, n) for n in own) + len(own) * headroom, p["own_split"]) + len(own)
    assert turned == {0, 1, 2}
