"""The split of the ragged attentions (host only): it covers every key, fits the lanes that join it, and the row tiles of
any starts lie inside the launch; the workspace query says what the launch uses."""
import random

import pytest

from ragged_plans import plan


def test_every_plan_covers_the_keys_and_can_be_joined():
    rng = random.Random(7)
    for _ in range(20000):
        R, T = int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 17))
        Hkv = rng.choice([1, 2, 3, 5, 8, 40])
        Hq, Dh = Hkv * rng.choice([1, 2, 5, 8]), rng.choice([64, 128])
        max_k = rng.choice([0, 1, 127, 128, 129, int(2 ** rng.uniform(0, 30)), 1 << 30])
        p = plan(R, T, Hq, Hkv, Dh, max_k)
        assert p["rows"] in (16, 32, 128) and p["groups"] in (1, 2) and 1 <= p["splits"] <= 64
        assert p["keys"] % 128 == 0 and p["keys"] >= 128 and p["keys"] * p["splits"] >= max_k
        assert p["keys"] < 2 ** 31 and (p["splits"] - 1) * p["keys"] < max(max_k, 1)
        assert p["groups"] == 1 or (p["rows"] == 128 and R == 1)
        if p["splits"] == 1:
            assert p["ws"] == 0
        else:
            assert p["ws"] >= T * Hq * p["splits"] * (Dh * 4 + 8)


def test_row_tiles_of_any_starts_lie_in_the_launch():
    """Request r's first tile is floor(start G / rows) + r; the tiles of two requests never meet, and the last is below
    the count that is launched."""
    rng = random.Random(8)
    for _ in range(5000):
        R, G, rows = rng.randint(1, 9), rng.choice([1, 2, 3, 8, 40]), rng.choice([16, 32, 128])
        T = rng.randint(1, 700)
        cuts = sorted(rng.randint(0, T) for _ in range(R + 1))
        if rng.random() < 0.5:
            cuts[0], cuts[-1] = 0, T
        first = [c * G // rows + r for r, c in enumerate(cuts[:-1])]
        last = [f + -(-(b - a) * G // rows) - 1 for f, a, b in zip(first, cuts, cuts[1:])]
        assert all(x < y for x, y in zip(last, first[1:]))
        assert max(last) < -(-T * G // rows) + R - 1


@pytest.mark.parametrize("args,want", [
    ((48, 48, 32, 8, 128, 16001), dict(rows=16, splits=16, keys=1024)),     # single tokens
    ((1, 32, 5, 5, 128, 1120), dict(rows=32, splits=5, keys=256)),          # one robot's action tokens
    ((2, 6304, 40, 40, 128, 15760), dict(rows=128, groups=1, splits=1)),    # two 480p chunks
    ((1, 544, 40, 40, 128, 1632), dict(rows=128, groups=2, splits=1)),      # a 256-pixel camera's chunk
    ((1, 3152, 5, 5, 128, 12608), dict(rows=128, groups=2, splits=2)),      # one rank's heads of a 480p chunk
    ((12, 2394, 8, 2, 64, 3401), dict(rows=128, groups=1, splits=4)),       # a ragged prefill
])
def test_documented_plans(args, want):
    p = plan(*args)
    assert {k: p[k] for k in want} == want


def test_workspace_query_agrees():
    import ctypes as C
    import paper_2602_15922_amd as w
    b = w.binding
    for R, T, Hq, Hkv, Dh, k in ((48, 48, 32, 8, 128, 16001), (1, 3152, 5, 5, 128, 12608), (2, 6304, 40, 40, 128, 512), (7, 900, 8, 2, 64, 4000)):
        need = plan(R, T, Hq, Hkv, Dh, k)["ws"]
        assert w.wam_attn_cross_workspace_bytes(R=R, T=T, Hq=Hq, Hkv=Hkv, Dh=Dh, max_k=k) == need
        c = b.wam_paged_cache(Hkv=Hkv, Dh=Dh)
        assert w.wam_attn_paged_workspace_bytes(c, R=R, T=T, Hq=Hq, max_kv=k) == need
        if need:  # a workspace one byte short, or none, is refused before any launch
            d = b.wam_attn_cross_desc(R=R, T=T, S=k, Hq=Hq, Hkv=Hkv, Dh=Dh, max_k=k, q_tok_stride=Hq * Dh,
                                      kv_tok_stride=Hkv * Dh, o_tok_stride=Hq * Dh)
            for ws, n in ((None, 0), (4096, need - 1), (4097, need)):
                assert w.lib().wam_attn_cross(C.byref(d), 4096, 4096, 4096, 4096, None, 4096, None, 4096, ws, n, None) == b.WAM_EWORKSPACE
