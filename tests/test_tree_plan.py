"""The split of the tree attention's key axis (csrc/ragged_plan.h, compiled with the host compiler): it covers every key, fits the
lanes that join it, the launch holds every row tile and part, and the workspace query says what the launch uses."""
import ctypes
import functools
import os
import random
import subprocess
import tempfile

import pytest

from ragged_plans import CSRC, plan

ENTRY = """#include "ragged_plan.h"
extern "C" void tree(long R, long T, long Hq, long Hkv, long Dh, long max_k, long* out) {
  const wam::RaggedPlan p = wam::plan_tree(R, T, Hq, Hkv, Dh, max_k);
  out[0] = p.rows; out[1] = p.groups; out[2] = p.splits; out[3] = p.split_keys; out[4] = p.turns;
  out[5] = wam::ragged_tiles(R, T, Hq, Hkv, p.rows); out[6] = (long)wam::ragged_ws_bytes(p, T, Hq, Dh, wam::ragged_tiles(R, T, Hq, Hkv, p.rows));
  out[8] = p.hull;
  out[7] = wam::ragged_blocks(p, R, T, Hq, Hkv);
}
"""


@functools.lru_cache(maxsize=None)
def _lib():
    with tempfile.TemporaryDirectory() as tmp:
        src, so = os.path.join(tmp, "plan.cpp"), os.path.join(tmp, "plan.so")
        with open(src, "w") as f:
            f.write(ENTRY)
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, src, "-o", so], check=True)
        return ctypes.CDLL(so)


def tree(*args):
    out = (ctypes.c_long * 9)()
    _lib().tree(*(ctypes.c_long(x) for x in args), out)
    return dict(zip(("rows", "groups", "splits", "keys", "turns", "tiles", "ws", "blocks", "hull"), out))


def test_every_plan_covers_the_keys_and_can_be_joined():
    rng = random.Random(7)
    for _ in range(20000):
        R, T = int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 17))
        Hkv = rng.choice([1, 2, 3, 5, 8, 40])
        Hq, Dh = Hkv * rng.choice([1, 2, 5, 8]), rng.choice([64, 128])
        max_k = rng.choice([0, 1, 127, 128, 129, int(2 ** rng.uniform(0, 30)), 1 << 30])
        p = tree(R, T, Hq, Hkv, Dh, max_k)
        assert p["rows"] in (16, 32, 128) and p["groups"] in (1, 2) and 1 <= p["splits"] <= 64
        assert p["keys"] % 128 == 0 and p["keys"] >= 128 and p["keys"] * p["splits"] >= max_k
        assert (p["splits"] - 1) * p["keys"] < max(max_k, 1)
        assert p["groups"] == 1 or (p["rows"] == 128 and R == 1)
        hull = 12 * p["tiles"] if p["hull"] else 0
        assert p["ws"] == hull if p["splits"] == 1 else p["ws"] >= T * Hq * p["splits"] * (Dh * 4 + 8) + hull
        assert not p["hull"] or (p["rows"] == 128 and p["groups"] == 1)
        # every (row tile, part, head) has its workgroup
        assert p["blocks"] >= p["tiles"] * p["splits"] * Hkv and (not p["turns"] or p["blocks"] % (8 * Hkv) == 0)


def test_one_request_and_few_rows_are_the_paged_attentions():
    for args in ((1, 300, 8, 2, 128, 5000), (9, 40, 8, 8, 128, 700), (1, 200, 40, 40, 128, 12608), (40, 40, 32, 8, 64, 9000)):
        p, want = tree(*args), plan(*args)
        assert {k: p[k] for k in want} == want and p["turns"] == 0


@pytest.mark.parametrize("args,want", [
    ((16, 681, 32, 8, 128, 16064), dict(rows=128, splits=8, keys=2048, turns=1)),   # drafted trees, a shared-head decoder
    ((48, 225, 40, 8, 128, 32012), dict(rows=128, splits=16, keys=2048, turns=1)),              # small trees over long histories
    ((2, 12608, 40, 40, 128, 18912), dict(rows=128, splits=1, turns=0, hull=1))])           # two robots' video branches
def test_documented_plans(args, want):
    p = tree(*args)
    assert {k: p[k] for k in want} == want, p


def test_workspace_query_agrees():
    import paper_2602_15922_amd as w
    for R, T, Hq, Hkv, Dh, k in ((48, 225, 40, 8, 128, 32012), (1, 3152, 5, 5, 128, 12608), (16, 681, 32, 8, 128, 16064), (7, 900, 8, 2, 64, 4000)):
        c = w.binding.wam_paged_cache(Hkv=Hkv, Dh=Dh)
        assert w.wam_attn_tree_workspace_bytes(c, R=R, T=T, Hq=Hq, max_kv=k) == tree(R, T, Hq, Hkv, Dh, k)["ws"]
    assert w.wam_attn_tree_workspace_bytes(w.binding.wam_paged_cache(Hkv=2, Dh=128), R=-1, T=5, Hq=4, max_kv=100) == 0
