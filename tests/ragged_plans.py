"""The ragged attentions' split of the key axis as a host function: csrc/ragged_plan.h, which holds it and no HIP code,
compiled with the host compiler."""
import ctypes
import functools
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_15922_amd", "csrc")
ENTRY = """#include "ragged_plan.h"
extern "C" void plan(long R, long T, long Hq, long Hkv, long Dh, long max_k, long* out) {
  const wam::RaggedPlan p = wam::plan_ragged(R, T, Hq, Hkv, Dh, max_k);
  out[0] = p.rows; out[1] = p.groups; out[2] = p.splits; out[3] = p.split_keys;
  out[4] = wam::ragged_tiles(R, T, Hq, Hkv, p.rows); out[5] = (long)wam::ragged_ws_bytes(p, T, Hq, Dh);
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


def plan(R, T, Hq, Hkv, Dh, max_k):
    """dict(rows, groups, splits, keys, tiles, ws)."""
    out = (ctypes.c_long * 6)()
    _lib().plan(*(ctypes.c_long(x) for x in (R, T, Hq, Hkv, Dh, max_k)), out)
    return dict(zip(("rows", "groups", "splits", "keys", "tiles", "ws"), out))
