// How the ragged attentions split the key axis: the choice alone, host code with no HIP in it.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace wam {

constexpr int RAGGED_ROWS = 128;     // rows (token, head of a KV head's group) of a workgroup of the tile kernel,
constexpr int RAGGED_STREAM = 32;    // where requests of at most so many rows take the streaming path
constexpr int RAGGED_MAX_SPLITS = 64;

struct RaggedPlan {
  int rows = RAGGED_ROWS;  // rows of a workgroup: 128 (tile kernel), 16 or 32 (streaming kernel)
  int splits = 1;          // workgroups along the key axis, at most
  int split_keys = 0;      // keys of each (a multiple of 128)
};

// From what the host knows: R requests with T rows together (packed or padded), at most max_k keys.
inline RaggedPlan plan_ragged(int64_t R, int64_t T, int64_t Hq, int64_t Hkv, int64_t max_k) {
  RaggedPlan p;
  const int64_t rows = T * (Hq / Hkv);
  p.rows = rows <= 16 * R ? 16 : rows <= 32 * R ? 32 : RAGGED_ROWS;
  const bool few = p.rows < RAGGED_ROWS;
  const int64_t per = (rows + p.rows - 1) / p.rows, least_tiles = R < T ? R : T;
  const int64_t tiles = least_tiles > per ? least_tiles : per;
  const int64_t items = tiles * Hkv > 0 ? tiles * Hkv : 1;
  const auto parts = [&](int64_t keys) { return items * ((max_k + keys - 1) / keys); };
  int64_t keys, most;
  if (few) {
    // The parts of ragged requests have to be many and alike, or the longest run alone at the end, and the fewer,
    // the less is written and joined.  us at 256, 512, 1024, 1536 keys: 48 requests of 212-16001 keys, 8 heads 176, 158,
    // 157, 170; the same of 64 dims 86, 79, 83, 87; 32 requests of 328-4000 keys 52, 54, 62, 62.  32 rows write and
    // join eight times as much as 4 (32 rows, 40 heads, 9488 keys 68, 63, 72, 66; 5 heads, 1120 keys 13, 15, 20).
    keys = parts(1024) >= 4096 ? 1024 : parts(512) >= (p.rows == 16 ? 4096 : 512) ? 512 : 256;
    most = 16384;
  } else {
    keys = 512;
    most = 512;
  }
  // not more parts than `most` (the workspace grows with them), or than a wavefront has lanes to join them
  int64_t s = (most + items - 1) / items;
  if (s > RAGGED_MAX_SPLITS) s = RAGGED_MAX_SPLITS;
  const int64_t longer = ((max_k + s - 1) / s + 127) / 128 * 128;
  if (keys < longer) keys = longer;
  p.split_keys = (int)keys;
  p.splits = (int)((max_k + keys - 1) / keys);
  if (p.splits < 1) p.splits = 1;
  return p;
}

// Row tiles of a launch: floor(q_start G / rows) + r is the first of request r, so the last lies below this.
inline int64_t ragged_tiles(int64_t R, int64_t T, int64_t Hq, int64_t Hkv, int rows) { return T * (Hq / Hkv) / rows + R; }

// Workspace: per row and split the reference and the sum (8 bytes), then Dh partial outputs.
inline size_t ragged_ml_bytes(const RaggedPlan& p, int64_t T, int64_t Hq) {
  return ((size_t)T * Hq * p.splits * 8 + 255) / 256 * 256;
}
inline size_t ragged_ws_bytes(const RaggedPlan& p, int64_t T, int64_t Hq, int64_t Dh) {
  return p.splits <= 1 ? 0 : ragged_ml_bytes(p, T, Hq) + (size_t)T * Hq * p.splits * Dh * 4;
}

}  // namespace wam
