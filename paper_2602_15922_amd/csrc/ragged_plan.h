// How the ragged attentions split the key axis: the choice alone, host code with no HIP in it.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace wam {

constexpr int RAGGED_ROWS = 128;     // rows (token, head of a KV head's group) of a workgroup
constexpr int RAGGED_STREAM = 32;    // requests of at most so many rows take the streaming path
constexpr int RAGGED_MAX_SPLITS = 64;

struct RaggedPlan {
  int splits = 1;      // workgroups along the key axis, at most
  int split_keys = 0;  // keys of each (a multiple of 128)
  bool few = false;    // the requests have few rows on average
};

// From what the host knows: R requests with T rows together (packed or padded), at most max_k keys.
inline RaggedPlan plan_ragged(int64_t R, int64_t T, int64_t Hq, int64_t Hkv, int64_t max_k) {
  RaggedPlan p;
  const int64_t rows = T * (Hq / Hkv), per = (rows + RAGGED_ROWS - 1) / RAGGED_ROWS;
  const int64_t tiles = (R < T ? R : T) > per ? (R < T ? R : T) : per;
  p.few = rows <= RAGGED_STREAM * R;
  const int64_t items = tiles * Hkv > 0 ? tiles * Hkv : 1;
  const int64_t want = p.few ? 4096 : 512, least = p.few ? 256 : 512;
  int64_t s = (want + items - 1) / items;
  if (s > RAGGED_MAX_SPLITS) s = RAGGED_MAX_SPLITS;
  int64_t keys = ((max_k + s - 1) / s + 127) / 128 * 128;
  if (keys < least) keys = least;
  p.split_keys = (int)keys;
  p.splits = (int)((max_k + keys - 1) / keys);
  if (p.splits < 1) p.splits = 1;
  return p;
}

// Row tiles of a launch: floor(q_start G / 128) + r is the first of request r, so the last lies below this.
inline int64_t ragged_tiles(int64_t R, int64_t T, int64_t Hq, int64_t Hkv) { return T * (Hq / Hkv) / RAGGED_ROWS + R; }

// Workspace: per row and split the reference and the sum (8 bytes), then Dh partial outputs.
inline size_t ragged_ml_bytes(const RaggedPlan& p, int64_t T, int64_t Hq) {
  return ((size_t)T * Hq * p.splits * 8 + 255) / 256 * 256;
}
inline size_t ragged_ws_bytes(const RaggedPlan& p, int64_t T, int64_t Hq, int64_t Dh) {
  return p.splits <= 1 ? 0 : ragged_ml_bytes(p, T, Hq) + (size_t)T * Hq * p.splits * Dh * 4;
}

}  // namespace wam
