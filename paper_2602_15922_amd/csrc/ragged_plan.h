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
  int groups = 1;          // groups of four wavefronts of a workgroup of the tile kernel
  int splits = 1;          // workgroups along the key axis, at most
  int split_keys = 0;      // keys of each (a multiple of 128)
};

// From what the host knows: R requests with T rows together (packed or padded), at most max_k keys.
inline RaggedPlan plan_ragged(int64_t R, int64_t T, int64_t Hq, int64_t Hkv, int64_t Dh, int64_t max_k) {
  constexpr int64_t CUS = 256;
  RaggedPlan p;
  const int64_t rows = T * (Hq / Hkv);
  p.rows = rows <= 16 * R ? 16 : rows <= 32 * R ? 32 : RAGGED_ROWS;
  const int64_t per = (rows + p.rows - 1) / p.rows, least_tiles = R < T ? R : T;
  const int64_t tiles = least_tiles > per ? least_tiles : per;
  const int64_t items = tiles * Hkv > 0 ? tiles * Hkv : 1;
  int64_t n, keys;  // parts that the machine asks for, keys that a part has at least
  if (p.rows < RAGGED_ROWS) {
    // The parts of ragged requests have to be many and alike, or the longest run alone at the end, and the fewer,
    // the less is written and joined.  us at 256, 512, 1024, 1536 keys: 48 requests of 212-16001 keys, 8 heads 162, 152,
    // 139, 148; the same of 64 dims 85, 79, 78, 86; 32 requests of 328-4000 keys 48, 46, 54, 52.  32 rows write and
    // join eight times as much as 4 (32 rows, 40 heads, 9488 keys 61, 56, 64, 58; 5 heads, 1120 keys 12, 14, 17, 19).
    const auto parts = [&](int64_t k) { return items * ((max_k + k - 1) / k); };
    keys = parts(1024) >= 4096 ? 1024 : parts(512) >= (p.rows == 16 ? 4096 : 512) ? 512 : 256;
    n = (16384 + items - 1) / items;
  } else if (R == 1 && items <= CUS) {
    // One request that leaves CUs idle: as many parts as there are CUs for, each a workgroup of eight wavefronts that has
    // its CU alone.  544 rows, 1632 keys, 40 heads: 38 us; with workgroups of four wavefronts in one part 44, two 48, four
    // 64.  3152 rows, 12608 keys, 5 heads: 132 us; 257, 152, 128.
    keys = 512;
    n = CUS / items;
  } else {
    // About one workgroup per CU (64 dims: two, three fit), unless the parts get short.  At 256, 384, 512, 768
    // workgroups: 3 x 700 rows, 10 heads 90, 106, 99, 97 us; 20 x 10-100 rows, 16/4 heads 77, 88, 91, 85; 12 ragged prefills
    // of 64 dims 39, 38, 33, 33 (in parts of 448 keys 46).
    // All requests get one length of part, from the average of their rows: where a few have many rows and most have one, the
    // single tokens over long histories are hardly split, and two calls are faster than one (one request of 512 rows with 47
    // single tokens of 212-16001 keys, 32/8 heads 408 us, apart 181 and 133; 2000 rows with 8 tokens of 32000 keys 430,
    // apart 58 and 186).
    keys = 1024;
    n = ((Dh == 64 ? 2 : 1) * CUS + items - 1) / items;
  }
  // not more parts than a wavefront has lanes to join them; all of one length
  const int64_t by_keys = (max_k + keys - 1) / keys;
  if (n > RAGGED_MAX_SPLITS) n = RAGGED_MAX_SPLITS;
  if (n > by_keys) n = by_keys;
  if (n < 1) n = 1;
  keys = ((max_k + n - 1) / n + 127) / 128 * 128;
  p.split_keys = (int)(keys < 128 ? 128 : keys);
  p.splits = (int)((max_k + p.split_keys - 1) / p.split_keys);
  if (p.splits < 1) p.splits = 1;
  p.groups = p.rows == RAGGED_ROWS && R == 1 && items * p.splits <= CUS ? 2 : 1;
  return p;
}

// Row tiles of a launch.  Request r's first is floor(a) + r, a = q_start G / rows, and it has ceil(b) with a + b <= T G /
// rows; so its last is floor(a) + ceil(b) + r - 1 <= ceil(T G / rows) + R - 2.
inline int64_t ragged_tiles(int64_t R, int64_t T, int64_t Hq, int64_t Hkv, int rows) {
  return (T * (Hq / Hkv) + rows - 1) / rows + R - 1;
}

// Workgroups of the launch (256 threads per group of four wavefronts): one per row tile, part and KV head; of the streaming
// kernel, row tiles and parts in eights, one to each XCD.
inline int64_t ragged_blocks(const RaggedPlan& p, int64_t R, int64_t T, int64_t Hq, int64_t Hkv) {
  const int64_t parts = ragged_tiles(R, T, Hq, Hkv, p.rows) * p.splits;
  return (p.rows == RAGGED_ROWS ? parts : (parts + 7) / 8 * 8) * Hkv;
}

// Workspace: per row and split the reference and the sum (8 bytes), then Dh partial outputs.
inline size_t ragged_ml_bytes(const RaggedPlan& p, int64_t T, int64_t Hq) {
  return ((size_t)T * Hq * p.splits * 8 + 255) / 256 * 256;
}
inline size_t ragged_ws_bytes(const RaggedPlan& p, int64_t T, int64_t Hq, int64_t Dh) {
  return p.splits <= 1 ? 0 : ragged_ml_bytes(p, T, Hq) + (size_t)T * Hq * p.splits * Dh * 4;
}

}  // namespace wam
