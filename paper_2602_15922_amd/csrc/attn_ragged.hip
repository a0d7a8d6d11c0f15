// Attention of ragged rows over a paged KV cache, or over packed states of other lengths (bf16
// MFMA, fp32 online softmax).
//
// The rows of a request and KV head are its tokens times the query heads that share the KV head,
// token by token; a workgroup owns 128 (16, 32) of them, so a shared head's keys are read once for its
// whole group.  Row tile x of the launch belongs to the last request r with floor(q_start[r] G / 128)
// + r <= x: every request has room for its tiles there, the launch needs only T, G and R, and a
// workgroup finds its request by ballots over q_start, 64 starts at a time.
//
// Two paths by the request's rows (a kernel for calls whose requests have few on average, 16 or 32 to a workgroup, and
// one for the others, which streams those that have few all the same):
//  stream  few rows (single tokens): bound by reading the cache.  Each wavefront takes every
//          fourth 32-key tile on its own: whole rows into registers, the next tile's 16 KB in flight while
//          one is used, and through a private piece of LDS into the matrix operands' order (V's with the
//          transposing read); nothing waits for another wavefront until the four states are joined at the end.
//  tile    more rows: 32 per wavefront against 64-key tiles shared in LDS, as in attn.hip (whose tile
//          code it shares); the page of a wavefront's 16 keys of a tile is one entry of the
//          block table (a page holds a multiple of 16 keys).
// Where rows are few and keys many the key axis is split over workgroups (ragged_plan.h); the parts
// are joined in a fixed order by a second kernel.
//
// Held in fewer than 32 bits: the probabilities, rounded to bf16 (each off by 2^-8 of itself at most) since a matrix
// instruction takes both operands in one type and V is bf16; their sum is that of the rounded ones, so that what they have in
// common cancels.  Scores, references, sums and outputs are in 32 bits until the one rounding of the stored output.
#include "attn_tile.h"
#include "kernels.h"
#include "ragged_plan.h"

namespace wam {
namespace {

typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

struct Parts {
  float* ml;  // [row][splits][2]: reference and sum
  float* o;   // [row][splits][Dh]
  int splits, split_keys, tiles;
  FastDiv by_splits, by_tiles, by_heads;
};

WAM_DEV int fdiv(const FastDiv& f, int n) {
  return f.d == 1 ? n : (int)(__umulhi((uint32_t)n, f.mul) >> f.shift);
}
WAM_DEV int fdiv_rest(const FastDiv& f, int n) { return n - fdiv(f, n) * (int)f.d; }
WAM_DEV int clampi(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }
WAM_DEV int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// A request's rows and keys, cut to what the call names.
struct Req {
  int q0, n;       // first token row, tokens
  int kv, keys;    // length that positions count from; keys there are (at most max_k)
  int64_t k0;      // packed states: first key row
};
template <bool PAGED>
WAM_DEV Req request(const RaggedArgs& a, int r) {
  // every load before any use: one trip to memory
  const int32_t* qn = a.q_len ? a.q_len : a.q_start;
  const int32_t* kn = PAGED || a.k_len ? a.k_len + r : a.k_start + r + 1;
  const int32_t* kf = PAGED ? a.k_len : a.k_start;
  const int q0 = a.q_start[r], q1 = a.q_start[r + 1], n = qn[r], klen = *kn, kfirst = kf[r];
  Req q;
  const int end = clampi(q1, 0, a.T), room = q0 < 0 || q0 >= end ? 0 : end - q0;
  q.q0 = q0;
  q.n = a.q_len ? clampi(n, 0, room) : room;
  if (PAGED) {
    q.k0 = 0;
    q.kv = klen;
    q.keys = clampi(klen, 0, a.max_k);
  } else {
    const int k0 = clampi(kfirst, 0, a.S), most = a.S - k0 < a.max_k ? a.S - k0 : a.max_k;
    const int64_t len = a.k_len ? klen : (int64_t)klen - k0;
    q.k0 = k0;
    q.kv = q.keys = len < 0 ? 0 : (len < most ? (int)len : most);
  }
  return q;
}
// keys that token i of the request sees (a prefix)
template <bool PAGED>
WAM_DEV int kend_of(const RaggedArgs& a, const Req& q, int i) {
  if (!PAGED || a.chunk.d == 0) return q.keys;
  const int64_t p = (int64_t)q.kv - q.n + i;
  if (p < 0) return 0;
  const int64_t e = ((int64_t)fdiv(a.chunk, (int)p) + 1) * a.chunk.d;
  return e < q.keys ? (int)e : q.keys;
}

// page of the 16 keys from `key` on (a multiple of 16), -1 where there is none (or the table ends)
template <bool PAGED>
WAM_DEV int page_of(const RaggedArgs& a, int r, int key) {
  if (key >= a.max_k) return -1;
  if (!PAGED) return 0;
  const int p = a.table[r * a.table_stride + fdiv(a.ps, key)];
  return (unsigned)p < (unsigned)a.n_pages ? p : -1;
}
// element offset of the row of `key` in page `page`
template <bool PAGED>
WAM_DEV int64_t row_at(const RaggedArgs& a, const Req& q, int page, int key, int hk) {
  if (!PAGED) return (q.k0 + key) * a.tok_stride + hk * a.head_stride;
  const int in = key - fdiv(a.ps, key) * (int)a.ps.d;
  return (int64_t)page * a.page_stride + (int64_t)in * a.tok_stride + hk * a.head_stride;
}

// 8 E4M3 codes times the power of two sc, exactly, as bf16
WAM_DEV bf16x8 decode8(uint32_t lo, uint32_t hi, float sc) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, sc, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, sc, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, sc, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, sc, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
WAM_DEV float exp_scale(uint32_t biased) { return __uint_as_float(biased << 23); }

// Values that are not finite.  The value product gives every row 0 * V of the keys it does not see, which is NaN where V is
// not finite.  Keys past a part's last one and of absent pages are zeros in LDS; what is left are the keys that some of a
// workgroup's rows see and others do not, in the tiles at the mask's edge.  Those tiles are searched, and where one holds an
// infinity or a NaN the workgroup's rows are done once more on the streaming path, in a form whose product leaves such
// values out, while two products of ones count for every row and dim those that the row sees: (infinity or NaN) and
// (-infinity or NaN), added as infinities of both signs (a NaN as their sum).  Done anew and not within the tile, for its
// vector registers: a product by key in the tile spilt 100 and more.  The search and the second pass take hardly any of them
// (paged, head size 128: 252 -> 253; E4M3, which spilt 7 of them without, 12), but scalar ones, of which the tile kernels keep
// some in vector lanes (0 -> 93).  With the search alone left out one causal request of 500 rows over 3000 keys takes 38.6 us
// (a form of the kernel that spills; 29.2 with it), the 12 causal requests of 1 to 901 rows 32.4 (32.9), two samples' 3152
// rows 1842 (1835).
// x + 0 * (every bf16 of v): NaN from the first that is not finite on
WAM_DEV float zero_times(u32x4v v, float x) {
  const bf16x2 zeros = {(bf16)0.f, (bf16)0.f};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t two = v[e];
    x = __builtin_amdgcn_fdot2_f32_bf16(*reinterpret_cast<const bf16x2*>(&two), zeros, x, false);
  }
  return x;
}
// of 8 bf16: kind 0 themselves, where they are finite; kind 1 a one where infinity or NaN is; kind 2 where -infinity or NaN is
WAM_DEV bf16x8 of_kind(bf16x8 v, int kind) {
  u32x4v x = *reinterpret_cast<const u32x4v*>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t y = 0;
#pragma unroll
    for (int sh = 0; sh < 32; sh += 16) {
      const uint32_t h = x[i] >> sh & 0xffff;
      const bool odd = (h & 0x7f80) == 0x7f80, other = h == (kind == 1 ? 0xff80u : 0x7f80u);
      y |= (kind == 0 ? (odd ? 0u : h) : (odd && !other ? 0x3f80u : 0u)) << sh;
    }
    x[i] = y;
  }
  return *reinterpret_cast<const bf16x8*>(&x);
}

// ---------------------------------------------------------------------------------
// stream path
// ---------------------------------------------------------------------------------
// 16x16x32 bf16 MFMA.  Lane l, g = l / 16: A[m = l % 16][8 k's of group g], B[8 k's of group g][n =
// l % 16], D register r: D[m = 4 g + r][n = l % 16]; both operands' k order is free as long as it is one.
WAM_DEV f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Bytes between V rows of a tile in a wavefront's LDS: 32 more than a row, so that the 8 rows x 32 bytes that 32 lanes
// of the transposing read touch lie in different banks, at constant distances; and between the K rows of a group (as they are
// stored): 16 more, so that 16 rows' chunks do.
constexpr int spitch(int dh) { return dh * 2 + 32; }
constexpr int kpitch(int dh, bool fp8) { return dh * (fp8 ? 1 : 2) + 16; }
constexpr int stream_wave_lds(int dh, bool fp8) { return 32 * spitch(dh) + 16 * kpitch(dh, fp8); }

// One 32-key tile of a wavefront in registers: two groups of 16 keys.
template <int DH, bool FP8>
struct StreamRegs {
  static constexpr int N = FP8 ? 2 : DH / 32;  // 16-byte chunks of a group's K (and V) per lane
  u32x4v k[2][N], v[2][N];
  uint32_t ex[2];
  int nv[2];  // keys there are of each group (wave-uniform)
};

// (Whole rows, marked as used once: only this workgroup reads them, and they should not push others out of the caches.
// us for 48 single tokens, 8 heads of 128 / the same of 64 / 64 tokens, 8 heads, E4M3: 139 / 78 / 255; not marked 153 / 87 /
// 268; V of a group right after its K instead of after both groups' 140 / 79 / 255.)
template <int DH, bool PAGED, bool FP8>
WAM_DEV void stream_load(StreamRegs<DH, FP8>& x, const RaggedArgs& a, const Req& q, int hk, int key0, int end, int pg0,
                         int pg1, int lane, int off) {
  constexpr int EB = FP8 ? 1 : 2, CPR = DH * EB / 16, RPI = 64 / CPR;  // chunks per row, rows per instruction
  const int ts = (int)a.tok_stride * EB, n16 = lane & 15;
  constexpr int N = StreamRegs<DH, FP8>::N;
  const char *kp[2], *vp[2], *ep[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int key = key0 + 16 * u, pg = u ? pg1 : pg0;
    x.nv[u] = pg < 0 ? 0 : clampi(end - key, 0, 16);
    const int64_t at = x.nv[u] > 0 ? row_at<PAGED>(a, q, pg, key, hk) : 0;
    kp[u] = static_cast<const char*>(a.k) + at * EB;
    vp[u] = static_cast<const char*>(a.v) + at * EB;
    ep[u] = FP8 ? static_cast<const char*>(a.k_exp) + at / 32 : nullptr;
  }
  if (x.nv[0] == 16 && x.nv[1] == 16) {  // uniform bases, one lane offset
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        x.k[u][i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4v*>(kp[u] + RPI * i * ts + off));
      if (FP8) x.ex[u] = *reinterpret_cast<const uint32_t*>(ep[u] + (n16 * ts >> 5));
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < N; ++i)
        x.v[u][i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4v*>(vp[u] + RPI * i * ts + off));
    return;
  }
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int nv = x.nv[u];
    if (nv == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) x.k[u][i] = x.v[u][i] = u32x4v{0, 0, 0, 0};
      x.ex[u] = 0;
      continue;
    }
    // rows past the last key re-read it (their scores are masked, their values zeroed)
    if (FP8) x.ex[u] = *reinterpret_cast<const uint32_t*>(ep[u] + ((n16 < nv ? n16 : nv - 1) * ts >> 5));
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = RPI * i + lane / CPR, at_row = (row < nv ? row : nv - 1) * ts + 16 * (lane % CPR);
      x.k[u][i] = *reinterpret_cast<const u32x4v*>(kp[u] + at_row);
      x.v[u][i] = *reinterpret_cast<const u32x4v*>(vp[u] + at_row);
    }
  }
}

// Keeps LDS accesses of other lanes' rows in their order: the compiler moves none across, and a wavefront's LDS operations
// run in order, so nothing has to wait.
WAM_DEV void lds_order() { asm volatile("" ::: "memory"); }

// a group's K rows, as they are stored
template <int DH, bool FP8>
WAM_DEV void stream_store_k(const StreamRegs<DH, FP8>& x, int u, char* ks, int lane) {
  constexpr int EB = FP8 ? 1 : 2, CPR = DH * EB / 16, RPI = 64 / CPR;
#pragma unroll
  for (int i = 0; i < StreamRegs<DH, FP8>::N; ++i)
    *reinterpret_cast<u32x4v*>(ks + (RPI * i + lane / CPR) * kpitch(DH, FP8) + 16 * (lane % CPR)) = x.k[u][i];
}
// a tile's V rows as bf16; rows from nv on as zeros
template <int DH, bool FP8>
WAM_DEV void stream_store_v(const StreamRegs<DH, FP8>& x, char* vs, int lane) {
  constexpr int EB = FP8 ? 1 : 2, CPR = DH * EB / 16, RPI = 64 / CPR;
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int i = 0; i < StreamRegs<DH, FP8>::N; ++i) {
      const int row = RPI * i + lane / CPR, ch = lane % CPR;
      u32x4v v = x.v[u][i];
      if (x.nv[u] < 16 && row >= x.nv[u]) v = u32x4v{0, 0, 0, 0};
      char* dst = vs + (16 * u + row) * spitch(DH);
      if constexpr (FP8) {
        *reinterpret_cast<bf16x8*>(dst + 32 * ch) = decode8(v[0], v[1], 1.0f);
        *reinterpret_cast<bf16x8*>(dst + 32 * ch + 16) = decode8(v[2], v[3], 1.0f);
      } else {
        *reinterpret_cast<u32x4v*>(dst + 16 * ch) = v;
      }
    }
}

// key of the group whose page lane l holds, from the wavefront's first key on
WAM_DEV int stream_key(int lane) { return 128 * (lane >> 1) + 16 * (lane & 1); }

// LDS of the streaming path: four wavefronts' tiles, or their 16 rows each of the join
constexpr int stream_lds(int dh, bool fp8) {
  const int join = (4 * 16 * (dh + 4) + 128) * 4, tiles = 4 * stream_wave_lds(dh, fp8);
  return join > tiles ? join : tiles;
}

// a V operand of the value product: k slots are the four keys 4 g .. of group 0, then of group 1
template <int DH>
WAM_DEV bf16x8 stream_v(const char* at) {
  const s16x4 v2[2] = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at),
                       __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 16 * spitch(DH)))};
  return *reinterpret_cast<const bf16x8*>(v2);
}
// the value product of a tile whose V may hold values that are not finite
template <int DH, int NQ>
WAM_DEV void stream_value_odd(const char* vr, const bf16x8* pb, f32x4 (*acc)[DH / 16], int key0, const int* row_kend, int g) {
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    bf16x8 sees;
#pragma unroll
    for (int i = 0; i < 8; ++i) sees[i] = (bf16)(key0 + 16 * (i >> 2) + 4 * g + (i & 3) < row_kend[n] ? 1.f : 0.f);
#pragma unroll
    for (int d = 0; d < DH / 16; ++d) {
      const bf16x8 v = stream_v<DH>(vr + 32 * d);
      const f32x4 none = {0.f, 0.f, 0.f, 0.f};
      acc[n][d] = mfma16(of_kind(v, 0), pb[n], acc[n][d]);
      const f32x4 up = mfma16(of_kind(v, 1), sees, none), down = mfma16(of_kind(v, 2), sees, none);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (up[e] > 0.f) acc[n][d][e] += INFINITY;
        if (down[e] > 0.f) acc[n][d][e] -= INFINITY;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

template <int DH, bool PAGED, bool FP8, int NQ>
WAM_DEV void stream_rows(const RaggedArgs& a, const Parts& pt, const Req& q, int r, int hk, int G, int m0, int split,
                         bool whole, int start, int end, int meta, char* smem) {
  constexpr int KS = DH / 32, DT = DH / 16;
  const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6), g = lane >> 4, n16 = lane & 15;
  const int rows = q.n * G;
  bf16x8 qf[NQ][KS];
  int row_kend[NQ];
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    const int row = m0 + 16 * i + n16 < rows ? m0 + 16 * i + n16 : rows - 1, tok = fdiv(a.group, row);
    const bf16* qp = static_cast<const bf16*>(a.q) + (q.q0 + tok) * a.q_ts + (hk * G + row - tok * G) * DH;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[i][ks] = load_bf16x8(qp + (FP8 ? 32 * g + 8 * ks : 32 * ks + 8 * g));
    row_kend[i] = kend_of<PAGED>(a, q, tok);
  }
  const int kmin = kend_of<PAGED>(a, q, fdiv(a.group, m0));
  f32x4 acc[NQ][DT];
  float m_ref[NQ], l_part[NQ];
  char* vs = smem + w * stream_wave_lds(DH, FP8);
  char* kl = vs + 32 * spitch(DH);
  // transposing read: lane j of a group points at row 4 g + j / 4, 4 dims from 4 (j % 4) of each 16
  const char* vr = vs + (4 * g + (n16 >> 2)) * spitch(DH) + 8 * (n16 & 3);
  const int ts = (int)a.tok_stride * (FP8 ? 1 : 2), cpr = DH * (FP8 ? 1 : 2) / 16;
  const int off = lane / cpr * ts + 16 * (lane % cpr);
  // K operand of a group: row n16; bf16: dims 32 ks + 8 g ..; codes: dims 32 g + 8 ks .. (one block's exponent per lane)
  const char* kr = kl + n16 * kpitch(DH, FP8) + (FP8 ? 32 : 16) * g;
  const float c = a.c, thr = RESCALE_LOG2 / c;

  // tile i of this wavefront: keys start + 128 i + 32 w; lane l holds the page of group l % 2 of tile
  // base + l / 2, for 32 tiles at a time
  const int first = start + 32 * w;
  const int n_tiles = end > first ? (end - first + 127) / 128 : 0;
  auto pages = [&](int base) { meta = page_of<PAGED>(a, r, first + 128 * base + stream_key(lane)); };
  StreamRegs<DH, FP8> x;
  auto load = [&](int i) {
    if (i > 0 && (i & 31) == 0) pages(i);
    const int at = 2 * (i & 31);
    stream_load<DH, PAGED, FP8>(x, a, q, hk, first + 128 * i, end, __builtin_amdgcn_readlane(meta, at),
                                __builtin_amdgcn_readlane(meta, at + 1), lane, off);
  };
  // odd: V may hold values that are not finite; else true is returned if so
  auto sweep = [&](auto odd) __attribute__((always_inline)) {
    constexpr bool ODD = decltype(odd)::value;
    bool bad = false;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      m_ref[n] = -INFINITY;
      l_part[n] = 0.f;
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[n][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (!ODD && n_tiles > 0) load(0);
    for (int i = 0; i < n_tiles; ++i) {
      const int key0 = first + 128 * i;
      if (ODD) load(i);
      f32x4 s[NQ][2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        lds_order();
        stream_store_k<DH, FP8>(x, u, kl, lane);
        if (u == 0) stream_store_v<DH, FP8>(x, vs, lane);
        lds_order();
        const float sc = FP8 ? exp_scale((x.ex[u] >> (8 * g)) & 255) : 1.f;
#pragma unroll
        for (int n = 0; n < NQ; ++n) s[n][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          bf16x8 kf;
          if constexpr (FP8) {
            const u32x2 c8 = *reinterpret_cast<const u32x2*>(kr + 8 * ks);
            kf = decode8(c8[0], c8[1], sc);
          } else {
            kf = *reinterpret_cast<const bf16x8*>(kr + 64 * ks);
          }
#pragma unroll
          for (int n = 0; n < NQ; ++n) s[n][u] = mfma16(kf, qf[n][ks], s[n][u]);
        }
      }
      const int nv0 = x.nv[0], nv1 = x.nv[1];
      if (!ODD && i + 1 < n_tiles) load(i + 1);
      if (nv0 < 16 || nv1 < 16 || key0 + 32 > kmin) {
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int kk = 4 * g + e;
              if (kk >= (u ? nv1 : nv0) || key0 + 16 * u + kk >= row_kend[n]) s[n][u][e] = -INFINITY;
            }
      }
      bf16x8 pb[NQ];
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        float mx = s[n][0][0];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[n][u][e]);
        if (__any(mx > m_ref[n] + thr || (m_ref[n] == -INFINITY && mx != -INFINITY))) {
          // the four lanes of a query raise their common reference together
          mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
          mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
          const bool raise = mx > m_ref[n] + thr || (m_ref[n] == -INFINITY && mx != -INFINITY);
          const float m_new = raise ? mx : m_ref[n];
          const float alpha = m_ref[n] == -INFINITY ? 0.f : exp2_fast((m_ref[n] - m_new) * c);
          m_ref[n] = m_new;
          l_part[n] *= alpha;
#pragma unroll
          for (int d = 0; d < DT; ++d) acc[n][d] *= alpha;
        }
        const float ms = m_ref[n] == -INFINITY ? 0.f : m_ref[n] * c;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) pb[n][4 * u + e] = (bf16)exp2_fast(__builtin_fmaf(s[n][u][e], c, -ms));
        // the sum of exactly the bf16 probabilities the value product uses
        const bf16x2 ones = {(bf16)1.0f, (bf16)1.0f};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          l_part[n] = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pb[n][2 * e], pb[n][2 * e + 1]}, ones, l_part[n], false);
      }
      if constexpr (ODD) {
        stream_value_odd<DH, NQ>(vr, pb, acc, key0, row_kend, g);
        continue;
      }
      if (kmin < end && key0 + 32 > kmin) {
        float z = 0.f;
#pragma unroll 2
        for (int k = 0; k < DH / 16; ++k) {  // 32 rows of DH / 8 chunks
          const int u = 64 * k + lane;
          z = zero_times(*reinterpret_cast<const u32x4v*>(vs + u / (DH / 8) * spitch(DH) + u % (DH / 8) * 16), z);
        }
        if (__any(z != 0.f)) bad = true;
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const bf16x8 vf = stream_v<DH>(vr + 32 * d);
#pragma unroll
        for (int n = 0; n < NQ; ++n) acc[n][d] = mfma16(vf, pb[n], acc[n][d]);
      }
    }
    return bad;
  };
  if (sweep(std::false_type{})) {
    pages(0);
    sweep(std::true_type{});
  }

  // join the four wavefronts: common reference, scaled sums, 16 rows at a time through LDS
  constexpr int PITCH = DH + 4;
  float* red = reinterpret_cast<float*>(smem);                // [4][16][PITCH]
  float* wml = red + 4 * 16 * PITCH;                          // [4][16][2]
  static_assert(stream_lds(DH, FP8) <= 4 * BN * DH * 2, "fits the tile kernel's LDS");
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    float l = l_part[n];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    __syncthreads();  // the V tiles (the rows before) are no longer read
    if (g == 0) {
      wml[(w * 16 + n16) * 2] = m_ref[n];
      wml[(w * 16 + n16) * 2 + 1] = l;
    }
    __syncthreads();
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) top = fmaxf(top, wml[(k * 16 + n16) * 2]);
    const float f = m_ref[n] == -INFINITY ? 0.f : exp2_fast((m_ref[n] - top) * c);
#pragma unroll
    for (int d = 0; d < DT; ++d)
      *reinterpret_cast<f32x4*>(red + (w * 16 + n16) * PITCH + 16 * d + 4 * g) = acc[n][d] * f;
    __syncthreads();
    // thread: row tid / 16, DH / 16 dims
    constexpr int PER = DH / 16;
    const int rr = tid >> 4, d0 = (tid & 15) * PER, row = m0 + 16 * n + rr;
    top = -INFINITY;
#pragma unroll
    for (int k = 0; k < 4; ++k) top = fmaxf(top, wml[(k * 16 + rr) * 2]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float mk = wml[(k * 16 + rr) * 2];
      sum += mk == -INFINITY ? 0.f : wml[(k * 16 + rr) * 2 + 1] * exp2_fast((mk - top) * c);
    }
    float y[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) y[e] = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int e = 0; e < PER; ++e) y[e] += red[(k * 16 + rr) * PITCH + d0 + e];
    if (row < rows) {
      const int tok = fdiv(a.group, row), h = hk * G + row - tok * G;
      if (whole) {
        const float inv = sum > 0.f ? (FP8 ? a.v_scale : 1.f) / sum : 0.f;
        bf16* op = static_cast<bf16*>(a.o) + (q.q0 + tok) * a.o_ts + h * DH + d0;
#pragma unroll
        for (int e = 0; e < PER; e += 4)
          *reinterpret_cast<bf16x4*>(op + e) =
              bf16x4{(bf16)(y[e] * inv), (bf16)(y[e + 1] * inv), (bf16)(y[e + 2] * inv), (bf16)(y[e + 3] * inv)};
      } else {
        const int64_t id = ((int64_t)(q.q0 + tok) * a.Hq + h) * pt.splits + split;
        if ((tid & 15) == 0) {
          pt.ml[2 * id] = top;
          pt.ml[2 * id + 1] = sum;
        }
#pragma unroll
        for (int e = 0; e < PER; e += 4)
          *reinterpret_cast<f32x4*>(pt.o + id * DH + d0 + e) = f32x4{y[e], y[e + 1], y[e + 2], y[e + 3]};
      }
    }
  }
}

// ---------------------------------------------------------------------------------
// tile path
// ---------------------------------------------------------------------------------
// What a wavefront needs to fetch its 16 rows (16 w .. 16 w + 15) of a 64-key tile.
template <int DH, bool PAGED, bool FP8>
struct Fetch {
  static constexpr int EB = FP8 ? 1 : 2, CPR = DH * EB / 16, N = 16 * CPR / 64;  // 16-byte chunks per lane
  int koff[N], voff[N], row[N];
  u32x4v kr[FP8 ? N : 1], vr[FP8 ? N : 1];  // FP8: the tile's codes on their way to LDS
  uint32_t ex[FP8 ? N : 1];

  WAM_DEV void init(const RaggedArgs& a, int lane) {
    const int ts = (int)a.tok_stride * EB;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int u = i * 64 + lane, rw = u / CPR, ch = u % CPR;
      row[i] = rw;
      // (16 w does not change either swizzle)
      koff[i] = rw * ts + (FP8 ? ch : kswz<DH>(rw, ch)) * 16;
      voff[i] = rw * ts + (FP8 ? ch : vswz<DH>(rw, ch)) * 16;
    }
  }
  // bf16: into LDS; rows from nv on as zeros.  FP8: into registers.
  WAM_DEV void load(const RaggedArgs& a, const Req& q, bf16* tile, int key, int pg, int nv, int hk, int w, int lane) {
    bf16* Ks = tile + 16 * w * DH;
    bf16* Vs = Ks + BN * DH;
    const int64_t at = nv > 0 ? row_at<PAGED>(a, q, pg, key, hk) * EB : 0;
    char* kp = const_cast<char*>(static_cast<const char*>(a.k)) + at;
    char* vp = const_cast<char*>(static_cast<const char*>(a.v)) + at;
    if constexpr (FP8) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        kr[i] = vr[i] = u32x4v{0, 0, 0, 0};
        ex[i] = 0;
        if (row[i] < nv) {
          kr[i] = *reinterpret_cast<const u32x4v*>(kp + koff[i]);
          vr[i] = *reinterpret_cast<const u32x4v*>(vp + voff[i]);
          ex[i] = *reinterpret_cast<const uint32_t*>(static_cast<const char*>(a.k_exp) + at / 32 + (koff[i] & ~127) / 32);
        }
      }
    } else if (nv == 16) {
      const __amdgpu_buffer_rsrc_t kres = __builtin_amdgcn_make_buffer_rsrc(kp, (short)0, 0x7fffffff, 0x00020000);
      const __amdgpu_buffer_rsrc_t vres = __builtin_amdgcn_make_buffer_rsrc(vp, (short)0, 0x7fffffff, 0x00020000);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(kres, (lds_void*)(Ks + i * 512), 16, koff[i], 0, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(vres, (lds_void*)(Vs + i * 512), 16, voff[i], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        u32x4v kk = {0, 0, 0, 0}, vv = {0, 0, 0, 0};
        if (row[i] < nv) {
          kk = *reinterpret_cast<const u32x4v*>(kp + koff[i]);
          vv = *reinterpret_cast<const u32x4v*>(vp + voff[i]);
        }
        *reinterpret_cast<u32x4v*>(Ks + i * 512 + lane * 8) = kk;
        *reinterpret_cast<u32x4v*>(Vs + i * 512 + lane * 8) = vv;
      }
    }
  }
  // FP8: the codes decoded into LDS (chunk ch of 16 dims: two 16-byte chunks of bf16)
  WAM_DEV void store(bf16* tile, int w, int lane) {
    if constexpr (FP8) {
      bf16* Ks = tile + 16 * w * DH;
      bf16* Vs = Ks + BN * DH;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int ch = (i * 64 + lane) % CPR;
        const float sc = exp_scale((ex[i] >> (8 * (ch >> 1))) & 255);
        bf16 *kd = Ks + row[i] * DH, *vd = Vs + row[i] * DH;
        *reinterpret_cast<bf16x8*>(kd + 8 * kswz<DH>(row[i], 2 * ch)) = decode8(kr[i][0], kr[i][1], sc);
        *reinterpret_cast<bf16x8*>(kd + 8 * kswz<DH>(row[i], 2 * ch + 1)) = decode8(kr[i][2], kr[i][3], sc);
        *reinterpret_cast<bf16x8*>(vd + 8 * vswz<DH>(row[i], 2 * ch)) = decode8(vr[i][0], vr[i][1], 1.0f);
        *reinterpret_cast<bf16x8*>(vd + 8 * vswz<DH>(row[i], 2 * ch + 1)) = decode8(vr[i][2], vr[i][3], 1.0f);
      }
    }
  }
};

// does any of a tile's 64 V rows hold an infinity or a NaN?  (Reads with their wait in one block: the compiler's own would wait
// for the next tile's direct loads.)
template <int DH>
WAM_DEV bool any_not_finite(const char* Vs, int lane) {
  const unsigned at = lds_addr(Vs) + 16 * lane;
  float z = 0.f;
#pragma unroll
  for (int i = 0; i < DH / 32; ++i) {
    u32x4v a, b, c, d;
    asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:1024\n\tds_read_b128 %2, %4 offset:2048\n\t"
                 "ds_read_b128 %3, %4 offset:3072\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(a), "=&v"(b), "=&v"(c), "=&v"(d)
                 : "v"(at + 4096 * i));
    z = zero_times(d, zero_times(c, zero_times(b, zero_times(a, z))));
  }
  return __any(z != 0.f);
}

// scores, mask (row_kend: the lane's prefix; groups: which of the tile's four 16-key groups have a page), softmax,
// value product
template <int DH, bool MASK>
WAM_DEV void ragged_tile(const char* Ks, const bf16x8* qf, f32x16* acc, float& m_ref, float& l_part, const int* kofs,
                         const int* vofs, float c, float thr, int kb, int row_kend, int groups, int hh) {
  f32x16 s[2] = {f32x16{}, f32x16{}};
  __builtin_amdgcn_s_setprio(1);
  scores_tile<DH>(Ks, kofs, qf, s);
  __builtin_amdgcn_s_setprio(0);
  if (MASK) {
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int key = kb + 32 * nt + 8 * (r >> 2) + 4 * hh + (r & 3);
        if (key >= row_kend || !((groups >> (2 * nt + (r >> 3))) & 1)) s[nt][r] = -INFINITY;
      }
  }
  softmax_pv<DH>(s, Ks + BN * DH * 2, acc, m_ref, l_part, vofs, c, thr);
}

// Wait for this wavefront's part of a tile (direct loads and LDS stores), then for the workgroup.
WAM_DEV void tile_arrived() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// GROUPS = 2: the key tiles go in turn to two groups of four wavefronts, each with its own pair of LDS buffers, and the
// groups' states are joined in LDS at the end: two wavefronts per SIMD where there are too few workgroups for two on a
// CU, without parts in memory.
// False, and nothing is written: V of keys that only some of the rows see holds values that are not finite.
template <int DH, bool PAGED, bool FP8, int GROUPS>
WAM_DEV bool tile_rows(const RaggedArgs& a, const Parts& pt, const Req& q, int r, int hk, int G, int m0, int split,
                       bool whole, int start, int end, int meta, bf16* smem_all) {
  constexpr int KS = DH / 16, MT = DH / 32, TILE = 2 * BN * DH;
  const int tid = threadIdx.x, lane = tid & 63, hh = lane >> 5, l32 = lane & 31;
  const int w = uniform(tid >> 6) & 3, grp = GROUPS == 1 ? 0 : uniform(tid >> 8);
  bf16* smem = smem_all + grp * 2 * TILE;
  const int rows = q.n * G;
  const int qrow = m0 + 32 * w + l32, qc = qrow < rows ? qrow : rows - 1, tok = fdiv(a.group, qc), head = hk * G + qc - tok * G;
  const int row_kend = kend_of<PAGED>(a, q, tok);
  const int kmin = kend_of<PAGED>(a, q, fdiv(a.group, m0));
  bf16x8 qf[KS];
  {
    const bf16* qp = static_cast<const bf16*>(a.q) + (q.q0 + tok) * a.q_ts + head * DH + 8 * hh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = load_bf16x8(qp + 16 * ks);
  }
  // LDS operand offsets, as in attn.hip
  int kofs[KS], vofs[MT];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) kofs[ks] = l32 * DH * 2 + kswz<DH>(l32, 2 * ks + hh) * 16;
  {
    const int l16 = lane >> 4, j16 = lane & 15, r0 = 4 * (l16 >> 1) + (j16 >> 2);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int col = 32 * mt + 16 * (l16 & 1) + 4 * (j16 & 3);
      vofs[mt] = r0 * DH * 2 + vswz<DH>(r0, col >> 3) * 16 + 8 * ((col >> 2) & 1);
    }
  }
  f32x16 acc[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) acc[mt] = f32x16{};
  float m_ref = -INFINITY, l_part = 0.f;
  const float c = a.c, thr = RESCALE_LOG2 / c;

  const int t0 = start / BN, nt = end > start ? (end + BN - 1) / BN : t0;
  const int n_plain = kmin / BN;  // tiles before it hide no key from any row
  Fetch<DH, PAGED, FP8> f;
  f.init(a, lane);
  // meta: the pages of a window of 16 tiles, lane l keys 16 l .. of it; and of the next window
  int meta_next = -1;
  auto fetch = [&](int t, int cur, int wend) {
    const int key = t * BN + 16 * w, pg = __builtin_amdgcn_readlane(t < wend ? meta : meta_next, (4 * (t - t0) + w) & 63);
    const int nv = pg < 0 ? 0 : clampi(end - key, 0, 16);
    f.load(a, q, smem + cur * TILE, key, pg, nv, hk, w, lane);
  };
  bool bad = false;
  // this group's tiles: t0 + grp, then every GROUPS-th; two at a time, one per buffer
  if (t0 + grp < nt) {
    fetch(t0 + grp, 0, t0 + 16);
    f.store(smem, w, lane);
  }
  tile_arrived();
  for (int wb = t0; wb < nt; wb += 16) {
    const int we = wb + 16 < nt ? wb + 16 : nt;
    meta_next = page_of<PAGED>(a, r, (wb + 16) * BN + 16 * lane);
    // (groups past the end count as present: the rows' prefixes hide them)
    const uint64_t there = __ballot(meta >= 0 || wb * BN + 16 * lane >= end);
    const int plain = ~there == 0 ? (n_plain < we ? n_plain : we) : wb;
    int tb = wb;  // the groups' tiles tb .. tb + GROUPS - 1
    auto step = [&](int cur, auto mask) {
      const int t = tb + grp;
      if (GROUPS == 1 || t < nt) {
        if (t + GROUPS < nt) fetch(t + GROUPS, cur ^ 1, wb + 16);
        const char* Ks = reinterpret_cast<const char*>(smem + cur * TILE);
        // (keys that the first row does not see: the same answer in every wavefront of the group)
        if (decltype(mask)::value && kmin < end && t * BN + BN > kmin && any_not_finite<DH>(Ks + BN * DH * 2, lane)) bad = true;
        ragged_tile<DH, decltype(mask)::value>(Ks, qf, acc, m_ref, l_part, kofs, vofs, c, thr, t * BN, row_kend,
                                               (int)(there >> (4 * (t - wb))) & 15, hh);
        if (t + GROUPS < nt) f.store(smem + (cur ^ 1) * TILE, w, lane);
      }
      tile_arrived();
      tb += GROUPS;
    };
    while (tb + 2 * GROUPS <= plain) {
      step(0, std::false_type{});
      step(1, std::false_type{});
    }
    while (tb < we) step((tb - t0) / GROUPS & 1, std::true_type{});
    meta = meta_next;
  }

  float l = l_part + other_half(l_part);
  if constexpr (GROUPS == 2) {
    // the second group's state through the first's buffers, register by register (the same lanes hold the same rows)
    float* mine = reinterpret_cast<float*>(smem_all) + w * (16 * MT * 64) + lane;
    float* stat = reinterpret_cast<float*>(smem_all + 2 * TILE) + w * 128 + lane;
    int* theirs = reinterpret_cast<int*>(smem_all + 2 * TILE) + 512;  // (the same of all of its wavefronts)
    if (grp == 1) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int e = 0; e < 16; ++e) mine[(16 * mt + e) * 64] = acc[mt][e];
      stat[0] = m_ref;
      stat[64] = l;
      *theirs = bad;
    }
    __syncthreads();
    if (grp == 1) return true;
    if (uniform(*theirs)) bad = true;
    const float m2 = stat[0], l2 = stat[64], top = fmaxf(m_ref, m2);
    const float f1 = m_ref == -INFINITY ? 0.f : exp2_fast((m_ref - top) * c);
    const float f2 = m2 == -INFINITY ? 0.f : exp2_fast((m2 - top) * c);
    m_ref = top;
    l = l * f1 + l2 * f2;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[mt][e] = acc[mt][e] * f1 + mine[(16 * mt + e) * 64] * f2;
    lds_order();  // (each wavefront reads and then overwrites its own quarter)
  }
  if (bad) return false;
  // The output through LDS (the key tiles are done with), so that a row leaves in whole lines: a lane holds 4 dims here and
  // there of one row; the wavefront's 32 rows go to its quarter of LDS, 16-byte chunks XOR-swizzled by the row (written
  // 8 bytes per lane, 32 rows; read back one row per 16 lanes).  whole: bf16; else fp32, in two halves of the dims.
  char* my = reinterpret_cast<char*>(smem) + w * (BN * DH * 2);
  constexpr int CH = DH / 8, RPI = 64 / CH;  // 16-byte chunks of a row of DH bf16 (or DH / 2 fp32), rows per instruction
  const auto put = [&](auto&& chunk_out) {  // chunk_out(row's index, token, head, chunk, 16 bytes)
    lds_order();
#pragma unroll
    for (int i = 0; i < 32 / RPI; ++i) {
      const int rr = RPI * i + lane / CH, ch = lane % CH, row = m0 + 32 * w + rr;
      const u32x4v v = *reinterpret_cast<const u32x4v*>(my + rr * DH * 2 + 16 * (ch ^ (rr & (CH - 1))));
      if (row < rows) {
        const int tk = fdiv(a.group, row);
        chunk_out((int64_t)q.q0 + tk, hk * G + row - tk * G, ch, v);
      }
    }
    lds_order();
  };
  if (whole) {
    const float inv = l > 0.f ? (FP8 ? a.v_scale : 1.f) / l : 0.f;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int rr = 0; rr < 4; ++rr) {
        const int ch = 4 * mt + rr;  // dims 8 ch + 4 hh ..
        *reinterpret_cast<bf16x4*>(my + l32 * DH * 2 + 16 * (ch ^ (l32 & (CH - 1))) + 8 * hh) =
            bf16x4{(bf16)(acc[mt][4 * rr + 0] * inv), (bf16)(acc[mt][4 * rr + 1] * inv),
                   (bf16)(acc[mt][4 * rr + 2] * inv), (bf16)(acc[mt][4 * rr + 3] * inv)};
      }
    // (not to be kept in the caches: two samples' 3152 rows against 512 and 248 keys 93 -> 73 to 86 us)
    put([&](int64_t tk, int h, int ch, u32x4v v) {
      __builtin_nontemporal_store(v, reinterpret_cast<u32x4v*>(static_cast<bf16*>(a.o) + tk * a.o_ts + h * DH + 8 * ch));
    });
  } else {
    if (hh == 0 && qrow < rows) {
      const int64_t id = ((int64_t)(q.q0 + tok) * a.Hq + head) * pt.splits + split;
      pt.ml[2 * id] = m_ref;
      pt.ml[2 * id + 1] = l;
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int mt = half * MT / 2; mt < (half + 1) * MT / 2; ++mt)
#pragma unroll
        for (int rr = 0; rr < 4; ++rr) {
          const int ch = 8 * (mt - half * MT / 2) + 2 * rr + hh;  // dims DH / 2 half + 4 ch ..
          *reinterpret_cast<f32x4*>(my + l32 * DH * 2 + 16 * (ch ^ (l32 & (CH - 1)))) =
              f32x4{acc[mt][4 * rr + 0], acc[mt][4 * rr + 1], acc[mt][4 * rr + 2], acc[mt][4 * rr + 3]};
        }
      put([&](int64_t tk, int h, int ch, u32x4v v) {
        const int64_t id = (tk * a.Hq + h) * pt.splits + split;
        *reinterpret_cast<u32x4v*>(pt.o + id * DH + half * (DH / 2) + 4 * ch) = v;
      });
    }
  }
  return true;
}

// last request whose start is not past x, or -1; by row tiles (2^shift rows each) the first tile of request r is
// floor(q_start[r] G / 2^shift) + r
WAM_DEV int find_request(const RaggedArgs& a, int x, int G, int shift, int lane) {
  if (a.R == 1) return 0;  // (rows before it or past it are none of its)
  // 64 requests at a time; of more, first every so-manieth, then those between two (the starts do not fall)
  int lo = 0, n = a.R;
  for (;;) {
    const int step = (n + 63) >> 6, r = lo + lane * step;
    bool in = false;
    if (lane * step < n) in = shift ? (((int64_t)a.q_start[r] * G) >> shift) + r <= x : a.q_start[r] <= x;
    const int cnt = __popcll(__ballot(in));
    if (step == 1 || cnt == 0) return lo + cnt - 1;
    lo += (cnt - 1) * step;
    n = n - (cnt - 1) * step < step ? n - (cnt - 1) * step : step;
  }
}

// A workgroup's work: its request, KV head, first row, and keys.
struct Work {
  Req q;
  int r, hk, G, m0, split, start, end;
  int meta;    // lane: page of a group of the first keys
  bool whole;  // the request has one part: the output itself is written
};
template <bool PAGED, int SHIFT>
WAM_DEV bool find_work(const RaggedArgs& a, const Parts& pt, int block, Work& k) {
  const int lane = threadIdx.x & 63;
  k.G = (int)a.group.d;
  int x;
  if (SHIFT == 7) {
    // rows share keys with their neighbours: each XCD a contiguous range of (row tile, head) pairs
    const int nblk = gridDim.x, bi = block, xcd = bi & 7, per = nblk >> 3, rem = nblk & 7;
    const int lid = xcd * per + (xcd < rem ? xcd : rem) + (bi >> 3);
    const int column = fdiv(pt.by_tiles, lid);
    x = lid - column * pt.tiles;
    k.split = fdiv(pt.by_heads, column);
    k.hk = column - k.split * a.Hkv;
  } else {
    // the heads of the same keys, neighbours in memory, one after another on one XCD; parts and requests in turn over
    // the XCDs
    const int slot = block >> 3, column = fdiv(pt.by_heads, slot), part = column * 8 + (block & 7);
    k.hk = slot - column * a.Hkv;
    x = fdiv(pt.by_splits, part);
    const int turned = part - x * pt.splits + fdiv_rest(pt.by_splits, x);
    k.split = turned < pt.splits ? turned : turned - pt.splits;  // (by the request: no XCD has all of the late, rarer parts)
  }
  if (x >= pt.tiles) return false;
  k.r = uniform(find_request(a, x, k.G, SHIFT, lane));
  if (k.r < 0) return false;
  k.start = k.split * pt.split_keys;
  // the first keys' pages, before the request's own lengths are there (the table's row is)
  const int w = uniform(threadIdx.x >> 6);
  k.meta = page_of<PAGED>(a, k.r, k.start + (SHIFT == 7 ? 16 * lane : 32 * w + stream_key(lane)));
  k.q = request<PAGED>(a, k.r);
  const int64_t m0 = ((int64_t)x - k.r - (((int64_t)k.q.q0 * k.G) >> SHIFT)) * (1 << SHIFT);
  const int rows = k.q.n * k.G;
  if (m0 < 0 || m0 >= rows) return false;
  k.m0 = (int)m0;
  if (k.split > 0 && k.start >= k.q.keys) return false;
  k.whole = k.q.keys <= pt.split_keys;
  const int last = rows - k.m0 > (1 << SHIFT) ? k.m0 + (1 << SHIFT) - 1 : rows - 1;
  const int kmax = kend_of<PAGED>(a, k.q, fdiv(a.group, last));
  k.end = kmax - k.start < pt.split_keys ? kmax : k.start + pt.split_keys;
  return true;
}

// Requests with more than a few rows on average: 128 rows per workgroup; those with at most 32 are streamed.
// (Head size 64: 168 registers, three wavefronts per SIMD; with two 12 causal requests of 1 to 901 rows 33 -> 38 us.)
template <int DH, bool PAGED, bool FP8, int GROUPS>
__global__ __launch_bounds__(NT * GROUPS, DH == 64 ? 3 : 2) void ragged_tile_kernel(const RaggedArgs a, const Parts pt) {
  __shared__ __attribute__((aligned(16))) bf16 smem[GROUPS * 4 * BN * DH];
  static_assert(RAGGED_ROWS == 128, "2^7 rows");
  Work k;
  if (!find_work<PAGED, 7>(a, pt, blockIdx.x, k)) return;
  int last = k.m0 + 1;  // streamed: the rows m0 .. last - 1, 32 at a time
  if (GROUPS == 2 || k.q.n * k.G > RAGGED_STREAM) {
    if (tile_rows<DH, PAGED, FP8, GROUPS>(a, pt, k.q, k.r, k.hk, k.G, k.m0, k.split, k.whole, k.start, k.end, k.meta, smem))
      return;
    int block = blockIdx.x;  // (found anew, so that nothing is kept for it: two samples' 3152 rows 1861 -> 1831 us)
    asm volatile("" : "+s"(block) : : "memory");
    find_work<PAGED, 7>(a, pt, block, k);
    last = k.q.n * k.G < k.m0 + RAGGED_ROWS ? k.q.n * k.G : k.m0 + RAGGED_ROWS;
  }
  const int meta = page_of<PAGED>(a, k.r, k.start + 32 * uniform(threadIdx.x >> 6) + stream_key(threadIdx.x & 63));
#pragma unroll 1
  for (int m = k.m0; m < last; m += RAGGED_STREAM) {
    __syncthreads();  // (LDS of what was before)
    stream_rows<DH, PAGED, FP8, 2>(a, pt, k.q, k.r, k.hk, k.G, m, k.split, k.whole, k.start, k.end, meta,
                                   reinterpret_cast<char*>(smem));
  }
}

// Few rows per request: 16 NQ per workgroup.  (Wavefronts per SIMD as the registers come out: of 128 dims and 16 rows three
// over pages and two over packed states, 168 and 170 registers; two for 32 rows.)
template <int DH, bool PAGED, bool FP8, int NQ>
__global__ __launch_bounds__(NT, 2) void ragged_stream_kernel(const RaggedArgs a, const Parts pt) {
  __shared__ __attribute__((aligned(16))) char smem[stream_lds(DH, FP8)];
  Work k;
  if (!find_work<PAGED, NQ == 1 ? 4 : 5>(a, pt, blockIdx.x, k)) return;
  stream_rows<DH, PAGED, FP8, NQ>(a, pt, k.q, k.r, k.hk, k.G, k.m0, k.split, k.whole, k.start, k.end, k.meta, smem);
}

// The join: o = sum_s 2^(c (m_s - m)) o_s / sum_s 2^(c (m_s - m)) l_s over the parts s of a row, in their order.
// Two forms: for few rows a workgroup for each, its parts over four wavefronts (the chain of loads is what takes the
// time); for many a thread for four dims of a row, a workgroup for some heads of a token.
// Every part of a row is written, also where the row sees none of its keys (sum and outputs 0), so a part of weight 0
// is added like the others: a NaN or an infinity in its outputs reaches the row, as it does within one part.
template <bool PAGED>
WAM_DEV int parts_of(const RaggedArgs& a, const Parts& pt, int t, int lane) {  // 0: nothing to join
  const int r = uniform(find_request(a, t, 1, 0, lane));
  if (r < 0) return 0;
  const Req q = request<PAGED>(a, r);
  if (t < q.q0 || t - q.q0 >= q.n || q.keys <= pt.split_keys) return 0;
  return (q.keys + pt.split_keys - 1) / pt.split_keys;
}

template <int DH, bool PAGED, bool FP8>
__global__ __launch_bounds__(256) void ragged_join_few_kernel(const RaggedArgs a, const Parts pt) {
  __shared__ float red[4][DH];
  constexpr int PER = DH / 64;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t id = blockIdx.x;
  const int t = (int)(id / a.Hq), h = (int)(id - (int64_t)t * a.Hq);
  const int n = parts_of<PAGED>(a, pt, t, lane);
  if (n == 0) return;
  float m = -INFINITY, l = 0.f;
  if (lane < n) {
    m = pt.ml[2 * (id * pt.splits + lane)];
    l = pt.ml[2 * (id * pt.splits + lane) + 1];
  }
  float top = m;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) top = fmaxf(top, __shfl_xor(top, s, 64));
  const float f = l != 0.f ? exp2_fast((m - top) * a.c) : 0.f;
  const float sum = wave_sum(f * l);
  float y[PER] = {};
  const float* o = pt.o + id * pt.splits * DH + lane * PER;
  for (int s0 = w; s0 < n; s0 += 16) {
    float v[4][PER];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int s = s0 + 4 * j < n ? s0 + 4 * j : s0;
#pragma unroll
      for (int e = 0; e < PER; ++e) v[j][e] = o[(int64_t)s * DH + e];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool there = s0 + 4 * j < n;
      const float fs = __shfl(f, there ? s0 + 4 * j : s0, 64);
#pragma unroll
      for (int e = 0; e < PER; ++e) y[e] += there ? fs * v[j][e] : 0.f;
    }
  }
#pragma unroll
  for (int e = 0; e < PER; ++e) red[w][lane * PER + e] = y[e];
  __syncthreads();
  if (w > 0) return;
  // (a NaN among a part's sums makes the row NaN, also where the part's own weight is 0: all of its scores were NaN)
  const float inv = sum != 0.f ? (FP8 ? a.v_scale : 1.f) / sum : 0.f;
  bf16* op = static_cast<bf16*>(a.o) + t * a.o_ts + h * DH + lane * PER;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const int i = lane * PER + e;
    op[e] = (bf16)(((red[0][i] + red[1][i]) + (red[2][i] + red[3][i])) * inv);
  }
}

template <int DH, bool PAGED, bool FP8>
__global__ __launch_bounds__(256) void ragged_join_kernel(const RaggedArgs a, const Parts pt) {
  constexpr int LPH = DH / 4, HEADS = 256 / LPH;  // threads of a head, heads of a workgroup
  const int t = blockIdx.x, n = parts_of<PAGED>(a, pt, t, threadIdx.x & 63), d = threadIdx.x % LPH * 4;
  if (n == 0) return;
  const int h = blockIdx.y * HEADS + threadIdx.x / LPH;
  if (h < a.Hq) {
    const int64_t id = ((int64_t)t * a.Hq + h) * pt.splits;
    float top = -INFINITY, sum = 0.f;
#pragma unroll 4
    for (int s = 0; s < n; ++s) top = fmaxf(top, pt.ml[2 * (id + s)]);
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < n; ++s) {
      const float m = pt.ml[2 * (id + s)], l = pt.ml[2 * (id + s) + 1], f = l != 0.f ? exp2_fast((m - top) * a.c) : 0.f;
      const f32x4 v = *reinterpret_cast<const f32x4*>(pt.o + (id + s) * DH + d);
      sum += f * l;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] += f * v[e];
    }
    const float inv = sum != 0.f ? (FP8 ? a.v_scale : 1.f) / sum : 0.f;
    *reinterpret_cast<bf16x4*>(static_cast<bf16*>(a.o) + t * a.o_ts + h * DH + d) =
        bf16x4{(bf16)(y[0] * inv), (bf16)(y[1] * inv), (bf16)(y[2] * inv), (bf16)(y[3] * inv)};
  }
}

template <int DH, bool PAGED, bool FP8>
hipError_t launch(const RaggedArgs& a, const Parts& pt, const RaggedPlan& p, hipStream_t s) {
  const dim3 grid((unsigned)ragged_blocks(p, a.R, a.T, a.Hq, a.Hkv)), block(NT);
  if (p.rows == 16) hipLaunchKernelGGL((ragged_stream_kernel<DH, PAGED, FP8, 1>), grid, block, 0, s, a, pt);
  else if (p.rows == 32) hipLaunchKernelGGL((ragged_stream_kernel<DH, PAGED, FP8, 2>), grid, block, 0, s, a, pt);
  else if (p.groups == 1) hipLaunchKernelGGL((ragged_tile_kernel<DH, PAGED, FP8, 1>), grid, block, 0, s, a, pt);
  else hipLaunchKernelGGL((ragged_tile_kernel<DH, PAGED, FP8, 2>), grid, dim3(2 * NT), 0, s, a, pt);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || pt.splits == 1) return e;
  const int64_t out = (int64_t)a.T * a.Hq;
  constexpr int HEADS = 256 / (DH / 4);
  if (out <= 4096) hipLaunchKernelGGL((ragged_join_few_kernel<DH, PAGED, FP8>), dim3((unsigned)out), block, 0, s, a, pt);
  else hipLaunchKernelGGL((ragged_join_kernel<DH, PAGED, FP8>), dim3((unsigned)a.T, (unsigned)((a.Hq + HEADS - 1) / HEADS)), block, 0, s, a,
                          pt);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_ragged(const RaggedArgs& a, const RaggedPlan& p, void* ws, hipStream_t s) {
  Parts pt;
  pt.ml = static_cast<float*>(ws);
  pt.o = reinterpret_cast<float*>(static_cast<char*>(ws) + ragged_ml_bytes(p, a.T, a.Hq));
  pt.splits = p.splits;
  pt.split_keys = p.split_keys;
  pt.tiles = (int)ragged_tiles(a.R, a.T, a.Hq, a.Hkv, p.rows);
  pt.by_splits = fast_div(p.splits);
  pt.by_tiles = fast_div(pt.tiles);
  pt.by_heads = fast_div(a.Hkv);
  if (a.table) {
    if (a.k_exp) return launch<128, true, true>(a, pt, p, s);
    return a.Dh == 128 ? launch<128, true, false>(a, pt, p, s) : launch<64, true, false>(a, pt, p, s);
  }
  return a.Dh == 128 ? launch<128, false, false>(a, pt, p, s) : launch<64, false, false>(a, pt, p, s);
}

}  // namespace wam
