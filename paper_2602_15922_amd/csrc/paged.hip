// The KV cache in pages: block tables and slot maps from request lengths, and rotary
// positions with the append through a slot map.
#include "common.h"
#include "kernels.h"

namespace wam {
namespace {

WAM_DEV int fdiv(const FastDiv& f, int n) {
  return f.d == 1 ? n : (int)(__umulhi((uint32_t)n, f.mul) >> f.shift);
}
WAM_DEV int clampi(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }

// ---------------------------------------------------------------------------------
// Page plan.  Every workgroup forms the same three exclusive sums over the requests (new
// tokens, pages to take, surplus pages) in LDS, then fills its share of the rows; so one
// launch does it all and no workgroup waits for another.  The stack of free pages is never
// read where it is written: surplus pages lie on top of it, a page taken is either
// entry [n_free - ...] of the list as it came or, found by a search in the sums, an entry of the
// table row that gives it up, and only what stays on the stack is stored.
//
// Bound by latency, a chain of dependent loads (lengths, sums, search, table entry), so: the sums
// are in 32 bits (tokens saturate at T) and in registers but for one exchange through LDS, and workgroups
// are small and many, each with one kind of output.  6 requests with 5600 rows: 5.0 us, 1000 with 196000 rows and
// 27000 pages that change hands 11.7 us (1000 with a row each 11.8); 1030 and 1900 requests, which read the lengths again
// instead of keeping them in LDS, 17 and 18 us.  With one kind of workgroup for all outputs the first two 5.7 and 13.4; with
// 64-bit sums by lane exchange, 1024 threads, and a search and a 64-bit division per token 27.6 and 43.1.
// ---------------------------------------------------------------------------------
constexpr int PLAN_NT = 256;

WAM_DEV uint32_t udiv(const FastDiv& f, uint32_t n) { return n < 0x80000000u ? (uint32_t)fdiv(f, (int)n) : n / f.d; }

struct PlanReq {
  int cache, fresh, held, need;
  uint32_t over;  // pages past the table's width
  bool bad;
};
WAM_DEV PlanReq plan_req(const PagePlanArgs& a, int r) {
  const int c = a.cache_len[r], n = a.new_len[r], h = a.held[r];
  PlanReq q;
  q.cache = c < 0 ? 0 : c;
  q.fresh = n < 0 ? 0 : n;
  q.held = clampi(h, 0, a.d.max_pages);
  q.bad = c < 0 || n < 0 || q.held != h;
  const uint32_t len = (uint32_t)q.cache + (uint32_t)q.fresh, full = udiv(a.ps, len);
  const uint32_t whole = full + (full * (uint32_t)a.d.page_size < len ? 1 : 0);
  q.need = whole < (uint32_t)a.d.max_pages ? (int)whole : a.d.max_pages;
  q.over = whole - (uint32_t)q.need;
  return q;
}

// last r in [0, n) with at[r] <= x (at[0] = 0, non-decreasing, x >= 0)
WAM_DEV int last_at_most(const int* at, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (at[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// inclusive sums over the wavefront, cut to `most` (all values in [0, most])
#define WAM_SCAN_STEP(ctrl, rows)                                                   \
  {                                                                                 \
    const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, rows, 0xf, false) + v; \
    v = y < most ? y : most;                                                        \
  }
WAM_DEV uint32_t row_scan(uint32_t v, uint32_t most) {
  WAM_SCAN_STEP(0x111, 0xf)  // row_shr 1, 2, 4, 8: within rows of 16 lanes
  WAM_SCAN_STEP(0x112, 0xf)
  WAM_SCAN_STEP(0x114, 0xf)
  WAM_SCAN_STEP(0x118, 0xf)
  return v;
}
WAM_DEV uint32_t wave_scan(uint32_t v, uint32_t most) {
  v = row_scan(v, most);
  WAM_SCAN_STEP(0x142, 0xa)  // row_bcast 15: rows 1 and 3 take the last of the row before
  WAM_SCAN_STEP(0x143, 0xc)  // row_bcast 31: rows 2 and 3 take the last of row 1
  return v;
}
#undef WAM_SCAN_STEP

// What the fill threads need of a request, from LDS where all of it fits (E small), else from memory again.
template <int E>
struct PlanLds {
  alignas(16) int q_at[E * PLAN_NT], take_at[E * PLAN_NT], back_at[E * PLAN_NT];
  int cache[E <= 4 ? E * PLAN_NT : 1], held[E <= 4 ? E * PLAN_NT : 1], need[E <= 4 ? E * PLAN_NT : 1];
  uint32_t wave[3][PLAN_NT / 64];
  uint64_t total[3][PLAN_NT / 64];  // status: new tokens, pages past the width, invalid inputs of each wavefront
};

// E requests per thread: R <= 256 E.  The first `rows` workgroups fill the new tokens' rows, the last the requests'
// outputs and the status, those between them the pages that change hands.
template <int E>
__global__ __launch_bounds__(PLAN_NT) void page_plan_kernel(const PagePlanArgs a, int rows) {
  __shared__ PlanLds<E> L;
  const int R = a.d.R, T = a.d.T, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int nf_in = a.n_free[0], nf = clampi(nf_in, 0, a.d.n_pages);
  const bool status = blockIdx.x == gridDim.x - 1;
  uint32_t fresh[E], take[E], back[E], sum[3] = {0, 0, 0};
  uint64_t all_new = 0, all_over = 0, all_bad = 0;
  const uint32_t most[3] = {(uint32_t)T, 0x7fffffffu, 0x7fffffffu};
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int r = tid * E + e;
    fresh[e] = take[e] = back[e] = 0;
    if (r < R) {
      const PlanReq q = plan_req(a, r);
      fresh[e] = (uint32_t)(q.fresh < T ? q.fresh : T);
      take[e] = q.need > q.held ? q.need - q.held : 0;
      back[e] = q.held > q.need ? q.held - q.need : 0;
      if (status) {
        all_new += q.fresh;
        all_over += q.over;
        all_bad += q.bad;
      }
      if constexpr (E <= 4) {
        L.cache[r] = q.cache;
        L.held[r] = q.held;
        L.need[r] = q.need;
      }
    }
    sum[0] = sum[0] + fresh[e] < most[0] ? sum[0] + fresh[e] : most[0];
    sum[1] += take[e];
    sum[2] += back[e];
  }
  uint32_t at[3], all[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const uint32_t incl = wave_scan(sum[i], most[i]);
    at[i] = (uint32_t)__shfl_up((int)incl, 1, 64);
    if (lane == 0) at[i] = 0;
    if (lane == 63) L.wave[i][w] = incl;
  }
  if (status) {
    const uint64_t total[3] = {all_new, all_over, all_bad};
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      // (may pass 32 bits: the low 16 bits and the rest apart)
      const uint32_t lo = wave_scan((uint32_t)total[i] & 0xffffu, ~0u), hi = wave_scan((uint32_t)(total[i] >> 16), ~0u);
      if (lane == 63) L.total[i][w] = ((uint64_t)hi << 16) + lo;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    uint32_t before = 0;
    all[i] = 0;
#pragma unroll
    for (int k = 0; k < PLAN_NT / 64; ++k) {
      const uint32_t x = L.wave[i][k];
      if (k == w) before = all[i];
      all[i] = all[i] + x < most[i] ? all[i] + x : most[i];
    }
    at[i] = before + at[i] < most[i] ? before + at[i] : most[i];
  }
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int r = tid * E + e;
    L.q_at[r] = (int)at[0];
    L.take_at[r] = (int)at[1];
    L.back_at[r] = (int)at[2];
    at[0] = at[0] + fresh[e] < most[0] ? at[0] + fresh[e] : most[0];
    at[1] += take[e];
    at[2] += back[e];
  }
  __syncthreads();
  const int tokens = (int)all[0], takes = (int)all[1], backs = (int)all[2];
  const int64_t top = (int64_t)nf + backs;  // height of the stack with the surplus pages on it
  const int64_t left = top - takes;

  struct Three { int cache, held, need; };
  auto req = [&](int r) {
    if constexpr (E <= 4) return Three{L.cache[r], L.held[r], L.need[r]};
    const PlanReq q = plan_req(a, r);
    return Three{q.cache, q.held, q.need};
  };
  // surplus page number j, in order of requests and entries
  auto back_page = [&](int j) {
    const int r = last_at_most(L.back_at, R, j);
    return a.table[(int64_t)r * a.d.table_stride + req(r).need + (j - L.back_at[r])];
  };
  // the k-th page taken, -1 where the stack is empty
  auto taken_page = [&](int k) {
    const int64_t i = top - 1 - k;
    if (i < 0) return -1;
    return i >= nf ? back_page((int)(i - nf)) : a.free_list[i];
  };

  if (status) {
    for (int r = tid; r < R; r += PLAN_NT) {
      const Three q = req(r);
      const int want = q.need > q.held ? q.need - q.held : 0;
      const int64_t room = top - L.take_at[r];
      const int end = r + 1 < R ? L.q_at[r + 1] : tokens;
      a.held_out[r] = (q.need < q.held ? q.need : q.held) + (int)(room < 0 ? 0 : (room < want ? room : want));
      a.q_start[r] = L.q_at[r];
      const int64_t kv = (int64_t)q.cache + (end - L.q_at[r]);
      a.kv_len[r] = (int)(kv < INT32_MAX ? kv : INT32_MAX);
    }
    if (tid == 0) {
      uint64_t v[3];
#pragma unroll
      for (int i = 0; i < 3; ++i) v[i] = L.total[i][0] + L.total[i][1] + L.total[i][2] + L.total[i][3];
      const uint64_t cut = v[0] - tokens, big = 0x7fffffffu;
      a.q_start[R] = tokens;
      a.n_free_out[0] = (int)(left < 0 ? 0 : (left < a.d.n_pages ? left : a.d.n_pages));
      a.status[0] = (int)(left < 0 ? -left : 0);
      a.status[1] = (int)(v[1] < big ? v[1] : big);
      a.status[2] = (int)(cut < big ? cut : big);
      a.status[3] = (int)v[2] + (nf != nf_in);
    }
    return;
  }

  if ((int)blockIdx.x >= rows) {
    const int id = ((int)blockIdx.x - rows) * PLAN_NT + tid, n_threads = ((int)gridDim.x - 1 - rows) * PLAN_NT;
    for (int k = id; k < takes; k += n_threads) {
      const int r = last_at_most(L.take_at, R, k);
      a.table[(int64_t)r * a.d.table_stride + req(r).held + (k - L.take_at[r])] = taken_page(k);
    }
    for (int j = id; j < backs - takes; j += n_threads)
      if (nf + (int64_t)j < a.d.n_pages) a.free_list[nf + j] = back_page(j);
    return;
  }

  const bool wide = ((reinterpret_cast<uintptr_t>(a.slots) | reinterpret_cast<uintptr_t>(a.token_pos)) & 15) == 0;
  for (int64_t t0 = 4 * ((int64_t)blockIdx.x * PLAN_NT + tid); t0 < T; t0 += 4 * (int64_t)rows * PLAN_NT) {
    int slot[4], pos[4], r = 0, next = -1, page = -1;  // tokens below `next` belong to request r
    uint32_t entry = 0xffffffffu;                      // the entry that `page` is
    Three q{0, 0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int t = (int)t0 + j;
      slot[j] = pos[j] = -1;
      if (t0 + j >= tokens) continue;
      if (t >= next) {
        r = last_at_most(L.q_at, R, t);
        q = req(r);
        next = r + 1 < R ? L.q_at[r + 1] : tokens;
        entry = 0xffffffffu;
      }
      const uint32_t p = (uint32_t)q.cache + (uint32_t)(t - L.q_at[r]);
      pos[j] = (int)(p < 0x7fffffffu ? p : 0x7fffffffu);
      const uint32_t e = udiv(a.ps, p);
      if (e >= (uint32_t)q.need) continue;
      if (e != entry) {
        entry = e;
        page = (int)e < q.held ? a.table[(int64_t)r * a.d.table_stride + e] : taken_page(L.take_at[r] + (int)e - q.held);
      }
      if (page >= 0 && page < a.d.n_pages) slot[j] = page * a.d.page_size + (int)(p - e * (uint32_t)a.d.page_size);
    }
    if (wide && t0 + 4 <= T) {
      *reinterpret_cast<int4*>(a.slots + t0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
      if (a.token_pos) *reinterpret_cast<int4*>(a.token_pos + t0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
    } else {
      for (int j = 0; j < 4 && t0 + j < T; ++j) {
        a.slots[t0 + j] = slot[j];
        if (a.token_pos) a.token_pos[t0 + j] = pos[j];
      }
    }
  }
}

// ---------------------------------------------------------------------------------
// Rotary positions and the append.  A workgroup owns a token: its first threads form the
// cosine and sine of every pair once for all heads (fp64 angle in revolutions, reduced to
// [-1/2, 1/2] there, then fp32), the rest is one pass over the row, 16 dims per item in two 16-byte
// chunks: neighbouring chunks, or the two halves' chunks whose dims turn together.  Bound by memory, each byte
// moved once; a thread's first item is on its way while the angles are formed.  3152 tokens, 40 heads: 44.0 us for
// 194 MB (4.4 TB/s; a large copy reaches 4.85); without the loads' mark as used once 46.1 (but 1120 tokens into an E4M3
// cache 14.9, and 18.5 with it).  Two or four items on their way at once: 46 and 47 us, E4M3 15 and 17.  Rows of up to 128
// items share a workgroup: 8000 tokens of 8/2 heads of 64 11.9 -> 8.6 us.
// ---------------------------------------------------------------------------------
// dims (2p, 2p + 1) of pairs pair0 .. pair0 + 3; pairs from n on are kept
WAM_DEV void turn8(float* y, const float* cs, const float* sn, int pair0, int n) {
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    if (pair0 + p >= n) continue;
    const float c = cs[pair0 + p], s = sn[pair0 + p], x0 = y[2 * p], x1 = y[2 * p + 1];
    y[2 * p] = __builtin_fmaf(x0, c, -(x1 * s));
    y[2 * p + 1] = __builtin_fmaf(x0, s, x1 * c);
  }
}

// 16 dims of a head in two 16-byte chunks
struct RopeItem {
  int head, u, ca, cb;
  bool rot, split;
};
template <int DH>
WAM_DEV RopeItem rope_item(const RopePagedArgs& a, int i) {
  constexpr int U = DH / 16;  // items per head
  RopeItem x;
  x.head = i / U;
  x.u = i % U;
  x.rot = x.head < a.Hq + a.c.Hkv;
  x.split = a.halves && x.rot && x.u < a.n >> 3;
  x.ca = x.split ? x.u : 2 * x.u;
  x.cb = x.split ? x.u + (a.n >> 3) : 2 * x.u + 1;  // (u from n / 8 on: past the rotated dims)
  return x;
}

// An item's chunks xa, xb turned and stored.  dst: the token's row in the cache (elements).
template <int DH, bool FP8>
WAM_DEV void rope_store(const RopePagedArgs& a, const RopeItem& it, bf16x8 xa, bf16x8 xb, const float* cs, const float* sn,
                        int t, int64_t dst) {
  const int Hkv = a.c.Hkv;
  const int head = it.head, u = it.u, ca = it.ca, cb = it.cb;
  const bool rot = it.rot, split = it.split;
  float ya[8], yb[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    ya[j] = (float)xa[j];
    yb[j] = (float)xb[j];
  }
  if (split) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float c = cs[8 * u + j], s = sn[8 * u + j], x = ya[j], y = yb[j];
      ya[j] = __builtin_fmaf(x, c, -(y * s));
      yb[j] = __builtin_fmaf(x, s, y * c);
    }
  } else if (rot && !a.halves) {
    turn8(ya, cs, sn, 4 * ca, a.n);
    turn8(yb, cs, sn, 4 * cb, a.n);
  }
  if (FP8 && head >= a.Hq) {
    const int hk = head - a.Hq - (rot ? 0 : Hkv);
    const int64_t at = dst + hk * a.c.head_stride;
    if (rot) {
      // a block of 32 dims is four chunks: of two items side by side, or, of the halves, the first
      // (second) chunks of four; items of a head are eight lanes in order, so all of a block's are active
      float ma = 0.f, mb = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        ma = fmaxf(ma, fabsf(ya[j]));
        mb = fmaxf(mb, fabsf(yb[j]));
      }
      if (!split) ma = mb = fmaxf(ma, mb);
      ma = fmaxf(ma, __shfl_xor(ma, 1, 64));
      mb = fmaxf(mb, __shfl_xor(mb, 1, 64));
      const float ma2 = __shfl_xor(ma, 2, 64), mb2 = __shfl_xor(mb, 2, 64);
      if (split) {
        ma = fmaxf(ma, ma2);
        mb = fmaxf(mb, mb2);
      }
      const int ea = mx_exp_biased(ma), eb = mx_exp_biased(mb);
      *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.c.k) + at + 8 * ca) = e4m3x8(ya, ldexpf(1.0f, 127 - ea));
      *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.c.k) + at + 8 * cb) = e4m3x8(yb, ldexpf(1.0f, 127 - eb));
      uint8_t* ex = static_cast<uint8_t*>(a.c.k_exp) + at / 32;  // 4 bytes per row of 128 codes
      if ((ca & 3) == 0) ex[ca >> 2] = (uint8_t)ea;
      if ((cb & 3) == 0) ex[cb >> 2] = (uint8_t)eb;
    } else {
      *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.c.v) + at + 8 * ca) = e4m3x8(ya, a.v_inv);
      *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.c.v) + at + 8 * cb) = e4m3x8(yb, a.v_inv);
    }
  } else {
    bf16x8 oa, ob;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      oa[j] = (bf16)ya[j];
      ob[j] = (bf16)yb[j];
    }
    bf16* out;
    if (head < a.Hq) out = static_cast<bf16*>(a.q_out) + t * a.q_ts + head * DH;
    else if (rot) out = static_cast<bf16*>(a.c.k) + dst + (head - a.Hq) * a.c.head_stride;
    else out = static_cast<bf16*>(a.c.v) + dst + (head - a.Hq - Hkv) * a.c.head_stride;
    *reinterpret_cast<bf16x8*>(out + 8 * ca) = oa;
    *reinterpret_cast<bf16x8*>(out + 8 * cb) = ob;
  }
}

// TPT threads per token: 64 or 128 where a row has no more items, so that short rows share a workgroup.
template <int DH, bool FP8, int TPT>
__global__ __launch_bounds__(256) void rope_paged_kernel(const RopePagedArgs a) {
  constexpr int U = DH / 16;
  __shared__ float cs_all[256 / TPT][DH / 2], sn_all[256 / TPT][DH / 2];
  const int tid = threadIdx.x % TPT, sub = threadIdx.x / TPT;
  const int64_t tok = (int64_t)blockIdx.x * (256 / TPT) + sub;
  const int t = (int)(tok < a.T ? tok : a.T - 1);
  const int slot = a.slots[t];
  const bf16* src = static_cast<const bf16*>(a.qkv) + t * a.qkv_ts;
  const int first = a.q_out ? 0 : a.Hq * U, items = (a.Hq + 2 * a.c.Hkv) * U;
  const bool on = tok < a.T && slot >= 0 && slot < a.c.n_pages * a.c.page_size;
  float *cs = cs_all[sub], *sn = sn_all[sub];
  bf16x8 xa, xb;
  auto load = [&](int i) {
    const RopeItem it = rope_item<DH>(a, i);
    const bf16x8 *pa = reinterpret_cast<const bf16x8*>(src + it.head * DH + 8 * it.ca),
                 *pb = reinterpret_cast<const bf16x8*>(src + it.head * DH + 8 * it.cb);
    xa = FP8 ? *pa : __builtin_nontemporal_load(pa);
    xb = FP8 ? *pb : __builtin_nontemporal_load(pb);
  };
  int i = first + tid;
  if (on && i < items) load(i);
  if (on && tid < a.n) {
    const double x = a.pos[(int64_t)t * a.n_axes + a.axis[tid]] * a.turns[tid];
    sincospif(2.0f * (float)(x - rint(x)), &sn[tid], &cs[tid]);
  }
  __syncthreads();
  if (!on) return;
  const int page = fdiv(a.ps, slot), row = slot - page * a.c.page_size;
  const int64_t dst = (int64_t)page * a.c.page_stride + (int64_t)row * a.c.tok_stride;
  while (i < items) {
    rope_store<DH, FP8>(a, rope_item<DH>(a, i), xa, xb, cs, sn, t, dst);
    i += TPT;
    if (i < items) load(i);
  }
}

}  // namespace

hipError_t launch_page_plan(const PagePlanArgs& a, hipStream_t s) {
  // four rows per thread, a page that changes hands per thread (those that the new rows need, and some 16 of each request
  // that ends or shrinks), at most eight workgroups per CU each; and one
  const auto groups = [](int64_t n) { return (int)(n < 1 ? 1 : (n > 2048 ? 2048 : n)); };
  const int rows = groups(((int64_t)a.d.T + 4 * PLAN_NT - 1) / (4 * PLAN_NT));
  const int pages = groups(((int64_t)a.d.T / a.d.page_size + 16 * (int64_t)a.d.R + PLAN_NT - 1) / PLAN_NT);
  const dim3 grid((unsigned)(rows + pages + 1)), block(PLAN_NT);
  static_assert(16 * PLAN_NT >= WAM_PLAN_MAX_REQUESTS, "requests per thread");
  if (a.d.R <= PLAN_NT) hipLaunchKernelGGL(page_plan_kernel<1>, grid, block, 0, s, a, rows);
  else if (a.d.R <= 4 * PLAN_NT) hipLaunchKernelGGL(page_plan_kernel<4>, grid, block, 0, s, a, rows);
  else hipLaunchKernelGGL(page_plan_kernel<16>, grid, block, 0, s, a, rows);
  return hipGetLastError();
}

template <int DH, bool FP8>
static void launch_rope(const RopePagedArgs& a, hipStream_t s) {
  const int tpt = rope_threads(a.Hq, a.c.Hkv, DH);
  const dim3 grid((unsigned)(((int64_t)a.T * tpt + 255) / 256)), block(256);
  if (tpt == 64) hipLaunchKernelGGL((rope_paged_kernel<DH, FP8, 64>), grid, block, 0, s, a);
  else if (tpt == 128) hipLaunchKernelGGL((rope_paged_kernel<DH, FP8, 128>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((rope_paged_kernel<DH, FP8, 256>), grid, block, 0, s, a);
}

hipError_t launch_rope_paged(const RopePagedArgs& a, hipStream_t s) {
  if (a.c.k_exp) launch_rope<128, true>(a, s);
  else if (a.c.Dh == 128) launch_rope<128, false>(a, s);
  else launch_rope<64, false>(a, s);
  return hipGetLastError();
}

}  // namespace wam
