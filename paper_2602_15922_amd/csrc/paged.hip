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
// ---------------------------------------------------------------------------------
constexpr int PLAN_NT = 1024;

struct PlanReq {
  int cache, held, need;
  int64_t whole;  // pages its tokens fill, past the table's width too
  int fresh;      // new tokens
  bool bad;
};
WAM_DEV PlanReq plan_req(const PagePlanArgs& a, int r) {
  const int c = a.cache_len[r], n = a.new_len[r], h = a.held[r];
  PlanReq q;
  q.cache = c < 0 ? 0 : c;
  q.fresh = n < 0 ? 0 : n;
  q.held = clampi(h, 0, a.d.max_pages);
  q.bad = c < 0 || n < 0 || q.held != h;
  q.whole = ((int64_t)q.cache + q.fresh + a.d.page_size - 1) / a.d.page_size;
  q.need = (int)(q.whole < a.d.max_pages ? q.whole : a.d.max_pages);
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

__global__ __launch_bounds__(PLAN_NT) void page_plan_kernel(const PagePlanArgs a) {
  __shared__ int q_at[WAM_PLAN_MAX_REQUESTS], take_at[WAM_PLAN_MAX_REQUESTS], back_at[WAM_PLAN_MAX_REQUESTS];
  __shared__ int64_t wsum[PLAN_NT / 64][5];
  const int R = a.d.R, T = a.d.T, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int nf_in = a.n_free[0], nf = clampi(nf_in, 0, a.d.n_pages);
  int64_t run[5] = {0, 0, 0, 0, 0};  // tokens, takes, backs, pages past the width, invalid inputs
  for (int base = 0; base < R; base += PLAN_NT) {
    const int r = base + tid;
    int64_t v[5] = {0, 0, 0, 0, 0};
    if (r < R) {
      const PlanReq q = plan_req(a, r);
      v[0] = q.fresh;
      v[1] = q.need > q.held ? q.need - q.held : 0;
      v[2] = q.held > q.need ? q.held - q.need : 0;
      v[3] = q.whole - q.need;
      v[4] = q.bad;
    }
    int64_t x[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) {
      x[i] = v[i];
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) {
        const int64_t y = __shfl_up(x[i], s, 64);
        if (lane >= s) x[i] += y;
      }
      if (lane == 63) wsum[w][i] = x[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 5; ++i) {
      int64_t before = 0, all = 0;
      for (int k = 0; k < PLAN_NT / 64; ++k) {
        if (k < w) before += wsum[k][i];
        all += wsum[k][i];
      }
      x[i] += run[i] + before - v[i];
      run[i] += all;
    }
    if (r < R) {
      q_at[r] = (int)(x[0] < T ? x[0] : T);
      take_at[r] = (int)x[1];
      back_at[r] = (int)x[2];
    }
    __syncthreads();
  }
  const int tokens = (int)(run[0] < T ? run[0] : T), takes = (int)run[1], backs = (int)run[2];
  const int64_t top = (int64_t)nf + backs;  // height of the stack with the surplus pages on it

  // surplus page number j, in order of requests and entries
  auto back_page = [&](int j) {
    const int r = last_at_most(back_at, R, j);
    return a.table[(int64_t)r * a.d.table_stride + plan_req(a, r).need + (j - back_at[r])];
  };
  // the k-th page taken, -1 where the stack is empty
  auto taken_page = [&](int k) {
    const int64_t at = top - 1 - k;
    if (at < 0) return -1;
    return at >= nf ? back_page((int)(at - nf)) : a.free_list[at];
  };

  const int id = blockIdx.x * PLAN_NT + tid, n_threads = gridDim.x * PLAN_NT;
  for (int r = id; r < R; r += n_threads) {
    const PlanReq q = plan_req(a, r);
    const int take = q.need > q.held ? q.need - q.held : 0;
    const int64_t room = top - take_at[r];
    const int end = r + 1 < R ? q_at[r + 1] : tokens;
    a.held_out[r] = (q.need < q.held ? q.need : q.held) + (int)(room < 0 ? 0 : (room < take ? room : take));
    a.q_start[r] = q_at[r];
    const int64_t kv = (int64_t)q.cache + (end - q_at[r]);
    a.kv_len[r] = (int)(kv < INT32_MAX ? kv : INT32_MAX);
  }
  if (id == 0) {
    a.q_start[R] = tokens;
    const int64_t left = top - takes;
    a.n_free_out[0] = (int)(left < 0 ? 0 : (left < a.d.n_pages ? left : a.d.n_pages));
    a.status[0] = (int)(left < 0 ? -left : 0);
    a.status[1] = (int)(run[3] < INT32_MAX ? run[3] : INT32_MAX);
    a.status[2] = (int)(run[0] - tokens < INT32_MAX ? run[0] - tokens : INT32_MAX);
    a.status[3] = (int)run[4] + (nf != nf_in);
  }
  for (int k = id; k < takes; k += n_threads) {
    const int r = last_at_most(take_at, R, k);
    a.table[(int64_t)r * a.d.table_stride + plan_req(a, r).held + (k - take_at[r])] = taken_page(k);
  }
  for (int j = id; j < backs - takes; j += n_threads)
    if (nf + j < a.d.n_pages) a.free_list[nf + j] = back_page(j);
  for (int t = id; t < T; t += n_threads) {
    int slot = -1, pos = -1;
    if (t < tokens) {
      const int r = last_at_most(q_at, R, t);
      const PlanReq q = plan_req(a, r);
      const int64_t p = (int64_t)q.cache + (t - q_at[r]);
      pos = (int)(p < INT32_MAX ? p : INT32_MAX);
      const int64_t e = p / a.d.page_size;
      if (e < q.need) {
        const int page = e < q.held ? a.table[(int64_t)r * a.d.table_stride + e]
                                    : taken_page(take_at[r] + (int)e - q.held);
        if (page >= 0 && page < a.d.n_pages) slot = page * a.d.page_size + (int)(p - e * a.d.page_size);
      }
    }
    a.slots[t] = slot;
    if (a.token_pos) a.token_pos[t] = pos;
  }
}

// ---------------------------------------------------------------------------------
// Rotary positions and the append.  A workgroup owns a token: its first threads form the
// cosine and sine of every pair once for all heads (fp64 angle in revolutions, reduced to
// [-1/2, 1/2] there, then fp32), the rest is one pass over the row, 16 dims per item in two 16-byte
// chunks: neighbouring chunks, or the two halves' chunks whose dims turn together.
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

template <int DH, bool FP8>
__global__ __launch_bounds__(256) void rope_paged_kernel(const RopePagedArgs a) {
  constexpr int U = DH / 16;  // items per head
  __shared__ float cs[DH / 2], sn[DH / 2];
  const int t = blockIdx.x, tid = threadIdx.x;
  const int slot = a.slots[t];
  if (slot < 0 || slot >= a.c.n_pages * a.c.page_size) return;
  if (tid < a.n) {
    const double x = a.pos[(int64_t)t * a.n_axes + a.axis[tid]] * a.turns[tid];
    sincospif(2.0f * (float)(x - rint(x)), &sn[tid], &cs[tid]);
  }
  __syncthreads();
  const int page = fdiv(a.ps, slot), row = slot - page * a.c.page_size;
  const int64_t dst = (int64_t)page * a.c.page_stride + (int64_t)row * a.c.tok_stride;
  const int Hkv = a.c.Hkv, n8 = a.n >> 3;
  const bf16* src = static_cast<const bf16*>(a.qkv) + t * a.qkv_ts;
  const int first = a.q_out ? 0 : a.Hq * U, items = (a.Hq + 2 * Hkv) * U;
  for (int i = first + tid; i < items; i += 256) {
    const int head = i / U, u = i % U;
    const bool rot = head < a.Hq + Hkv, split = a.halves && rot && u < n8;
    const int ca = split ? u : 2 * u, cb = split ? u + n8 : 2 * u + 1;  // (n8 <= u: past the rotated dims)
    const bf16x8 xa = load_bf16x8(src + head * DH + 8 * ca), xb = load_bf16x8(src + head * DH + 8 * cb);
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
}

}  // namespace

hipError_t launch_page_plan(const PagePlanArgs& a, hipStream_t s) {
  // about four rows per thread, at most one workgroup per CU
  const int64_t want = ((int64_t)a.d.T + 4 * PLAN_NT - 1) / (4 * PLAN_NT);
  const int grid = want < 1 ? 1 : (want > 256 ? 256 : (int)want);
  hipLaunchKernelGGL(page_plan_kernel, dim3(grid), dim3(PLAN_NT), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_rope_paged(const RopePagedArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.T), block(256);
  if (a.c.k_exp) hipLaunchKernelGGL((rope_paged_kernel<128, true>), grid, block, 0, s, a);
  else if (a.c.Dh == 128) hipLaunchKernelGGL((rope_paged_kernel<128, false>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((rope_paged_kernel<64, false>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace wam
