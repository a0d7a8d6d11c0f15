// Attention of ragged rows over a paged KV cache, or over packed states of other lengths.
#include "common.h"
#include "kernels.h"

namespace wam {
namespace {

WAM_DEV int fdiv(const FastDiv& f, int n) {
  return f.d == 1 ? n : (int)(__umulhi((uint32_t)n, f.mul) >> f.shift);
}
WAM_DEV int clampi(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }

// One decoded value of a K or V row.
template <bool FP8>
WAM_DEV float value(const void* p, int64_t at) {
  if constexpr (FP8)
    return __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(p)[at], 0);
  else
    return (float)static_cast<const bf16*>(p)[at];
}

// One wavefront per (token, query head), 64 keys at a time: a lane forms the score of a key, the
// wavefront keeps the running maximum and sum, and a lane sums the output dims it owns.
template <int DH, bool PAGED, bool FP8>
__global__ __launch_bounds__(64) void attn_ragged_kernel(const RaggedArgs a) {
  __shared__ float qs[DH], ps[64];
  const int t = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
  // the request of row t: the last whose start is not past it
  int cnt = 0;
  for (int b = 0; b < a.R; b += 64) {
    const bool in = b + lane < a.R && a.q_start[b + lane] <= t;
    cnt += __popcll(__ballot(in));
  }
  const int r = cnt - 1;
  if (r < 0) return;
  const int q0 = a.q_start[r], room = clampi(a.q_start[r + 1], 0, a.T) - q0;
  int n = a.q_len ? a.q_len[r] : room;
  n = n < room ? n : room;
  if (q0 < 0 || t - q0 >= n) return;
  int64_t k0 = 0;
  int kv, kend;
  if (PAGED) {
    kv = a.k_len[r];
    kend = kv;
    const int64_t p = (int64_t)kv - n + (t - q0);
    if (a.chunk) {
      const int64_t e = p < 0 ? 0 : (p / a.chunk + 1) * a.chunk;
      kend = e < kend ? (int)e : kend;
    }
  } else {
    k0 = clampi(a.k_start[r], 0, a.S);
    kend = a.k_len ? a.k_len[r] : a.k_start[r + 1] - (int)k0;
    kend = kend < a.S - k0 ? kend : a.S - (int)k0;
  }
  kend = clampi(kend, 0, a.max_k);
  const int hk = h / (a.Hq / a.Hkv);
  for (int i = lane; i < DH; i += 64) qs[i] = (float)(static_cast<const bf16*>(a.q)[t * a.q_ts + h * DH + i]);
  __syncthreads();
  float m = -INFINITY, l = 0.f, acc[DH / 64] = {};
  for (int kb = 0; kb < kend; kb += 64) {
    const int j = kb + lane;
    int64_t at = -1;
    if (j < kend) {
      if (PAGED) {
        const int e = fdiv(a.ps, j), page = a.table[r * a.table_stride + e];
        if (page >= 0 && page < a.n_pages)
          at = page * a.page_stride + (int64_t)(j - e * (int)a.ps.d) * a.tok_stride + hk * a.head_stride;
      } else {
        at = (k0 + j) * a.tok_stride + hk * DH;
      }
    }
    float s = -INFINITY;
    if (at >= 0) {
      s = 0.f;
      const uint32_t ex = FP8 ? static_cast<const uint32_t*>(a.k_exp)[at / 128] : 0;
      for (int b = 0; b < DH / 32; ++b) {
        float part = 0.f;
        for (int i = 32 * b; i < 32 * b + 32; ++i) part += qs[i] * value<FP8>(a.k, at + i);
        s += FP8 ? ldexpf(part, (int)((ex >> (8 * b)) & 255) - 127) : part;
      }
    }
    float mx = s;
    for (int x = 1; x < 64; x <<= 1) mx = fmaxf(mx, __shfl_xor(mx, x, 64));
    const float mn = fmaxf(m, mx), ref = mn == -INFINITY ? 0.f : mn;
    const float alpha = exp2_fast((m - ref) * a.c);
    const float p = exp2_fast((s - ref) * a.c);
    float sum = p;
    for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x, 64);
    m = mn;
    l = l * alpha + sum;
    ps[lane] = p;
    __syncthreads();
    for (int i = 0; i < DH / 64; ++i) acc[i] *= alpha;
    for (int jj = 0; jj < 64; ++jj) {
      const int64_t row = __shfl(at, jj, 64);
      if (row < 0) continue;
      for (int i = 0; i < DH / 64; ++i) acc[i] += ps[jj] * value<FP8>(a.v, row + lane + 64 * i);
    }
    __syncthreads();
  }
  const float inv = l > 0.f ? (FP8 ? a.v_scale : 1.f) / l : 0.f;
  for (int i = 0; i < DH / 64; ++i)
    static_cast<bf16*>(a.o)[t * a.o_ts + h * DH + lane + 64 * i] = (bf16)(acc[i] * inv);
}

}  // namespace

hipError_t launch_attn_ragged(const RaggedArgs& a, void*, hipStream_t s) {
  const dim3 grid((unsigned)a.T, (unsigned)a.Hq), block(64);
  if (a.table) {
    if (a.k_exp) hipLaunchKernelGGL((attn_ragged_kernel<128, true, true>), grid, block, 0, s, a);
    else if (a.Dh == 128) hipLaunchKernelGGL((attn_ragged_kernel<128, true, false>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((attn_ragged_kernel<64, true, false>), grid, block, 0, s, a);
  } else {
    if (a.Dh == 128) hipLaunchKernelGGL((attn_ragged_kernel<128, false, false>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((attn_ragged_kernel<64, false, false>), grid, block, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace wam
