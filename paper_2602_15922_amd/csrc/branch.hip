// Requests that branch over a paged KV cache: block tables of forks, the copies of their last pages, the pages that no
// request names any more, and the rows of a chosen branch moved together.
#include "common.h"
#include "kernels.h"

namespace wam {
namespace {

typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));

WAM_DEV int fdiv(const FastDiv& f, int n) {
  return f.d == 1 ? n : (int)(__umulhi((uint32_t)n, f.mul) >> f.shift);
}
WAM_DEV int clampi(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }

// inclusive sum over the wavefront
WAM_DEV int wave_scan(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const int y = __shfl_up(v, s, 64);
    if (lane >= s) v += y;
  }
  return v;
}

// ---------------------------------------------------------------------------------
// Fork.  Every workgroup finds in LDS which forks hold (the first to name a destination, which holds no page) and how many
// of those before each need a page of their own; so one launch does it and none waits for another.  Rows that are
// written belong to requests without pages and rows that are read to requests with some, so no order matters.
// ---------------------------------------------------------------------------------
constexpr int FORK_NT = 256;

struct Fork {
  int src, dst, first, whole, tail;
};

template <int E>  // forks per thread: N <= 256 E
__global__ __launch_bounds__(FORK_NT) void page_fork_kernel(const PageForkArgs a, int chunks) {
  __shared__ int owner[WAM_PLAN_MAX_REQUESTS], at[E * FORK_NT], wave[FORK_NT / 64], bad_of[FORK_NT / 64];
  const int R = a.d.R, N = a.d.N, ps = a.d.page_size, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int nf_in = a.n_free[0], nf = clampi(nf_in, 0, a.d.n_pages);
  for (int r = tid; r < R; r += FORK_NT) owner[r] = INT32_MAX;
  __syncthreads();
  for (int i = tid; i < N; i += FORK_NT)
    if ((unsigned)a.dst[i] < (unsigned)R) atomicMin(&owner[a.dst[i]], i);
  __syncthreads();
  const auto held = [&](int r) { return clampi(a.held[r], 0, a.d.max_pages); };
  // whether fork i holds
  const auto get = [&](int i, Fork& f) {
    f.src = a.src[i];
    f.dst = a.dst[i];
    f.first = a.first ? a.first[i] : 0;
    const int len = a.len[i];
    if ((unsigned)f.src >= (unsigned)R || (unsigned)f.dst >= (unsigned)R || f.first < 0 || len < 0) return false;
    if (owner[f.dst] != i || held(f.dst) != 0) return false;
    if ((int64_t)f.first * ps + len > (int64_t)held(f.src) * ps) return false;
    f.whole = fdiv(a.ps, len);
    f.tail = len - f.whole * ps;
    return true;
  };
  int tails = 0, bad = 0;
#pragma unroll 1
  for (int e = 0; e < E; ++e) {
    const int i = tid * E + e;
    Fork f;
    const bool ok = i < N && get(i, f);
    bad += i < N && !ok;
    if (i < N) at[i] = ok ? tails : -1;
    tails += ok && f.tail > 0;
  }
  const int incl = wave_scan(tails);
  const int bads = wave_scan(bad);
  if (lane == 63) {
    wave[w] = incl;
    bad_of[w] = bads;
  }
  __syncthreads();
  int before = incl - tails, all = 0;
#pragma unroll
  for (int k = 0; k < FORK_NT / 64; ++k) {
    if (k < w) before += wave[k];
    all += wave[k];
  }
#pragma unroll 1
  for (int e = 0; e < E; ++e) {
    const int i = tid * E + e;
    if (i < N && at[i] >= 0) at[i] += before;
  }
  __syncthreads();

  if (blockIdx.x == gridDim.x - 1) {
    int wrong = 0;
    for (int r = tid; r < R; r += FORK_NT) {
      const int h = held(r), i = owner[r];
      wrong += h != a.held[r];
      Fork f;
      a.held_out[r] = i < N && at[i] >= 0 && get(i, f) ? f.whole + (f.tail > 0 && at[i] < nf) : h;
    }
    __syncthreads();
    const int w2 = wave_scan(wrong);
    if (lane == 63) wave[w] = w2;
    __syncthreads();
    if (tid == 0) {
      a.n_free_out[0] = nf > all ? nf - all : 0;
      a.status[0] = all > nf ? all - nf : 0;
      a.status[1] = bad_of[0] + bad_of[1] + bad_of[2] + bad_of[3] + wave[0] + wave[1] + wave[2] + wave[3] + (nf != nf_in);
    }
    return;
  }

  // `chunks` items of 256 entries for each fork
  for (int64_t item = blockIdx.x; item < (int64_t)N * chunks; item += gridDim.x - 1) {
    const int i = (int)(item / chunks), part = (int)(item - (int64_t)i * chunks), j = part * FORK_NT + tid;
    Fork f;
    const bool ok = at[i] >= 0 && get(i, f);
    int page = -1, last = -1;
    if (ok) {
      const int32_t* from = a.table + (int64_t)f.src * a.d.table_stride + f.first;
      int32_t* to = a.table + (int64_t)f.dst * a.d.table_stride;
      if (j < f.whole) to[j] = from[j];
      if (part == 0 && tid == 0 && f.tail > 0) {
        if (at[i] < nf) {
          page = a.free_list[nf - 1 - at[i]];
          last = from[f.whole];
        }
        to[f.whole] = page;
      }
    }
    if (part == 0 && tid == 0) {
      const bool copied = ok && f.tail > 0 && at[i] < nf;
      a.copies[3 * i] = copied ? last : -1;
      a.copies[3 * i + 1] = copied ? page : -1;
      a.copies[3 * i + 2] = copied ? f.tail : 0;
    }
  }
}

// ---------------------------------------------------------------------------------
// Copies of pages' first rows: 16-byte chunks of K and V in the order of the rows, four of each per thread on their way.
// ---------------------------------------------------------------------------------
constexpr int COPY_NT = 256, COPY_PER = 4;

__global__ __launch_bounds__(COPY_NT) void page_copy_kernel(const PageCopyArgs a) {
  const int i = fdiv(a.by_blocks, blockIdx.x), block = blockIdx.x - i * (int)a.by_blocks.d;
  const int src = a.copies[3 * (int64_t)i], dst = a.copies[3 * (int64_t)i + 1], rows = clampi(a.copies[3 * (int64_t)i + 2], 0, a.c.page_size);
  if ((unsigned)src >= (unsigned)a.c.n_pages || (unsigned)dst >= (unsigned)a.c.n_pages) return;
  const int EB = a.c.k_exp ? 1 : 2, cpr = a.c.Dh * EB / 16, per_row = (int)a.by_row.d, n = rows * per_row;
  u32x4v k[COPY_PER], v[COPY_PER];
  int64_t off[COPY_PER];
#pragma unroll
  for (int u = 0; u < COPY_PER; ++u) {
    const int x = (block * COPY_PER + u) * COPY_NT + threadIdx.x;
    off[u] = -1;
    if (x >= n) continue;
    const int tok = fdiv(a.by_row, x), rest = x - tok * per_row, head = rest / cpr, ch = rest - head * cpr;
    off[u] = (tok * a.c.tok_stride + head * a.c.head_stride) * EB + 16 * ch;
    const int64_t at = (int64_t)src * a.c.page_stride * EB + off[u];
    k[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4v*>(static_cast<const char*>(a.c.k) + at));
    v[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4v*>(static_cast<const char*>(a.c.v) + at));
  }
#pragma unroll
  for (int u = 0; u < COPY_PER; ++u) {
    if (off[u] < 0) continue;
    const int64_t at = (int64_t)dst * a.c.page_stride * EB + off[u], from = (int64_t)src * a.c.page_stride * EB + off[u];
    *reinterpret_cast<u32x4v*>(static_cast<char*>(a.c.k) + at) = k[u];
    *reinterpret_cast<u32x4v*>(static_cast<char*>(a.c.v) + at) = v[u];
    // (a row of 128 codes has one word of exponents)
    if (a.c.k_exp && (off[u] & 127) == 0)
      *reinterpret_cast<uint32_t*>(static_cast<char*>(a.c.k_exp) + at / 32) =
          *reinterpret_cast<const uint32_t*>(static_cast<const char*>(a.c.k_exp) + from / 32);
  }
}

// ---------------------------------------------------------------------------------
// Collect.  Every workgroup marks the pages that the requests keep in a bit map in LDS (n_pages bits, at most 128 KB), a
// wavefront per row of the table; then it knows how many free pages lie below its share of the pool and lists its own.
// ---------------------------------------------------------------------------------
constexpr int COLLECT_NT = 1024;

WAM_DEV int kept_pages(const PageCollectArgs& a, int r, bool* bad) {
  const int c = a.cache_len[r], h = a.held[r], len = c < 0 ? 0 : c, held = clampi(h, 0, a.d.max_pages);
  *bad = c < 0 || held != h;
  const int full = fdiv(a.ps, len), need = full + (full * a.d.page_size < len);
  return need < held ? need : held;
}

template <int WORDS>  // n_pages <= 32 WORDS
__global__ __launch_bounds__(COLLECT_NT) void page_collect_kernel(const PageCollectArgs a) {
  __shared__ uint32_t used[WORDS];
  __shared__ int wave[COLLECT_NT / 64], miss[COLLECT_NT / 64];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, n_pages = a.d.n_pages, words = (n_pages + 31) >> 5;
  for (int i = tid; i < words; i += COLLECT_NT) used[i] = 0;
  __syncthreads();
  int missing = 0, wrong = 0;
  for (int r = w; r < a.d.R; r += COLLECT_NT / 64) {
    bool bad;
    const int kept = kept_pages(a, r, &bad);
    const int32_t* row = a.table + (int64_t)r * a.d.table_stride;
    for (int j = lane; j < kept; j += 64) {
      const int p = row[j];
      if ((unsigned)p < (unsigned)n_pages) atomicOr(&used[p >> 5], 1u << (p & 31));
      else ++missing;
    }
    if (lane == 0) {
      wrong += bad;
      if (blockIdx.x == 0) a.held_out[r] = kept;
    }
  }
  const int m = wave_scan(missing), b = wave_scan(wrong);
  if (lane == 63) {
    wave[w] = b;
    miss[w] = m;
  }
  __syncthreads();
  if (blockIdx.x == 0 && tid == 0) {
    int x = 0, y = 0;
    for (int k = 0; k < COLLECT_NT / 64; ++k) {
      x += miss[k];
      y += wave[k];
    }
    a.status[0] = x;
    a.status[1] = y;
  }
  __syncthreads();
  // free pages below a word: those of the words before
  const auto free_of = [&](int i) {
    const int left = n_pages - 32 * i;
    return ~used[i] & (left >= 32 ? ~0u : (1u << left) - 1);
  };
  const int share = (words + gridDim.x - 1) / gridDim.x, lo = blockIdx.x * share < words ? blockIdx.x * share : words,
            hi = lo + share < words ? lo + share : words;
  int below = 0, all = 0;
  for (int i = tid; i < words; i += COLLECT_NT) {
    const int c = __popc(free_of(i));
    all += c;
    if (i < lo) below += c;
  }
  below = wave_scan(below);
  all = wave_scan(all);
  if (lane == 63) {
    wave[w] = below;
    miss[w] = all;
  }
  __syncthreads();
  int start = 0, total = 0;
  for (int k = 0; k < COLLECT_NT / 64; ++k) {
    start += wave[k];
    total += miss[k];
  }
  if (blockIdx.x == 0 && tid == 0) a.n_free_out[0] = total;
  // this share, 1024 words at a time
  for (int i0 = lo; i0 < hi; i0 += COLLECT_NT) {
    const int i = i0 + tid;
    uint32_t f = i < hi ? free_of(i) : 0;
    const int c = __popc(f), incl = wave_scan(c);
    __syncthreads();
    if (lane == 63) wave[w] = incl;
    __syncthreads();
    int at = start + incl - c;
    for (int k = 0; k < COLLECT_NT / 64; ++k) {
      if (k < w) at += wave[k];
      start += wave[k];
    }
    while (f) {
      a.free_list[at++] = 32 * i + __ffs(f) - 1;
      f &= f - 1;
    }
  }
}

// ---------------------------------------------------------------------------------
// Compact.  A workgroup owns one head of K or V of a request.  A row moves down or stays (the kept rows ascend), so what a
// group of rows overwrites has been read by then: by an earlier group, or by this one, whose loads end before its stores.
// ---------------------------------------------------------------------------------
constexpr int MOVE_NT = 256, MOVE_PER = 8;

template <int CPR>  // 16-byte chunks of a row
__global__ __launch_bounds__(MOVE_NT) void cache_compact_kernel(const CacheCompactArgs a) {
  constexpr int RPP = MOVE_NT / CPR;  // rows at once
  const int rv = fdiv(a.by_heads, blockIdx.x), head = blockIdx.x - rv * (int)a.by_heads.d, r = rv >> 1;
  const bool is_v = rv & 1;
  const int q0 = a.q_start[r], q1 = a.q_start[r + 1], n_in = a.q_len ? a.q_len[r] : 0, keep_in = a.n_keep[r], kv = a.kv_len[r];
  const int end = clampi(q1, 0, a.T), room = q0 < 0 || q0 >= end ? 0 : end - q0, n = a.q_len ? clampi(n_in, 0, room) : room;
  const int m = clampi(keep_in, 0, n);
  const int64_t hist = (int64_t)kv - n, width = (int64_t)a.max_pages * a.c.page_size;
  const int EB = a.c.k_exp ? 1 : 2, ch = threadIdx.x % CPR;
  char* base = static_cast<char*>(is_v ? a.c.v : a.c.k);
  char* ex = is_v ? nullptr : static_cast<char*>(a.c.k_exp);
  const int32_t* row = a.table + r * a.table_stride;
  // byte offset of a position's row, -1 where there is none
  const auto place = [&](int64_t p) -> int64_t {
    if (p < 0 || p >= width) return -1;
    const int e = fdiv(a.ps, (int)p), pg = row[e];
    if ((unsigned)pg >= (unsigned)a.c.n_pages) return -1;
    return ((int64_t)pg * a.c.page_stride + ((int)p - e * a.c.page_size) * a.c.tok_stride + head * a.c.head_stride) * EB;
  };
  for (int i0 = 0; i0 < m; i0 += RPP * MOVE_PER) {
    u32x4v x[MOVE_PER];
    uint32_t e4[MOVE_PER];
    int64_t to[MOVE_PER];
#pragma unroll
    for (int u = 0; u < MOVE_PER; ++u) {
      const int i = i0 + u * RPP + threadIdx.x / CPR;
      to[u] = -1;
      if (i >= m) continue;
      const int k = a.keep[q0 + i];
      if ((unsigned)k >= (unsigned)n || k == i) continue;
      const int64_t from = place(hist + k);
      to[u] = from < 0 ? -1 : place(hist + i);
      if (to[u] < 0) continue;
      x[u] = *reinterpret_cast<const u32x4v*>(base + from + 16 * ch);
      if (ex && ch == 0) e4[u] = *reinterpret_cast<const uint32_t*>(ex + from / 32);
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < MOVE_PER; ++u) {
      if (to[u] < 0) continue;
      *reinterpret_cast<u32x4v*>(base + to[u] + 16 * ch) = x[u];
      if (ex && ch == 0) *reinterpret_cast<uint32_t*>(ex + to[u] / 32) = e4[u];
    }
    __syncthreads();  // (also for lists that do not ascend: the same result every time)
  }
}

}  // namespace

hipError_t launch_page_fork(const PageForkArgs& a, hipStream_t s) {
  const int chunks = a.d.max_pages < 1 ? 1 : (a.d.max_pages + FORK_NT - 1) / FORK_NT;
  const int64_t items = (int64_t)a.d.N * chunks;
  const dim3 grid((unsigned)((items < 1024 ? items : 1024) + 1)), block(FORK_NT);
  if (a.d.N <= FORK_NT) hipLaunchKernelGGL(page_fork_kernel<1>, grid, block, 0, s, a, chunks);
  else if (a.d.N <= 4 * FORK_NT) hipLaunchKernelGGL(page_fork_kernel<4>, grid, block, 0, s, a, chunks);
  else hipLaunchKernelGGL(page_fork_kernel<16>, grid, block, 0, s, a, chunks);
  return hipGetLastError();
}

hipError_t launch_page_copy(const PageCopyArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(page_copy_kernel, dim3((unsigned)(a.N * (int64_t)a.by_blocks.d)), dim3(COPY_NT), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_page_collect(const PageCollectArgs& a, hipStream_t s) {
  const int words = (a.d.n_pages + 31) / 32, groups = words < 64 ? 1 : (words / 64 < 64 ? words / 64 : 64);
  const dim3 grid((unsigned)groups), block(COLLECT_NT);
  static_assert(WAM_COLLECT_MAX_PAGES <= 32 * 32768, "bits of the map");
  if (words <= 1024) hipLaunchKernelGGL(page_collect_kernel<1024>, grid, block, 0, s, a);
  else if (words <= 8192) hipLaunchKernelGGL(page_collect_kernel<8192>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(page_collect_kernel<32768>, grid, block, 0, s, a);
  return hipGetLastError();
}

hipError_t launch_cache_compact(const CacheCompactArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(2 * (int64_t)a.R * a.c.Hkv)), block(MOVE_NT);
  if (a.c.Dh == 128 && !a.c.k_exp) hipLaunchKernelGGL(cache_compact_kernel<16>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(cache_compact_kernel<8>, grid, block, 0, s, a);  // 64 bf16 or 128 codes
  return hipGetLastError();
}

}  // namespace wam
