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
// written belong to requests without pages and rows that are read to requests with some, so no order matters.  Bound by
// latency (starts -> lengths -> table; medians): 8 forks of 198 pages 4.1 us, 256 of up to 63 pages 5.8 (3.9 and 5.5 without the
// look at the last page's entry, which an absent page needs).
// ---------------------------------------------------------------------------------
constexpr int FORK_NT = 256;

struct Fork {
  int src, dst, first, whole, tail;
  int last;    // the source's entry of the tail's page
  bool takes;  // it needs a page of its own: of an absent page there is nothing to copy, and its entry is shared
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
    f.last = f.tail > 0 ? a.table[f.src * a.d.table_stride + f.first + f.whole] : -1;  // (a source's row is not written)
    f.takes = (unsigned)f.last < (unsigned)a.d.n_pages;
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
    tails += ok && f.takes;
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
      a.held_out[r] = i < N && at[i] >= 0 && get(i, f) ? f.whole + (f.tail > 0 && (!f.takes || at[i] < nf)) : h;
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
    const bool some = ok && f.tail > 0 && at[i] < nf, copied = some && f.takes;
    const int top = some ? a.free_list[nf - 1 - at[i]] : -1, page = copied ? top : -1;  // (on its way with the tail's entry)
    if (ok) {
      const int32_t* from = a.table + (int64_t)f.src * a.d.table_stride + f.first;
      int32_t* to = a.table + (int64_t)f.dst * a.d.table_stride;
      if (j < f.whole) to[j] = from[j];
      if (part == 0 && tid == 0 && f.tail > 0) to[f.whole] = f.takes ? page : f.last;
    }
    if (part == 0 && tid == 0) {
      a.copies[3 * i] = copied ? f.last : -1;
      a.copies[3 * i + 1] = page;
      a.copies[3 * i + 2] = copied ? f.tail : 0;
    }
  }
}

// ---------------------------------------------------------------------------------
// Copies of pages' first rows: 16-byte chunks of K and V in the order of the rows, four of each per thread on their way.  Bound
// by memory: 256 copies of 0 to 127 rows, 16 heads of 128, 55.6 us for 247 MB (4.4 TB/s; a large copy reaches 4.85), of E4M3 33.7
// for 126 (3.7: the exponents are a second trip, behind the stores).
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
// Collect.  Every workgroup marks the pages that the requests keep in LDS, a byte each (plain stores: lanes that meet store
// the same), so it knows how many free pages lie below its share of the pool and lists its own; one launch does
// it and none waits for another.  Pools of more bytes than LDS has go by segments, from the first on.
// Bound by the instructions that one CU issues for all marks (16 wavefronts, 4 cycles each): so no lane is masked off, 8 rows' first 64
// entries are on their way at once and then a longer row's, 512 at a time.  That marks places past a row's end too, and the
// wavefronts have their rows by number, not by length: 1000 requests that keep 0 to 1000 pages, 80078 of 144700 together, are 204288
// places, 160 to 256 rounds of 64 to a wavefront.  They take 28 us; with lanes masked 40, a wavefront per row with atomic marks of a
// bit 44; 12 requests, 2224 pages 7.4.
// ---------------------------------------------------------------------------------
constexpr int COLLECT_NT = 1024, COLLECT_SMALL = 32 << 10, COLLECT_LARGE = 152 << 10;

WAM_DEV int kept_pages(const PageCollectArgs& a, int r, bool* bad) {
  const int c = a.cache_len[r], h = a.held[r], len = c < 0 ? 0 : c, held = clampi(h, 0, a.d.max_pages);
  *bad = c < 0 || held != h;
  const int full = fdiv(a.ps, len), need = full + (full * a.d.page_size < len);
  return need < held ? need : held;
}

// sum over the workgroup, the same in every thread (tmp: an int per wavefront; barriers inside)
WAM_DEV int block_sum(int v, int* tmp) {
  // (the wavefronts' sums: a lane each)
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) v += __shfl_xor(v, k, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
  __syncthreads();
  int sum = tmp[threadIdx.x & 15];
#pragma unroll
  for (int k = 1; k < 16; k <<= 1) sum += __shfl_xor(sum, k, 64);
  return sum;
}

template <int SEGMENT>  // pages whose marks fit at once, a multiple of 16
__global__ __launch_bounds__(COLLECT_NT) void page_collect_kernel(const PageCollectArgs a, int share) {
  constexpr int WAVES = COLLECT_NT / 64;
  __shared__ __attribute__((aligned(16))) uint8_t used[SEGMENT + 16];  // 1: kept (or past the pool)
  __shared__ int tmp[WAVES];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), n_pages = a.d.n_pages;
  const bool last = blockIdx.x == gridDim.x - 1;  // counts all pages, and the status
  const int lo = (int)blockIdx.x * share, hi = last || n_pages - lo < share ? n_pages : lo + share;
  const int mine = a.d.R > w ? (a.d.R - w + WAVES - 1) / WAVES : 0;  // rows w + 16 i: 64 at a time, a lane each
  int at = 0, total = 0, missing = 0, wrong = 0;                     // at: free pages below what is listed next
  for (int seg = 0; seg == 0 || seg < hi; seg += SEGMENT) {
    const int pages = n_pages - seg < SEGMENT ? n_pages - seg : SEGMENT, groups = (pages + 15) >> 4;
    const auto lengths = [&](int base) {
      const int i = base + lane, r = w + WAVES * i;
      if (i >= mine) return 0;
      bool bad;
      const int kept = kept_pages(a, r, &bad);
      if (last && seg == 0) {
        wrong += bad;
        a.held_out[r] = kept;
      }
      return kept;
    };
    int kept = lengths(0);
    for (int i = tid; i < groups; i += COLLECT_NT) {
      u32x4v z = {0, 0, 0, 0};
      if (16 * i + 16 > pages)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (16 * i + e >= pages) z[e >> 2] |= 1u << (8 * (e & 3));
      *reinterpret_cast<u32x4v*>(used + 16 * i) = z;
    }
    __syncthreads();
    // (no lane is masked: entries that count for nothing are read, inside their row, and marked past the pages)
    const auto mark = [&](int v, bool in) {
      const unsigned p = (unsigned)v - (unsigned)seg;
      used[in && p < (unsigned)pages ? p : SEGMENT] = 1;
      if (last && seg == 0) missing += in && (unsigned)v >= (unsigned)n_pages;
    };
    const int64_t step = WAVES * a.d.table_stride;
    const int32_t* row = a.table + w * a.d.table_stride;
    const int end = a.d.max_pages - 1;  // (>= 0 where anything is kept)
    for (int base = 0; base < mine; base += 64, row += 64 * step) {
      if (base > 0) kept = lengths(base);
      const uint64_t any = __ballot(kept > 0);
      // the first 64 entries of 8 rows at once
#pragma unroll 1
      for (int g = 0; g < 64 && any >> g; g += 8) {
        int v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = row[(any >> (g + u) & 1 ? (g + u) * step : 0) + (lane < end ? lane : end)];
#pragma unroll
        for (int u = 0; u < 8; ++u) mark(v[u], lane < __builtin_amdgcn_readlane(kept, g + u));
      }
      // then what longer rows have, 512 at once
      for (uint64_t more = __ballot(kept > 64); more; more &= more - 1) {
        const int i = __ffsll((unsigned long long)more) - 1, n = __builtin_amdgcn_readlane(kept, i);
        const int32_t* at = row + i * step;
#pragma unroll 1
        for (int j = 64 + lane; j - lane < n; j += 512) {
          int v[8];
#pragma unroll
          for (int u = 0; u < 8; ++u) v[u] = at[j + 64 * u < end ? j + 64 * u : end];
#pragma unroll
          for (int u = 0; u < 8; ++u) mark(v[u], j + 64 * u < n);
        }
      }
    }
    __syncthreads();
    // free pages of this segment below the share, and all of them
    int below = 0, all = 0;
    for (int i = tid; i < groups; i += COLLECT_NT) {
      const u32x4v x = *reinterpret_cast<const u32x4v*>(used + 16 * i);
      const int c = 16 - (__popc(x[0]) + __popc(x[1]) + __popc(x[2]) + __popc(x[3]));
      all += c;
      if (seg + 16 * i < lo) below += c;
    }
    at += block_sum(below, tmp);
    if (last) total += block_sum(all, tmp);
    // the share's pages of this segment, 16 of them a thread
    const int g1 = hi - seg < pages ? (hi - seg + 15) >> 4 : groups;
    for (int g0 = lo > seg ? (lo - seg) >> 4 : 0; g0 < g1; g0 += COLLECT_NT) {
      const int g = g0 + tid;
      u32x4v x = {~0u, ~0u, ~0u, ~0u};
      int c = 0;
      if (g < g1) {
        x = *reinterpret_cast<const u32x4v*>(used + 16 * g);
        c = 16 - (__popc(x[0]) + __popc(x[1]) + __popc(x[2]) + __popc(x[3]));
      }
      const int incl = wave_scan(c);
      __syncthreads();
      if (lane == 63) tmp[w] = incl;
      __syncthreads();
      const int sums = wave_scan(lane < WAVES ? tmp[lane] : 0);
      int to = at + incl - c + (w > 0 ? __builtin_amdgcn_readlane(sums, w > 0 ? w - 1 : 0) : 0);
      at += __builtin_amdgcn_readlane(sums, WAVES - 1);
      int page = seg + 16 * g;
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll 1
        for (uint32_t f = ~x[k] & 0x01010101u; f; f &= f - 1) a.free_list[to++] = page + 4 * k + (__ffs(f) >> 3);
    }
    __syncthreads();
  }
  if (last) {
    const int m = block_sum(missing, tmp), b = block_sum(wrong, tmp);
    if (tid == 0) {
      a.n_free_out[0] = total;
      a.status[0] = m;
      a.status[1] = b;
    }
  }
}

// ---------------------------------------------------------------------------------
// Compact.  A workgroup owns one head of K or V of a request.  Row i's new place lies below what it holds (others are left
// out), so a group of rows overwrites nothing that a later one reads, and its own loads end before its stores.
// Bound by memory where lists are long (a group of 128 rows of 256 bytes, 32 KB, is on its way while the one before is stored;
// the rows' places are looked up 1024 at a time), by the chain lengths -> numbers -> table -> row where they are short.  4 x 1576
// of 3152 rows, 40 heads: 67 us for 258 MB (3.8 TB/s; groups of 256 rows 69.5, heads in a row on one XCD 68, marked as used once
// 69.5); looked up as they are moved, nothing ahead, 166; of E4M3 33 for 131 MB.  16 paths of 2 to 6 rows, 8 heads 3.3 (median).
// ---------------------------------------------------------------------------------
constexpr int MOVE_NT = 256, MOVE_PER = 8, MOVE_ROWS = 1024;

template <int CPR>  // 16-byte chunks of a row
__global__ __launch_bounds__(MOVE_NT) void cache_compact_kernel(const CacheCompactArgs a) {
  constexpr int RPP = MOVE_NT / CPR, GROUP = RPP * MOVE_PER;  // rows at once
  __shared__ int64_t from[MOVE_ROWS], to[MOVE_ROWS];  // byte offsets, -1: the row does not move
  const int rv = fdiv(a.by_heads, blockIdx.x), head = blockIdx.x - rv * (int)a.by_heads.d, r = rv >> 1;
  const bool is_v = rv & 1;
  const int q0 = a.q_start[r], q1 = a.q_start[r + 1], n_in = a.q_len ? a.q_len[r] : 0, keep_in = a.n_keep[r], kv = a.kv_len[r];
  const int end = clampi(q1, 0, a.T), room = q0 < 0 || q0 >= end ? 0 : end - q0, n = a.q_len ? clampi(n_in, 0, room) : room;
  const int m = clampi(keep_in, 0, n);
  const int64_t hist = (int64_t)kv - n, width = (int64_t)a.max_pages * a.c.page_size;
  const int EB = a.c.k_exp ? 1 : 2, ch = threadIdx.x % CPR, sub = threadIdx.x / CPR;
  char* base = static_cast<char*>(is_v ? a.c.v : a.c.k);
  char* ex = is_v ? nullptr : static_cast<char*>(a.c.k_exp);
  const int32_t* row = a.table + r * a.table_stride;
  // the page entry of a position (-1 where there is none), and its row's byte offset
  const auto page = [&](int64_t p) { return p < 0 || p >= width ? -1 : row[fdiv(a.ps, (int)p)]; };
  const auto place = [&](int64_t p, int pg) -> int64_t {
    if ((unsigned)pg >= (unsigned)a.c.n_pages) return -1;
    const int in = (int)p - fdiv(a.ps, (int)p) * a.c.page_size;
    return ((int64_t)pg * a.c.page_stride + in * a.c.tok_stride + head * a.c.head_stride) * EB;
  };
  for (int s0 = 0; s0 < m; s0 += MOVE_ROWS) {
    const int rows = m - s0 < MOVE_ROWS ? m - s0 : MOVE_ROWS;
    for (int i = threadIdx.x; i < rows; i += MOVE_NT) {
      const int k = a.keep[q0 + s0 + i];
      const int pt = page(hist + s0 + i);
      const bool moves = k > s0 + i && k < n;
      const int pf = moves ? page(hist + k) : -1;
      const int64_t x = moves ? place(hist + k, pf) : -1, y = moves ? place(hist + s0 + i, pt) : -1;
      from[i] = x < 0 || y < 0 ? -1 : x;
      to[i] = y;
    }
    __syncthreads();
    u32x4v x[MOVE_PER];
    uint32_t e4[MOVE_PER];
    const auto load = [&](int i0) {
#pragma unroll
      for (int u = 0; u < MOVE_PER; ++u) {
        const int i = i0 + u * RPP + sub;
        if (i >= rows || from[i] < 0) continue;
        x[u] = *reinterpret_cast<const u32x4v*>(base + from[i] + 16 * ch);
        if (ex && ch == 0) e4[u] = *reinterpret_cast<const uint32_t*>(ex + from[i] / 32);
      }
    };
    load(0);
    for (int i0 = 0; i0 < rows; i0 += GROUP) {
      // every thread's rows have arrived before any is overwritten
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      u32x4v y[MOVE_PER];
      uint32_t f4[MOVE_PER];
#pragma unroll
      for (int u = 0; u < MOVE_PER; ++u) {
        y[u] = x[u];
        f4[u] = e4[u];
      }
      if (i0 + GROUP < rows) load(i0 + GROUP);  // (later rows: nothing that is stored now)
#pragma unroll
      for (int u = 0; u < MOVE_PER; ++u) {
        const int i = i0 + u * RPP + sub;
        if (i >= rows || from[i] < 0) continue;
        *reinterpret_cast<u32x4v*>(base + to[i] + 16 * ch) = y[u];
        if (ex && ch == 0) *reinterpret_cast<uint32_t*>(ex + to[i] / 32) = f4[u];
      }
    }
    __syncthreads();  // (the places are looked up anew)
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
  // shares of 4096 pages (16 bytes of marks for a quarter of the threads), more of a pool that 64 workgroups do not cover so
  const int n = a.d.n_pages, share = n <= 64 * 4096 ? 4096 : ((n + 63) / 64 + 15) / 16 * 16;
  const dim3 grid((unsigned)(n <= share ? 1 : (n + share - 1) / share)), block(COLLECT_NT);
  if (n <= COLLECT_SMALL) hipLaunchKernelGGL(page_collect_kernel<COLLECT_SMALL>, grid, block, 0, s, a, share);
  else hipLaunchKernelGGL(page_collect_kernel<COLLECT_LARGE>, grid, block, 0, s, a, share);
  return hipGetLastError();
}

hipError_t launch_cache_compact(const CacheCompactArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(2 * (int64_t)a.R * a.c.Hkv)), block(MOVE_NT);
  if (a.c.Dh == 128 && !a.c.k_exp) hipLaunchKernelGGL(cache_compact_kernel<16>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(cache_compact_kernel<8>, grid, block, 0, s, a);  // 64 bf16 or 128 codes
  return hipGetLastError();
}

}  // namespace wam
