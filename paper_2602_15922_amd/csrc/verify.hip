// Verification of trees of drafted tokens against the target's probabilities, from given random numbers.
//
// At a node the target's distribution is P and the draft's Q.  The node's children are tried in their order: token x is taken
// if u s Q(x) < R(x), where R = P and s = 1 at first; after a rejection what is left of the target is
// max(R - s Q, 0), its sum the new s.  With R_i = max(P_i - c Q_i, 0) that is max(P_i - (c + s) Q_i, 0) again, so c alone
// says what is left, and only its sum takes a pass over the vocabulary.  (Drafts that were chosen, not drawn: Q is a one at
// the child's token, so R is P without the tokens rejected so far, and s, without a pass, one minus those.)  The token after
// the last node taken is drawn from R: the first one whose sum up to it exceeds u' times the whole.
//
// Bound by reading the vocabulary's rows at the last node, and before that by the chain lengths -> nodes -> probabilities of
// their tokens.  Every workgroup of a request walks its tree by itself (in each wavefront: 64 nodes at a time by
// ballots) to the place where a sum is needed, then sums 4096 entries; the next launch joins the sums and walks on.  All in
// 64 bits: what the inputs say in 32 is exact there, and a product or difference of them is off by 2^-53.
#include "common.h"
#include "kernels.h"

namespace wam {
namespace {

constexpr int MAX_NODES = WAM_TREE_MAX_NODES;
constexpr int SLICE = VERIFY_SLICE;

WAM_DEV int fdiv(const FastDiv& f, int n) {
  return f.d == 1 ? n : (int)(__umulhi((uint32_t)n, f.mul) >> f.shift);
}
WAM_DEV int clampi(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }

struct Tree {
  int q0, n;  // first row, nodes that are looked at
  int rows;   // nodes
};
WAM_DEV Tree tree_of(const VerifyArgs& a, int r) {
  const int q0 = a.q_start[r], q1 = a.q_start[r + 1], n = a.q_len ? a.q_len[r] : INT32_MAX;
  const int end = clampi(q1, 0, a.d.T), room = q0 < 0 || q0 >= end ? 0 : end - q0;
  Tree t;
  t.q0 = q0;
  t.rows = clampi(n, 0, room);
  t.n = t.rows < MAX_NODES ? t.rows : MAX_NODES;
  return t;
}

// the nodes of a request in LDS: parent (-1: never tried), token, random number, the probabilities of the token at the parent
struct Nodes {
  int parent[MAX_NODES], token[MAX_NODES];
  float u[MAX_NODES], p[MAX_NODES], q[MAX_NODES];
};
// Their probabilities come from the rows, from the workspace, where the first launch kept them (one trip to memory less), or
// are not needed (the walk has ended).
enum Chances { ROWS, KEPT, NONE };
template <bool DRAWN, int NT, int FROM>
WAM_DEV void load_nodes(const VerifyArgs& a, const Tree& t, Nodes& x, float2* keep) {
  for (int i = threadIdx.x; i < t.n; i += NT) {
    const int par = a.parent[t.q0 + i], tok = a.tokens[t.q0 + i];
    const float u = a.u[t.q0 + i];
    float2 pq = {0.f, 0.f};
    if (FROM == KEPT) pq = a.nodes[t.q0 + i];
    const bool ok = i > 0 && (unsigned)par < (unsigned)i && (unsigned)tok < (unsigned)a.d.V;
    if (FROM == ROWS && ok) {
      pq.x = a.p[(int64_t)(t.q0 + par) * a.d.p_stride + tok];
      if (DRAWN) pq.y = fmaxf(a.q[(int64_t)(t.q0 + par) * a.d.q_stride + tok], 0.f);
    }
    x.parent[i] = ok ? par : -1;
    x.token[i] = tok;
    x.u[i] = u;
    x.p[i] = pq.x;
    if (DRAWN) x.q[i] = pq.y;
    if (keep) keep[t.q0 + i] = pq;
  }
}

// what is left of a probability (NaN and negative ones of either count as 0)
WAM_DEV double left_of(float p, float q, double c) {
#pragma clang fp contract(off)
  const double x = (double)p - c * (double)fmaxf(q, 0.f);
  return x > 0.0 ? x : 0.0;
}
WAM_DEV double left_of(float p) { return p > 0.f ? (double)p : 0.0; }

// first child of `cur` from node i on, or n (the same in all lanes)
WAM_DEV int next_child(const Nodes& x, int n, int cur, int i) {
  const int lane = threadIdx.x & 63;
  for (int b = i & ~63; b < n; b += 64) {
    const int k = b + lane;
    const uint64_t hit = __ballot(k < n && k >= i && x.parent[k] == cur);
    if (hit) return b + __ffsll((unsigned long long)hit) - 1;
  }
  return n;
}

// whether the token of child i of `cur` is an earlier child's (the same in all lanes)
WAM_DEV bool tried(const Nodes& x, int cur, int i) {
  const int lane = threadIdx.x & 63, token = x.token[i];
  bool hit = false;
#pragma unroll 4
  for (int k = lane; k - lane < i; k += 64) hit |= k < i && x.parent[k] == cur && x.token[k] == token;
  return __any(hit);
}

// The walk from a state whose s is known, to the next sum that it needs or to its end.  Taken nodes go to `path` (may be
// NULL) from entry `count` on.
template <bool DRAWN>
WAM_DEV void walk(const Nodes& x, int n, VerifyState& st, int32_t* path) {
#pragma clang fp contract(off)
  for (;;) {
    const int i = next_child(x, n, st.cur, st.next);
    if (i >= n) break;
    const double r = DRAWN ? left_of(x.p[i], x.q[i], st.c) : left_of(x.p[i]);
    const double chance = !DRAWN && tried(x, st.cur, i) ? 0.0 : r;  // (0: a token that was rejected here before)
    const bool take = (double)x.u[i] * st.s * (DRAWN ? (double)x.q[i] : 1.0) < chance;
    st.next = i + 1;
    if (take) {
      if (path && (threadIdx.x & 63) == 0) path[st.count] = i;
      st.cur = i;
      st.count += 1;
      st.c = 0.0;
      st.s = 1.0;
    } else if (DRAWN) {
      st.c += st.s;
      if (next_child(x, n, st.cur, st.next) < n) return;
      break;
    } else {
      st.s -= chance;
    }
  }
  st.done = 1;
}

WAM_DEV double wave_sum_f64(double v) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) v += __shfl_xor(v, s, 64);
  return v;
}
WAM_DEV double wave_scan_f64(double v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const double y = __shfl_up(v, s, 64);
    if (lane >= s) v += y;
  }
  return v;
}

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

// 4 entries of a row from v on; those from V on as 0
WAM_DEV f32x4 load4(const float* row, int v, int V) {
  if (v + 4 <= V) {
    const f32x4u x = *reinterpret_cast<const f32x4u*>(row + v);
    return f32x4{x[0], x[1], x[2], x[3]};
  }
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (v + e < V) y[e] = row[v + e];
  return y;
}

// What is left of 4 entries with probabilities p and q.  gone: a bit for each entry of the slice, set where its token was
// rejected (NULL: none); at: the first one's place in the slice.
template <bool DRAWN>
WAM_DEV void left4(f32x4 p, f32x4 q, double c, const uint32_t* gone, int at, double* y) {
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = DRAWN ? left_of(p[e], q[e], c) : left_of(p[e]);
  if (!DRAWN && gone) {
    const uint32_t bits = gone[at >> 5] >> (at & 31);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (bits >> e & 1) y[e] = 0.0;
  }
}
// 4 entries of p and q (0 where nothing of it is taken away) at node row from v on
template <bool DRAWN>
WAM_DEV void load_pq(const VerifyArgs& a, int64_t row, int v, bool taken, f32x4& p, f32x4& q) {
  p = load4(a.p + row * a.d.p_stride, v, a.d.V);
  q = f32x4{0.f, 0.f, 0.f, 0.f};
  if (DRAWN && taken) q = load4(a.q + row * a.d.q_stride, v, a.d.V);
}

// marks the slice's tokens that were rejected at node st.cur (every thread of the workgroup, barriers inside)
template <int NT>
WAM_DEV void mark_gone(const Nodes& x, int n, const VerifyState& st, int v0, uint32_t* gone) {
  for (int i = threadIdx.x; i < SLICE / 32; i += NT) gone[i] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < n && i < st.next; i += NT) {
    const int v = x.token[i] - v0;
    if (x.parent[i] == st.cur && (unsigned)v < (unsigned)SLICE) atomicOr(&gone[v >> 5], 1u << (v & 31));
  }
  __syncthreads();
}

WAM_DEV VerifyState first_state() { return VerifyState{0.0, 1.0, 0, 1, 1, 0, 0, {0, 0, 0}}; }

// the sum of a request's slices, in a fixed order (the same in every lane)
WAM_DEV double join(const double* sums, int slices) {
  double s = 0.0;
  for (int i = threadIdx.x & 63; i < slices; i += 64) s += sums[i];
  return wave_sum_f64(s);
}

// One workgroup per request and slice: walks to the next sum, and sums its slice.  In a later round the rows of the node
// where the last one stopped are on their way while it walks (it stops there again where the next child is rejected too).
constexpr int SUM_NT = 256, SUM_PER = SLICE / (4 * SUM_NT);
template <bool DRAWN, bool LATER>
__global__ __launch_bounds__(SUM_NT) void verify_sum_kernel(const VerifyArgs a, int round) {
  __shared__ Nodes x;
  __shared__ uint32_t gone[SLICE / 32];
  __shared__ double part[SUM_NT];
  const int r = fdiv(a.by_slices, blockIdx.x), slice = blockIdx.x - r * a.slices, tid = threadIdx.x, w = tid >> 6;
  const int v0 = slice * SLICE;
  VerifyState st = first_state();
  double s = 1.0;
  if (LATER) {
    st = a.state[(int64_t)(round - 1) * a.d.R + r];
    s = join(a.sums + ((int64_t)(round - 1) * a.d.R + r) * a.slices, a.slices);
  }
  const Tree t = tree_of(a, r);
  if (t.n == 0) return;
  if (LATER && st.done) {
    if (slice == 0 && tid == 0) a.state[(int64_t)round * a.d.R + r] = st;
    return;
  }
  st.s = s;
  f32x4 p[SUM_PER], q[SUM_PER];
  const auto load = [&] {
#pragma unroll
    for (int k = 0; k < SUM_PER; ++k) load_pq<DRAWN>(a, t.q0 + st.cur, v0 + 4 * (k * SUM_NT + tid), st.c != 0.0, p[k], q[k]);
  };
  const int was = st.cur;
  if (LATER) load();  // (c > 0: it stopped at a rejection)
  load_nodes<DRAWN, SUM_NT, LATER ? KEPT : ROWS>(a, t, x, DRAWN && !LATER && slice == 0 ? a.nodes : nullptr);
  __syncthreads();
  int32_t* path = slice == 0 && w == 0 ? a.path + t.q0 : nullptr;
  if (path && !LATER && tid == 0) path[0] = 0;
  walk<DRAWN>(x, t.n, st, path);
  st.round = round;
  if (slice == 0 && tid == 0) a.state[(int64_t)round * a.d.R + r] = st;
  if (!LATER || st.cur != was) load();
  const bool some = !DRAWN && st.next > 1;
  if (some) mark_gone<SUM_NT>(x, t.n, st, v0, gone);
  double sum = 0.0;
#pragma unroll
  for (int k = 0; k < SUM_PER; ++k) {
    double y[4];
    left4<DRAWN>(p[k], q[k], st.c, some ? gone : nullptr, 4 * (k * SUM_NT + tid), y);
    sum += (y[0] + y[1]) + (y[2] + y[3]);
  }
  part[tid] = sum;
  __syncthreads();
  if (w > 0) return;
  sum = wave_sum_f64((part[tid] + part[tid + 64]) + (part[tid + 128] + part[tid + 192]));
  if (tid == 0) a.sums[((int64_t)round * a.d.R + r) * a.slices + slice] = sum;
}

// One workgroup per request: ends the walk (passes that are still needed are its own), and draws the last token.  Its
// chain of loads is what takes the time, so it is small where no pass can be left.
template <bool DRAWN>
__global__ __launch_bounds__(DRAWN ? 1024 : 256) void verify_end_kernel(const VerifyArgs a) {
  constexpr int END_NT = DRAWN ? 1024 : 256, QUADS = SLICE / (4 * END_NT);  // fours of a slice's entries per thread
  __shared__ Nodes x;
  __shared__ uint32_t gone[SLICE / 32];
  __shared__ double part[END_NT / 64], own[WAM_VERIFY_MAX_VOCAB / SLICE];
  __shared__ int found, last_of[END_NT / 64];
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  VerifyState st = a.state[(int64_t)(a.rounds - 1) * a.d.R + r];  // (of a request without rows: anything)
  const float u_next = a.u_next[r];
  const Tree t = tree_of(a, r);
  if (t.n == 0) {
    if (tid == 0) {
      a.n_path[r] = 0;
      a.next_token[r] = -1;
      if (a.cache_len) a.cache_len[r] = a.kv_len[r] - t.rows;
    }
    return;
  }
  const double* sums = a.sums + ((int64_t)st.round * a.d.R + r) * a.slices;
  if (!DRAWN) load_nodes<DRAWN, END_NT, NONE>(a, t, x, nullptr);
  else if (!st.done) load_nodes<DRAWN, END_NT, KEPT>(a, t, x, nullptr);
  // the sums of all slices, a wavefront for each, in the order of verify_sum_kernel (s[j]: what a lane of its wavefront j adds
  // up), so that it does not matter in which of the two a pass is made
  const auto sum_all = [&](bool whole_p) {
    for (int i = w; i < a.slices; i += END_NT / 64) {
      double s[4] = {0.0, 0.0, 0.0, 0.0};
      static_assert(SUM_NT == 4 * 64, "four wavefronts");
#pragma unroll 2
      for (int k = 0; k < SUM_PER; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          double y[4];
          f32x4 p, q;
          load_pq<DRAWN>(a, t.q0 + st.cur, i * SLICE + 4 * (k * SUM_NT + 64 * j + lane), !whole_p && st.c != 0.0, p, q);
          left4<DRAWN>(p, q, st.c, nullptr, 0, y);
          s[j] += (y[0] + y[1]) + (y[2] + y[3]);
        }
      const double sum = wave_sum_f64((s[0] + s[1]) + (s[2] + s[3]));
      if (lane == 0) own[i] = sum;
    }
    __syncthreads();
    sums = own;
  };
  __syncthreads();
  while (!st.done) {
    st.s = join(sums, a.slices);
    walk<DRAWN>(x, t.n, st, w == 0 ? a.path + t.q0 : nullptr);
    __syncthreads();  // (everybody has joined)
    sum_all(false);
  }
  double total = join(sums, a.slices);
  bool whole_p = false;  // nothing is left: the token is drawn from the target's probabilities themselves
  if (!(total > 0.0)) {
    whole_p = true;
    __syncthreads();
    sum_all(true);
    total = join(sums, a.slices);
  }
  // the first slice whose sum up to its end exceeds the threshold, or the last with any; by the first wavefront's lanes
  const double goal = (double)u_next * total;
  int slice = -1, some = -1;
  double before = 0.0, at = 0.0;
  for (int b = 0; b < a.slices && slice < 0; b += 64) {
    const double s = b + lane < a.slices ? sums[b + lane] : 0.0, incl = wave_scan_f64(s) + before;
    const uint64_t over = __ballot(incl > goal && s > 0.0), any = __ballot(s > 0.0);
    const int hit = over ? __ffsll((unsigned long long)over) - 1 : (any ? 63 - __clzll((long long)any) : -1);
    if (hit >= 0) {
      (over ? slice : some) = b + hit;
      at = __shfl(incl - s, hit, 64);
    }
    before = __shfl(incl, 63, 64);
  }
  if (slice < 0) slice = some;
  int token = -1;
  if (slice >= 0) {
    const int v0 = slice * SLICE;
    const bool marked = !DRAWN && !whole_p && st.next > 1;
    if (marked) mark_gone<END_NT>(x, t.n, st, v0, gone);
    double y[4 * QUADS], mine = 0.0;
    f32x4 p[QUADS], q[QUADS];
#pragma unroll
    for (int k = 0; k < QUADS; ++k) load_pq<DRAWN>(a, t.q0 + st.cur, v0 + 4 * (QUADS * tid + k), !whole_p && st.c != 0.0, p[k], q[k]);
#pragma unroll
    for (int k = 0; k < QUADS; ++k) {
      left4<DRAWN>(p[k], q[k], st.c, marked ? gone : nullptr, 4 * (QUADS * tid + k), y + 4 * k);
      mine += (y[4 * k] + y[4 * k + 1]) + (y[4 * k + 2] + y[4 * k + 3]);
    }
    const double incl = wave_scan_f64(mine);
    if (tid == 0) found = INT32_MAX;
    if (lane == 63) part[w] = incl;
    __syncthreads();
    double sum = at + (incl - mine);
    for (int k = 0; k < w; ++k) sum += part[k];
    int first = INT32_MAX, last = -1;
#pragma unroll
    for (int e = 0; e < 4 * QUADS; ++e) {
      sum += y[e];
      if (y[e] > 0.0) {
        last = v0 + 4 * QUADS * tid + e;
        if (sum > goal && first == INT32_MAX) first = last;
      }
    }
    if (first != INT32_MAX) atomicMin(&found, first);
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int o = __shfl_xor(last, s, 64);
      last = o > last ? o : last;
    }
    if (lane == 0) last_of[w] = last;
    __syncthreads();
    token = found;
    if (token == INT32_MAX) {
      token = -1;
      for (int k = 0; k < END_NT / 64; ++k) token = last_of[k] > token ? last_of[k] : token;
    }
  }
  if (tid == 0) {
    a.n_path[r] = st.count;
    a.next_token[r] = token;
    if (a.cache_len) a.cache_len[r] = a.kv_len[r] - t.rows + st.count;
  }
}

template <bool DRAWN>
hipError_t launch(const VerifyArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)a.d.R * a.slices)), block(SUM_NT);
  for (int i = 0; i < a.rounds; ++i) {
    if (i == 0) hipLaunchKernelGGL((verify_sum_kernel<DRAWN, false>), grid, block, 0, s, a, i);
    else if (DRAWN) hipLaunchKernelGGL((verify_sum_kernel<true, true>), grid, block, 0, s, a, i);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(verify_end_kernel<DRAWN>, dim3((unsigned)a.d.R), dim3(DRAWN ? 1024 : 256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_verify_tree(const VerifyArgs& a, hipStream_t s) {
  return a.d.drawn ? launch<true>(a, s) : launch<false>(a, s);
}

}  // namespace wam
