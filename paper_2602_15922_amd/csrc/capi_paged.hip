// C ABI of the paged KV cache: argument checks and launches of the page plan, the rotary
// append, the ragged attentions, and the operators of requests that branch.
#include <cmath>
#include <limits>

#include "capi_check.h"
#include "kernels.h"

using namespace wam;

namespace {

wam_status need_ints(const void* p, const char* name) {
  if (!p) return fail(WAM_EINVAL, "%s is NULL", name);
  if (!al4(p)) return fail(WAM_EINVAL, "%s is not 4-byte aligned", name);
  return WAM_OK;
}
wam_status opt_ints(const void* p, const char* name) {
  if (p && !al4(p)) return fail(WAM_EINVAL, "%s is not 4-byte aligned", name);
  return WAM_OK;
}

wam_status check_heads(int32_t Hq, int32_t Hkv, int32_t Dh) {
  CHECK(Dh == 64 || Dh == 128, WAM_EUNSUPPORTED, "Dh=%d (supported: 64, 128)", Dh);
  CHECK(Hkv >= 1 && Hq >= 1 && Hq <= 4096 && Hkv <= 4096, WAM_EINVAL, "Hq=%d, Hkv=%d outside [1, 4096]", Hq, Hkv);
  return WAM_OK;
}

wam_status check_page_size(int32_t page_size, int32_t n_pages) {
  CHECK(page_size >= 16 && page_size % 16 == 0, WAM_EUNSUPPORTED, "page_size=%d must be a positive multiple of 16",
        page_size);
  CHECK(n_pages >= 0, WAM_EINVAL, "n_pages=%d is negative", n_pages);
  CHECK((int64_t)n_pages * page_size <= INT32_MAX, WAM_EUNSUPPORTED, "n_pages * page_size = %lld must stay below 2^31",
        (long long)n_pages * page_size);
  return WAM_OK;
}

wam_status check_cache(const wam_paged_cache& c) {
  TRY(check_heads(1, c.Hkv, c.Dh));
  TRY(check_page_size(c.page_size, c.n_pages));
  CHECK(!c.k_exp || c.Dh == 128, WAM_EUNSUPPORTED, "an FP8 cache needs Dh=128 (got %d)", c.Dh);
  CHECK(!c.k_exp || (std::isfinite(c.v_scale) && c.v_scale > 0.f), WAM_EINVAL,
        "v_scale=%g must be positive and finite", (double)c.v_scale);
  if (c.n_pages > 0) {
    TRY(need_ptr(c.k, "cache k"));
    TRY(need_ptr(c.v, "cache v"));
    TRY(opt_ints(c.k_exp, "cache k_exp"));
  }
  const int unit = c.k_exp ? 128 : 8, bytes = c.k_exp ? 1 : 2;
  CHECK(c.page_stride >= c.Dh && c.tok_stride >= c.Dh && c.head_stride >= c.Dh, WAM_EINVAL,
        "cache strides must be >= Dh=%d", c.Dh);
  CHECK(c.page_stride % unit == 0 && c.tok_stride % unit == 0 && c.head_stride % unit == 0, WAM_EINVAL,
        "cache strides must be multiples of %d", unit);
  CHECK(c.tok_stride <= INT32_MAX / bytes / c.page_size && c.head_stride <= INT32_MAX / bytes / c.Hkv &&
            (c.page_size * c.tok_stride + c.Hkv * c.head_stride) * bytes <= INT32_MAX,
        WAM_EUNSUPPORTED, "one page's rows must span less than 2^31 bytes");
  CHECK(c.page_stride <= INT64_MAX / 4 / (c.n_pages + 1), WAM_EINVAL, "page_stride overflows");
  return WAM_OK;
}

// sizes shared by the two attentions
wam_status check_ragged(int32_t R, int32_t T, int32_t Hq, int32_t Hkv, int32_t Dh, int32_t max_k) {
  TRY(check_heads(Hq, Hkv, Dh));
  CHECK(Hq % Hkv == 0, WAM_EINVAL, "Hq=%d must be a multiple of Hkv=%d", Hq, Hkv);
  CHECK(R >= 0 && T >= 0 && max_k >= 0, WAM_EINVAL, "negative size (R=%d T=%d longest=%d)", R, T, max_k);
  CHECK(max_k <= 1 << 30, WAM_EUNSUPPORTED, "the longest key axis %d exceeds 2^30", max_k);
  CHECK((int64_t)T * Hq <= INT32_MAX && ragged_tiles(R, T, Hq, Hkv, 16) * Hkv <= INT32_MAX / RAGGED_MAX_SPLITS,
        WAM_EUNSUPPORTED, "T * Hq and (R + T * Hq / Hkv / 16) * Hkv * 64 must stay below 2^31");
  return WAM_OK;
}
// (a launch's threads are counted in 32 bits)
wam_status check_launch(int64_t threads) {
  CHECK(threads <= UINT32_MAX, WAM_EUNSUPPORTED, "%lld threads: more than one launch has (2^32); split the call",
        (long long)threads);
  return WAM_OK;
}
wam_status check_rows(const void* q, const void* o, int64_t q_ts, int64_t o_ts, int64_t hd) {
  TRY(need_ptr(q, "q"));
  TRY(need_ptr(o, "o"));
  CHECK(q_ts >= hd && o_ts >= hd && q_ts % 8 == 0 && o_ts % 8 == 0, WAM_EINVAL,
        "q and o token strides must be multiples of 8, >= Hq*Dh=%lld", (long long)hd);
  return WAM_OK;
}
// the factor of the scores in the exponent of 2
float exp2_scale(float scale, int32_t Dh) {
  return (scale > 0.f ? scale : 1.0f / std::sqrt((float)Dh)) * 1.4426950408889634f;
}
wam_status check_scale(float scale, int32_t Dh) {
  CHECK(std::isfinite(scale) && std::isfinite(exp2_scale(scale, Dh)), WAM_EINVAL, "scale=%g (times log2(e)) must be finite",
        (double)scale);
  return WAM_OK;
}
// A buffer of a call: `rows` rows of `n` ints, `stride` apart.
struct Ints {
  const char* name;
  const int32_t* p;
  int64_t n, rows, stride;
  bool written;
};
// (b has one row; both are 4-byte aligned, so whole ints count)
bool overlap(const Ints& a, const Ints& b) {
  if (!a.p || !b.p || a.n <= 0 || a.rows <= 0 || b.n <= 0) return false;
  const int64_t d = ((int64_t)reinterpret_cast<uintptr_t>(b.p) - (int64_t)reinterpret_cast<uintptr_t>(a.p)) / 4;
  // the first of a's rows that ends past b's first int
  const int64_t r = d < 0 ? 0 : a.rows == 1 ? d >= a.n : d / a.stride + (d % a.stride >= a.n);
  return r < a.rows && r * a.stride < d + b.n;
}
// a table of R rows, and R and the pool's sizes as the page plan takes them
wam_status check_table(int32_t R, int32_t max_pages, int64_t table_stride, const void* table) {
  CHECK(R >= 0 && max_pages >= 0, WAM_EINVAL, "negative size (R=%d max_pages=%d)", R, max_pages);
  CHECK((int64_t)R * max_pages <= INT32_MAX, WAM_EUNSUPPORTED, "R * max_pages must stay below 2^31");
  CHECK(table_stride >= max_pages && table_stride <= INT64_MAX / 8 / ((int64_t)R + 1), WAM_EINVAL,
        "table_stride=%lld must be >= max_pages=%d", (long long)table_stride, max_pages);
  if (R > 0 && max_pages > 0) TRY(need_ints(table, "block_table"));
  return WAM_OK;
}
template <size_t N>
wam_status check_apart(const Ints (&all)[N]) {
  for (const Ints& x : all)
    for (const Ints& y : all) {
      if (&x == &y || !x.written || (y.written && &y < &x)) continue;
      // (the one of several rows goes first)
      CHECK(!(y.rows > 1 ? overlap(y, x) : overlap(x, y)), WAM_EINVAL, "%s and %s overlap", x.name, y.name);
    }
  return WAM_OK;
}
wam_status check_ws(const void* ws, size_t have, size_t need) {
  CHECK(need == 0 || (ws && (reinterpret_cast<uintptr_t>(ws) & 255) == 0 && have >= need), WAM_EWORKSPACE,
        "workspace of %zu bytes (256-byte aligned) needed, got %zu", need, ws ? have : (size_t)0);
  return WAM_OK;
}

// attention over pages; a holds what says which keys a row sees
wam_status run_paged(const wam_attn_paged_desc& d, const wam_paged_cache& c, const void* q, const int32_t* block_table,
                     const int32_t* q_start, const int32_t* q_len, const int32_t* kv_len, void* o, void* ws, size_t ws_bytes,
                     RaggedArgs& a, RaggedPlan (*plan)(int64_t, int64_t, int64_t, int64_t, int64_t, int64_t),
                     hipError_t (*launch)(const RaggedArgs&, const RaggedPlan&, void*, hipStream_t),
                     hipStream_t stream) {
  TRY(check_cache(c));
  TRY(check_ragged(d.R, d.T, d.Hq, c.Hkv, c.Dh, d.max_kv));
  CHECK(d.chunk >= 0, WAM_EINVAL, "chunk=%d is negative", d.chunk);
  TRY(check_scale(d.scale, c.Dh));
  CHECK(d.max_pages >= 0 && d.table_stride >= d.max_pages && d.table_stride <= INT64_MAX / 8 / (d.R + 1), WAM_EINVAL,
        "table_stride=%lld must be >= max_pages=%d >= 0", (long long)d.table_stride, d.max_pages);
  if (d.R == 0 || d.T == 0) return WAM_OK;
  TRY(check_rows(q, o, d.q_tok_stride, d.o_tok_stride, (int64_t)d.Hq * c.Dh));
  TRY(need_ints(q_start, "q_start"));
  TRY(opt_ints(q_len, "q_len"));
  TRY(need_ints(kv_len, "kv_len"));
  if (d.max_pages > 0) TRY(need_ints(block_table, "block_table"));
  const RaggedPlan p = plan(d.R, d.T, d.Hq, c.Hkv, c.Dh, d.max_kv);
  TRY(check_ws(ws, ws_bytes, ragged_ws_bytes(p, d.T, d.Hq, c.Dh, ragged_tiles(d.R, d.T, d.Hq, c.Hkv, p.rows))));
  TRY(check_launch(ragged_blocks(p, d.R, d.T, d.Hq, c.Hkv) * 256 * p.groups));
  a.q = q; a.k = c.k; a.v = c.v; a.k_exp = c.k_exp; a.o = o;
  // (a table without columns is never read: no key is below max_k = 0; its address only says "paged")
  a.table = block_table ? block_table : q_start;
  a.q_start = q_start; a.q_len = q_len; a.k_len = kv_len;
  a.table_stride = d.table_stride; a.q_ts = d.q_tok_stride; a.o_ts = d.o_tok_stride;
  a.page_stride = c.page_stride; a.tok_stride = c.tok_stride; a.head_stride = c.head_stride;
  a.R = d.R; a.T = d.T; a.Hq = d.Hq; a.Hkv = c.Hkv; a.Dh = c.Dh; a.n_pages = c.n_pages;
  a.group = fast_div((uint32_t)(d.Hq / c.Hkv));
  const int64_t width = (int64_t)d.max_pages * c.page_size;
  a.max_k = (int32_t)(width < d.max_kv ? width : d.max_kv);
  a.ps = fast_div((uint32_t)c.page_size);
  a.c = exp2_scale(d.scale, c.Dh);
  a.v_scale = c.v_scale;
  HIPCHECK(launch(a, p, ws, stream));
  return WAM_OK;
}

wam_status check_verify(const wam_verify_tree_desc& d) {
  CHECK(d.R >= 0 && d.T >= 0, WAM_EINVAL, "negative size (R=%d T=%d)", d.R, d.T);
  CHECK(d.V >= 1, WAM_EINVAL, "V=%d must be positive", d.V);
  CHECK(d.V <= WAM_VERIFY_MAX_VOCAB, WAM_EUNSUPPORTED, "V=%d exceeds %d", d.V, WAM_VERIFY_MAX_VOCAB);
  CHECK(d.drawn == 0 || d.drawn == 1, WAM_EINVAL, "drawn=%d must be 0 or 1", d.drawn);
  CHECK(d.p_stride >= d.V && (!d.drawn || d.q_stride >= d.V), WAM_EINVAL, "the strides of p and q must be >= V=%d", d.V);
  CHECK(d.p_stride <= INT64_MAX / 8 / ((int64_t)d.T + 1) && (!d.drawn || d.q_stride <= INT64_MAX / 8 / ((int64_t)d.T + 1)),
        WAM_EINVAL, "a stride of p or q overflows");
  return check_launch((int64_t)d.R * verify_slices(d) * 256 > (int64_t)d.R * 1024 ? (int64_t)d.R * verify_slices(d) * 256
                                                                                 : (int64_t)d.R * 1024);
}

}  // namespace

extern "C" {

wam_status wam_page_plan(const wam_page_plan_desc* desc, const int32_t* cache_len, const int32_t* new_len,
                         const int32_t* held, const int32_t* n_free, int32_t* block_table, int32_t* free_list,
                         int32_t* held_out, int32_t* n_free_out, int32_t* q_start, int32_t* kv_len,
                         int32_t* slots, int32_t* token_pos, int32_t* status, hipStream_t stream) {
  CHECK(desc, WAM_EINVAL, "desc is NULL");
  const wam_page_plan_desc& d = *desc;
  CHECK(d.R >= 0 && d.T >= 0 && d.max_pages >= 0, WAM_EINVAL, "negative size (R=%d T=%d max_pages=%d)", d.R, d.T,
        d.max_pages);
  CHECK(d.R <= WAM_PLAN_MAX_REQUESTS, WAM_EUNSUPPORTED, "R=%d exceeds %d", d.R, WAM_PLAN_MAX_REQUESTS);
  TRY(check_page_size(d.page_size, d.n_pages));
  CHECK((int64_t)d.R * d.max_pages <= INT32_MAX, WAM_EUNSUPPORTED, "R * max_pages must stay below 2^31");
  CHECK(d.table_stride >= d.max_pages && d.table_stride <= INT64_MAX / 8 / (d.R + 1), WAM_EINVAL,
        "table_stride=%lld must be >= max_pages=%d", (long long)d.table_stride, d.max_pages);
  if (d.R > 0) {
    TRY(need_ints(cache_len, "cache_len"));
    TRY(need_ints(new_len, "new_len"));
    TRY(need_ints(held, "held"));
    TRY(need_ints(held_out, "held_out"));
    TRY(need_ints(kv_len, "kv_len"));
    if (d.max_pages > 0) TRY(need_ints(block_table, "block_table"));
  }
  if (d.n_pages > 0) TRY(need_ints(free_list, "free_list"));
  if (d.T > 0) TRY(need_ints(slots, "slots"));
  TRY(need_ints(n_free, "n_free"));
  TRY(need_ints(n_free_out, "n_free_out"));
  TRY(need_ints(q_start, "q_start"));
  TRY(need_ints(status, "status"));
  TRY(opt_ints(token_pos, "token_pos"));
  // Every workgroup reads the inputs while others store, so nothing written may lie on anything else.
  const Ints all[] = {{"block_table", block_table, d.max_pages, d.R, d.table_stride, true},
                      {"free_list", free_list, d.n_pages, 1, 0, true},
                      {"held_out", held_out, d.R, 1, 0, true},
                      {"n_free_out", n_free_out, 1, 1, 0, true},
                      {"q_start", q_start, d.R + 1, 1, 0, true},
                      {"kv_len", kv_len, d.R, 1, 0, true},
                      {"slots", slots, d.T, 1, 0, true},
                      {"token_pos", token_pos, d.T, 1, 0, true},
                      {"status", status, 4, 1, 0, true},
                      {"cache_len", cache_len, d.R, 1, 0, false},
                      {"new_len", new_len, d.R, 1, 0, false},
                      {"held", held, d.R, 1, 0, false},
                      {"n_free", n_free, 1, 1, 0, false}};
  for (const Ints& x : all)
    for (const Ints& y : all)
      CHECK(&x >= &y || !x.written || !overlap(x, y), WAM_EINVAL, "%s and %s overlap", x.name, y.name);
  PagePlanArgs a{};
  a.d = d;
  a.ps = fast_div((uint32_t)d.page_size);
  a.cache_len = cache_len; a.new_len = new_len; a.held = held; a.n_free = n_free;
  a.table = block_table; a.free_list = free_list; a.held_out = held_out; a.n_free_out = n_free_out;
  a.q_start = q_start; a.kv_len = kv_len; a.slots = slots; a.token_pos = token_pos; a.status = status;
  HIPCHECK(launch_page_plan(a, stream));
  return WAM_OK;
}

wam_status wam_rope_qkv_paged(const wam_rope_paged_desc* desc, const wam_paged_cache* cache, const void* qkv,
                              const int32_t* pos, const int32_t* slots, void* q_out, hipStream_t stream) {
  CHECK(desc && cache, WAM_EINVAL, "desc or cache is NULL");
  const wam_rope_paged_desc& d = *desc;
  TRY(check_cache(*cache));
  TRY(check_heads(d.Hq, cache->Hkv, cache->Dh));
  CHECK(d.T >= 0, WAM_EINVAL, "T=%d is negative", d.T);
  CHECK(d.n_axes >= 1 && d.n_axes <= WAM_ROPE_MAX_AXES, WAM_EINVAL, "n_axes=%d outside [1,%d]", d.n_axes,
        WAM_ROPE_MAX_AXES);
  CHECK(std::isfinite(d.theta) && d.theta > 0.0, WAM_EINVAL, "theta=%g must be positive and finite", d.theta);
  RopePagedArgs a{};
  for (int x = 0; x < d.n_axes; ++x) {
    CHECK(d.pairs[x] >= 0 && d.pairs[x] <= cache->Dh / 2 - a.n, WAM_EINVAL,
          "pairs[%d]=%d: the axes' pairs must be >= 0 and at most Dh/2=%d together", x, d.pairs[x], cache->Dh / 2);
    // theta^(-i / pairs) / (2 pi) by repeated products of 64-bit mantissas (2^-64 of the value each, at most 127), rounded to
    // fp64 once: a position of 2^31 multiplies what is off.  (Products in fp64 were off by up to 33 units in the last
    // place, 2^-18.4 rad at 2^31 and theta = 1.1.)
#ifndef __HIP_DEVICE_COMPILE__  // (the device's own long double is not used)
    static_assert(std::numeric_limits<long double>::digits >= 64, "extended precision");
#endif
    const long double step = d.pairs[x] ? std::pow((long double)d.theta, -1.0L / d.pairs[x]) : 1.0L;
    long double w = 0.15915494309189533576888376337251436L;
    for (int i = 0; i < d.pairs[x]; ++i, w *= step) {
      a.turns[a.n] = (double)w;
      a.axis[a.n++] = (uint8_t)x;
    }
  }
  CHECK(d.halves == 0 || d.halves == 1, WAM_EINVAL, "halves=%d must be 0 or 1", d.halves);
  const int unit = cache->k_exp ? 32 : 8;
  CHECK(!d.halves || a.n % unit == 0, WAM_EUNSUPPORTED, "pairs in halves: their number %d must be a multiple of %d", a.n,
        unit);
  if (d.T == 0) return WAM_OK;
  TRY(need_ptr(qkv, "qkv"));
  TRY(need_ints(pos, "pos"));
  TRY(need_ints(slots, "slots"));
  TRY(opt_ptr(q_out, "q_out"));
  const int64_t width = ((int64_t)d.Hq + 2 * cache->Hkv) * cache->Dh;
  CHECK(d.qkv_tok_stride >= width && d.qkv_tok_stride % 8 == 0, WAM_EINVAL,
        "qkv_tok_stride must be a multiple of 8, >= (Hq + 2 Hkv) * Dh=%lld", (long long)width);
  CHECK(!q_out || (d.q_tok_stride >= (int64_t)d.Hq * cache->Dh && d.q_tok_stride % 8 == 0), WAM_EINVAL,
        "q_tok_stride must be a multiple of 8, >= Hq * Dh");
  TRY(check_launch((int64_t)d.T * rope_threads(d.Hq, cache->Hkv, cache->Dh) + 255));
  a.c = *cache;
  a.ps = fast_div((uint32_t)cache->page_size);
  a.T = d.T; a.Hq = d.Hq; a.n_axes = d.n_axes; a.halves = d.halves;
  a.qkv_ts = d.qkv_tok_stride; a.q_ts = d.q_tok_stride;
  a.qkv = qkv; a.pos = pos; a.slots = slots; a.q_out = q_out;
  a.v_inv = cache->k_exp ? 1.0f / cache->v_scale : 1.0f;
  HIPCHECK(launch_rope_paged(a, stream));
  return WAM_OK;
}

size_t wam_attn_paged_workspace_bytes(const wam_attn_paged_desc* desc, const wam_paged_cache* cache) {
  if (!desc || !cache || check_ragged(desc->R, desc->T, desc->Hq, cache->Hkv, cache->Dh, desc->max_kv) != WAM_OK) return 0;
  return ragged_ws_bytes(plan_ragged(desc->R, desc->T, desc->Hq, cache->Hkv, cache->Dh, desc->max_kv), desc->T, desc->Hq, cache->Dh);
}

wam_status wam_attn_paged(const wam_attn_paged_desc* desc, const wam_paged_cache* cache, const void* q,
                          const int32_t* block_table, const int32_t* q_start, const int32_t* q_len,
                          const int32_t* kv_len, void* o, void* ws, size_t ws_bytes, hipStream_t stream) {
  CHECK(desc && cache, WAM_EINVAL, "desc or cache is NULL");
  RaggedArgs a{};
  if (desc->chunk > 0) a.chunk = fast_div((uint32_t)desc->chunk);
  return run_paged(*desc, *cache, q, block_table, q_start, q_len, kv_len, o, ws, ws_bytes, a, plan_ragged, launch_attn_ragged, stream);
}

size_t wam_attn_cross_workspace_bytes(const wam_attn_cross_desc* desc) {
  if (!desc || check_ragged(desc->R, desc->T, desc->Hq, desc->Hkv, desc->Dh, desc->max_k) != WAM_OK) return 0;
  return ragged_ws_bytes(plan_ragged(desc->R, desc->T, desc->Hq, desc->Hkv, desc->Dh, desc->max_k), desc->T, desc->Hq, desc->Dh);
}

wam_status wam_attn_cross(const wam_attn_cross_desc* desc, const void* q, const void* k, const void* v,
                          const int32_t* q_start, const int32_t* q_len, const int32_t* k_start,
                          const int32_t* k_len, void* o, void* ws, size_t ws_bytes, hipStream_t stream) {
  CHECK(desc, WAM_EINVAL, "desc is NULL");
  const wam_attn_cross_desc& d = *desc;
  TRY(check_ragged(d.R, d.T, d.Hq, d.Hkv, d.Dh, d.max_k));
  CHECK(d.S >= 0, WAM_EINVAL, "S=%d is negative", d.S);
  TRY(check_scale(d.scale, d.Dh));
  if (d.R == 0 || d.T == 0) return WAM_OK;
  TRY(check_rows(q, o, d.q_tok_stride, d.o_tok_stride, (int64_t)d.Hq * d.Dh));
  if (d.S > 0) {
    TRY(need_ptr(k, "k"));
    TRY(need_ptr(v, "v"));
    CHECK(d.kv_tok_stride >= (int64_t)d.Hkv * d.Dh && d.kv_tok_stride % 8 == 0 &&
              d.kv_tok_stride <= 1 << 25, WAM_EINVAL,
          "kv_tok_stride must be a multiple of 8, >= Hkv*Dh=%lld and at most 2^25", (long long)d.Hkv * d.Dh);
  }
  TRY(need_ints(q_start, "q_start"));
  TRY(opt_ints(q_len, "q_len"));
  TRY(need_ints(k_start, "k_start"));
  TRY(opt_ints(k_len, "k_len"));
  const RaggedPlan p = plan_ragged(d.R, d.T, d.Hq, d.Hkv, d.Dh, d.max_k);
  TRY(check_ws(ws, ws_bytes, ragged_ws_bytes(p, d.T, d.Hq, d.Dh)));
  TRY(check_launch(ragged_blocks(p, d.R, d.T, d.Hq, d.Hkv) * 256 * p.groups));
  RaggedArgs a{};
  a.q = q; a.k = k; a.v = v; a.o = o;
  a.q_start = q_start; a.q_len = q_len; a.k_start = k_start; a.k_len = k_len;
  a.q_ts = d.q_tok_stride; a.o_ts = d.o_tok_stride; a.tok_stride = d.kv_tok_stride; a.head_stride = d.Dh;
  a.R = d.R; a.T = d.T; a.S = d.S; a.Hq = d.Hq; a.Hkv = d.Hkv; a.Dh = d.Dh;
  a.max_k = d.max_k < d.S ? d.max_k : d.S;
  a.ps = fast_div(1);
  a.group = fast_div((uint32_t)(d.Hq / d.Hkv));
  a.c = exp2_scale(d.scale, d.Dh);
  HIPCHECK(launch_attn_ragged(a, p, ws, stream));
  return WAM_OK;
}

wam_status wam_page_fork(const wam_page_fork_desc* desc, const int32_t* src, const int32_t* dst, const int32_t* first,
                         const int32_t* len, const int32_t* held, const int32_t* n_free, int32_t* block_table,
                         const int32_t* free_list, int32_t* held_out, int32_t* n_free_out, int32_t* copies,
                         int32_t* status, hipStream_t stream) {
  CHECK(desc, WAM_EINVAL, "desc is NULL");
  const wam_page_fork_desc& d = *desc;
  CHECK(d.N >= 0, WAM_EINVAL, "N=%d is negative", d.N);
  CHECK(d.R <= WAM_PLAN_MAX_REQUESTS && d.N <= WAM_PLAN_MAX_REQUESTS, WAM_EUNSUPPORTED, "R=%d or N=%d exceeds %d", d.R, d.N,
        WAM_PLAN_MAX_REQUESTS);
  TRY(check_page_size(d.page_size, d.n_pages));
  TRY(check_table(d.R, d.max_pages, d.table_stride, block_table));
  if (d.N > 0) {
    TRY(need_ints(src, "src"));
    TRY(need_ints(dst, "dst"));
    TRY(opt_ints(first, "first"));
    TRY(need_ints(len, "len"));
    TRY(need_ints(copies, "copies"));
  }
  if (d.R > 0) {
    TRY(need_ints(held, "held"));
    TRY(need_ints(held_out, "held_out"));
  }
  if (d.n_pages > 0) TRY(need_ints(free_list, "free_list"));
  TRY(need_ints(n_free, "n_free"));
  TRY(need_ints(n_free_out, "n_free_out"));
  TRY(need_ints(status, "status"));
  const Ints all[] = {{"block_table", block_table, d.max_pages, d.R, d.table_stride, true},
                      {"held_out", held_out, d.R, 1, 0, true},
                      {"n_free_out", n_free_out, 1, 1, 0, true},
                      {"copies", copies, 3 * (int64_t)d.N, 1, 0, true},
                      {"status", status, 2, 1, 0, true},
                      {"src", src, d.N, 1, 0, false},
                      {"dst", dst, d.N, 1, 0, false},
                      {"first", first, d.N, 1, 0, false},
                      {"len", len, d.N, 1, 0, false},
                      {"held", held, d.R, 1, 0, false},
                      {"n_free", n_free, 1, 1, 0, false},
                      {"free_list", free_list, d.n_pages, 1, 0, false}};
  TRY(check_apart(all));
  PageForkArgs a{};
  a.d = d;
  a.ps = fast_div((uint32_t)d.page_size);
  a.src = src; a.dst = dst; a.first = first; a.len = len; a.held = held; a.n_free = n_free; a.free_list = free_list;
  a.table = block_table; a.held_out = held_out; a.n_free_out = n_free_out; a.copies = copies; a.status = status;
  HIPCHECK(launch_page_fork(a, stream));
  return WAM_OK;
}

wam_status wam_page_copy(const wam_paged_cache* cache, int32_t N, const int32_t* copies, hipStream_t stream) {
  CHECK(cache, WAM_EINVAL, "cache is NULL");
  TRY(check_cache(*cache));
  CHECK(N >= 0, WAM_EINVAL, "N=%d is negative", N);
  if (N == 0 || cache->n_pages == 0) return WAM_OK;
  TRY(need_ints(copies, "copies"));
  const int64_t blocks = page_copy_blocks(*cache);
  TRY(check_launch(N * blocks * 256));
  PageCopyArgs a{};
  a.c = *cache;
  a.by_blocks = fast_div((uint32_t)blocks);
  a.by_row = fast_div((uint32_t)(cache->Hkv * (cache->Dh * (cache->k_exp ? 1 : 2) / 16)));
  a.N = N;
  a.copies = copies;
  HIPCHECK(launch_page_copy(a, stream));
  return WAM_OK;
}

wam_status wam_page_collect(const wam_page_collect_desc* desc, const int32_t* cache_len, const int32_t* held,
                            const int32_t* block_table, int32_t* free_list, int32_t* held_out, int32_t* n_free_out,
                            int32_t* status, hipStream_t stream) {
  CHECK(desc, WAM_EINVAL, "desc is NULL");
  const wam_page_collect_desc& d = *desc;
  CHECK(d.R <= WAM_PLAN_MAX_REQUESTS, WAM_EUNSUPPORTED, "R=%d exceeds %d", d.R, WAM_PLAN_MAX_REQUESTS);
  TRY(check_page_size(d.page_size, d.n_pages));
  CHECK(d.n_pages <= WAM_COLLECT_MAX_PAGES, WAM_EUNSUPPORTED, "n_pages=%d exceeds %d", d.n_pages, WAM_COLLECT_MAX_PAGES);
  TRY(check_table(d.R, d.max_pages, d.table_stride, block_table));
  if (d.R > 0) {
    TRY(need_ints(cache_len, "cache_len"));
    TRY(need_ints(held, "held"));
    TRY(need_ints(held_out, "held_out"));
  }
  if (d.n_pages > 0) TRY(need_ints(free_list, "free_list"));
  TRY(need_ints(n_free_out, "n_free_out"));
  TRY(need_ints(status, "status"));
  const Ints all[] = {{"free_list", free_list, d.n_pages, 1, 0, true},
                      {"held_out", held_out, d.R, 1, 0, true},
                      {"n_free_out", n_free_out, 1, 1, 0, true},
                      {"status", status, 2, 1, 0, true},
                      {"block_table", block_table, d.max_pages, d.R, d.table_stride, false},
                      {"cache_len", cache_len, d.R, 1, 0, false},
                      {"held", held, d.R, 1, 0, false}};
  TRY(check_apart(all));
  PageCollectArgs a{};
  a.d = d;
  a.ps = fast_div((uint32_t)d.page_size);
  a.cache_len = cache_len; a.held = held; a.table = block_table;
  a.free_list = free_list; a.held_out = held_out; a.n_free_out = n_free_out; a.status = status;
  HIPCHECK(launch_page_collect(a, stream));
  return WAM_OK;
}

wam_status wam_cache_compact(const wam_cache_compact_desc* desc, const wam_paged_cache* cache, const int32_t* block_table,
                             const int32_t* q_start, const int32_t* q_len, const int32_t* kv_len, const int32_t* keep,
                             const int32_t* n_keep, hipStream_t stream) {
  CHECK(desc && cache, WAM_EINVAL, "desc or cache is NULL");
  const wam_cache_compact_desc& d = *desc;
  TRY(check_cache(*cache));
  CHECK(d.T >= 0, WAM_EINVAL, "T=%d is negative", d.T);
  TRY(check_table(d.R, d.max_pages, d.table_stride, block_table));
  if (d.R == 0 || d.T == 0 || d.max_pages == 0 || cache->n_pages == 0) return WAM_OK;
  TRY(need_ints(q_start, "q_start"));
  TRY(opt_ints(q_len, "q_len"));
  TRY(need_ints(kv_len, "kv_len"));
  TRY(need_ints(keep, "keep"));
  TRY(need_ints(n_keep, "n_keep"));
  TRY(check_launch(2 * (int64_t)d.R * cache->Hkv * 256));
  CacheCompactArgs a{};
  a.c = *cache;
  a.ps = fast_div((uint32_t)cache->page_size);
  a.by_heads = fast_div((uint32_t)cache->Hkv);
  a.R = d.R; a.T = d.T; a.max_pages = d.max_pages; a.table_stride = d.table_stride;
  a.table = block_table; a.q_start = q_start; a.q_len = q_len; a.kv_len = kv_len; a.keep = keep; a.n_keep = n_keep;
  HIPCHECK(launch_cache_compact(a, stream));
  return WAM_OK;
}

size_t wam_attn_tree_workspace_bytes(const wam_attn_tree_desc* desc, const wam_paged_cache* cache) {
  if (!desc || !cache || check_ragged(desc->R, desc->T, desc->Hq, cache->Hkv, cache->Dh, desc->max_kv) != WAM_OK) return 0;
  const RaggedPlan p = plan_tree(desc->R, desc->T, desc->Hq, cache->Hkv, cache->Dh, desc->max_kv);
  return ragged_ws_bytes(p, desc->T, desc->Hq, cache->Dh, ragged_tiles(desc->R, desc->T, desc->Hq, cache->Hkv, p.rows));
}

wam_status wam_attn_tree(const wam_attn_tree_desc* desc, const wam_paged_cache* cache, const void* q,
                         const int32_t* block_table, const int32_t* q_start, const int32_t* q_len,
                         const int32_t* kv_len, const uint32_t* mask, void* o, void* ws, size_t ws_bytes,
                         hipStream_t stream) {
  CHECK(desc && cache, WAM_EINVAL, "desc or cache is NULL");
  const wam_attn_tree_desc& d = *desc;
  CHECK(d.mask_words >= 0 && d.mask_stride >= d.mask_words && d.mask_stride <= INT64_MAX / 8 / ((int64_t)(d.T < 0 ? 0 : d.T) + 1),
        WAM_EINVAL, "mask_stride=%lld must be >= mask_words=%d >= 0", (long long)d.mask_stride, d.mask_words);
  if (d.R > 0 && d.T > 0 && d.mask_words > 0) TRY(need_ints(mask, "mask"));
  RaggedArgs a{};
  a.mask = mask;
  a.mask_stride = d.mask_stride;
  a.mask_words = d.mask_words;
  const wam_attn_paged_desc p{d.R, d.T, d.Hq, d.max_pages, d.max_kv, 0, d.table_stride, d.q_tok_stride, d.o_tok_stride, d.scale};
  return run_paged(p, *cache, q, block_table, q_start, q_len, kv_len, o, ws, ws_bytes, a, plan_tree, launch_attn_tree, stream);
}

size_t wam_verify_tree_workspace_bytes(const wam_verify_tree_desc* desc) {
  if (!desc || check_verify(*desc) != WAM_OK) return 0;
  return verify_ws_bytes(*desc);
}

wam_status wam_verify_tree(const wam_verify_tree_desc* desc, const float* p, const float* q, const int32_t* tokens,
                           const int32_t* parent, const float* u, const float* u_next, const int32_t* q_start,
                           const int32_t* q_len, const int32_t* kv_len, int32_t* path, int32_t* n_path,
                           int32_t* next_token, int32_t* cache_len, void* ws, size_t ws_bytes, hipStream_t stream) {
  CHECK(desc, WAM_EINVAL, "desc is NULL");
  const wam_verify_tree_desc& d = *desc;
  TRY(check_verify(d));
  // (without rows p and q have no address)
  CHECK(!d.drawn == !q || (d.drawn && d.T == 0), WAM_EINVAL, "q must be given where drawn is 1 and only there");
  CHECK(!kv_len == !cache_len, WAM_EINVAL, "kv_len and cache_len must be given both or neither");
  if (d.R == 0) return WAM_OK;
  if (d.T > 0) {
    TRY(need_ints(p, "p"));
    TRY(opt_ints(q, "q"));
    TRY(need_ints(tokens, "tokens"));
    TRY(need_ints(parent, "parent"));
    TRY(need_ints(u, "u"));
    TRY(need_ints(path, "path"));
  }
  TRY(need_ints(u_next, "u_next"));
  TRY(need_ints(q_start, "q_start"));
  TRY(opt_ints(q_len, "q_len"));
  TRY(opt_ints(kv_len, "kv_len"));
  TRY(need_ints(n_path, "n_path"));
  TRY(need_ints(next_token, "next_token"));
  TRY(opt_ints(cache_len, "cache_len"));
  const auto ints = [](const float* x) { return reinterpret_cast<const int32_t*>(x); };
  const Ints all[] = {{"path", path, d.T, 1, 0, true},
                      {"n_path", n_path, d.R, 1, 0, true},
                      {"next_token", next_token, d.R, 1, 0, true},
                      {"cache_len", cache_len, d.R, 1, 0, true},
                      {"p", ints(p), d.V, d.T, d.p_stride, false},
                      {"q", ints(q), d.V, d.T, d.q_stride, false},
                      {"tokens", tokens, d.T, 1, 0, false},
                      {"parent", parent, d.T, 1, 0, false},
                      {"u", ints(u), d.T, 1, 0, false},
                      {"u_next", ints(u_next), d.R, 1, 0, false},
                      {"q_start", q_start, (int64_t)d.R + 1, 1, 0, false},
                      {"q_len", q_len, d.R, 1, 0, false},
                      {"kv_len", kv_len, d.R, 1, 0, false}};
  TRY(check_apart(all));
  TRY(check_ws(ws, ws_bytes, verify_ws_bytes(d)));
  VerifyArgs a{};
  a.d = d;
  a.p = p; a.q = q; a.u = u; a.u_next = u_next;
  a.tokens = tokens; a.parent = parent; a.q_start = q_start; a.q_len = q_len; a.kv_len = kv_len;
  a.path = path; a.n_path = n_path; a.next_token = next_token; a.cache_len = cache_len;
  a.slices = verify_slices(d);
  a.rounds = verify_rounds(d);
  a.by_slices = fast_div((uint32_t)a.slices);
  a.state = static_cast<VerifyState*>(ws);
  a.sums = reinterpret_cast<double*>(a.state + (int64_t)a.rounds * d.R);
  a.nodes = reinterpret_cast<float2*>(a.sums + (int64_t)a.rounds * d.R * a.slices);
  HIPCHECK(launch_verify_tree(a, stream));
  return WAM_OK;
}

wam_status wam_tree_mask(const int32_t* parent, int32_t n, int32_t words, uint32_t* mask) {
  CHECK(n >= 0 && words >= 0 && n <= 32 * (int64_t)words, WAM_EINVAL, "n=%d nodes do not fit %d words", n, words);
  CHECK(n == 0 || (parent && mask), WAM_EINVAL, "parent or mask is NULL");
  for (int32_t i = 0; i < n; ++i)
    CHECK(parent[i] >= -1 && parent[i] < i, WAM_EINVAL, "parent[%d]=%d must be -1 or a node before it", i, parent[i]);
  for (int32_t i = 0; i < n; ++i) {
    uint32_t* row = mask + (int64_t)i * words;
    for (int32_t w = 0; w < words; ++w) row[w] = parent[i] < 0 ? 0u : mask[(int64_t)parent[i] * words + w];
    row[i >> 5] |= 1u << (i & 31);
  }
  return WAM_OK;
}

}  // extern "C"
