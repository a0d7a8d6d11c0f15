// C ABI of the paged KV cache: argument checks and launches of the page plan, the rotary
// append, and the ragged attentions.
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
wam_status check_ws(const void* ws, size_t have, size_t need) {
  CHECK(need == 0 || (ws && (reinterpret_cast<uintptr_t>(ws) & 255) == 0 && have >= need), WAM_EWORKSPACE,
        "workspace of %zu bytes (256-byte aligned) needed, got %zu", need, ws ? have : (size_t)0);
  return WAM_OK;
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
  const wam_attn_paged_desc& d = *desc;
  const wam_paged_cache& c = *cache;
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
  const RaggedPlan p = plan_ragged(d.R, d.T, d.Hq, c.Hkv, c.Dh, d.max_kv);
  TRY(check_ws(ws, ws_bytes, ragged_ws_bytes(p, d.T, d.Hq, c.Dh)));
  TRY(check_launch(ragged_blocks(p, d.R, d.T, d.Hq, c.Hkv) * 256 * p.groups));
  RaggedArgs a{};
  a.q = q; a.k = c.k; a.v = c.v; a.k_exp = c.k_exp; a.o = o;
  // (a table without columns is never read: no key is below max_k = 0; its address only says "paged")
  a.table = block_table ? block_table : q_start;
  a.q_start = q_start; a.q_len = q_len; a.k_len = kv_len;
  a.table_stride = d.table_stride; a.q_ts = d.q_tok_stride; a.o_ts = d.o_tok_stride;
  a.page_stride = c.page_stride; a.tok_stride = c.tok_stride; a.head_stride = c.head_stride;
  a.R = d.R; a.T = d.T; a.Hq = d.Hq; a.Hkv = c.Hkv; a.Dh = c.Dh; a.n_pages = c.n_pages;
  a.group = fast_div((uint32_t)(d.Hq / c.Hkv));
  if (d.chunk > 0) a.chunk = fast_div((uint32_t)d.chunk);
  const int64_t width = (int64_t)d.max_pages * c.page_size;
  a.max_k = (int32_t)(width < d.max_kv ? width : d.max_kv);
  a.ps = fast_div((uint32_t)c.page_size);
  a.c = exp2_scale(d.scale, c.Dh);
  a.v_scale = c.v_scale;
  HIPCHECK(launch_attn_ragged(a, p, ws, stream));
  return WAM_OK;
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

}  // extern "C"
