// Host side of the cache operators declared in include/evconv_ops.h: checks of the arguments, launches on the caller's stream.
#include "ops_host.h"

#include <algorithm>
#include <cmath>

using namespace evk;

namespace {

evconv_status check_cache(const char* what, const evconv_cache& c, const evconv_tokens& t) {
  if (c.kind != EVCONV_CACHE_BF16 && c.kind != EVCONV_CACHE_FP4) return refuse(EVCONV_ERR_INVALID_ARG, "%s: cache kind %d", what, c.kind);
  if (c.heads < 1 || c.d < 1 || c.n_pages < 1) return refuse(EVCONV_ERR_SHAPE, "%s: cache of %d pages, %d heads of %d", what, c.n_pages, c.heads, c.d);
  if (c.page != 32 && c.page != 64 && c.page != 128 && c.page != 256) return refuse(EVCONV_ERR_UNSUPPORTED, "%s: pages of %d tokens: 32, 64, 128 or 256", what, c.page);
  if (c.heads > 1024 || c.d > 256) return refuse(EVCONV_ERR_UNSUPPORTED, "%s: %d heads of %d: at most 1024 of 256", what, c.heads, c.d);
  if (t.n_seq < 1 || t.n_seq > 65535) return refuse(t.n_seq < 1 ? EVCONV_ERR_SHAPE : EVCONV_ERR_UNSUPPORTED, "%s: %d sequences", what, t.n_seq);
  if (t.n_tokens < 0 || (!t.seq_offsets && t.n_tokens % t.n_seq)) return refuse(EVCONV_ERR_SHAPE, "%s: %lld tokens for %d sequences", what, (long long)t.n_tokens, t.n_seq);
  if (t.n_tokens >= (1ll << 31) - 64) return refuse(EVCONV_ERR_UNSUPPORTED, "%s: %lld tokens", what, (long long)t.n_tokens);
  if (t.width < 1) return refuse(EVCONV_ERR_SHAPE, "%s: table rows of %d", what, t.width);
  if ((int64_t)t.width * c.page >= 1ll << 30) return refuse(EVCONV_ERR_UNSUPPORTED, "%s: table rows of %d pages of %d: a sequence has less than 2^30 tokens", what, t.width, c.page);
  if (!t.n_tokens) return EVCONV_OK;
  if (!c.k || !c.v || !t.table || !t.past) return refuse(EVCONV_ERR_INVALID_ARG, "%s: null cache, table or past", what);
  if (c.kind == EVCONV_CACHE_FP4 && (!c.k_scale || !c.v_scale)) return refuse(EVCONV_ERR_INVALID_ARG, "%s: a cache in 4 bits without scales", what);
  if (!aligned(c.k, 16) || !aligned(c.v, 16) || !aligned(c.k_scale, 16) || !aligned(c.v_scale, 16) || !aligned(c.bounds, 16))
    return refuse(EVCONV_ERR_INVALID_ARG, "%s: cache tensors at addresses that are no multiples of 16", what);
  return EVCONV_OK;
}

evconv_status check_head(const char* what, int abi_version, int dtype) {
  if (abi_version != EVCONV_OPS_ABI_VERSION) return refuse(EVCONV_ERR_BAD_DESC, "%s: abi_version %d, expected %d", what, abi_version, EVCONV_OPS_ABI_VERSION);
  if (!float_type(dtype)) return refuse(EVCONV_ERR_INVALID_ARG, "%s: dtype %d", what, dtype);
  return EVCONV_OK;
}

evconv_status check_query_heads(const char* what, int heads_q, int heads) {
  if (heads_q < 1 || heads_q % heads) return refuse(EVCONV_ERR_SHAPE, "%s: %d query heads for %d key heads", what, heads_q, heads);
  if (heads_q > 1024) return refuse(EVCONV_ERR_UNSUPPORTED, "%s: %d query heads: at most 1024", what, heads_q);
  return EVCONV_OK;
}

evconv_status check_append(const evconv_append_args* a) {
  const char* const what = "cache append";
  if (!a) return refuse(EVCONV_ERR_INVALID_ARG, "%s: null arguments", what);
  evconv_status st = check_head(what, a->abi_version, a->dtype);
  if (st == EVCONV_OK) st = check_cache(what, a->cache, a->tokens);
  if (st != EVCONV_OK) return st;
  if (a->heads_q < 0) return refuse(EVCONV_ERR_SHAPE, "%s: %d query heads", what, a->heads_q);
  if (a->heads_q > 1024) return refuse(EVCONV_ERR_UNSUPPORTED, "%s: %d query heads: at most 1024", what, a->heads_q);
  if (a->rot < 0 || a->rot % 2 || a->rot > a->cache.d) return refuse(EVCONV_ERR_SHAPE, "%s: %d channels of %d rotated", what, a->rot, a->cache.d);
  if (a->pairs != EVCONV_PAIRS_HALVES && a->pairs != EVCONV_PAIRS_NEIGHBOURS) return refuse(EVCONV_ERR_INVALID_ARG, "%s: pairs %d", what, a->pairs);
  if (!(a->eps >= 0.0f)) return refuse(EVCONV_ERR_INVALID_ARG, "%s: eps %g", what, a->eps);
  if (a->rot && !a->freqs) return refuse(EVCONV_ERR_INVALID_ARG, "%s: a rotation without freqs", what);
  if (a->tokens.n_tokens && (!a->k.data || !a->v.data || (a->heads_q && (!a->q.data || !a->q_out)))) return refuse(EVCONV_ERR_INVALID_ARG, "%s: null tensor", what);
  return EVCONV_OK;
}

evconv_status check_read(const evconv_read_args* a) {
  const char* const what = "cache read";
  if (!a) return refuse(EVCONV_ERR_INVALID_ARG, "%s: null arguments", what);
  evconv_status st = check_head(what, a->abi_version, a->dtype);
  if (st == EVCONV_OK) st = check_cache(what, a->cache, a->tokens);
  if (st != EVCONV_OK) return st;
  if (a->tokens.n_tokens && (!a->k || !a->v)) return refuse(EVCONV_ERR_INVALID_ARG, "%s: null tensor", what);
  return EVCONV_OK;
}

evconv_status plan(const evconv_attend_args* a, AttendParams* p, size_t* bytes) {
  const char* const what = "cache attend";
  if (!a) return refuse(EVCONV_ERR_INVALID_ARG, "%s: null arguments", what);
  evconv_status st = check_head(what, a->abi_version, a->dtype);
  if (st == EVCONV_OK) st = check_cache(what, a->cache, a->tokens);
  if (st == EVCONV_OK) st = check_query_heads(what, a->heads_q, a->cache.heads);
  if (st != EVCONV_OK) return st;
  if (a->causal != 0 && a->causal != 1) return refuse(EVCONV_ERR_INVALID_ARG, "%s: causal %d", what, a->causal);
  if (a->window < 0 || (a->window && (!a->causal || a->selected))) return refuse(EVCONV_ERR_INVALID_ARG, "%s: window %d%s", what, a->window, a->window < 0 ? "" : !a->causal ? " without causal" : " beside chosen pages");
  if (a->selected && (a->count < 1 || a->count > 65536)) return refuse(a->count < 1 ? EVCONV_ERR_SHAPE : EVCONV_ERR_UNSUPPORTED, "%s: %d chosen pages", what, a->count);
  if (a->max_len < 0) return refuse(EVCONV_ERR_INVALID_ARG, "%s: max_len %lld", what, (long long)a->max_len);
  if (!(a->scale > 0.0f) || std::isinf(a->scale)) return refuse(EVCONV_ERR_INVALID_ARG, "%s: scale %g", what, a->scale);
  if (a->tokens.n_tokens && (!a->q.data || !a->o)) return refuse(EVCONV_ERR_INVALID_ARG, "%s: null tensor", what);
  *p = AttendParams{};
  p->a = *a;
  p->vec = a->cache.d % 8 == 0 && wide(a->dtype, a->q);
  p->vec_o = a->cache.d % 4 == 0 && a->o_token_stride % 4 == 0 && a->o_head_stride % 4 == 0 && aligned(a->o, 4 * type_size(a->dtype));
  *bytes = a->tokens.n_tokens ? plan_attend(*p) : 0;
  return EVCONV_OK;
}

evconv_status plan(const evconv_select_args* a, SelectParams* p, size_t* bytes) {
  const char* const what = "cache select";
  if (!a) return refuse(EVCONV_ERR_INVALID_ARG, "%s: null arguments", what);
  evconv_status st = check_head(what, a->abi_version, a->dtype);
  if (st == EVCONV_OK) st = check_cache(what, a->cache, a->tokens);
  if (st == EVCONV_OK) st = check_query_heads(what, a->heads_q, a->cache.heads);
  if (st != EVCONV_OK) return st;
  if (a->count < 1 || a->count > 65536) return refuse(a->count < 1 ? EVCONV_ERR_SHAPE : EVCONV_ERR_UNSUPPORTED, "%s: %d pages to choose", what, a->count);
  if (a->first < 0 || a->last < 1 || (int64_t)a->first + a->last > a->count) return refuse(EVCONV_ERR_INVALID_ARG, "%s: the first %d and the last %d pages of %d", what, a->first, a->last, a->count);
  if (a->max_len < 0) return refuse(EVCONV_ERR_INVALID_ARG, "%s: max_len %lld", what, (long long)a->max_len);
  if (a->tokens.n_tokens && !a->cache.bounds) return refuse(EVCONV_ERR_INVALID_ARG, "%s: a cache without bounds", what);
  if (a->tokens.n_tokens && (!a->q.data || !a->selected)) return refuse(EVCONV_ERR_INVALID_ARG, "%s: null tensor", what);
  *p = SelectParams{};
  p->a = *a;
  *bytes = a->tokens.n_tokens ? plan_select(*p) : 0;
  return EVCONV_OK;
}

evconv_status check_workspace(const char* what, size_t bytes, const void* workspace, size_t workspace_bytes) {
  if (bytes && (!workspace || workspace_bytes < bytes || !aligned(workspace, 256)))
    return refuse(EVCONV_ERR_WORKSPACE, "%s: needs %zu bytes of workspace at a multiple of 256, got %zu", what, bytes, workspace ? workspace_bytes : 0);
  return EVCONV_OK;
}

}  // namespace

extern "C" {

evconv_status evconv_cache_append(const evconv_append_args* args, void* hip_stream) {
  const evconv_status st = check_append(args);
  if (st != EVCONV_OK || !args->tokens.n_tokens) return st;
  const evconv_append_args& a = *args;
  bool vec = a.cache.d % 8 == 0 && wide(a.dtype, a.k) && wide(a.dtype, a.v);
  if (a.heads_q) vec = vec && wide(a.dtype, a.q) && wide(a.dtype, a.q_out, a.q_out_token_stride) && wide(a.dtype, a.q_out, a.q_out_head_stride);
  launch_cache_append(a, vec, (hipStream_t)hip_stream);
  return launched("cache append");
}

evconv_status evconv_cache_read(const evconv_read_args* args, void* hip_stream) {
  const evconv_status st = check_read(args);
  if (st != EVCONV_OK || !args->tokens.n_tokens) return st;
  launch_cache_read(*args, (hipStream_t)hip_stream);
  return launched("cache read");
}

evconv_status evconv_cache_attend_workspace(const evconv_attend_args* args, size_t* bytes) {
  if (!bytes) return refuse(EVCONV_ERR_INVALID_ARG, "cache attend: null bytes");
  AttendParams p;
  size_t n;
  const evconv_status st = plan(args, &p, &n);
  if (st == EVCONV_OK) *bytes = n;
  return st;
}

evconv_status evconv_cache_attend(const evconv_attend_args* args, void* workspace, size_t workspace_bytes, void* hip_stream) {
  AttendParams p;
  size_t n;
  evconv_status st = plan(args, &p, &n);
  if (st == EVCONV_OK) st = check_workspace("cache attend", n, workspace, workspace_bytes);
  if (st != EVCONV_OK || !args->tokens.n_tokens) return st;
  if (n) place_attend(p, (char*)workspace);
  launch_attend(p, (hipStream_t)hip_stream);
  return launched("cache attend");
}

evconv_status evconv_cache_select_workspace(const evconv_select_args* args, size_t* bytes) {
  if (!bytes) return refuse(EVCONV_ERR_INVALID_ARG, "cache select: null bytes");
  SelectParams p;
  size_t n;
  const evconv_status st = plan(args, &p, &n);
  if (st == EVCONV_OK) *bytes = n;
  return st;
}

evconv_status evconv_cache_select(const evconv_select_args* args, void* workspace, size_t workspace_bytes, void* hip_stream) {
  SelectParams p;
  size_t n;
  evconv_status st = plan(args, &p, &n);
  if (st == EVCONV_OK) st = check_workspace("cache select", n, workspace, workspace_bytes);
  if (st != EVCONV_OK || !args->tokens.n_tokens) return st;
  p.score = (unsigned*)workspace;
  launch_select(p, (hipStream_t)hip_stream);
  return launched("cache select");
}

}  // extern "C"
