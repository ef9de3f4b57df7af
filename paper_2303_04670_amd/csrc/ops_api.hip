// Host side of the C ABI declared in include/evconv_ops.h: checks of the arguments, the choice of
// kernels, launches on the caller's stream.
#include "ops_kernels.h"

#include <algorithm>
#include <cstdarg>
#include <cstdio>

using namespace evk;

namespace {

evconv_status refuse(evconv_status st, const char* format, ...) {
  char text[256];
  va_list args;
  va_start(args, format);
  vsnprintf(text, sizeof text, format, args);
  va_end(args);
  set_call_error(text);
  return st;
}

evconv_status launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? EVCONV_OK : refuse(EVCONV_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

bool float_type(int dtype) { return dtype == EVCONV_F32 || dtype == EVCONV_BF16; }
size_t type_size(int dtype) { return dtype == EVCONV_F32 ? 4 : 2; }
bool aligned(const void* p, size_t to) { return (uintptr_t)p % to == 0; }
// Whether rows of `dtype` at this address and these distances may be read 16 bytes at a time.
bool wide(int dtype, const void* p, int64_t stride) { return aligned(p, 16) && stride * (int64_t)type_size(dtype) % 16 == 0; }
bool wide(int dtype, const evconv_heads& h) { return wide(dtype, h.data, h.token_stride) && wide(dtype, h.data, h.head_stride); }

// Sequences of up to this many tokens go token by token: of calls that the one-launch kernel takes otherwise, of others.  us for
// 16 sequences of 4 heads of 64 x 64, 64 of 16 of 128 x 128, token by token / in chunks: bf16, 6 tokens 18 / 14, 59 / 76, 8
// tokens 22 / 14, 70 / 76; fp32, 8 tokens 19 / 27, 61 / 128, 12 tokens 25 / 27, 77 / 128.
// Of calls with lengths of their own the chunks wait for the launch of the tokens (24 sequences of up to 700 tokens, 6 heads of
// 80 x 112, fp32: for 24 us at 12 tokens, 12 at 4): fewer there, where sequences are longer than that on average.  Where they are not, as
// many (256 sequences of 16 heads of 128 x 128 / of 4 of 64 x 64: 5 tokens each in bf16 207 / 35 us, in chunks 304 / 53; 12 in fp32 297 / 55,
// 521 / 82).
constexpr int kShortFused = 6, kShort = 12;

struct DeltaPlan {
  DeltaParams p;
  bool steps, chunks, fused;
  size_t off_k, off_t, off_scal, off_seq, bytes;
};

evconv_status plan_delta(const evconv_delta_args* a, DeltaPlan* out) {
  if (!a) return refuse(EVCONV_ERR_INVALID_ARG, "delta rule: null arguments");
  if (a->abi_version != EVCONV_OPS_ABI_VERSION) return refuse(EVCONV_ERR_BAD_DESC, "delta rule: abi_version %d, expected %d", a->abi_version, EVCONV_OPS_ABI_VERSION);
  if (!float_type(a->dtype) || !float_type(a->gate_dtype)) return refuse(EVCONV_ERR_INVALID_ARG, "delta rule: dtype %d, gate_dtype %d", a->dtype, a->gate_dtype);
  if (a->flags & ~(EVCONV_DELTA_NORMALIZE | EVCONV_DELTA_RAW_GATES)) return refuse(EVCONV_ERR_INVALID_ARG, "delta rule: unknown flags 0x%x", a->flags);
  if (a->heads_k < 1 || a->heads_v < 1 || a->heads_v % a->heads_k) return refuse(EVCONV_ERR_SHAPE, "delta rule: %d value heads for %d key heads", a->heads_v, a->heads_k);
  if (a->d_k < 1 || a->d_v < 1) return refuse(EVCONV_ERR_SHAPE, "delta rule: head sizes %d, %d", a->d_k, a->d_v);
  if (a->heads_v > 1024 || a->d_k > 256 || a->d_v > 256) return refuse(EVCONV_ERR_UNSUPPORTED, "delta rule: %d heads of %d x %d: at most 1024 of 256 x 256", a->heads_v, a->d_k, a->d_v);
  if (a->n_seq < 1 || a->n_seq > 65535) return refuse(a->n_seq < 1 ? EVCONV_ERR_SHAPE : EVCONV_ERR_UNSUPPORTED, "delta rule: %d sequences", a->n_seq);
  if (a->n_tokens < 0 || (!a->seq_offsets && a->n_tokens % a->n_seq)) return refuse(EVCONV_ERR_SHAPE, "delta rule: %lld tokens for %d sequences", (long long)a->n_tokens, a->n_seq);
  if (a->n_tokens >= (1ll << 31) - 64) return refuse(EVCONV_ERR_UNSUPPORTED, "delta rule: %lld tokens", (long long)a->n_tokens);
  if ((a->state_in || a->state_out) && a->n_slots < (a->slots ? 0 : a->n_seq)) return refuse(EVCONV_ERR_SHAPE, "delta rule: %d state slots for %d sequences", a->n_slots, a->n_seq);
  if ((a->flags & EVCONV_DELTA_RAW_GATES) && (!a->a_scale || !a->dt_bias)) return refuse(EVCONV_ERR_INVALID_ARG, "delta rule: raw gates without a_scale or dt_bias");
  if (a->n_tokens && (!a->q.data || !a->k.data || !a->v.data || !a->gate.data || !a->beta.data || !a->o)) return refuse(EVCONV_ERR_INVALID_ARG, "delta rule: null tensor");
  DeltaPlan& d = *out;
  d.p = DeltaParams{};
  d.p.a = *a;
  d.p.share = a->heads_v / a->heads_k;
  d.p.len = a->seq_offsets ? -1 : (int)(a->n_tokens / a->n_seq);
  d.p.dkp = a->d_k <= 64 ? 64 : a->d_k <= 128 ? 128 : 256;
  if (a->dtype == EVCONV_F32 && a->d_k <= 128) d.p.dkp = (a->d_k + 31) / 32 * 32;  // (its products are six times as many)
  d.p.vec = a->d_k % 8 == 0 && wide(a->dtype, a->q) && wide(a->dtype, a->k);
  d.p.vec_v = a->d_v % 8 == 0 && wide(a->dtype, a->v) && aligned(a->o, 8) && a->o_token_stride % 4 == 0 && a->o_head_stride % 4 == 0;
  const bool one_launch = delta_fused_supported(d.p);
  d.p.short_len = one_launch ? kShortFused : kShort;
  if (d.p.len < 0 && a->n_tokens > (int64_t)d.p.short_len * a->n_seq) d.p.short_len = kDeltaShortRagged;
  // (room for the sequences that can be in chunks, not for all: a call of single tokens with offsets has few)
  const int n = (int)a->n_tokens;
  d.p.slots_total = d.p.len >= 0 ? a->n_seq * ((d.p.len + kDeltaChunk - 1) / kDeltaChunk) : n / kDeltaChunk + std::min(a->n_seq, n / (kDeltaShortRagged + 1));
  d.steps = d.p.len < 0 || d.p.len <= d.p.short_len;
  d.chunks = d.p.len < 0 ? a->n_tokens > d.p.short_len : !d.steps;
  d.off_k = d.off_t = d.off_scal = d.off_seq = d.bytes = 0;
  d.fused = d.chunks && one_launch;
  if (d.chunks) d.bytes = plan_delta_segments(d.p, d.fused);
  if ((d.steps && delta_steps_threads(d.p) > kMostThreads) || (d.chunks && (d.fused ? delta_fused_threads(d.p) : delta_chunks_threads(d.p)) > kMostThreads))
    return refuse(EVCONV_ERR_UNSUPPORTED, "delta rule: %lld tokens of %d sequences and %d heads are more than one launch takes", (long long)a->n_tokens, a->n_seq, a->heads_v);
  if (d.chunks && !d.fused) {
    d.off_k = (d.bytes + 255) / 256 * 256;
    d.off_t = d.off_k + (size_t)d.p.slots_total * a->heads_k * delta_frag_k_bytes(a->dtype, d.p.dkp);
    d.off_scal = d.off_t + (size_t)d.p.slots_total * a->heads_v * delta_frag_t_bytes(a->dtype);
    d.off_seq = d.off_scal + (size_t)d.p.slots_total * a->heads_v * kDeltaScalars * sizeof(float);
    d.bytes = d.off_seq + (d.p.len < 0 ? (size_t)d.p.slots_total * sizeof(int) : 0);
  }
  return EVCONV_OK;
}

evconv_status check_norm(const evconv_norm_args* a) {
  if (!a) return refuse(EVCONV_ERR_INVALID_ARG, "block norm: null arguments");
  if (a->abi_version != EVCONV_OPS_ABI_VERSION) return refuse(EVCONV_ERR_BAD_DESC, "block norm: abi_version %d, expected %d", a->abi_version, EVCONV_OPS_ABI_VERSION);
  if (!float_type(a->dtype)) return refuse(EVCONV_ERR_INVALID_ARG, "block norm: dtype %d", a->dtype);
  if (a->norm != EVCONV_NORM_RMS && a->norm != EVCONV_NORM_LAYER) return refuse(EVCONV_ERR_INVALID_ARG, "block norm: norm %d", a->norm);
  if (a->gate_act < EVCONV_GATE_NONE || a->gate_act > EVCONV_GATE_SILU) return refuse(EVCONV_ERR_INVALID_ARG, "block norm: gate_act %d", a->gate_act);
  if (a->rows < 0 || a->dim < 1 || a->group < 1 || a->dim % a->group) return refuse(EVCONV_ERR_SHAPE, "block norm: %lld rows of %d in groups of %d", (long long)a->rows, a->dim, a->group);
  if (a->rows >= 1ll << 31 || a->dim > 16384 || (a->group != a->dim && (a->group < 8 || a->group > 512)) || block_norm_vectors(*a) > kNormVectors)
    return refuse(EVCONV_ERR_UNSUPPORTED, "block norm: %lld rows of %d in groups of %d", (long long)a->rows, a->dim, a->group);
  if (!(a->eps >= 0.0f)) return refuse(EVCONV_ERR_INVALID_ARG, "block norm: eps %g", a->eps);
  if (!a->rows) return EVCONV_OK;
  if (!a->x && !a->branch) return refuse(EVCONV_ERR_INVALID_ARG, "block norm: neither x nor branch");
  if (!a->x_out && !a->h_out && !a->q) return refuse(EVCONV_ERR_INVALID_ARG, "block norm: no output");
  if ((a->gate != nullptr) != (a->gate_act != EVCONV_GATE_NONE)) return refuse(EVCONV_ERR_INVALID_ARG, "block norm: gate_act %d %s a gate", a->gate_act, a->gate ? "beside" : "without");
  if (!a->branch && (a->gate || a->post_weight || a->post_bias || a->res_scale)) return refuse(EVCONV_ERR_INVALID_ARG, "block norm: gate, weight or scale of a branch that is null");
  if (!a->pre_norm && (a->pre_weight || a->pre_bias)) return refuse(EVCONV_ERR_INVALID_ARG, "block norm: weights of a norm that is off");
  if (a->q) {
    if (!a->q_scale) return refuse(EVCONV_ERR_INVALID_ARG, "block norm: q without q_scale");
    if (a->q_stride % 128 || a->q_stride < a->dim || a->q_stride >= (int64_t)a->dim + 128 || !aligned(a->q, 16))
      return refuse(EVCONV_ERR_SHAPE, "block norm: q rows of %lld bytes for %d values", (long long)a->q_stride, a->dim);
  }
  return EVCONV_OK;
}

evconv_status check_quant(const evconv_quant_args* a) {
  if (!a) return refuse(EVCONV_ERR_INVALID_ARG, "quantised product: null arguments");
  if (a->abi_version != EVCONV_OPS_ABI_VERSION) return refuse(EVCONV_ERR_BAD_DESC, "quantised product: abi_version %d, expected %d", a->abi_version, EVCONV_OPS_ABI_VERSION);
  if (!float_type(a->dtype)) return refuse(EVCONV_ERR_INVALID_ARG, "quantised product: dtype %d", a->dtype);
  if (a->act < EVCONV_ACT_NONE || a->act > EVCONV_ACT_TANH) return refuse(EVCONV_ERR_INVALID_ARG, "quantised product: act %d", a->act);
  if (a->m < 0 || a->n < 1 || a->k < 1) return refuse(EVCONV_ERR_SHAPE, "quantised product: %lld x %d x %d", (long long)a->m, a->n, a->k);
  if (a->m >= 1ll << 31 || a->k > 131072 || a->n > 1 << 24 || ((a->m + 255) / 256) * ((a->n + 255) / 256) * 512 > kMostThreads) return refuse(EVCONV_ERR_UNSUPPORTED, "quantised product: %lld x %d x %d", (long long)a->m, a->n, a->k);
  if (!a->m) return EVCONV_OK;
  if (!a->a || !a->b || !a->a_scale || !a->b_scale || !a->y) return refuse(EVCONV_ERR_INVALID_ARG, "quantised product: null tensor");
  const int64_t row = (a->k + 127) / 128 * 128;
  if (a->a_stride % 128 || a->b_stride % 128 || a->a_stride < row || a->b_stride < row || !aligned(a->a, 16) || !aligned(a->b, 16))
    return refuse(EVCONV_ERR_SHAPE, "quantised product: rows of %lld and %lld bytes for %d values", (long long)a->a_stride, (long long)a->b_stride, a->k);
  if (a->y_stride < a->n) return refuse(EVCONV_ERR_SHAPE, "quantised product: y rows of %lld for %d columns", (long long)a->y_stride, a->n);
  return EVCONV_OK;
}

}  // namespace

extern "C" {

evconv_status evconv_delta_rule_workspace(const evconv_delta_args* args, size_t* bytes) {
  if (!bytes) return refuse(EVCONV_ERR_INVALID_ARG, "delta rule: null bytes");
  DeltaPlan d;
  const evconv_status st = plan_delta(args, &d);
  if (st == EVCONV_OK) *bytes = d.bytes;
  return st;
}

evconv_status evconv_delta_rule(const evconv_delta_args* args, void* workspace, size_t workspace_bytes, void* hip_stream) {
  DeltaPlan d;
  const evconv_status st = plan_delta(args, &d);
  if (st != EVCONV_OK) return st;
  if (d.bytes && (!workspace || workspace_bytes < d.bytes || !aligned(workspace, 256)))
    return refuse(EVCONV_ERR_WORKSPACE, "delta rule: needs %zu bytes of workspace at a multiple of 256, got %zu", d.bytes, workspace ? workspace_bytes : 0);
  if (d.chunks && d.p.segs > 1) place_delta_segments(d.p, (char*)workspace);
  if (d.chunks && !d.fused) {
    d.p.frag_k = (char*)workspace + d.off_k;
    d.p.frag_t = (char*)workspace + d.off_t;
    d.p.scal = (float*)((char*)workspace + d.off_scal);
    if (d.p.len < 0) d.p.slot_seq = (int*)((char*)workspace + d.off_seq);
  }
  if (d.steps && (args->n_tokens || args->state_out)) launch_delta_steps(d.p, (hipStream_t)hip_stream);
  if (d.fused) launch_delta_fused(d.p, (hipStream_t)hip_stream);
  else if (d.chunks) launch_delta_chunks(d.p, (hipStream_t)hip_stream);
  return launched("delta rule");
}

evconv_status evconv_block_norm(const evconv_norm_args* args, void* hip_stream) {
  const evconv_status st = check_norm(args);
  if (st != EVCONV_OK || !args->rows) return st;
  const evconv_norm_args& a = *args;
  auto fits = [&](const void* p, int64_t stride) { return !p || wide(a.dtype, p, stride); };
  const bool vec = a.group % 8 == 0 && fits(a.x, a.x_stride) && fits(a.branch, a.branch_stride) && fits(a.gate, a.gate_stride) &&
                   fits(a.x_out, a.x_out_stride) && fits(a.h_out, a.h_out_stride) && aligned(a.post_weight, 16) && aligned(a.post_bias, 16) &&
                   aligned(a.res_scale, 16) && aligned(a.pre_weight, 16) && aligned(a.pre_bias, 16);
  launch_block_norm(a, vec, (hipStream_t)hip_stream);
  return launched("block norm");
}

evconv_status evconv_quant_matmul(const evconv_quant_args* args, void* hip_stream) {
  const evconv_status st = check_quant(args);
  if (st != EVCONV_OK || !args->m) return st;
  launch_quant_matmul(*args, (hipStream_t)hip_stream);
  return launched("quantised product");
}

}  // extern "C"
