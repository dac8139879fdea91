// seq_api.hip -- the entry points of include/ntk_seq.h: argument checks and launches.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdio.h>

#include "seq/attn_cached.hpp"
#include "seq/launch_attn.hpp"
#include "seq/launch_cache.hpp"
#include "seq/launch_seq.hpp"
#include "ntk_seq.h"

namespace ntk {
int call_error(int code, const char* what) noexcept;   // ntk_api.hip: the message of ntk_last_error(NULL)
}

namespace {

using namespace ntk;

int bad(int code, const char* what) { return call_error(code, what); }
int hip_bad(hipError_t e) {
  char what[160];
  snprintf(what, sizeof what, "kernel launch: %s", hipGetErrorString(e));
  return bad(NTK_E_HIP, what);
}

int elem(int dtype) { return dtype == NTK_F32 ? 4 : 2; }
bool type_ok(int dtype) { return dtype == NTK_F32 || dtype == NTK_BF16 || dtype == NTK_F16; }
bool whole16(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool aligned(const void* p, int e) { return ((uintptr_t)p & (uintptr_t)(e - 1)) == 0; }
// a grid of `blocks` workgroups of `threads` fits a launch
bool grid_ok(long long blocks, int threads) { return blocks < (1LL << 31) && blocks * threads < (1LL << 32); }

int norm_args(int dtype, int wtype, long long rows, int width, float eps) {
  if (!type_ok(dtype)) return bad(NTK_E_ARG, "rms_norm: dtype");
  if (wtype != dtype && wtype != NTK_F32) return bad(NTK_E_ARG, "rms_norm: wtype is dtype or NTK_F32");
  if (rows < 0 || width < 1) return bad(NTK_E_ARG, "rms_norm: rows < 0 or width < 1");
  if (!(eps >= 0.f)) return bad(NTK_E_ARG, "rms_norm: eps < 0");
  if (width > 32768) return bad(NTK_E_UNSUPPORTED, "rms_norm: width over 32768");
  return NTK_OK;
}

bool view_ok(const ntk_view* v, int e) {
  return v && v->data && aligned(v->data, e) && v->stride_batch >= 0 && v->stride_position >= 0 && v->stride_head >= 0;
}
bool view_vec(const ntk_view* v, int e) {
  const long long k = 16 / e;
  return whole16(v->data) && v->stride_batch % k == 0 && v->stride_position % k == 0 && v->stride_head % k == 0;
}
// An output's elements share no memory: a stride below the head size would lay rows over each other.
bool apart(const ntk_view* v, int batch, int positions, int heads, int dim) {
  return (batch == 1 || v->stride_batch >= dim) && (positions == 1 || v->stride_position >= dim) && (heads == 1 || v->stride_head >= dim);
}
bool same_place(const ntk_view* a, const ntk_view* b) { return a->data == b->data; }

// Checks a descriptor for the pass asked for; `plan` as the forward pass runs it.  `cached`: over pages, which has a plan of its own.
int attn_args(const ntk_attention_desc* d, AttnPlan* plan, bool backward, bool cached = false) {
  if (!d) return bad(NTK_E_ARG, "attention: the descriptor is NULL");
  if (!type_ok(d->dtype)) return bad(NTK_E_ARG, "attention: dtype");
  if (d->batch < 0 || d->q_len < 0 || d->k_len < 0) return bad(NTK_E_ARG, "attention: batch, q_len or k_len < 0");
  if (d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads)
    return bad(NTK_E_SHAPE, "attention: heads must be a multiple of kv_heads, both > 0");
  if (d->head_dim < 1) return bad(NTK_E_ARG, "attention: head_dim < 1");
  if (d->head_dim > 128) return bad(NTK_E_UNSUPPORTED, "attention: head_dim over 128");
  if (!(d->scale > 0.f) || !isfinite(d->scale)) return bad(NTK_E_ARG, "attention: scale must be positive and finite");
  if (!(d->softcap >= 0.f) || !isfinite(d->softcap)) return bad(NTK_E_ARG, "attention: softcap must be >= 0 and finite");
  // the kernels' constants: scale log2(e), softcap log2(e) and 2 scale log2(e) / softcap
  if (!isfinite(d->scale * kLog2e) || !isfinite(d->softcap * kLog2e) || (d->softcap > 0.f && !isfinite(2.f * kLog2e * d->scale / d->softcap)))
    return bad(NTK_E_ARG, "attention: scale, softcap or scale / softcap leaves fp32's range in units of log2");
  if (d->prefix && !d->causal) return bad(NTK_E_ARG, "attention: a prefix needs causal");
  // rows and grids are 32-bit; a margin for the last tile
  const long long G = d->heads / d->kv_heads, R = (long long)d->q_len * G, bh = (long long)d->batch * d->kv_heads;
  if (R >= (1LL << 29) - 1024 || d->k_len >= (1LL << 31) - 1024 || bh >= (1LL << 31))
    return bad(NTK_E_UNSUPPORTED, "attention: q_len * group reaches 2^29 or k_len 2^31");
  if (cached) return NTK_OK;
  if (R > 0 && bh > 0) {
    *plan = attn_plan_fwd(d->dtype, d->batch, d->kv_heads, (int)R, d->k_len, d->head_dim);
    const int dp = d->head_dim <= 64 ? 64 : 128;
    const long long rows = bh * R, keys = bh * d->k_len, spr = 256 / (dp / 4);   // rows a workgroup of the ranges' sums
    bool fits;
    if (backward) {
      const AttnBwdPlan back = attn_plan_bwd(d->dtype, d->batch, d->kv_heads, (int)R, d->k_len, d->head_dim, d->causal != 0);
      fits = grid_ok(bh * back.dq_tiles * back.dq_splits, 256) && grid_ok(bh * back.dkv_tiles * back.dkv_splits, 256) &&
             grid_ok(rows / 16 + 1, 256) && (back.dq_splits == 1 || grid_ok(rows / spr + 1, 256)) &&
             (back.dkv_splits == 1 || grid_ok(keys / spr + 1, 256));
    } else {
      fits = grid_ok(bh * (plan->tokens ? 1 : plan->tiles) * plan->splits, 256) && (plan->splits == 1 || grid_ok(rows, dp));
    }
    if (!fits)
      return bad(NTK_E_UNSUPPORTED, "attention: too many rows for one launch");
  } else {
    *plan = AttnPlan{};
  }
  return NTK_OK;
}

AttnBwdPlan bwd_plan(const ntk_attention_desc* d) {
  return attn_plan_bwd(d->dtype, d->batch, d->kv_heads, d->q_len * (d->heads / d->kv_heads), d->k_len, d->head_dim, d->causal != 0);
}

void set_view(AttnView& to, const ntk_view* v) {
  to.p = v->data;
  to.sb = v->stride_batch;
  to.ss = v->stride_position;
  to.sh = v->stride_head;
}

void set_desc(AttnArgs& a, const ntk_attention_desc* d) {
  a.B = d->batch;
  a.Sq = d->q_len;
  a.Sk = d->k_len;
  a.H = d->heads;
  a.Hk = d->kv_heads;
  a.G = d->heads / d->kv_heads;
  a.D = d->head_dim;
  a.R = d->q_len * a.G;
  a.causal = d->causal != 0;
  a.lens = d->k_lens;
  a.prefix = d->prefix;
  a.docs = d->docs;
  a.slopes = d->slopes;
  a.scale = d->scale;
  a.c = d->scale * kLog2e;
  a.cap_in = d->softcap > 0.f ? 2.f * kLog2e * d->scale / d->softcap : 0.f;
  a.cap_out = d->softcap * kLog2e;
  a.gdiv = FastDiv((uint32_t)a.G);
  a.splits = 1;
}

// A tile of `rows` positions (times the group's heads) lies within 2 GiB of its first element.
bool span_ok(const ntk_view* v, int rows, int G, int D, int e) {
  const long long lim = (1LL << 31) - (1 << 16);
  if (v->stride_position > lim / (rows + 1) / e || v->stride_head > lim / (G + 1) / e) return false;
  return ((rows + 1) * v->stride_position + G * v->stride_head + D) * e < lim;
}

// A cache that calls of type `dtype` use; `what` names the call.
int cache_args(const ntk_cache* c, int dtype, int batch, const char* what) {
  char text[160];
  auto no = [&](int code, const char* why) {
    snprintf(text, sizeof text, "%s: %s", what, why);
    return bad(code, text);
  };
  if (!c) return no(NTK_E_ARG, "the cache is NULL");
  if (c->dtype != NTK_E4M3 && c->dtype != dtype) return no(NTK_E_ARG, "the cache's dtype is the call's or NTK_E4M3");
  if (c->pages < 0 || c->max_pages < 0) return no(NTK_E_ARG, "pages or max_pages < 0");
  if (c->page_size < 8 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)))
    return no(NTK_E_UNSUPPORTED, "page_size must be a power of two from 8 to 1024");
  if (c->kv_heads < 1) return no(NTK_E_SHAPE, "kv_heads < 1");
  if (c->head_dim < 1) return no(NTK_E_ARG, "head_dim < 1");
  if (c->head_dim > 128) return no(NTK_E_UNSUPPORTED, "head_dim over 128");
  if ((long long)c->max_pages * c->page_size >= (1LL << 31) - 1024) return no(NTK_E_UNSUPPORTED, "max_pages * page_size reaches 2^31");
  if (batch > 0 && c->max_pages > 0 && (!c->page_table || !aligned(c->page_table, 4))) return no(NTK_E_ARG, "page_table is NULL or unaligned");
  if (c->pages > 0) {
    const int e = c->dtype == NTK_E4M3 ? 1 : elem(dtype);
    if (!view_ok(&c->k, e) || !view_ok(&c->v, e)) return no(NTK_E_ARG, "the cache's k or v is missing, unaligned or has a negative stride");
    if (c->dtype == NTK_E4M3 && (!c->k_scale || !c->v_scale || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4) || c->k_scale == c->v_scale))
      return no(NTK_E_ARG, "k_scale or v_scale is NULL, unaligned, or the other one");
  }
  return NTK_OK;
}
int shift_of(int page_size) {
  int s = 0;
  while ((1 << s) < page_size) ++s;
  return s;
}
PageTable page_table(const ntk_cache* c) {
  PageTable t;
  t.table = c->page_table;
  t.most = c->max_pages;
  t.pages = c->pages;
  t.shift = shift_of(c->page_size);
  return t;
}

int logprob_args(int dtype, long long rows, int vocab, int top) {
  if (!type_ok(dtype)) return bad(NTK_E_ARG, "logprobs: dtype");
  if (rows < 0 || vocab < 1) return bad(NTK_E_ARG, "logprobs: rows < 0 or vocab < 1");
  if (top < 0 || top > vocab) return bad(NTK_E_ARG, "logprobs: top < 0 or over vocab");
  if (top > 64) return bad(NTK_E_UNSUPPORTED, "logprobs: top over 64");
  // element numbers of a row are 32-bit, with a margin for the last workgroup's
  if (vocab >= (1 << 30)) return bad(NTK_E_UNSUPPORTED, "logprobs: vocab reaches 2^30");
  if (rows >= (1LL << 31) || (rows > 0 && (!grid_ok(rows * logprob_splits(dtype, rows, vocab), 256) || !grid_ok(rows * logprob_bwd_chunks(dtype, vocab), 256))))
    return bad(NTK_E_UNSUPPORTED, "logprobs: too many rows for one launch");
  return NTK_OK;
}

}  // namespace

extern "C" int ntk_rms_norm(int dtype, int wtype, long long rows, int width, const void* x, long long x_stride,
                            const void* residual, long long residual_stride, const void* weight, float eps, void* y, void* h,
                            float* scale, void* hip_stream) {
  if (int rc = norm_args(dtype, wtype, rows, width, eps)) return rc;
  if (rows == 0) return NTK_OK;
  const int rpb = norm_rows_per_block(width);
  if (!grid_ok(rows / rpb + 1, norm_threads(width))) return bad(NTK_E_UNSUPPORTED, "rms_norm: too many rows for one launch");
  const int e = elem(dtype), we = elem(wtype);
  if (!x || !weight || !y) return bad(NTK_E_ARG, "rms_norm: x, weight or y is NULL");
  if (x_stride < width || (residual && residual_stride < width)) return bad(NTK_E_ARG, "rms_norm: a row stride is below width");
  if (!aligned(x, e) || !aligned(residual, e) || !aligned(weight, we) || (!scale && !aligned(y, e)) || !aligned(h, e) || !aligned(scale, 4))
    return bad(NTK_E_ARG, "rms_norm: a pointer is not aligned to its type");
  NormArgs a{x, residual, weight, x_stride, residual_stride, y, h, scale, rows, width, eps};
  const bool vec = width % 8 == 0 && whole16(x) && whole16(residual) && whole16(weight) && whole16(y) && whole16(h) &&
                   x_stride % 8 == 0 && (!residual || residual_stride % 8 == 0);
  const hipError_t err = launch_rms_norm((hipStream_t)hip_stream, dtype, wtype, a, vec);
  return err == hipSuccess ? NTK_OK : hip_bad(err);
}

extern "C" long long ntk_rms_norm_workspace(long long rows, int width) {
  if (rows < 0 || width < 1) return bad(NTK_E_ARG, "rms_norm: rows < 0 or width < 1");
  if (width > 32768) return bad(NTK_E_UNSUPPORTED, "rms_norm: width over 32768");
  return rows == 0 ? 0 : (long long)norm_bwd_parts(rows, width) * width * 4;
}

extern "C" int ntk_rms_norm_bwd(int dtype, int wtype, long long rows, int width, const void* dy, long long dy_stride, const void* h,
                                long long h_stride, const void* weight, const void* dh, long long dh_stride, float eps, void* dx,
                                void* dweight, void* workspace, long long workspace_bytes, void* hip_stream) {
  if (int rc = norm_args(dtype, wtype, rows, width, eps)) return rc;
  if (!dweight) return bad(NTK_E_ARG, "rms_norm_bwd: dweight is NULL");
  const int e = elem(dtype), we = elem(wtype);
  if (rows > 0) {
    if (!dy || !h || !weight || !dx) return bad(NTK_E_ARG, "rms_norm_bwd: dy, h, weight or dx is NULL");
    if (dy_stride < width || h_stride < width || (dh && dh_stride < width))
      return bad(NTK_E_ARG, "rms_norm_bwd: a row stride is below width");
    if (!workspace || !whole16(workspace) || workspace_bytes < ntk_rms_norm_workspace(rows, width))
      return bad(NTK_E_ARG, "rms_norm_bwd: the workspace is missing, unaligned or too small");
  }
  if (!aligned(dy, e) || !aligned(h, e) || !aligned(weight, we) || !aligned(dh, e) || !aligned(dx, e) || !aligned(dweight, we))
    return bad(NTK_E_ARG, "rms_norm_bwd: a pointer is not aligned to its type");
  NormBwdArgs a{dy, h, dh, weight, dy_stride, h_stride, dh_stride, dx, dweight, (float*)workspace, rows, width, eps};
  const bool vec = width % 8 == 0 && whole16(dy) && whole16(h) && whole16(weight) && whole16(dh) && whole16(dx) &&
                   dy_stride % 8 == 0 && h_stride % 8 == 0 && (!dh || dh_stride % 8 == 0);
  const hipError_t err = launch_rms_norm_bwd((hipStream_t)hip_stream, dtype, wtype, a, vec);
  return err == hipSuccess ? NTK_OK : hip_bad(err);
}

extern "C" int ntk_rotary_table(int max_pos, int rot, double base, const ntk_rotary_scaling* scaling, float* table,
                                void* hip_stream) {
  if (max_pos < 1 || rot < 2 || rot % 2) return bad(NTK_E_ARG, "rotary_table: max_pos < 1, or rot odd or < 2");
  if (!(base > 1.0) || !isfinite(base)) return bad(NTK_E_ARG, "rotary_table: base must be over 1");
  if (!table || !aligned(table, 4)) return bad(NTK_E_ARG, "rotary_table: table is NULL or unaligned");
  RotaryTableArgs a{table, max_pos, rot, NTK_ROTARY_PLAIN, base, 1.0, 1.0, 0.0, 1.0};
  if (scaling && scaling->kind != NTK_ROTARY_PLAIN) {
    a.scaling = scaling->kind;
    a.factor = scaling->factor;
    if (a.scaling < 0 || a.scaling > NTK_ROTARY_RAMP) return bad(NTK_E_ARG, "rotary_table: unknown scaling");
    if (!(a.factor >= 1.0) || !isfinite(a.factor)) return bad(NTK_E_ARG, "rotary_table: factor must be >= 1");
    if (a.scaling == NTK_ROTARY_RAMP) {
      a.original = scaling->original;
      a.lo = scaling->low;
      a.hi = scaling->high;
      if (!(a.original >= 1.0) || !(a.lo >= 0.0) || !(a.hi > a.lo) || !isfinite(a.original) || !isfinite(a.hi))
        return bad(NTK_E_ARG, "rotary_table: the ramp needs original >= 1 and 0 <= low < high");
    }
  }
  if (!grid_ok(((long long)max_pos * (rot / 2) + 255) / 256, 256)) return bad(NTK_E_UNSUPPORTED, "rotary_table: too large");
  const hipError_t err = launch_rotary_table((hipStream_t)hip_stream, a);
  return err == hipSuccess ? NTK_OK : hip_bad(err);
}

extern "C" int ntk_rotary(int dtype, int batch, int length, int q_heads, int k_heads, int dim, int rot, int interleaved,
                          int inverse, const ntk_view* q, const ntk_view* k, const float* table, int max_pos, const int* positions,
                          int first_position, const ntk_view* q_out, const ntk_view* k_out, void* hip_stream) {
  if (!type_ok(dtype)) return bad(NTK_E_ARG, "rotary: dtype");
  if (batch < 0 || length < 0 || q_heads < 0 || k_heads < 0 || dim < 1) return bad(NTK_E_ARG, "rotary: a size is negative");
  if (rot < 2 || rot % 2 || rot > dim) return bad(NTK_E_SHAPE, "rotary: rot must be even, 2 <= rot <= dim");
  if (!k) k_heads = 0;
  if (max_pos < 1 || !table || !aligned(table, 4) || !aligned(positions, 4)) return bad(NTK_E_ARG, "rotary: table or positions");
  if (!positions && (first_position < 0 || first_position > 2147483647 - length)) return bad(NTK_E_ARG, "rotary: first_position");
  const long long heads = (long long)q_heads + k_heads;
  if (batch == 0 || length == 0 || heads == 0) return NTK_OK;
  const int e = elem(dtype);
  if ((q_heads && (!view_ok(q, e) || !view_ok(q_out, e))) || (k_heads && (!view_ok(k, e) || !view_ok(k_out, e))))
    return bad(NTK_E_ARG, "rotary: a view is missing, unaligned or has a negative stride");
  const long long rows = (long long)batch * length, items = heads * (dim / 16 + 2);
  if (rows >= (1LL << 31) || heads >= (1LL << 20) || items >= (1LL << 20)) return bad(NTK_E_UNSUPPORTED, "rotary: too large for one launch");
  RotaryArgs a{};
  bool vec = rot % 16 == 0 && dim % 8 == 0 && whole16(table);
  const ntk_view* in[2] = {q, k};
  const ntk_view* out[2] = {q_out, k_out};
  const int n[2] = {q_heads, k_heads};
  for (int i = 0; i < 2; ++i) {
    a.heads[i] = n[i];
    if (!n[i]) continue;
    if (!apart(out[i], batch, length, n[i], dim) || (n[1 - i] && (same_place(out[i], out[1 - i]) || same_place(out[i], in[1 - i]))))
      return bad(NTK_E_ARG, "rotary: an output overlaps itself or another array");
    a.x[i] = in[i]->data;
    a.xb[i] = in[i]->stride_batch;
    a.xs[i] = in[i]->stride_position;
    a.xh[i] = in[i]->stride_head;
    a.y[i] = out[i]->data;
    a.yb[i] = out[i]->stride_batch;
    a.ys[i] = out[i]->stride_position;
    a.yh[i] = out[i]->stride_head;
    vec = vec && view_vec(in[i], e) && view_vec(out[i], e);
  }
  a.table = table;
  a.positions = positions;
  a.first = first_position;
  a.max_pos = max_pos;
  a.batch = batch;
  a.length = length;
  a.dim = dim;
  a.rot = rot;
  a.interleaved = interleaved != 0;
  a.sign = inverse ? -1.f : 1.f;
  if (!grid_ok(rotary_blocks(a), 256)) return bad(NTK_E_UNSUPPORTED, "rotary: too large for one launch");
  const hipError_t err = launch_rotary((hipStream_t)hip_stream, dtype, a, vec);
  return err == hipSuccess ? NTK_OK : hip_bad(err);
}

extern "C" long long ntk_attention_workspace(const ntk_attention_desc* desc, int backward) {
  AttnPlan plan;
  if (int rc = attn_args(desc, &plan, backward != 0)) return rc;
  if (!backward) return (plan.part_floats + plan.flag_ints) * 4;
  const AttnBwdPlan back = bwd_plan(desc);
  return (back.part_floats + back.flag_ints + 2 * (long long)desc->batch * desc->heads * desc->q_len) * 4;
}

extern "C" int ntk_attention(const ntk_attention_desc* desc, const ntk_view* q, const ntk_view* k, const ntk_view* v,
                             const ntk_view* o, float* lse, void* workspace, long long workspace_bytes, void* hip_stream) {
  AttnPlan plan;
  if (int rc = attn_args(desc, &plan, false)) return rc;
  if (desc->batch == 0 || desc->q_len == 0) return NTK_OK;
  const int e = elem(desc->dtype), G = desc->heads / desc->kv_heads;
  if (!view_ok(q, e) || !view_ok(o, e) || (desc->k_len && (!view_ok(k, e) || !view_ok(v, e))))
    return bad(NTK_E_ARG, "attention: a view is missing, unaligned or has a negative stride");
  if (!aligned(lse, 4) || !aligned(desc->k_lens, 4) || !aligned(desc->prefix, 4) || !aligned(desc->docs, 4) || !aligned(desc->slopes, 4))
    return bad(NTK_E_ARG, "attention: a pointer is not aligned to its type");
  const long long need = (plan.part_floats + plan.flag_ints) * 4;
  if (need && (!workspace || !whole16(workspace) || workspace_bytes < need))
    return bad(NTK_E_ARG, "attention: the workspace is missing, unaligned or too small");
  if (!apart(o, desc->batch, desc->q_len, desc->heads, desc->head_dim) || same_place(o, q) ||
      (desc->k_len && (same_place(o, k) || same_place(o, v))))
    return bad(NTK_E_ARG, "attention: o overlaps itself, q, k or v");
  AttnArgs a{};
  set_desc(a, desc);
  set_view(a.q, q);
  set_view(a.o, o);
  bool vec = desc->head_dim * e % 16 == 0 && view_vec(q, e) && view_vec(o, e);
  if (desc->k_len) {
    set_view(a.k, k);
    set_view(a.v, v);
    vec = vec && view_vec(k, e) && view_vec(v, e) && span_ok(k, 128, 0, desc->head_dim, e) && span_ok(v, 128, 0, desc->head_dim, e);
  }
  a.lse = lse;
  a.part = (float*)workspace;
  a.flags = (int*)workspace + plan.part_floats;
  a.tiles = plan.tiles;
  a.splits = plan.splits;
  const hipError_t err = launch_attn_fwd((hipStream_t)hip_stream, desc->dtype, a, plan.tokens, vec);
  return err == hipSuccess ? NTK_OK : hip_bad(err);
}

extern "C" int ntk_attention_bwd(const ntk_attention_desc* desc, const ntk_view* dout, const ntk_view* q, const ntk_view* k,
                                 const ntk_view* v, const ntk_view* o, const float* lse, const ntk_view* dq, const ntk_view* dk,
                                 const ntk_view* dv, void* workspace, long long workspace_bytes, void* hip_stream) {
  AttnPlan plan;
  if (int rc = attn_args(desc, &plan, true)) return rc;
  if (desc->batch == 0) return NTK_OK;
  const int e = elem(desc->dtype), G = desc->heads / desc->kv_heads;
  const ntk_view* views[8] = {dout, q, o, dq, k, v, dk, dv};   // four of the queries' axis, four of the keys'
  bool vec = desc->head_dim * e % 16 == 0;
  for (int i = 0; i < 8; ++i) {
    if ((i < 4 ? desc->q_len : desc->k_len) == 0) continue;
    if (!view_ok(views[i], e)) return bad(NTK_E_ARG, "attention_bwd: a view is missing, unaligned or has a negative stride");
    vec = vec && view_vec(views[i], e) && span_ok(views[i], 128, G, desc->head_dim, e);
  }
  if ((desc->q_len && !lse) || !aligned(lse, 4) || !aligned(desc->k_lens, 4) || !aligned(desc->prefix, 4) || !aligned(desc->docs, 4) || !aligned(desc->slopes, 4))
    return bad(NTK_E_ARG, "attention_bwd: lse is NULL, or a pointer is not aligned to its type");
  const long long need = ntk_attention_workspace(desc, 1);
  if (need && (!workspace || !whole16(workspace) || workspace_bytes < need))
    return bad(NTK_E_ARG, "attention_bwd: the workspace is missing, unaligned or too small");
  for (const int out : {3, 6, 7}) {                             // dq, dk, dv
    const bool keys = out > 3;
    if ((keys ? desc->k_len : desc->q_len) == 0) continue;
    bool clear = apart(views[out], desc->batch, keys ? desc->k_len : desc->q_len, keys ? desc->kv_heads : desc->heads, desc->head_dim);
    for (int i = 0; i < 8; ++i)
      clear = clear && (i == out || (i < 4 ? desc->q_len : desc->k_len) == 0 || !same_place(views[out], views[i]));
    if (!clear) return bad(NTK_E_ARG, "attention_bwd: dq, dk or dv overlaps itself or another array");
  }
  AttnArgs a{};
  set_desc(a, desc);
  if (desc->q_len) {
    set_view(a.dout, dout);
    set_view(a.q, q);
    set_view(a.o, o);
    set_view(a.dq, dq);
  }
  if (desc->k_len) {
    set_view(a.k, k);
    set_view(a.v, v);
    set_view(a.dk, dk);
    set_view(a.dv, dv);
  }
  a.lse = const_cast<float*>(lse);
  const hipError_t err = launch_attn_bwd((hipStream_t)hip_stream, desc->dtype, a, bwd_plan(desc), (float*)workspace, vec);
  return err == hipSuccess ? NTK_OK : hip_bad(err);
}

extern "C" int ntk_cache_append(int dtype, int batch, int length, int q_heads, const ntk_cache* cache, const int* lens,
                                const int* new_lens, const ntk_view* k, const ntk_view* v, const ntk_view* q, const ntk_view* q_out,
                                const float* table, int max_pos, int rot, int interleaved, const int* positions, void* hip_stream) {
  if (!type_ok(dtype)) return bad(NTK_E_ARG, "cache_append: dtype");
  if (batch < 0 || length < 0 || q_heads < 0) return bad(NTK_E_ARG, "cache_append: a size is negative");
  if (int rc = cache_args(cache, dtype, batch, "cache_append")) return rc;
  const int dim = cache->head_dim, kv = cache->kv_heads, e = elem(dtype);
  const bool e4m3 = cache->dtype == NTK_E4M3;
  if (rot < 0 || rot % 2 || rot > dim) return bad(NTK_E_SHAPE, "cache_append: rot must be even, 0 <= rot <= head_dim");
  if (rot && (max_pos < 1 || !table || !aligned(table, 4))) return bad(NTK_E_ARG, "cache_append: table is NULL or unaligned, or max_pos < 1");
  if (!q) q_heads = 0;
  if (batch == 0 || length == 0) return NTK_OK;
  if (!lens || !aligned(lens, 4) || !aligned(new_lens, 4) || !aligned(positions, 4))
    return bad(NTK_E_ARG, "cache_append: lens is NULL, or a pointer is not aligned to its type");
  if (!view_ok(k, e) || !view_ok(v, e) || (q_heads && (!view_ok(q, e) || !view_ok(q_out, e))))
    return bad(NTK_E_ARG, "cache_append: a view is missing, unaligned or has a negative stride");
  if (cache->pages > 0) {
    const ntk_view* cells[2] = {&cache->k, &cache->v};
    for (const ntk_view* c : cells)
      if (!apart(c, cache->pages, cache->page_size, kv, dim) || same_place(c, k) || same_place(c, v) || (q_heads && (same_place(c, q) || same_place(c, q_out))))
        return bad(NTK_E_ARG, "cache_append: the cache overlaps itself or another array");
    if (same_place(cells[0], cells[1])) return bad(NTK_E_ARG, "cache_append: the cache overlaps itself or another array");
  }
  if (q_heads && (!apart(q_out, batch, length, q_heads, dim) || same_place(q_out, q) || same_place(q_out, k) || same_place(q_out, v)))
    return bad(NTK_E_ARG, "cache_append: q_out overlaps itself or another array");
  const long long rows = (long long)batch * length, heads = (long long)q_heads + 2LL * kv;
  if (rows >= (1LL << 31) || heads * (dim / 16 + 2) >= (1LL << 20) || (long long)cache->max_pages * cache->page_size + length >= (1LL << 31) - 1024)
    return bad(NTK_E_UNSUPPORTED, "cache_append: too large for one launch");
  AppendArgs a{};
  const ntk_view* in[3] = {q_heads ? q : k, k, v};
  bool vec = dim % 8 == 0 && rot % 16 == 0 && whole16(table);
  for (int i = 0; i < 3; ++i) {
    a.x[i] = in[i]->data;
    a.xb[i] = in[i]->stride_batch;
    a.xs[i] = in[i]->stride_position;
    a.xh[i] = in[i]->stride_head;
    vec = vec && view_vec(in[i], e);
  }
  if (q_heads) {
    a.qo = q_out->data;
    a.qb = q_out->stride_batch;
    a.qs = q_out->stride_position;
    a.qh = q_out->stride_head;
    vec = vec && view_vec(q_out, e);
  }
  const ntk_view* cells[2] = {&cache->k, &cache->v};
  for (int i = 0; i < 2 && cache->pages > 0; ++i) {
    a.cell[i] = cells[i]->data;
    a.cb[i] = cells[i]->stride_batch;
    a.cs[i] = cells[i]->stride_position;
    a.ch[i] = cells[i]->stride_head;
    vec = vec && view_vec(cells[i], e4m3 ? 1 : e);
  }
  a.scale[0] = e4m3 ? cache->k_scale : nullptr;
  a.scale[1] = e4m3 ? cache->v_scale : nullptr;
  a.quantize = e4m3;
  a.pages = page_table(cache);
  a.lens = lens;
  a.news = new_lens;
  a.positions = positions;
  a.table = table;
  a.max_pos = max_pos;
  a.rot = rot;
  a.interleaved = interleaved != 0;
  a.batch = batch;
  a.length = length;
  a.heads = q_heads;
  a.kv_heads = kv;
  a.dim = dim;
  const long long blocks = append_blocks(a);
  if (blocks == 0) return NTK_OK;
  if (!grid_ok(blocks, 256) || (long long)batch * append_pages(length, a.pages.shift) >= (1LL << 31))
    return bad(NTK_E_UNSUPPORTED, "cache_append: too large for one launch");
  const hipError_t err = launch_append((hipStream_t)hip_stream, dtype, a, vec);
  return err == hipSuccess ? NTK_OK : hip_bad(err);
}

namespace {

int cached_args(const ntk_attention_desc* d, int cells, CachedPlan* plan) {
  if (!d) return bad(NTK_E_ARG, "attention_cached: the descriptor is NULL");
  if (cells != NTK_E4M3 && cells != d->dtype) return bad(NTK_E_ARG, "attention_cached: the cache's dtype is the call's or NTK_E4M3");
  if (d->prefix || d->docs) return bad(NTK_E_ARG, "attention_cached: prefix and docs must be NULL");
  if (int rc = attn_args(d, nullptr, false, true)) return rc;
  *plan = CachedPlan{};
  if (d->batch == 0 || d->q_len == 0) return NTK_OK;
  *plan = attn_plan_cached(d->dtype, cells == NTK_E4M3, d->batch, d->kv_heads, d->q_len * (d->heads / d->kv_heads), d->k_len, d->head_dim);
  if (!grid_ok(plan->blocks, 256)) return bad(NTK_E_UNSUPPORTED, "attention_cached: too many rows for one launch");
  return NTK_OK;
}

}  // namespace

extern "C" long long ntk_attention_cached_workspace(const ntk_attention_desc* desc, int cache_dtype) {
  CachedPlan plan;
  if (int rc = cached_args(desc, cache_dtype, &plan)) return rc;
  return (plan.part_floats + plan.ints) * 4;
}

extern "C" int ntk_attention_cached(const ntk_attention_desc* desc, const ntk_cache* cache, const int* q_lens, const ntk_view* q,
                                    const ntk_view* o, float* lse, void* workspace, long long workspace_bytes, void* hip_stream) {
  CachedPlan plan;
  if (!cache) return bad(NTK_E_ARG, "attention_cached: the cache is NULL");
  if (int rc = cached_args(desc, cache->dtype, &plan)) return rc;
  if (int rc = cache_args(cache, desc->dtype, desc->batch, "attention_cached")) return rc;
  if (cache->kv_heads != desc->kv_heads || cache->head_dim != desc->head_dim || (long long)cache->max_pages * cache->page_size != desc->k_len)
    return bad(NTK_E_SHAPE, "attention_cached: kv_heads, head_dim or k_len is not the cache's");
  if (desc->batch == 0 || desc->q_len == 0) return NTK_OK;
  const bool e4m3 = cache->dtype == NTK_E4M3;
  const int e = elem(desc->dtype);
  if (!view_ok(q, e) || !view_ok(o, e)) return bad(NTK_E_ARG, "attention_cached: a view is missing, unaligned or has a negative stride");
  if (!desc->k_lens || !aligned(desc->k_lens, 4) || !aligned(q_lens, 4) || !aligned(lse, 4) || !aligned(desc->slopes, 4))
    return bad(NTK_E_ARG, "attention_cached: k_lens is NULL, or a pointer is not aligned to its type");
  const long long need = (plan.part_floats + plan.ints) * 4;
  if (need && (!workspace || !whole16(workspace) || workspace_bytes < need))
    return bad(NTK_E_ARG, "attention_cached: the workspace is missing, unaligned or too small");
  if (!apart(o, desc->batch, desc->q_len, desc->heads, desc->head_dim) || same_place(o, q) ||
      (cache->pages > 0 && (same_place(o, &cache->k) || same_place(o, &cache->v))))
    return bad(NTK_E_ARG, "attention_cached: o overlaps itself, q or the cache");
  CachedArgs a{};
  set_desc(a, desc);
  set_view(a.q, q);
  set_view(a.o, o);
  bool vec = desc->head_dim * (e4m3 ? 1 : e) % 16 == 0 && view_vec(q, e) && view_vec(o, e);
  if (cache->pages > 0) {
    set_view(a.k, &cache->k);
    set_view(a.v, &cache->v);
    const int ce = e4m3 ? 1 : e;
    for (const ntk_view* c : {&cache->k, &cache->v}) vec = vec && view_vec(c, ce) && narrow_slots(c->stride_position, ce, cache->page_size);
  }
  a.k_scale = cache->k_scale;
  a.v_scale = cache->v_scale;
  a.q_lens = q_lens;
  a.pages = page_table(cache);
  a.lse = lse;
  a.part = (float*)workspace;
  a.heads = (int*)workspace + plan.part_floats;
  a.flags = a.heads + 4LL * plan.workers;
  a.tiles = plan.tiles;
  a.workers = plan.workers;
  a.least = plan.least;
  const hipError_t err = launch_attn_cached((hipStream_t)hip_stream, desc->dtype, a, e4m3, plan.waves, vec);
  return err == hipSuccess ? NTK_OK : hip_bad(err);
}

extern "C" long long ntk_logprobs_workspace(int dtype, long long rows, int vocab, int top) {
  if (int rc = logprob_args(dtype, rows, vocab, top)) return rc;
  return logprob_work_bytes(rows, top, logprob_splits(dtype, rows, vocab));
}

extern "C" int ntk_logprobs(int dtype, long long rows, int vocab, const void* logits, long long stride, const int* tokens, float scale,
                            int top, float* logp, float* entropy, float* lse, float* top_logp, int* top_tokens, void* workspace,
                            long long workspace_bytes, void* hip_stream) {
  if (int rc = logprob_args(dtype, rows, vocab, top)) return rc;
  if (!(scale > 0.f) || !isfinite(scale * kLog2e)) return bad(NTK_E_ARG, "logprobs: scale must be positive and finite");
  if (rows == 0) return NTK_OK;
  if (!logits || !tokens || !logp || (top && (!top_logp || !top_tokens))) return bad(NTK_E_ARG, "logprobs: an array is NULL");
  if (stride < vocab) return bad(NTK_E_ARG, "logprobs: the row stride is below vocab");
  for (const void* p : {(const void*)tokens, (const void*)logp, (const void*)entropy, (const void*)lse, (const void*)top_logp, (const void*)top_tokens})
    if (!aligned(p, 4)) return bad(NTK_E_ARG, "logprobs: a pointer is not aligned to its type");
  if (!aligned(logits, elem(dtype))) return bad(NTK_E_ARG, "logprobs: a pointer is not aligned to its type");
  LogprobArgs a{logits, stride, tokens, logp, entropy, lse, top_logp, top_tokens, workspace, rows, vocab, top,
                logprob_splits(dtype, rows, vocab), scale};
  const long long need = logprob_work_bytes(rows, top, a.splits);
  if (need && (!workspace || !whole16(workspace) || workspace_bytes < need))
    return bad(NTK_E_ARG, "logprobs: the workspace is missing, unaligned or too small");
  const hipError_t err = launch_logprobs((hipStream_t)hip_stream, dtype, a);
  return err == hipSuccess ? NTK_OK : hip_bad(err);
}

extern "C" int ntk_logprobs_bwd(int dtype, long long rows, int vocab, const void* logits, long long stride, const int* tokens,
                                float scale, const float* lse, const float* entropy, const float* dlogp, const float* dentropy,
                                void* dlogits, long long dlogits_stride, void* hip_stream) {
  if (int rc = logprob_args(dtype, rows, vocab, 0)) return rc;
  if (!(scale > 0.f) || !isfinite(scale * kLog2e)) return bad(NTK_E_ARG, "logprobs_bwd: scale must be positive and finite");
  if (rows == 0) return NTK_OK;
  if (!logits || !tokens || !lse || (dentropy && !entropy) || !dlogits) return bad(NTK_E_ARG, "logprobs_bwd: an array is NULL");
  if (stride < vocab || dlogits_stride < vocab) return bad(NTK_E_ARG, "logprobs_bwd: a row stride is below vocab");
  if (dlogits == logits && dlogits_stride != stride) return bad(NTK_E_ARG, "logprobs_bwd: in place, the strides have to agree");
  for (const void* p : {(const void*)tokens, (const void*)lse, (const void*)entropy, (const void*)dlogp, (const void*)dentropy})
    if (!aligned(p, 4)) return bad(NTK_E_ARG, "logprobs_bwd: a pointer is not aligned to its type");
  if (!aligned(logits, elem(dtype)) || !aligned(dlogits, elem(dtype))) return bad(NTK_E_ARG, "logprobs_bwd: a pointer is not aligned to its type");
  LogprobBwdArgs a{logits, dlogits, stride, dlogits_stride, tokens, lse, entropy, dlogp, dentropy, rows, vocab,
                   logprob_bwd_chunks(dtype, vocab), scale};
  const hipError_t err = launch_logprobs_bwd((hipStream_t)hip_stream, dtype, a);
  return err == hipSuccess ? NTK_OK : hip_bad(err);
}
