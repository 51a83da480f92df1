// extern "C" calls of the token models' operators (declared in include/ckpt.h, "units
// of token models").  Every argument is validated before anything is launched.
#include <hip/hip_runtime.h>

#include <cmath>
#include <string>

#include "capi_args.h"
#include "capi_internal.h"
#include "seq.h"

static_assert(CKPT_TYPE_F32 == ckpt::SEQ_F32 && CKPT_TYPE_BF16 == ckpt::SEQ_BF16 && CKPT_TYPE_E4M3 == ckpt::SEQ_E4M3,
              "type codes of the C ABI and the kernels agree");

namespace {

using ckpt::launched;
using ckpt::need_ptr;
using ckpt::product;
using ckpt::refuse;

constexpr int64_t kRows = int64_t(1) << 31;

uintptr_t size_of(int32_t type) { return type == CKPT_TYPE_F32 ? 4 : type == CKPT_TYPE_BF16 ? 2 : 1; }

void need_type(int32_t type, const char *fn, bool e4m3 = false) {
  if (type != CKPT_TYPE_F32 && type != CKPT_TYPE_BF16 && !(e4m3 && type == CKPT_TYPE_E4M3))
    refuse(CKPT_E_INVALID, fn, ": unknown type");
}

// a row stride (0: the width) of a matrix whose elements 64 bits number
int64_t stride_of(int64_t ld, int64_t width, int64_t rows, const char *fn) {
  if (!ld) ld = width;
  if (ld < width) refuse(CKPT_E_INVALID, fn, ": a stride is smaller than its row");
  const int64_t e = rows ? product(rows, ld) : 0;
  if (e < 0 || e > (int64_t(1) << 60)) refuse(CKPT_E_UNSUPPORTED, fn, ": tensor too large");
  return ld;
}

void need_workspace(const void *ws, uint64_t have, uint64_t want, const char *fn) {
  if (!want) return;
  need_ptr(ws, fn, "workspace", 16);
  if (have < want) refuse(CKPT_E_WORKSPACE, fn, ": workspace smaller than its workspace_bytes call says");
}

// ---------------------------------------------------------------- RMS norm --
struct Rms {
  int64_t ldx, ldh, ldy, ldg, ldd;
  int groups, dw_groups, cpad;
};

Rms rms_of(const ckpt_rms_desc *d, const char *fn) {
  need_ptr(d, fn, "desc");
  if (d->rows < 1 || d->c < 1) refuse(CKPT_E_INVALID, fn, ": rows and c must be positive");
  if (d->rows >= kRows) refuse(CKPT_E_UNSUPPORTED, fn, ": rows must stay below 2^31");
  if (d->c > 16384) refuse(CKPT_E_UNSUPPORTED, fn, ": c must not exceed 16384");
  for (int32_t t : {d->xtype, d->htype, d->gtype, d->dtype}) need_type(t, fn);
  need_type(d->ytype, fn, true);
  if (!(d->eps > 0.f) || !std::isfinite(d->eps)) refuse(CKPT_E_INVALID, fn, ": eps must be positive");
  const int32_t q = d->qgroup;
  if (q && (d->ytype != CKPT_TYPE_E4M3 || q < 8 || q > 512 || (q & (q - 1))))
    refuse(CKPT_E_INVALID, fn, ": qgroup is 0, or for an 8-bit y a power of two from 8 to 512");
  Rms r;
  r.ldx = stride_of(d->ldx, d->c, d->rows, fn);
  r.ldh = stride_of(d->ldh, d->c, d->rows, fn);
  r.ldy = stride_of(d->ldy, d->c, d->rows, fn);
  r.ldg = stride_of(d->ldg, d->c, d->rows, fn);
  r.ldd = stride_of(d->ldd, d->c, d->rows, fn);
  r.groups = q ? (d->c + q - 1) / q : 1;
  r.dw_groups = ckpt::rms_backward_groups(d->rows, d->c);
  r.cpad = (d->c + 3) / 4 * 4;
  return r;
}

ckpt::RmsArgs rms_args(const ckpt_rms_desc *d, const Rms &r, const float *w, void *y, float *ys, float *st,
                       const char *fn) {
  need_ptr(w, fn, "w", 4);
  need_ptr(y, fn, "y", size_of(d->ytype));
  need_ptr(st, fn, "st", 4);
  if (d->ytype == CKPT_TYPE_E4M3) need_ptr(ys, fn, "ys", 4);
  else if (ys) refuse(CKPT_E_INVALID, fn, ": ys goes with an 8-bit y alone");
  ckpt::RmsArgs a{};
  a.w = w;
  a.y = y;
  a.ys = ys;
  a.st = st;
  a.ldx = r.ldx;
  a.ldh = r.ldh;
  a.ldy = r.ldy;
  a.rows = int(d->rows);
  a.c = d->c;
  a.qgroup = d->qgroup;
  a.groups = r.groups;
  a.eps = d->eps;
  a.inv_c = 1.f / float(d->c);
  return a;
}

// --------------------------------------------------------------- embedding --
ckpt::EmbedArgs embed_of(const ckpt_embed_desc *d, bool backward, const char *fn) {
  need_ptr(d, fn, "desc");
  if (d->tokens < 1 || d->vocab < 1 || d->c < 1) refuse(CKPT_E_INVALID, fn, ": tokens, vocab and c must be positive");
  if (d->tokens > kRows / 2) refuse(CKPT_E_UNSUPPORTED, fn, ": tokens must not exceed 2^30");
  if (d->vocab >= kRows) refuse(CKPT_E_UNSUPPORTED, fn, ": vocab must stay below 2^31");
  if (d->c > (1 << 20)) refuse(CKPT_E_UNSUPPORTED, fn, ": c must not exceed 2^20");
  // a launch has fewer than 2^32 threads
  if (product(d->tokens, d->c) >= (int64_t(1) << 36)) refuse(CKPT_E_UNSUPPORTED, fn, ": tokens*c must stay below 2^36");
  for (int32_t t : {d->wtype, d->ytype, d->gtype, d->dtype}) need_type(t, fn);
  if ((d->ids64 != 0 && d->ids64 != 1) || (d->accumulate != 0 && d->accumulate != 1))
    refuse(CKPT_E_INVALID, fn, ": ids64 and accumulate are 0 or 1");
  if (!std::isfinite(d->scale)) refuse(CKPT_E_INVALID, fn, ": scale must be finite");
  ckpt::EmbedArgs a{};
  const int64_t ldw = stride_of(d->ldw, d->c, d->vocab, fn), ldy = stride_of(d->ldy, d->c, d->tokens, fn),
                ldg = stride_of(d->ldg, d->c, d->tokens, fn);
  a.lds = backward ? ldg : ldw;
  a.ldd = backward ? ldw : ldy;
  a.tokens = d->tokens;
  a.vocab = d->vocab;
  a.c = d->c;
  a.ids64 = d->ids64;
  a.accumulate = d->accumulate;
  a.scale = d->scale;
  return a;
}

// --------------------------------------------------------------- attention --
ckpt::AttnArgs attn_of(const ckpt_attn_desc *d, const char *fn) {
  need_ptr(d, fn, "desc");
  if (d->tq < 0 || d->tk < 0 || d->seqs < 1 || d->heads < 1 || d->kv_heads < 1 || d->dim < 1)
    refuse(CKPT_E_INVALID, fn, ": tq and tk must not be negative, seqs, heads, kv_heads and dim positive");
  if (d->heads % d->kv_heads) refuse(CKPT_E_INVALID, fn, ": kv_heads must divide heads");
  if (d->dim % 8 || d->dim > 128) refuse(CKPT_E_UNSUPPORTED, fn, ": dim must be a multiple of 8, at most 128");
  if (d->causal != 0 && d->causal != 1) refuse(CKPT_E_INVALID, fn, ": causal is 0 or 1");
  if (!(d->scale >= 0.f) || !std::isfinite(d->scale)) refuse(CKPT_E_INVALID, fn, ": scale must be positive, or 0");
  if (d->tq > kRows / 2 || d->tk > kRows / 2) refuse(CKPT_E_UNSUPPORTED, fn, ": tq and tk must not exceed 2^30");
  if (d->seqs >= (1 << 20) || d->heads > 4096) refuse(CKPT_E_UNSUPPORTED, fn, ": too many sequences or heads");
  // workgroups of 256 threads, of which a launch has fewer than 2^32: tiles of 128 rows, or of 32 if
  // that takes no more than one for each sequence besides its last, partly filled one
  if ((d->tq * d->heads + d->tk * d->kv_heads) / 128 + 2 * int64_t(d->seqs) * d->kv_heads >= (int64_t(1) << 24))
    refuse(CKPT_E_UNSUPPORTED, fn, ": more than 2^24 tiles of 128 rows");
  ckpt::AttnArgs a{};
  const int64_t h = d->heads, kv = d->kv_heads, dim = d->dim;
  auto strides = [&](int64_t ld, int64_t hs, int64_t n, int64_t rows, int64_t &lo, int64_t &ho) {
    lo = ld ? ld : n * dim;
    ho = hs ? hs : dim;
    if (lo < dim || ho < dim) refuse(CKPT_E_INVALID, fn, ": a stride is smaller than a head's row");
    if (lo % 8 || ho % 8) refuse(CKPT_E_UNSUPPORTED, fn, ": strides must be multiples of 8");
    const int64_t e = rows ? product(rows, lo) : 0, f = product(n, ho);
    if (e < 0 || f < 0 || e > (int64_t(1) << 60) || f > (int64_t(1) << 60))
      refuse(CKPT_E_UNSUPPORTED, fn, ": tensor too large");
  };
  strides(d->ldq, d->hsq, h, d->tq, a.ldq, a.hsq);
  strides(d->ldk, d->hsk, kv, d->tk, a.ldk, a.hsk);
  strides(d->ldv, d->hsv, kv, d->tk, a.ldv, a.hsv);
  strides(d->ldo, d->hso, h, d->tq, a.ldo, a.hso);
  a.tq = d->tq;
  a.tk = d->tk;
  a.seqs = d->seqs;
  a.heads = d->heads;
  a.kv_heads = d->kv_heads;
  a.rep = d->heads / d->kv_heads;
  a.dim = d->dim;
  a.causal = d->causal;
  a.scale = d->scale == 0.f ? float(1.0 / std::sqrt(double(d->dim))) : d->scale;
  return a;
}

// tensors of no rows may be null
void need_rows(const void *p, int64_t rows, const char *fn, const char *arg) {
  if (rows || p) need_ptr(p, fn, arg, 16);
}

const __bf16 *bf16(const void *p) { return static_cast<const __bf16 *>(p); }
__bf16 *bf16(void *p) { return static_cast<__bf16 *>(p); }

}  // namespace

extern "C" {

int op_rms_forward(const ckpt_rms_desc *desc, const void *x, const void *res, const float *w, void *h, void *y,
                   float *ys, float *st, void *stream) {
  return ckpt::guarded([&] {
    const char *const fn = "op_rms_forward";
    const Rms r = rms_of(desc, fn);
    ckpt::RmsArgs a = rms_args(desc, r, w, y, ys, st, fn);
    need_ptr(x, fn, "x", size_of(desc->xtype));
    if (!res != !h) refuse(CKPT_E_INVALID, fn, ": res and h go together");
    if (res) {
      need_ptr(res, fn, "res", size_of(desc->htype));
      need_ptr(h, fn, "h", size_of(desc->htype));
    } else if (desc->xtype != desc->htype) {
      refuse(CKPT_E_INVALID, fn, ": without a residual x is of htype");
    }
    a.x = x;
    a.res = res;
    a.h = h;
    ckpt::rms_forward(static_cast<hipStream_t>(stream), a, desc->xtype, desc->htype, desc->ytype, false);
    launched(fn);
  });
}

int op_rms_apply(const ckpt_rms_desc *desc, const void *h, const float *st, const float *w, void *y, float *ys,
                 void *stream) {
  return ckpt::guarded([&] {
    const char *const fn = "op_rms_apply";
    const Rms r = rms_of(desc, fn);
    ckpt::RmsArgs a = rms_args(desc, r, w, y, ys, const_cast<float *>(st), fn);
    need_ptr(h, fn, "h", size_of(desc->htype));
    a.x = h;
    ckpt::rms_forward(static_cast<hipStream_t>(stream), a, desc->htype, desc->htype, desc->ytype, true);
    launched(fn);
  });
}

int op_rms_workspace_bytes(const ckpt_rms_desc *desc, uint64_t *bytes) {
  return ckpt::guarded([&] {
    need_ptr(bytes, "op_rms_workspace_bytes", "bytes");
    const Rms r = rms_of(desc, "op_rms_workspace_bytes");
    *bytes = 4 * uint64_t(r.dw_groups) * r.cpad;
  });
}

int op_rms_backward(const ckpt_rms_desc *desc, const void *g, const void *gh, const void *h, const float *st,
                    const float *w, void *d, float *dw, void *workspace, uint64_t workspace_bytes, void *stream) {
  return ckpt::guarded([&] {
    const char *const fn = "op_rms_backward";
    const Rms r = rms_of(desc, fn);
    need_ptr(g, fn, "g", size_of(desc->gtype));
    if (gh) need_ptr(gh, fn, "gh", size_of(desc->dtype));
    need_ptr(h, fn, "h", size_of(desc->htype));
    need_ptr(st, fn, "st", 4);
    need_ptr(w, fn, "w", 4);
    need_ptr(d, fn, "d", size_of(desc->dtype));
    need_ptr(dw, fn, "dw", 4);
    need_workspace(workspace, workspace_bytes, 4 * uint64_t(r.dw_groups) * r.cpad, fn);
    ckpt::RmsBwdArgs a{g, gh, h, st, w, d, static_cast<float *>(workspace), dw, r.ldg, r.ldh, r.ldd, int(desc->rows),
                       desc->c, r.cpad, 1.f / float(desc->c)};
    ckpt::rms_backward(static_cast<hipStream_t>(stream), a, r.dw_groups, desc->gtype, desc->htype, desc->dtype);
    launched(fn);
  });
}

int op_embed_forward(const ckpt_embed_desc *desc, const void *ids, const void *w, void *y, void *stream) {
  return ckpt::guarded([&] {
    const char *const fn = "op_embed_forward";
    ckpt::EmbedArgs a = embed_of(desc, false, fn);
    need_ptr(ids, fn, "ids", desc->ids64 ? 8 : 4);
    need_ptr(w, fn, "w", size_of(desc->wtype));
    need_ptr(y, fn, "y", size_of(desc->ytype));
    a.ids = ids;
    a.src = w;
    a.dst = y;
    ckpt::embed_forward(static_cast<hipStream_t>(stream), a, desc->wtype, desc->ytype);
    launched(fn);
  });
}

int op_embed_workspace_bytes(const ckpt_embed_desc *desc, uint64_t *bytes) {
  return ckpt::guarded([&] {
    need_ptr(bytes, "op_embed_workspace_bytes", "bytes");
    ckpt::EmbedArgs a = embed_of(desc, true, "op_embed_workspace_bytes");
    *bytes = ckpt::embed_plan(a, nullptr);
  });
}

int op_embed_backward(const ckpt_embed_desc *desc, const void *ids, const void *g, void *dw, void *workspace,
                      uint64_t workspace_bytes, void *stream) {
  return ckpt::guarded([&] {
    const char *const fn = "op_embed_backward";
    ckpt::EmbedArgs a = embed_of(desc, true, fn);
    need_ptr(ids, fn, "ids", desc->ids64 ? 8 : 4);
    need_ptr(g, fn, "g", size_of(desc->gtype));
    need_ptr(dw, fn, "dw", size_of(desc->dtype));
    a.ids = ids;
    a.src = g;
    a.dst = dw;
    need_workspace(workspace, workspace_bytes, ckpt::embed_plan(a, static_cast<char *>(workspace)), fn);
    ckpt::embed_backward(static_cast<hipStream_t>(stream), a, desc->gtype, desc->dtype);
    launched(fn);
  });
}

int op_attn_workspace_bytes(const ckpt_attn_desc *desc, int32_t backward, uint64_t *bytes) {
  return ckpt::guarded([&] {
    need_ptr(bytes, "op_attn_workspace_bytes", "bytes");
    ckpt::AttnArgs a = attn_of(desc, "op_attn_workspace_bytes");
    *bytes = ckpt::attn_plan(a, backward != 0, nullptr);
  });
}

int op_attn_forward(const ckpt_attn_desc *desc, const void *q, const void *k, const void *v, const int32_t *qoff,
                    const int32_t *koff, void *o, float *lse, void *workspace, uint64_t workspace_bytes, void *stream) {
  return ckpt::guarded([&] {
    const char *const fn = "op_attn_forward";
    ckpt::AttnArgs a = attn_of(desc, fn);
    need_rows(q, a.tq, fn, "q");
    need_rows(k, a.tk, fn, "k");
    need_rows(v, a.tk, fn, "v");
    need_ptr(qoff, fn, "qoff", 4);
    need_ptr(koff, fn, "koff", 4);
    need_rows(o, a.tq, fn, "o");
    if (a.tq || lse) need_ptr(lse, fn, "lse", 4);
    need_workspace(workspace, workspace_bytes, ckpt::attn_plan(a, false, static_cast<char *>(workspace)), fn);
    a.q = bf16(q);
    a.k = bf16(k);
    a.v = bf16(v);
    a.qoff = qoff;
    a.koff = koff;
    a.o = bf16(o);
    a.lse = lse;
    ckpt::attn_forward(static_cast<hipStream_t>(stream), a);
    launched(fn);
  });
}

int op_attn_backward(const ckpt_attn_desc *desc, const void *g, const void *q, const void *k, const void *v,
                     const void *o, const float *lse, const int32_t *qoff, const int32_t *koff, void *dq, void *dk,
                     void *dv, void *workspace, uint64_t workspace_bytes, void *stream) {
  return ckpt::guarded([&] {
    const char *const fn = "op_attn_backward";
    ckpt::AttnArgs a = attn_of(desc, fn);
    need_rows(g, a.tq, fn, "g");
    need_rows(q, a.tq, fn, "q");
    need_rows(k, a.tk, fn, "k");
    need_rows(v, a.tk, fn, "v");
    need_rows(o, a.tq, fn, "o");
    if (a.tq || lse) need_ptr(lse, fn, "lse", 4);
    need_ptr(qoff, fn, "qoff", 4);
    need_ptr(koff, fn, "koff", 4);
    need_rows(dq, a.tq, fn, "dq");
    need_rows(dk, a.tk, fn, "dk");
    need_rows(dv, a.tk, fn, "dv");
    need_workspace(workspace, workspace_bytes, ckpt::attn_plan(a, true, static_cast<char *>(workspace)), fn);
    a.g = bf16(g);
    a.q = bf16(q);
    a.k = bf16(k);
    a.v = bf16(v);
    a.out = bf16(o);
    a.lse = const_cast<float *>(lse);
    a.qoff = qoff;
    a.koff = koff;
    a.dq = bf16(dq);
    a.dk = bf16(dk);
    a.dv = bf16(dv);
    ckpt::attn_backward(static_cast<hipStream_t>(stream), a);
    launched(fn);
  });
}

}  // extern "C"
