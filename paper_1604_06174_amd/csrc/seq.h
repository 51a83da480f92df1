// Problems and launches of the token models' operators (RMS norm, embedding, attention
// over packed sequences), as capi_seq.cpp has checked them.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace ckpt {

enum { SEQ_F32 = 0, SEQ_BF16 = 1, SEQ_E4M3 = 2 };

struct RmsArgs {
  const void *x, *res;  // forward: the summands (res null: none); re-run: x = h
  void *h, *y;          // h null: not stored
  float *ys, *st;
  const float *w;
  int64_t ldx, ldh, ldy;
  int rows, c, qgroup, groups;
  float eps, inv_c;
};

struct RmsBwdArgs {
  const void *g, *gh, *h;
  const float *st, *w;
  void *d;
  float *part;  // [workgroups][cpad] sums of g xhat
  float *dw;
  int64_t ldg, ldh, ldd;
  int rows, c, cpad;
  float inv_c;
};

// apply: x is h and st is read
void rms_forward(hipStream_t s, const RmsArgs &a, int xtype, int htype, int ytype, bool apply);
int rms_backward_groups(int64_t rows, int c);
void rms_backward(hipStream_t s, const RmsBwdArgs &a, int groups, int gtype, int htype, int dtype);

struct EmbedArgs {
  const void *ids;
  const void *src;  // the table, or the looked-up rows' gradient
  void *dst;        // the rows, or the table's gradient
  int64_t lds, ldd;
  int64_t tokens, vocab;
  int c, ids64, accumulate;
  float scale;
  // backward's workspace
  int *start;   // [vocab + 1] first sorted position of each id
  int *perm;    // [tokens] token at each sorted position
  int *key;     // [tokens] its id
  int *tail;    // [chunks] the id in pieces that begins in a chunk, or -1
  float *part;  // [2 chunks][cpad] sums of the pieces that begin in a chunk: a later piece, a first one
  int chunk, chunks, cpad;
};

void embed_forward(hipStream_t s, const EmbedArgs &a, int wtype, int ytype);
// fills in chunk, chunks and cpad; the workspace's bytes, and its places if ws is not null
uint64_t embed_plan(EmbedArgs &a, char *ws);
void embed_backward(hipStream_t s, const EmbedArgs &a, int gtype, int dtype);

struct AttnArgs {
  const __bf16 *q, *k, *v;
  const int *qoff, *koff;
  __bf16 *o;
  float *lse;
  // backward
  const __bf16 *g, *out;
  __bf16 *dq, *dk, *dv;
  float *delta, *lse2;  // [heads, tq] sums of g o; lse in base 2
  int parts;            // workgroups that share a key head's query heads
  float *pkv;           // [2][parts][tk][kv_heads][dim] their dk and dv, if more than one
  int64_t tq, tk;
  int64_t ldq, hsq, ldk, hsk, ldv, hsv, ldo, hso;
  int seqs, heads, kv_heads, rep, dim, causal;  // rep: heads / kv_heads
  float scale;
  // forward over split keys
  int splits;
  float *po;   // [splits][heads][tq][dimension] partial outputs, each with its own maximum
  float *pml;  // [splits][heads][tq][2] maximum and sum of exponentials
};

// the workspace's bytes, and its places if ws is not null
uint64_t attn_plan(AttnArgs &a, bool backward, char *ws);
void attn_forward(hipStream_t s, const AttnArgs &a);
void attn_backward(hipStream_t s, const AttnArgs &a);

}  // namespace ckpt
