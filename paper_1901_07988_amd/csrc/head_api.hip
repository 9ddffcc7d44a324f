// C ABI of the losses over a vocabulary: argument validation in front of the launchers.  No device code here.

#include <math.h>

#include "head.h"

using namespace abl;

namespace {

inline bool off(const void* p, size_t size) { return (reinterpret_cast<uintptr_t>(p) & (size - 1)) != 0; }
inline bool bad(const void* p, size_t size) { return p == nullptr || off(p, size); }
inline bool finite_number(float v) { return fabsf(v) <= 3.402823466e38f; }

// p: the call's numbers with those of the other operator at their defaults.
int check_head(const abl_head* head, bool backward, bool teacher, abl_head& p) {
  if (head == nullptr) return ABL_ERR_ARG;
  p = *head;
  if (p.dtype != ABL_F32 && p.dtype != ABL_BF16) return ABL_ERR_ARG;
  if (!backward) p.dw_dtype = p.dtype;
  if (p.dw_dtype != ABL_F32 && p.dw_dtype != p.dtype) return ABL_ERR_ARG;
  if ((p.flags & ~(uint32_t)(ABL_MATH_BF16 | (backward ? ABL_ACCUM_DW : 0))) != 0) return ABL_ERR_ARG;
  if (!teacher) p.T = 0, p.temperature = 1.0f, p.label_weight = 1.0f, p.teacher_weight = 0.0f;
  if (!finite_number(p.scale) || !(p.smoothing >= 0.0f && p.smoothing < 1.0f) || !finite_number(p.z_weight)) return ABL_ERR_ARG;
  if (!(p.temperature > 0.0f) || !finite_number(p.temperature) || !finite_number(1.0f / p.temperature)) return ABL_ERR_ARG;
  if (1.0f / p.temperature == 1.0f) p.temperature = 1.0f;
  if (!finite_number(p.label_weight) || !finite_number(p.teacher_weight)) return ABL_ERR_ARG;
  if (p.M < 0 || p.M > (int64_t)1 << 23 || p.C < 1 || p.C > 1 << 16 || p.V < 1 || p.V > 1 << 26) return ABL_ERR_SHAPE;
  if (p.M * p.V > (int64_t)1 << 44 || p.T > kTopEntries || p.T < (teacher ? 1 : 0)) return ABL_ERR_SHAPE;
  return ABL_OK;
}

int check_operands(const HeadCall& c, const void* scratch, size_t scratch_bytes, bool backward) {
  const size_t t = (size_t)size_of(c.p.dtype);
  if (bad(c.h.p, t) || c.h.ld < c.p.C || bad(c.W.p, t) || c.W.ld < c.p.C) return ABL_ERR_ARG;
  if (c.p.T == 0 ? bad(c.labels, 8) : off(c.labels, 8) || bad(c.ids, 8) || bad(c.logits, 4)) return ABL_ERR_ARG;
  if (scratch == nullptr || (reinterpret_cast<uintptr_t>(scratch) & 15u) != 0) return ABL_ERR_ARG;
  return scratch_bytes < head_scratch_bytes(c.p, backward) ? ABL_ERR_SCRATCH : ABL_OK;
}

// Whether the log-sum at temperature one is part of the loss.
inline bool needs_lse(const HeadCall& c) { return c.labels != nullptr || c.p.z_weight != 0.0f; }

int forward(hipStream_t st, const HeadCall& c, void* scratch, size_t scratch_bytes) {
  if (c.p.M == 0) return ABL_OK;
  if (int e = check_operands(c, scratch, scratch_bytes, false)) return e;
  if (bad(c.loss, 4) || (needs_lse(c) ? bad(c.lse, 4) : off(c.lse, 4))) return ABL_ERR_ARG;
  if (c.p.T != 0 && (bad(c.lse_t, 4) || bad(c.z_top, 4))) return ABL_ERR_ARG;
  return launch_head_forward(st, c, scratch, scratch_bytes);
}

int backward(hipStream_t st, const HeadCall& c, void* scratch, size_t scratch_bytes) {
  const size_t t = (size_t)size_of(c.p.dtype), d = (size_t)size_of(c.p.dw_dtype);
  if (off(c.dW, d)) return ABL_ERR_ARG;
  if (c.p.M > 0) {
    if (int e = check_operands(c, scratch, scratch_bytes, true)) return e;
    if ((c.dh.p == nullptr && c.dW == nullptr) || off(c.dh.p, t) || (c.dh.p != nullptr && c.dh.ld < c.p.C)) return ABL_ERR_ARG;
    if (bad(c.dloss, 4) || (needs_lse(c) ? bad(c.in_lse, 4) : off(c.in_lse, 4))) return ABL_ERR_ARG;
    if (c.p.T != 0 && (bad(c.in_lse_t, 4) || bad(c.in_z_top, 4))) return ABL_ERR_ARG;
  }
  return launch_head_backward(st, c, scratch, scratch_bytes);
}

}  // namespace

extern "C" {

// No part of the interface: what a call lays out in its workspace, for the tests of abl_head_scratch_bytes.
size_t abl_head_layout_bytes(const abl_head* head, int backward, int copied) {
  abl_head p;
  if (check_head(head, backward != 0, head != nullptr && head->T != 0, p) != ABL_OK) return 0;
  return head_layout_bytes(p, backward != 0, copied != 0);
}

size_t abl_head_scratch_bytes(const abl_head* head, int backward) {
  abl_head p;
  if (check_head(head, backward != 0, head != nullptr && head->T != 0, p) != ABL_OK) return 0;
  return head_scratch_bytes(p, backward != 0);
}

int abl_xent_forward(void* stream, const abl_head* head, const void* h, int64_t ldh, const void* W, int64_t ldw, const int64_t* labels,
                     void* scratch, size_t scratch_bytes, float* loss, float* lse) {
  HeadCall c{};
  if (int e = check_head(head, false, false, c.p)) return e;
  c.h = {h, ldh}, c.W = {W, ldw}, c.labels = labels, c.loss = loss, c.lse = lse;
  return forward((hipStream_t)stream, c, scratch, scratch_bytes);
}

int abl_xent_backward(void* stream, const abl_head* head, const void* h, int64_t ldh, const void* W, int64_t ldw, const int64_t* labels,
                      const float* lse, const float* dloss, void* scratch, size_t scratch_bytes, void* dh, int64_t lddh, void* dW) {
  HeadCall c{};
  if (int e = check_head(head, true, false, c.p)) return e;
  c.h = {h, ldh}, c.W = {W, ldw}, c.labels = labels, c.in_lse = lse, c.dloss = dloss, c.dh = {dh, lddh}, c.dW = dW;
  return backward((hipStream_t)stream, c, scratch, scratch_bytes);
}

int abl_distill_forward(void* stream, const abl_head* head, const void* h, int64_t ldh, const void* W, int64_t ldw, const int64_t* labels,
                        const int64_t* top_ids, const float* top_logits, void* scratch, size_t scratch_bytes, float* loss, float* lse,
                        float* lse_t, float* z_top) {
  HeadCall c{};
  if (int e = check_head(head, false, true, c.p)) return e;
  c.h = {h, ldh}, c.W = {W, ldw}, c.labels = labels, c.ids = top_ids, c.logits = top_logits;
  c.loss = loss, c.lse = lse, c.lse_t = lse_t, c.z_top = z_top;
  return forward((hipStream_t)stream, c, scratch, scratch_bytes);
}

int abl_distill_backward(void* stream, const abl_head* head, const void* h, int64_t ldh, const void* W, int64_t ldw, const int64_t* labels,
                         const int64_t* top_ids, const float* top_logits, const float* lse, const float* lse_t, const float* z_top,
                         const float* dloss, void* scratch, size_t scratch_bytes, void* dh, int64_t lddh, void* dW) {
  HeadCall c{};
  if (int e = check_head(head, true, true, c.p)) return e;
  c.h = {h, ldh}, c.W = {W, ldw}, c.labels = labels, c.ids = top_ids, c.logits = top_logits;
  c.in_lse = lse, c.in_lse_t = lse_t, c.in_z_top = z_top, c.dloss = dloss, c.dh = {dh, lddh}, c.dW = dW;
  return backward((hipStream_t)stream, c, scratch, scratch_bytes);
}

}  // extern "C"
