// C ABI of the operators on rows of channels (block stores, residual norms, gated units, their weight gradients): argument
// validation in front of the launchers.  No device code here.

#include "block_store.h"

using namespace abl;

namespace {

constexpr int64_t kBlocks = (int64_t)1 << 29;   // of a store (four pieces each: a launch's threads are counted in 32 bits)
constexpr int64_t kNormRows = (int64_t)1 << 25;

inline bool bad_store(const void* p) { return p == nullptr || (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
// elements of `size` bytes
inline bool off(const void* p, size_t size) { return (reinterpret_cast<uintptr_t>(p) & (size - 1)) != 0; }
inline bool bad(const void* p, size_t size) { return p == nullptr || off(p, size); }
inline bool bad_rows(const void* p, size_t size, int64_t ld, int32_t C) { return bad(p, size) || ld < C; }

inline int check_dtype(int d) { return d == ABL_F32 || d == ABL_BF16 ? ABL_OK : ABL_ERR_ARG; }
inline int check_k(int K) { return K == 4 || K == 8 ? ABL_OK : ABL_ERR_ARG; }
inline int check_k0(int K) { return K == 0 ? ABL_OK : check_k(K); }
int check_rows(int64_t M, int32_t C) {
  if (M < 0 || C < 1 || M >= kBlocks) return ABL_ERR_SHAPE;
  return M * store_blocks(C) < kBlocks ? ABL_OK : ABL_ERR_SHAPE;
}
// dtype, K, sizes
int check(int dtype, int K, bool none, int64_t M, int32_t C) {
  if (int e = check_dtype(dtype)) return e;
  if (int e = none ? check_k0(K) : check_k(K)) return e;
  return check_rows(M, C);
}
int check_step(const abl_resnorm* s, bool none) {
  if (s == nullptr) return ABL_ERR_ARG;
  if (int e = check(s->dtype, s->K, none, s->M, s->C)) return e;
  if ((s->flags & ~(uint32_t)ABL_NORM_CENTER) != 0) return ABL_ERR_ARG;
  if (s->C > kNormChannels || s->M > kNormRows) return ABL_ERR_SHAPE;
  return ABL_OK;
}

}  // namespace

extern "C" {

size_t abl_ckpt_bytes(int64_t M, int32_t C, int K) {
  if (check_k(K) != ABL_OK || check_rows(M, C) != ABL_OK) return 0;
  const size_t used = (size_t)(store_code_bytes(M, C, K) + M * store_blocks(C));
  return used == 0 ? 128 : (used + 127) / 128 * 128;
}

int abl_ckpt_pack(void* stream, int dtype, const void* x, int64_t ldx, int64_t M, int32_t C, int K, void* ckpt) {
  if (int e = check(dtype, K, false, M, C)) return e;
  if (M == 0) return ABL_OK;
  if (bad_rows(x, (size_t)size_of(dtype), ldx, C) || bad_store(ckpt)) return ABL_ERR_ARG;
  return launch_ckpt_pack((hipStream_t)stream, dtype, {x, ldx}, M, C, K, ckpt);
}

int abl_ckpt_unpack(void* stream, int dtype, const void* ckpt, int64_t M, int32_t C, int K, void* x, int64_t ldx) {
  if (int e = check(dtype, K, false, M, C)) return e;
  if (M == 0) return ABL_OK;
  if (bad_rows(x, (size_t)size_of(dtype), ldx, C) || bad_store(ckpt)) return ABL_ERR_ARG;
  return launch_ckpt_unpack((hipStream_t)stream, dtype, ckpt, M, C, K, {x, ldx});
}

int abl_resnorm_forward(void* stream, const abl_resnorm* step, const void* r, const void* b, const void* gate,
                        const void* w_post, const void* w_pre, void* r_out, void* n, void* ckpt_b, float* rstd_b,
                        void* ckpt_n, float* rstd_n) {
  if (int e = check_step(step, true)) return e;
  if (!(step->eps > 0.0f) || (gate != nullptr && step->gate_rows < 1)) return ABL_ERR_ARG;
  if (step->M == 0) return ABL_OK;
  if (b == nullptr && (gate != nullptr || w_post != nullptr)) return ABL_ERR_ARG;
  const size_t t = (size_t)size_of(step->dtype);
  if (bad(r, t) || off(b, t) || off(gate, t) || off(w_post, t) || bad(w_pre, t) || off(r_out, t) || bad(n, t)) return ABL_ERR_ARG;
  if (step->K != 0) {
    if (bad_store(ckpt_n) || bad(rstd_n, 4)) return ABL_ERR_ARG;
    if ((w_post != nullptr || gate != nullptr) && bad_store(ckpt_b)) return ABL_ERR_ARG;
    if (w_post != nullptr && bad(rstd_b, 4)) return ABL_ERR_ARG;
  }
  const bool keep = step->K != 0, keep_b = keep && (w_post != nullptr || gate != nullptr);
  return launch_resnorm_forward((hipStream_t)stream, *step, r, b, gate, w_post, w_pre, r_out, n, keep_b ? ckpt_b : nullptr,
                                keep && w_post != nullptr ? rstd_b : nullptr, keep ? ckpt_n : nullptr, keep ? rstd_n : nullptr);
}

size_t abl_resnorm_scratch_bytes(int64_t M, int32_t C) {
  if (check_rows(M, C) != ABL_OK || C > kNormChannels || M > kNormRows) return 0;
  return resnorm_scratch_bytes(M, C);
}

int abl_resnorm_backward(void* stream, const abl_resnorm* step, int has_b, const void* dn, const void* dr_out, const void* gate,
                         const void* w_post, const void* w_pre, const void* ckpt_b, const float* rstd_b,
                         const void* ckpt_n, const float* rstd_n, void* scratch, size_t scratch_bytes,
                         void* dr, void* db, float* dgate, float* dw_post, float* dw_pre) {
  if (int e = check_step(step, false)) return e;
  if (gate != nullptr && step->gate_rows < 1) return ABL_ERR_ARG;
  if (!has_b && (gate != nullptr || w_post != nullptr || db != nullptr)) return ABL_ERR_ARG;
  if ((step->M > 0 && (gate != nullptr) != (dgate != nullptr)) || (w_post != nullptr) != (dw_post != nullptr)) return ABL_ERR_ARG;
  if (bad(dw_pre, 4) || off(dw_post, 4) || off(dgate, 4)) return ABL_ERR_ARG;
  const size_t t = (size_t)size_of(step->dtype);
  if (step->M > 0) {
    if (bad(dn, t) || off(dr_out, t) || off(gate, t) || off(w_post, t) || bad(w_pre, t) || off(dr, t) || off(db, t)) return ABL_ERR_ARG;
    if (bad_store(ckpt_n) || bad(rstd_n, 4) || bad_store(scratch)) return ABL_ERR_ARG;
    if ((w_post != nullptr || gate != nullptr) && bad_store(ckpt_b)) return ABL_ERR_ARG;
    if (w_post != nullptr && bad(rstd_b, 4)) return ABL_ERR_ARG;
    if (scratch_bytes < resnorm_scratch_bytes(step->M, step->C)) return ABL_ERR_SCRATCH;
  }
  return launch_resnorm_backward((hipStream_t)stream, *step, dn, dr_out, gate, w_post, w_pre,
                                 w_post != nullptr || gate != nullptr ? ckpt_b : nullptr, rstd_b, ckpt_n, rstd_n, scratch, dr, db,
                                 dgate, dw_post, dw_pre);
}

int abl_glu_forward(void* stream, int dtype, int act, const void* g, int64_t ldg, const void* u, int64_t ldu, int64_t M,
                    int32_t C, int K, void* h, int64_t ldh, void* ckpt_g, void* ckpt_u) {
  if (int e = check(dtype, K, true, M, C)) return e;
  if (act != ABL_ACT_SILU && act != ABL_ACT_GELU) return ABL_ERR_ARG;
  if (M == 0) return ABL_OK;
  const size_t t = (size_t)size_of(dtype);
  if (bad_rows(g, t, ldg, C) || bad_rows(u, t, ldu, C) || bad_rows(h, t, ldh, C)) return ABL_ERR_ARG;
  if (K != 0 && (bad_store(ckpt_g) || bad_store(ckpt_u))) return ABL_ERR_ARG;
  return launch_glu_forward((hipStream_t)stream, dtype, act, {g, ldg}, {u, ldu}, M, C, K, {h, ldh}, ckpt_g, ckpt_u);
}

int abl_glu_backward(void* stream, int dtype, int act, const void* dh, int64_t lddh, const void* ckpt_g,
                     const void* ckpt_u, int64_t M, int32_t C, int K, void* dg, int64_t lddg, void* du, int64_t lddu,
                     void* ckpt_h) {
  if (int e = check(dtype, K, false, M, C)) return e;
  if (act != ABL_ACT_SILU && act != ABL_ACT_GELU) return ABL_ERR_ARG;
  if (M == 0) return ABL_OK;
  const size_t t = (size_t)size_of(dtype);
  if (bad_rows(dh, t, lddh, C) || bad_rows(dg, t, lddg, C) || bad_rows(du, t, lddu, C)) return ABL_ERR_ARG;
  if (bad_store(ckpt_g) || bad_store(ckpt_u) || (ckpt_h != nullptr && bad_store(ckpt_h))) return ABL_ERR_ARG;
  return launch_glu_backward((hipStream_t)stream, dtype, act, {dh, lddh}, ckpt_g, ckpt_u, M, C, K, {dg, lddg}, {du, lddu}, ckpt_h);
}

static int check_wgrad(int dtype, int64_t M, int32_t Cin, int32_t Cout) {
  if (int e = check_dtype(dtype)) return e;
  if (int e = check_rows(M, Cin)) return e;
  if (int e = check_rows(M, Cout)) return e;
  return Cin <= 1 << 20 && Cout <= 1 << 20 && (int64_t)Cin * Cout <= 2147483647LL ? ABL_OK : ABL_ERR_SHAPE;
}

size_t abl_ckpt_wgrad_scratch_bytes(int64_t M, int32_t Cin, int32_t Cout, int dtype) {
  return check_wgrad(dtype, M, Cin, Cout) == ABL_OK ? store_wgrad_scratch_bytes(M, Cin, Cout, dtype) : 0;
}

int abl_ckpt_wgrad(void* stream, int dtype, uint32_t flags, const void* ckpt, int64_t M, int32_t Cin, int K,
                   const void* scale, const void* dy, int64_t lddy, int32_t Cout, void* scratch,
                   size_t scratch_bytes, float* dW) {
  if (int e = check_wgrad(dtype, M, Cin, Cout)) return e;
  if (int e = check_k(K)) return e;
  if ((flags & ~(uint32_t)(ABL_MATH_BF16 | ABL_ACCUM_DW)) != 0) return ABL_ERR_ARG;
  const size_t t = (size_t)size_of(dtype);
  if (off(scale, t) || bad(dW, 4)) return ABL_ERR_ARG;
  if (M > 0) {
    if (bad_store(ckpt) || bad_rows(dy, t, lddy, Cout) || bad_store(scratch)) return ABL_ERR_ARG;
    if (scratch_bytes < store_wgrad_scratch_bytes(M, Cin, Cout, dtype)) return ABL_ERR_SCRATCH;
  }
  return launch_store_wgrad((hipStream_t)stream, dtype, flags, ckpt, M, Cin, K, scale, {dy, lddy}, Cout, scratch, dW);
}

}  // extern "C"
