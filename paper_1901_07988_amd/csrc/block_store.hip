// Block stores (abl_ckpt_pack / abl_ckpt_unpack) and the gated unit that makes and reads them (abl_glu_*): passes in which every
// thread takes one piece of eight channels (block_store.h).
//
//   pack        codes and scales of x                 reads t bytes an element (2 in bf16), writes K / 8 + 1 / 32
//   unpack      x~ = 2^e code                         the other way round
//   glu_fwd     h = g s(g) u, codes of g and u        reads 2 t, writes t and two stores
//   glu_bwd     dg = dh u a'(g), du = dh a(g), codes of a(g) u      reads t and two stores, writes 2 t and an 8-bit store
//
// with s(g) = 1 / (1 + exp(-q(g))), a = g s and a' = s + g s (1 - s) q': q = g for SiLU, and for the tanh form of GELU
// q = 2 sqrt(2 / pi) (g + 0.044715 g^3), since (1 + tanh z) / 2 = 1 / (1 + exp(-2 z)).
//
// All are bound by memory (a copy of 2 GB reaches 6.2 TB/s); without the choice of a scale or without the scales' stores they take the
// same time within 4 %.  bf16, 16384 x 8192: pack 62 us at K = 4 and 74 at K = 8 (5.5 TB/s), unpack 47.5 and 67 (7.1 and 6.0); 8192 x 12288:
// glu_fwd 139 us with 8-bit stores (5.8) and 95 without (6.4), glu_bwd 149 (6.1).
// One piece a thread: a block of 256 threads has the loads of all its pieces on their way at once, and blocks of 128 to 1024 threads
// measure alike.  The large tensors pass by the caches (kStreamBytes), the codes do not: glu_fwd would gain 7 us by that, and what reads
// the stores next would lose 12.

#include "block_store.h"

namespace abl {
namespace {

constexpr int kThreads = 256;

// Where the pieces of a pass lie: 4 B pieces per row, the blocks of threads one after the other.
struct Pieces {
  int64_t total, per_row;
  int C;
  Divisor by_row;   // (of numbers below 4 B + the threads of a block)
  Pieces(int64_t M, int c) : total(M * store_blocks(c) * 4), per_row(store_blocks(c) * 4), C(c), by_row((int)(store_blocks(c) * 4)) {}
  int64_t grid() const { return (total + kThreads - 1) / kThreads; }
};

struct Place {
  int64_t piece, row;
  int c, n;   // first channel, channels that exist (may be negative)
};
__device__ inline Place place_of(const Pieces& g) {
  const int64_t first = (int64_t)blockIdx.x * kThreads;
  const int64_t row = first / g.per_row;
  const int rel = (int)(first - row * g.per_row) + (int)threadIdx.x;
  const int more = g.by_row.of(rel);
  Place p;
  p.piece = first + threadIdx.x;
  p.row = row + more;
  p.c = (rel - more * (int)g.per_row) * 8;
  p.n = g.C - p.c;
  return p;
}

template <typename T, int K, bool STREAM>
__global__ __launch_bounds__(kThreads) void pack_kernel(Pieces g, const T* __restrict__ x, int64_t ldx, unsigned char* __restrict__ store) {
  if (blockIdx.x == 0) zero_tail(store, g.total, K);
  const Place p = place_of(g);
  if (p.piece >= g.total) return;
  float v[8];
  load_piece<STREAM>(x + p.row * ldx + p.c, p.n, v);
  keep_piece<K>(store, store + g.total * K, p.piece, v);
}

template <typename T, int K, bool STREAM>
__global__ __launch_bounds__(kThreads) void unpack_kernel(Pieces g, const unsigned char* __restrict__ store, T* __restrict__ x, int64_t ldx) {
  const Place p = place_of(g);
  if (p.piece >= g.total) return;
  float v[8];
  decode<K>(load_codes<K>(store, p.piece), store[g.total * K + (p.piece >> 2)], v);
  store_piece<STREAM>(x + p.row * ldx + p.c, p.n, v);
}

template <int ACT>
__device__ inline void gate(float g, float& s, float& dq) {
  float q = g;
  dq = 1.0f;
  if constexpr (ACT == ABL_ACT_GELU) {
    const float k = 1.5957691216057308f, k3 = 0.071354816272600f;   // 2 sqrt(2 / pi), 0.044715 of it
    const float g2 = fminf(g * g, 1e30f);   // (beyond it s is 0 or 1, and dq only has to stay finite)
    q = g * __builtin_fmaf(k3, g2, k);
    dq = __builtin_fmaf(3.0f * k3, g2, k);
  }
  s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * q));
}

template <typename T, int ACT, int K, bool STREAM>
__global__ __launch_bounds__(kThreads) void glu_fwd_kernel(Pieces pc, const T* g, int64_t ldg, const T* u, int64_t ldu, T* h, int64_t ldh,
                                                           unsigned char* __restrict__ store_g, unsigned char* __restrict__ store_u) {
  if (K != 0 && blockIdx.x == 0) {
    zero_tail(store_g, pc.total, K);
    zero_tail(store_u, pc.total, K);
  }
  const Place p = place_of(pc);
  if (p.piece >= pc.total) return;
  float a[8], b[8], o[8];
  load_piece<STREAM>(g + p.row * ldg + p.c, p.n, a);
  load_piece<STREAM>(u + p.row * ldu + p.c, p.n, b);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float s, dq;
    gate<ACT>(a[i], s, dq);
    o[i] = a[i] * s * b[i];
  }
  store_piece<STREAM>(h + p.row * ldh + p.c, p.n, o);
  if constexpr (K != 0) {
    keep_piece<K>(store_g, store_g + pc.total * K, p.piece, a);
    keep_piece<K>(store_u, store_u + pc.total * K, p.piece, b);
  }
}

template <typename T, int ACT, int K, bool STREAM>
__global__ __launch_bounds__(kThreads) void glu_bwd_kernel(Pieces pc, const T* dh, int64_t lddh, const unsigned char* __restrict__ store_g,
                                                           const unsigned char* __restrict__ store_u, T* dg, int64_t lddg, T* du, int64_t lddu,
                                                           unsigned char* __restrict__ store_h) {
  if (store_h != nullptr && blockIdx.x == 0) zero_tail(store_h, pc.total, 8);
  const Place p = place_of(pc);
  if (p.piece >= pc.total) return;
  float d[8], a[8], b[8], o[8];
  load_piece<STREAM>(dh + p.row * lddh + p.c, p.n, d);
  decode<K>(load_codes<K>(store_g, p.piece), store_g[pc.total * K + (p.piece >> 2)], a);
  decode<K>(load_codes<K>(store_u, p.piece), store_u[pc.total * K + (p.piece >> 2)], b);
  float x[8], y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float s, dq;
    gate<ACT>(a[i], s, dq);
    const float act = a[i] * s;
    x[i] = d[i] * b[i] * __builtin_fmaf(act * (1.0f - s), dq, s);
    y[i] = d[i] * act;
    o[i] = act * b[i];
  }
  store_piece<STREAM>(dg + p.row * lddg + p.c, p.n, x);
  store_piece<STREAM>(du + p.row * lddu + p.c, p.n, y);
  if (store_h != nullptr) keep_piece<8>(store_h, store_h + pc.total * 8, p.piece, o);
}

// f(type, STREAM): with the dtype as a type, and whether the pass goes by the caches.
template <typename F>
void by_dtype(int dtype, int64_t bytes, F&& f) {
  auto stream = [&](auto t) {
    if (bytes > kStreamBytes)
      f(t, std::true_type{});
    else
      f(t, std::false_type{});
  };
  if (dtype == ABL_F32)
    stream(float{});
  else
    stream(bf16_t{});
}

}  // namespace

int launch_ckpt_pack(hipStream_t st, int dtype, Rows x, int64_t M, int C, int K, void* ckpt) {
  const Pieces g(M, C);
  by_dtype(dtype, g.total * (8 * size_of(dtype) + K), [&](auto t, auto s) {
    using T = decltype(t);
    constexpr bool S = decltype(s)::value;
    auto kern = K == 8 ? pack_kernel<T, 8, S> : pack_kernel<T, 4, S>;
    kern<<<dim3((unsigned)g.grid()), kThreads, 0, st>>>(g, (const T*)x.p, x.ld, (unsigned char*)ckpt);
  });
  return hip_status();
}

int launch_ckpt_unpack(hipStream_t st, int dtype, const void* ckpt, int64_t M, int C, int K, RowsOut x) {
  const Pieces g(M, C);
  by_dtype(dtype, g.total * (8 * size_of(dtype) + K), [&](auto t, auto s) {
    using T = decltype(t);
    constexpr bool S = decltype(s)::value;
    auto kern = K == 8 ? unpack_kernel<T, 8, S> : unpack_kernel<T, 4, S>;
    kern<<<dim3((unsigned)g.grid()), kThreads, 0, st>>>(g, (const unsigned char*)ckpt, (T*)x.p, x.ld);
  });
  return hip_status();
}

int launch_glu_forward(hipStream_t st, int dtype, int act, Rows g, Rows u, int64_t M, int C, int K, RowsOut h, void* ckpt_g,
                       void* ckpt_u) {
  const Pieces pc(M, C);
  by_dtype(dtype, pc.total * (3 * 8 * size_of(dtype) + 2 * K), [&](auto t, auto s) {
    using T = decltype(t);
    constexpr bool S = decltype(s)::value;
    auto pick = [&](auto a) {
      constexpr int A = decltype(a)::value;
      return K == 0 ? glu_fwd_kernel<T, A, 0, S> : K == 8 ? glu_fwd_kernel<T, A, 8, S> : glu_fwd_kernel<T, A, 4, S>;
    };
    auto kern = act == ABL_ACT_SILU ? pick(std::integral_constant<int, ABL_ACT_SILU>{}) : pick(std::integral_constant<int, ABL_ACT_GELU>{});
    kern<<<dim3((unsigned)pc.grid()), kThreads, 0, st>>>(pc, (const T*)g.p, g.ld, (const T*)u.p, u.ld, (T*)h.p, h.ld,
                                                         (unsigned char*)ckpt_g, (unsigned char*)ckpt_u);
  });
  return hip_status();
}

int launch_glu_backward(hipStream_t st, int dtype, int act, Rows dh, const void* ckpt_g, const void* ckpt_u, int64_t M, int C, int K,
                        RowsOut dg, RowsOut du, void* ckpt_h) {
  const Pieces pc(M, C);
  by_dtype(dtype, pc.total * (3 * 8 * size_of(dtype) + 2 * K), [&](auto t, auto s) {
    using T = decltype(t);
    constexpr bool S = decltype(s)::value;
    auto pick = [&](auto a) {
      constexpr int A = decltype(a)::value;
      return K == 8 ? glu_bwd_kernel<T, A, 8, S> : glu_bwd_kernel<T, A, 4, S>;
    };
    auto kern = act == ABL_ACT_SILU ? pick(std::integral_constant<int, ABL_ACT_SILU>{}) : pick(std::integral_constant<int, ABL_ACT_GELU>{});
    kern<<<dim3((unsigned)pc.grid()), kThreads, 0, st>>>(pc, (const T*)dh.p, dh.ld, (const unsigned char*)ckpt_g,
                                                         (const unsigned char*)ckpt_u, (T*)dg.p, dg.ld, (T*)du.p, du.ld,
                                                         (unsigned char*)ckpt_h);
  });
  return hip_status();
}

}  // namespace abl
