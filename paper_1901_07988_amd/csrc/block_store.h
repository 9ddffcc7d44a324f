// Device helpers of the kernels on rows of channels (block_store.hip, resnorm.hip, store_wgrad.hip): pieces of eight channels
// and the block store's codes.
//
// A thread works on a piece: eight consecutive channels of one row.  Four pieces are a block of 32 channels with one scale, held by
// four neighbouring lanes (a quad), so the block's maximum is two register moves between lanes.  Pieces are numbered through
// the whole tensor, 4 B of them per row (B blocks): piece p has its codes at byte K p and its scale at byte p / 4 of the scales.
#pragma once

#include <type_traits>

#include "abl_internal.h"

namespace abl {

typedef __bf16 bf16_t;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// (aligned to elements only: rows of odd width start anywhere, and the memory system takes such accesses)
typedef uint32_t u32x4_any2 __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_any4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2_any2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32_any2 __attribute__((aligned(2)));

__host__ __device__ inline int64_t store_blocks(int C) { return (C + 31) / 32; }
__host__ __device__ inline int64_t store_code_bytes(int64_t M, int C, int K) { return M * store_blocks(C) * 4 * K; }

__device__ inline float low_bf16(uint32_t u) { return __uint_as_float(u << 16); }
__device__ inline float high_bf16(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }
__device__ inline uint32_t two_bf16(float a, float b) {   // rounded to nearest even
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}

// ---- accesses through buffer descriptors: an offset beyond the descriptor's bytes reads zero and stores nothing ----
constexpr uint32_t kNowhere = 0x80000000u;   // (stays beyond with a row's offset added: descriptors hold less than 2^31 bytes)
__device__ inline __amdgpu_buffer_rsrc_t descriptor(const void* p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, p != nullptr ? (int)bytes : 0, 0x00027000);
}

// ---- a piece as it lies in memory ----
template <typename T>
struct Raw;
template <>
struct Raw<float> {
  f32x4_any4 a, b;
};
template <>
struct Raw<bf16_t> {
  u32x4 a;
};

// (T is one of the types above: a type that only differs in its alignment cannot be a template's argument)
#define ABL_FETCH(T, p) (STREAM ? __builtin_nontemporal_load(reinterpret_cast<const T*>(p)) : *reinterpret_cast<const T*>(p))
#define ABL_WRITE(T, p, v)                                             \
  do {                                                                 \
    if constexpr (STREAM)                                              \
      __builtin_nontemporal_store(v, reinterpret_cast<T*>(p));         \
    else                                                               \
      *reinterpret_cast<T*>(p) = v;                                    \
  } while (0)

// STREAM: past the caches, for passes that move more than the last-level cache holds (256 MB): nothing of them would stay there for the
// next pass, and what else lies there does.  Measured on 16384 x 8192 bf16, K = 4: unpack 65 -> 47 us, pack 63 -> 61; 8192 x 12288 gated unit
// without stores 103 -> 95, its backward 158 -> 150; on tensors that fit the cache the next pass would lose.
constexpr int64_t kStreamBytes = (int64_t)256 << 20;

// n: channels that exist (a piece at the end of a row may have fewer than eight, down to none); the others read as zero.  A short
// piece is taken as four, two and one of them, all on their way together and in few registers.
template <bool STREAM = false>
__device__ inline Raw<float> load_raw(const float* p, int n) {
  Raw<float> r{};
  if (n >= 8) {
    r.a = ABL_FETCH(f32x4_any4, p);
    r.b = ABL_FETCH(f32x4_any4, p + 4);
  } else if (n > 0) {
    f32x4_any4 four{};
    float x = 0.0f, y = 0.0f, z = 0.0f;
    if (n & 4) four = *reinterpret_cast<const f32x4_any4*>(p);
    if (n & 2) x = p[n & 4], y = p[(n & 4) + 1];
    if (n & 1) z = p[n & 6];
    const f32x4_any4 rest = n & 2 ? f32x4_any4{x, y, z, 0.0f} : f32x4_any4{z, 0.0f, 0.0f, 0.0f};
    r.a = n & 4 ? four : rest;
    if (n & 4) r.b = rest;
  }
  return r;
}
template <bool STREAM = false>
__device__ inline Raw<bf16_t> load_raw(const bf16_t* p, int n) {
  Raw<bf16_t> r{};
  if (n >= 8) {
    r.a = ABL_FETCH(u32x4_any2, p);
  } else if (n > 0) {
    const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
    u32x2_any2 four{};
    uint32_t two = 0, one = 0;
    if (n & 4) four = *reinterpret_cast<const u32x2_any2*>(h);
    if (n & 2) two = *reinterpret_cast<const u32_any2*>(h + (n & 4));
    if (n & 1) one = h[n & 6];
    const u32x2 rest = n & 2 ? u32x2{two, one} : u32x2{one, 0u};
    r.a = n & 4 ? u32x4{four[0], four[1], rest[0], rest[1]} : u32x4{rest[0], rest[1], 0u, 0u};
  }
  return r;
}
__device__ inline void expand(const Raw<float>& r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = r.a[i], v[i + 4] = r.b[i];
}
__device__ inline void expand(const Raw<bf16_t>& r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[2 * i] = low_bf16(r.a[i]), v[2 * i + 1] = high_bf16(r.a[i]);
}
template <bool STREAM = false, typename T>
__device__ inline void load_piece(const T* p, int n, float (&v)[8]) {
  expand(load_raw<STREAM>(p, n), v);
}
template <bool STREAM = false>
__device__ inline void store_piece(float* p, int n, const float (&v)[8]) {
  if (n >= 8) {
    ABL_WRITE(f32x4_any4, p, (f32x4_any4{v[0], v[1], v[2], v[3]}));
    ABL_WRITE(f32x4_any4, p + 4, (f32x4_any4{v[4], v[5], v[6], v[7]}));
  } else if (n > 0) {
    if (n & 4) *reinterpret_cast<f32x4_any4*>(p) = f32x4_any4{v[0], v[1], v[2], v[3]};
    const float a = v[0], b = v[1], c = v[2], d = v[4], e = v[5], f = v[6];   // (not chosen by address: v stays in registers)
    if (n & 2) p[n & 4] = n & 4 ? d : a, p[(n & 4) + 1] = n & 4 ? e : b;
    if (n & 1) p[n & 6] = n & 4 ? (n & 2 ? f : d) : (n & 2 ? c : a);
  }
}
template <bool STREAM = false>
__device__ inline void store_piece(bf16_t* p, int n, const float (&v)[8]) {
  const u32x4 w{two_bf16(v[0], v[1]), two_bf16(v[2], v[3]), two_bf16(v[4], v[5]), two_bf16(v[6], v[7])};
  if (n >= 8) {
    ABL_WRITE(u32x4_any2, p, (u32x4_any2)w);
  } else if (n > 0) {
    uint16_t* h = reinterpret_cast<uint16_t*>(p);
    if (n & 4) *reinterpret_cast<u32x2_any2*>(h) = u32x2_any2{w[0], w[1]};
    if (n & 2) *reinterpret_cast<u32_any2*>(h + (n & 4)) = n & 4 ? w[2] : w[0];
    if (n & 1) h[n & 6] = (uint16_t)(n & 4 ? (n & 2 ? w[3] : w[2]) : (n & 2 ? w[1] : w[0]));
  }
}

// Here the loads of a value have to have come: what is loaded in a branch or before a loop is waited for there, and not, together with
// all that was asked for since, where it is used.
__device__ inline void settle(Raw<bf16_t>& r) { asm volatile("" : "+v"(r.a)); }
__device__ inline void settle(Raw<float>& r) { asm volatile("" : "+v"(r.a), "+v"(r.b)); }

// ---- scale of a block ----
template <int CTRL>
__device__ inline uint32_t dpp_u32(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false);
}
__device__ inline uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// The scale byte of the block that the four lanes of a quad hold.  Magnitudes are compared as integers, in which infinities
// and NaN are the largest.  2^e is the maximum's exponent less that of the largest code, one more where the maximum's fraction
// would round beyond that code (127.5 = 1.9921875 2^6, 7 = 1.75 2^2): one addition to the bits, which carries into the exponent.
template <int K>
__device__ inline uint32_t scale_byte(const float (&v)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = umax(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  top = umax(top, dpp_u32<0xB1>(top));   // quad_perm [1,0,3,2]
  top = umax(top, dpp_u32<0x4E>(top));   // quad_perm [2,3,0,1]
  const int byte = (int)((top + (K == 8 ? 0x010000u : 0x200000u)) >> 23) - (K == 8 ? 6 : 2);
  return top >= 0x7F800000u ? 255u : (uint32_t)(byte < 8 ? 8 : byte);
}
__device__ inline float scale_of(uint32_t byte) {
  return byte == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float(byte << 23);
}

// ---- codes of a piece ----
template <int K>
struct Codes;   // K = 8: eight bytes, K = 4: four
template <>
struct Codes<8> {
  u32x2 w;
};
template <>
struct Codes<4> {
  uint32_t w;
};

// K = 8: x 2^-e + 1.5 2^23 in one rounding is the nearest integer, ties to even, in the low bits of the sum.
// K = 4: the conversion instruction (nearest, ties to even); it takes the scale itself.
template <int K>
__device__ inline Codes<K> encode(const float (&v)[8], uint32_t byte) {
  Codes<K> c;
  if constexpr (K == 8) {
    const float inv = __uint_as_float((254u - (byte == 255u ? 127u : byte)) << 23);
    uint32_t u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = __float_as_uint(__builtin_fmaf(v[i], inv, 12582912.0f));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t lo = __builtin_amdgcn_perm(u[4 * h + 1], u[4 * h], 0x0C0C0400u);
      const uint32_t hi = __builtin_amdgcn_perm(u[4 * h + 3], u[4 * h + 2], 0x04000C0Cu);
      c.w[h] = byte == 255u ? 0u : lo | hi;
    }
  } else {
    const float s = __uint_as_float((byte == 255u ? 127u : byte) << 23);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], s, 3);
    c.w = byte == 255u ? 0u : w;
  }
  return c;
}

template <int K>
__device__ inline void decode(const Codes<K>& c, uint32_t byte, float (&v)[8]) {
  const float s = scale_of(byte);
  if constexpr (K == 8) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)(int8_t)(c.w[i / 4] >> (8 * (i % 4))) * s;
  } else {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c.w, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c.w, 1.0f, 1);
    const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c.w, 1.0f, 2), f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c.w, 1.0f, 3);
    v[0] = a[0] * s, v[1] = a[1] * s, v[2] = b[0] * s, v[3] = b[1] * s;
    v[4] = d[0] * s, v[5] = d[1] * s, v[6] = f[0] * s, v[7] = f[1] * s;
  }
}

template <int K, typename I>
__device__ inline Codes<K> load_codes(const unsigned char* codes, I piece) {
  return *reinterpret_cast<const Codes<K>*>(codes + piece * K);
}
// Writes the codes of a piece and, from the quad's first lane, the block's scale.
template <int K, typename I>
__device__ inline void keep_piece(unsigned char* codes, unsigned char* scales, I piece, const float (&v)[8]) {
  const uint32_t byte = scale_byte<K>(v);
  *reinterpret_cast<Codes<K>*>(codes + piece * K) = encode<K>(v, byte);
  if ((threadIdx.x & 3u) == 0) scales[piece >> 2] = (unsigned char)byte;
}

// The zeros behind the scales, up to a multiple of 128 bytes: by the threads of one block, 128 or more.
__device__ inline void zero_tail(unsigned char* store, int64_t pieces, int K) {
  const int64_t used = pieces * K + (pieces >> 2);
  const int64_t all = (used + 127) / 128 * 128;
  if (used + threadIdx.x < all) store[used + threadIdx.x] = 0;
}

// ---- sums ----
// Sum over the 64 lanes, the same for all of them; of the four rows of 16 in S.
template <typename S = float>
__device__ inline S wave_sum(float v) {
  v += __uint_as_float(dpp_u32<0xB1>(__float_as_uint(v)));    // quad_perm [1,0,3,2]
  v += __uint_as_float(dpp_u32<0x4E>(__float_as_uint(v)));    // quad_perm [2,3,0,1]
  v += __uint_as_float(dpp_u32<0x141>(__float_as_uint(v)));   // row_half_mirror
  v += __uint_as_float(dpp_u32<0x140>(__float_as_uint(v)));   // row_mirror
  const int u = __float_as_int(v);
  return ((S)__int_as_float(__builtin_amdgcn_readlane(u, 0)) + (S)__int_as_float(__builtin_amdgcn_readlane(u, 16))) +
         ((S)__int_as_float(__builtin_amdgcn_readlane(u, 32)) + (S)__int_as_float(__builtin_amdgcn_readlane(u, 48)));
}

// ---- launchers ----
inline int64_t size_of(int dtype) { return dtype == ABL_F32 ? 4 : 2; }
struct Rows {   // a matrix of rows: elements from one row to the next
  const void* p;
  int64_t ld;
};
struct RowsOut {
  void* p;
  int64_t ld;
};
int launch_ckpt_pack(hipStream_t st, int dtype, Rows x, int64_t M, int C, int K, void* ckpt);
int launch_ckpt_unpack(hipStream_t st, int dtype, const void* ckpt, int64_t M, int C, int K, RowsOut x);
int launch_glu_forward(hipStream_t st, int dtype, int act, Rows g, Rows u, int64_t M, int C, int K, RowsOut h, void* ckpt_g,
                       void* ckpt_u);
int launch_glu_backward(hipStream_t st, int dtype, int act, Rows dh, const void* ckpt_g, const void* ckpt_u, int64_t M, int C, int K,
                        RowsOut dg, RowsOut du, void* ckpt_h);
int launch_resnorm_forward(hipStream_t st, const abl_resnorm& s, const void* r, const void* b, const void* gate, const void* w_post,
                           const void* w_pre, void* r_out, void* n, void* ckpt_b, float* rstd_b, void* ckpt_n, float* rstd_n);
size_t resnorm_scratch_bytes(int64_t M, int C);
int launch_resnorm_backward(hipStream_t st, const abl_resnorm& s, const void* dn, const void* dr_out, const void* gate, const void* w_post,
                            const void* w_pre, const void* ckpt_b, const float* rstd_b, const void* ckpt_n,
                            const float* rstd_n, void* scratch, void* dr, void* db, float* dgate, float* dw_post, float* dw_pre);
size_t store_wgrad_scratch_bytes(int64_t M, int Cin, int Cout, int dtype);
int launch_store_wgrad(hipStream_t st, int dtype, uint32_t flags, const void* ckpt, int64_t M, int Cin, int K, const void* scale,
                       Rows dy, int Cout, void* scratch, float* dW);

constexpr int kNormChannels = 16384;   // of a row of abl_resnorm_* at most

}  // namespace abl
