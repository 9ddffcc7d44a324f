// The step between two blocks of a residual network (abl_resnorm_forward / abl_resnorm_backward):
//
//   y = N(b),  p = gate (w_post y),  r' = alpha r + beta p,  z = N(r'),  n = w_pre z          stores of y and z
//
//   D  = dr' + rstd_r (v - z mean(v z)),   v = dn w_pre           (ABL_NORM_CENTER: less the mean of v too)
//   dr = alpha D,   e = beta D,   dgate = sum e w_post y,   dw_post = sum e gate y,   dw_pre = sum dn z
//   db = rstd_b (v - y mean(v y)),   v = e gate w_post
//
// Both are bound by memory: an element of bf16 costs 8 bytes and its two stores (10.1 at K = 8).  8192 x 4096 bf16 with a gate for
// 2048 rows, K = 8 (338 MB): forward 55 us (6.2 TB/s, as a copy; 66 after passes whose output the caches still have to write),
// backward 60 with the second launch (5.6); calls of a few rows are the launch: 8 rows 3.9 us.  That is the width
// whose pieces are as many as a team's threads: 8192 x 2560 takes 45 and 54 us (4.7 and 3.9 TB/s), 4096 x 5120 46 and 56 (4.6 and
// 3.7), 2048 x 12288, with four pieces a thread, 57 and 78 (4.5 and 3.2).  A team of threads holds a row in registers, so that every
// tensor is read once; the sums over a row go through the waves' registers and, between waves, LDS.  In the backward a team takes
// consecutive rows and keeps its share of the sums over rows in registers as well; the teams' sums are added in a fixed order by a
// second launch.

#include <utility>

#include "block_store.h"

namespace abl {
namespace {

// Channels that exist from channel c on (none or fewer for a thread beyond the row's end).
__device__ inline int left(int C, uint32_t c) { return C - (int)c; }

// ---- a team's rows in memory ----
// A team has consecutive rows, and accesses go through buffer descriptors of them: a lane beyond the row's end has an offset beyond
// the descriptor, and a tensor that is not there has a descriptor of no bytes; both read zero and store nothing.  (An access is out of
// range where its own offset is not below the descriptor's bytes less the scalar offset.  So that this difference is never
// negative, what may be absent takes no row's offset where it is.)  Without branches
// around them the compiler can count the accesses on their way, so waiting for the next row's loads does not wait for
// this row's stores, and from row to row only three scalar offsets change.  (A store takes the sum of its offsets in a vector register:
// with the row's in the instruction's scalar operand the compiler lets the next instruction overwrite the store's data, and wrong
// words have been written here.)
//
// A row of a multiple of eight channels is whole pieces (kWhole).  Where it is not (kRagged), the lane of the last piece loads the row's last eight
// channels and shifts them down, so that nothing beyond the row is read, and stores four, two and one of them, as many as there are.
// Rows of fewer than eight channels (kShort) are taken in parts (load_raw, store_piece).
// kStream: whole pieces past the caches (kStreamBytes).  8192 x 4096 bf16, K = 8, which moves 338 MB: forward 70 -> 57 us,
// backward 79 -> 66 (both with 1024 threads a unit).  Only for teams of 256 threads and more: with it narrower rows of bf16 take
// 0.99 to 1.02 of the time forward and 0.95 to 0.98 backward (131072 x 512 140 and 137 us instead of 139 and 144), 200000 x 128 fp32
// 124 and 183 us instead of 123 and 202, but 30000 x 1536 fp32 195 and 196 instead of 181 and 184.  Ragged rows are stored in parts, which past the caches would be
// parts of lines; they were not timed so.
enum Form { kWhole, kRagged, kShort, kStream };

// Where a lane's piece of a row lies: byte offsets in the row, kNowhere where there is nothing of the kind.
template <typename T, Form FORM>
struct Lane {
  uint32_t q, at;               // piece; whole pieces, and the loads of the last one
  uint32_t four, two, one, n;   // kRagged: stores of the last piece, its channels (8 for others)
  __device__ inline Lane(uint32_t piece, int C) : q(piece) {
    const uint32_t size = sizeof(T), c = piece * 8;
    const int left = C - (int)c;
    at = left > 0 ? c * size : kNowhere;
    four = two = one = kNowhere, n = 8;
    if constexpr (FORM == kRagged) {
      if (left > 0 && left < 8) {
        n = (uint32_t)left;
        at = (uint32_t)(C - 8) * size;
        if (n & 4) four = c * size;
        if (n & 2) two = (c + (n & 4)) * size;
        if (n & 1) one = (c + (n & 6)) * size;
      }
    }
  }
};

__device__ inline void shift_down(Raw<bf16_t>& r, uint32_t by) {   // by so many channels, zeros from above
  u32x4 w = r.a;
  const uint32_t bits = (by & 1) * 16;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_alignbit(i < 3 ? w[i + 1] : 0u, w[i], bits);
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = by & 2 ? (i < 3 ? w[i + 1] : 0u) : w[i];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = by & 4 ? (i < 2 ? w[i + 2] : 0u) : w[i];
  r.a = w;
}
__device__ inline void shift_down(Raw<float>& r, uint32_t by) {
  float w[8];
  expand(r, w);
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = by & 4 ? (i < 4 ? w[i + 4] : 0.0f) : w[i];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = by & 2 ? (i < 6 ? w[i + 2] : 0.0f) : w[i];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = by & 1 ? (i < 7 ? w[i + 1] : 0.0f) : w[i];
  r.a = f32x4_any4{w[0], w[1], w[2], w[3]}, r.b = f32x4_any4{w[4], w[5], w[6], w[7]};
}

// Rows of T from `first` on.  MAYBE: may be absent.
template <typename T, Form FORM, bool MAYBE = false>
struct TeamRows {
  const T* p;
  int C;
  __amdgpu_buffer_rsrc_t d;
  static constexpr int kAux = FORM == kStream ? 2 : 0;   // (non-temporal)
  __device__ inline TeamRows(const void* base, int64_t first, int64_t rows, int c)
      : p(base != nullptr ? (const T*)base + first * c : nullptr), C(c), d(descriptor(p, rows * c * (int64_t)sizeof(T))) {}
  // What lies in memory; `unpack` makes the channels of it.
  template <typename L>
  __device__ inline Raw<T> load(uint32_t k, const L& l) const {
    if constexpr (FORM == kShort) {
      return p != nullptr ? load_raw(p + (int64_t)k * C + l.q * 8, left(C, l.q * 8)) : Raw<T>{};
    } else {
      uint32_t row = k * (uint32_t)C * (uint32_t)sizeof(T);
      if constexpr (MAYBE) row = p != nullptr ? row : 0;
      if constexpr (std::is_same_v<T, float>) {
        Raw<float> r;
        r.a = __builtin_bit_cast(f32x4_any4, __builtin_amdgcn_raw_buffer_load_b128(d, l.at, row, kAux));
        r.b = __builtin_bit_cast(f32x4_any4, MAYBE ? __builtin_amdgcn_raw_buffer_load_b128(d, l.at + 16, row, kAux)
                                                   : __builtin_amdgcn_raw_buffer_load_b128(d, l.at, row + 16, kAux));
        return r;
      } else {
        return Raw<bf16_t>{__builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(d, l.at, row, kAux))};
      }
    }
  }
  __device__ inline void store(uint32_t k, const Lane<T, FORM>& l, const float (&v)[8]) const {
    if constexpr (FORM == kShort) {
      if (p != nullptr) store_piece(const_cast<T*>(p) + (int64_t)k * C + l.q * 8, left(C, l.q * 8), v);
    } else {
      const uint32_t row = k * (uint32_t)C * (uint32_t)sizeof(T);
      const uint32_t at = (FORM == kRagged && l.n < 8 ? kNowhere : l.at) + row;
      const bool n4 = l.n & 4, n2 = l.n & 2;
      if constexpr (std::is_same_v<T, float>) {
        const u32x4 lo = __builtin_bit_cast(u32x4, f32x4_any4{v[0], v[1], v[2], v[3]});
        const u32x4 hi = __builtin_bit_cast(u32x4, f32x4_any4{v[4], v[5], v[6], v[7]});
        __builtin_amdgcn_raw_buffer_store_b128(lo, d, at, 0, kAux);
        __builtin_amdgcn_raw_buffer_store_b128(hi, d, at + 16, 0, kAux);
        if constexpr (FORM == kRagged) {
          __builtin_amdgcn_raw_buffer_store_b128(lo, d, l.four + row, 0, 0);
          __builtin_amdgcn_raw_buffer_store_b64(u32x2{n4 ? hi[0] : lo[0], n4 ? hi[1] : lo[1]}, d, l.two + row, 0, 0);
          __builtin_amdgcn_raw_buffer_store_b32(n4 ? (n2 ? hi[2] : hi[0]) : (n2 ? lo[2] : lo[0]), d, l.one + row, 0, 0);
        }
      } else {
        const u32x4 w{two_bf16(v[0], v[1]), two_bf16(v[2], v[3]), two_bf16(v[4], v[5]), two_bf16(v[6], v[7])};
        __builtin_amdgcn_raw_buffer_store_b128(w, d, at, 0, kAux);
        if constexpr (FORM == kRagged) {
          __builtin_amdgcn_raw_buffer_store_b64(u32x2{w[0], w[1]}, d, l.four + row, 0, 0);
          __builtin_amdgcn_raw_buffer_store_b32(n4 ? w[2] : w[0], d, l.two + row, 0, 0);
          __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(n4 ? (n2 ? w[3] : w[2]) : (n2 ? w[1] : w[0])), d, l.one + row, 0, 0);
        }
      }
    }
  }
};
template <typename T, Form FORM>
__device__ inline void unpack(Raw<T> r, const Lane<T, FORM>& l, float (&v)[8]) {
  if constexpr (FORM == kRagged) shift_down(r, 8 - l.n);
  expand(r, v);
}

// The rows of a store: `pieces` = 4 B of each.
struct StoreLane {   // byte offsets in a row of a lane's codes (over K) and scale, and of the scale that it writes
  uint32_t q, scale, own;
  __device__ inline StoreLane(uint32_t piece, int pieces) {
    const bool in = piece < (uint32_t)pieces;
    q = in ? piece : kNowhere / 8;
    scale = in ? piece >> 2 : kNowhere;
    own = in && (piece & 3u) == 0 ? piece >> 2 : kNowhere;
  }
};
template <int K, bool MAYBE = false>
struct StoreRows {
  __amdgpu_buffer_rsrc_t codes, scales;
  uint32_t pieces;
  bool there;
  __device__ inline StoreRows(const unsigned char* store, int64_t M, int n, int64_t first, int64_t rows)
      : codes(descriptor(store != nullptr ? store + first * n * K : nullptr, rows * n * K)),
        scales(descriptor(store != nullptr ? store + M * n * K + (first * n >> 2) : nullptr, rows * n >> 2)),
        pieces((uint32_t)n), there(!MAYBE || store != nullptr) {}
  static __device__ inline uint32_t at(const StoreLane& l) { return l.q < kNowhere / 8 ? l.q * K : kNowhere; }
  __device__ inline void load(uint32_t k, const StoreLane& l, Codes<K>& c, uint32_t& byte) const {
    const uint32_t of = there ? k * pieces * K : 0, of_scale = there ? k * (pieces >> 2) : 0;
    if constexpr (K == 8)
      c.w = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(codes, at(l), of, 0));
    else
      c.w = __builtin_amdgcn_raw_buffer_load_b32(codes, at(l), of, 0);
    byte = __builtin_amdgcn_raw_buffer_load_b8(scales, l.scale, of_scale, 0);
  }
  __device__ inline void keep(uint32_t k, const StoreLane& l, const float (&v)[8]) const {
    const uint32_t byte = scale_byte<K>(v);
    const Codes<K> c = encode<K>(v, byte);
    if constexpr (K == 8)
      __builtin_amdgcn_raw_buffer_store_b64(c.w, codes, at(l) + k * pieces * 8, 0, 0);
    else
      __builtin_amdgcn_raw_buffer_store_b32(c.w, codes, at(l) + k * pieces * 4, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b8((unsigned char)byte, scales, l.own + k * (pieces >> 2), 0, 0);
  }
};

// A vector over the channels (a row of the gate): ones where there is none, zeros beyond the channels.  Shifted already where that is needed.
template <typename T, Form FORM>
__device__ inline Raw<T> load_weights(const void* w, int64_t row, int C, const Lane<T, FORM>& l) {
  Raw<T> r;
  if (w != nullptr) {
    r = TeamRows<T, FORM == kStream ? kWhole : FORM>(w, row, 1, C).load(0, l);   // (all rows read it: through the caches)
    if constexpr (FORM == kRagged) shift_down(r, 8 - l.n);
  } else if constexpr (std::is_same_v<T, float>) {
    r.a = r.b = f32x4_any4{1.0f, 1.0f, 1.0f, 1.0f};
  } else {
    r.a = u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
  }
  return r;
}

template <typename T, Form FORM, int NV>
struct Lanes {
  Lane<T, FORM> l[NV];
  StoreLane s[NV];
};
template <typename T, Form FORM, int TEAM, int... I>
__device__ inline Lanes<T, FORM, sizeof...(I)> lanes(uint32_t t, int C, int pieces, std::integer_sequence<int, I...>) {
  return {{Lane<T, FORM>(t + TEAM * I, C)...}, {StoreLane(t + TEAM * I, pieces)...}};
}

// ---- a team's sums over a row ----
// S: of the sums over the waves; a lane's and a row of 16 lanes' are in fp32.
template <int TEAM, typename S>
struct TeamSum {
  S* slots;   // [2][TEAM / 64], used in turn: the barrier of one sum keeps the next from overwriting what is still read
  int turn = 0;
  __device__ explicit TeamSum(S* s) : slots(s) {}
  __device__ inline S operator()(float w) {
    S v = wave_sum<S>(w);
    if constexpr (TEAM > 64) {
      S* s = slots + turn * (TEAM / 64);
      turn ^= 1;
      if ((threadIdx.x & 63u) == 0) s[threadIdx.x >> 6] = v;
      __syncthreads();
      v = 0;
#pragma unroll
      for (int i = 0; i < TEAM / 64; ++i) v += s[i];
    }
    return v;
  }
};

struct FwdArgs {
  int64_t M, gate_rows;
  const void *r, *b, *gate, *w_post, *w_pre;
  void *r_out, *n;
  unsigned char *ckpt_b, *ckpt_n;
  float *rstd_b, *rstd_n;
  int64_t rows;    // of a team
  int C, pieces;   // pieces of a row
  int center;
  float alpha, beta, eps;
  double inv_c;
};

// v <- N(v); returns 1 / sqrt(mean square + eps).  Channels that do not exist hold zeros and stay zero.
// A normalized value should be off by its own rounding only: the rounding of the factor, common to a row, would shift all values that lie near the
// middle of two codes to one side.  So the sums over waves, the mean and a Newton step on the instruction's root are in 64 bits, and the
// factor is applied as a float and what it lacks.
template <int TEAM, int NV>
__device__ inline float normalize(float (&v)[NV][8], const FwdArgs& a, TeamSum<TEAM, double>& sum, uint32_t t) {
  if (a.center) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) m += v[i][j];
    m = (float)(sum(m) * a.inv_c);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if ((t + TEAM * i) * 8 + j < (uint32_t)a.C) v[i][j] -= m;
  }
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) s = __builtin_fmaf(v[i][j], v[i][j], s);
  const double x = __builtin_fma(sum(s), a.inv_c, (double)a.eps);
  const float root = (float)__builtin_amdgcn_rsq(x);   // (that of 32 bits takes numbers below the least normal one for zero)
  const double e = __builtin_fma(-x * root, root, 1.0);
  const float more = finite((float)x) ? (float)(0.5 * root * e) : 0.0f;   // (an infinite or NaN sum: zero or NaN)
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = __builtin_fmaf(v[i][j], root, v[i][j] * more);
  return root + more;
}

// Blocks of teams of 64 hold four of them.
template <int TEAM>
constexpr int kBlock = TEAM == 64 ? 256 : TEAM;
template <int TEAM>
__device__ inline int64_t team_index() {
  return TEAM == 64 ? (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : (int64_t)blockIdx.x;
}

// A team takes consecutive rows and asks for the next one's elements before it works on this one's: the sums over a row are two
// waits for all waves of the team, during which nothing else would be on its way.
template <typename T, int K, Form FORM, int TEAM, int NV>
__global__ __launch_bounds__(kBlock<TEAM>, NV >= 2 ? 2 : 4) void resnorm_fwd_kernel(FwdArgs a) {
  __shared__ double slots[2 * (TEAM / 64)];
  TeamSum<TEAM, double> sum(slots);
  const uint32_t t = threadIdx.x % TEAM;
  if (K != 0 && blockIdx.x == 0) {
    zero_tail(a.ckpt_n, a.M * a.pieces, K);
    if (a.ckpt_b != nullptr) zero_tail(a.ckpt_b, a.M * a.pieces, K);
  }
  const int64_t first = team_index<TEAM>() * a.rows;
  if (first >= a.M) return;   // (a whole wave; blocks of larger teams are as many as teams)
  const uint32_t rows = (uint32_t)(first + a.rows < a.M ? a.rows : a.M - first);
  using In = TeamRows<T, FORM>;
  const TeamRows<T, FORM, true> from_b(a.b, first, rows, a.C);
  const In from_r(a.r, first, rows, a.C), to_r(a.r_out, first, rows, a.C), to_n(a.n, first, rows, a.C);
  const StoreRows<K == 0 ? 8 : K> keep_b(K != 0 ? a.ckpt_b : nullptr, a.M, a.pieces, first, rows);
  const StoreRows<K == 0 ? 8 : K> keep_n(K != 0 ? a.ckpt_n : nullptr, a.M, a.pieces, first, rows);
  const auto lane = lanes<T, FORM, TEAM>(t, a.C, a.pieces, std::make_integer_sequence<int, NV>{});
  Raw<T> r[NV], b[NV], w_post[NV], w_pre[NV], gate[NV];
  auto fetch = [&](uint32_t k) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      r[i] = from_r.load(k, lane.l[i]);
      b[i] = from_b.load(k, lane.l[i]);
    }
  };
  int64_t group = a.gate != nullptr ? first / a.gate_rows : 0;
  int64_t group_end = a.gate != nullptr ? (group + 1) * a.gate_rows : a.M;
  fetch(0);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    w_pre[i] = load_weights<T, FORM>(a.w_pre, 0, a.C, lane.l[i]);
    w_post[i] = load_weights<T, FORM>(a.w_post, 0, a.C, lane.l[i]);
    gate[i] = load_weights<T, FORM>(a.gate, group, a.C, lane.l[i]);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) settle(w_pre[i]), settle(w_post[i]), settle(gate[i]);
  for (uint32_t k = 0; k < rows; ++k) {
    float v[NV][8], x[NV][8], w[8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      unpack(r[i], lane.l[i], x[i]);
      unpack(b[i], lane.l[i], v[i]);
    }
    if (k + 1 < rows) fetch(k + 1);
    if (a.w_post != nullptr) {
      const float rstd = normalize<TEAM, NV>(v, a, sum, t);
      if (K != 0 && t == 0) a.rstd_b[first + k] = rstd;
    }
    if constexpr (K != 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i) keep_b.keep(k, lane.s[i], v[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      expand(w_post[i], w);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] *= w[j];
      expand(gate[i], w);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = a.alpha * x[i][j] + a.beta * (v[i][j] * w[j]);   // (v is zero where there is no b)
      to_r.store(k, lane.l[i], v[i]);
    }
    if (first + k + 1 == group_end && k + 1 < rows) {   // the next row has the next gate
      ++group;
      group_end += a.gate_rows;
#pragma unroll
      for (int i = 0; i < NV; ++i) gate[i] = load_weights<T, FORM>(a.gate, group, a.C, lane.l[i]);
#pragma unroll
      for (int i = 0; i < NV; ++i) settle(gate[i]);
    }
    const float rstd = normalize<TEAM, NV>(v, a, sum, t);
    if constexpr (K != 0) {
      if (t == 0) a.rstd_n[first + k] = rstd;
#pragma unroll
      for (int i = 0; i < NV; ++i) keep_n.keep(k, lane.s[i], v[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      expand(w_pre[i], w);
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] *= v[i][j];
      to_n.store(k, lane.l[i], w);
    }
  }
}

// ---- backward ----
// How the rows go to the teams.  A row of the gate's gradient is a sum over gate_rows rows: either a team's share holds whole groups of
// them (the team writes those sums itself), or a group holds whole shares.
struct Shares {
  int64_t rows = 1;       // of a team
  int64_t teams = 1;
  int64_t per_group = 0;  // teams of a group of rows (0: teams hold whole groups)
};

// Threads of a launch at most (256 compute units).  The backward: what stays on the units at once where a thread has two pieces,
// and half as many sums for the second launch where it has one: 1024 / 512 threads a unit take 108 / 92 us at 4096 x 8192 bf16
// with a gate a row, 64.4 / 59.4 at 8192 x 4096 (256: 84), 17.6 / 17.5 at 1500 x 1111 fp32 (with teams of 256);
// 19.8 / 21 at 16384 x 200.
constexpr int64_t kBwdThreads = 128 * 1024;   // (1500 x 1111: K = 8, a gate a row, means taken out; counted with a team's idle threads)
// The forward, 2048 / 1024 threads a unit: 53.5 / 55.2 us at 8192 x 4096 bf16 and 9.4 / 10.3 at 1500 x 1112 fp32; rows of more
// pieces than threads take the smaller launch (48 / 40 us at 1024 x 16384 bf16).
constexpr int64_t fwd_threads(int pieces_a_thread) { return (pieces_a_thread == 1 ? 512 : 256) * 1024; }
Shares shares_of(int64_t M, int64_t gate_rows, int team, bool gate) {
  const int64_t most = kBwdThreads / team;   // up to twice as many where groups are cut
  const int64_t block = team == 64 ? 4 : 1;   // teams of a block: of one group, where a group is cut
  Shares s;
  s.rows = (M + most - 1) / most;
  if (gate && gate_rows <= s.rows) {
    s.rows = (s.rows + gate_rows - 1) / gate_rows * gate_rows;
  } else if (gate) {
    const int64_t group = gate_rows < M ? gate_rows : M;
    s.per_group = ((group + s.rows - 1) / s.rows + block - 1) / block * block;
    s.rows = (group + s.per_group - 1) / s.per_group;
    s.teams = (M + group - 1) / group * s.per_group;
    return s;
  }
  s.teams = (M + s.rows - 1) / s.rows;
  return s;
}

struct BwdArgs {
  int64_t M, gate_rows;
  const void *dn, *dr_out, *gate, *w_post, *w_pre;
  const unsigned char *ckpt_b, *ckpt_n;
  const float *rstd_b, *rstd_n;
  void *dr, *db;
  float* dgate;
  float* part;   // [3][teams][pieces * 8]: shares of dw_pre, dw_post, dgate
  Shares share;
  int C, pieces, center;
  float alpha, beta, inv_c;
};

// v <- rstd (v - y mean(v y)) + more (less rstd times the mean of v where the norm took the mean out)
template <int TEAM, int NV, typename More>
__device__ inline void norm_gradient(float (&v)[NV][8], const float (&y)[NV][8], float rstd, const BwdArgs& a, TeamSum<TEAM, float>& sum, More&& more) {
  float s = 0.0f, m = 0.0f;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) s = __builtin_fmaf(v[i][j], y[i][j], s);
  s = sum(s) * a.inv_c;
  if (a.center) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) m += v[i][j];
    m = sum(m) * a.inv_c;
  }
  const float rs = -rstd * s;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float t[8];
    more(i, t);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = __builtin_fmaf(rstd, v[i][j], __builtin_fmaf(rs, y[i][j], t[j]));
  }
  if (a.center) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = __builtin_fmaf(-rstd, m, v[i][j]);
  }
}

// What a thread reads of a row.
template <typename T, int K, int NV>
struct RowIn {
  Raw<T> dn[NV], dr[NV];
  Codes<K> z[NV], y[NV];
  uint32_t sz[NV], sy[NV];
  float rstd_n, rstd_b;
};

// As in the forward, the next row's elements are asked for before this one's are worked on.
// The bound of four waves a SIMD, 128 registers, costs a piece a thread some spills to scratch: 2 to 22 registers in teams of 64 threads, 10 to 19 in
// fp32 teams of 512, up to 6 in fp32 teams of 192 and 256 and in ragged bf16 ones of 512, none elsewhere.  Four pieces a thread spill 5 to 94 of
// 256 registers here, and 16 to 60 in the forward (fp32, and ragged bf16 with stores).  Not priced.
template <typename T, int K, Form FORM, int TEAM, int NV>
__global__ __launch_bounds__(kBlock<TEAM>, NV == 1 ? 4 : 2) void resnorm_bwd_kernel(BwdArgs a) {
  constexpr bool kHold = NV < 4;   // registers for the weights and for the next row; rows of four pieces a thread read the weights again
  __shared__ float slots[2 * (TEAM / 64)];
  TeamSum<TEAM, float> sum(slots);
  const uint32_t t = threadIdx.x % TEAM;
  const int64_t team = team_index<TEAM>();
  if (TEAM > 64 && team >= a.share.teams) return;   // (teams of a wave meet at the end)
  int64_t row, end;
  if (a.share.per_group > 0) {
    const int64_t group = team / a.share.per_group, last = (group + 1) * a.gate_rows;
    row = group * a.gate_rows + (team - group * a.share.per_group) * a.share.rows;
    end = row + a.share.rows < last ? row + a.share.rows : last;
  } else {
    row = team * a.share.rows;
    end = row + a.share.rows;
  }
  end = end < a.M ? end : a.M;
  if (team >= a.share.teams) end = row;

  const int64_t first = row;
  const uint32_t rows = row < end ? (uint32_t)(end - row) : 0;
  using In = TeamRows<T, FORM>;
  const TeamRows<T, FORM, true> from_dr(a.dr_out, first, rows, a.C);
  const In from_dn(a.dn, first, rows, a.C), to_r(a.dr, first, rows, a.C), to_b(a.db, first, rows, a.C);
  const StoreRows<K> kept_n(a.ckpt_n, a.M, a.pieces, first, rows);
  const StoreRows<K, true> kept_b(a.ckpt_b, a.M, a.pieces, first, rows);
  const auto lane = lanes<T, FORM, TEAM>(t, a.C, a.pieces, std::make_integer_sequence<int, NV>{});
  RowIn<T, K, NV> in;
  auto fetch = [&](uint32_t k) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      in.dn[i] = from_dn.load(k, lane.l[i]);
      in.dr[i] = from_dr.load(k, lane.l[i]);
      kept_n.load(k, lane.s[i], in.z[i], in.sz[i]);
      kept_b.load(k, lane.s[i], in.y[i], in.sy[i]);
    }
    in.rstd_n = a.rstd_n[first + k];
    in.rstd_b = a.w_post != nullptr ? a.rstd_b[first + k] : 0.0f;
  };
  float pre[NV][8] = {}, post[NV][8] = {}, both[NV][8] = {};   // sums of dn z; of e gate y; of D y over the rows of a group
  Raw<T> w_pre[kHold ? NV : 1], w_post[kHold ? NV : 1], gate[kHold ? NV : 1];
  auto weights = [&](const Raw<T>* held, const void* from, int64_t row, int i, float (&w)[8]) __attribute__((always_inline)) {
    if constexpr (kHold)
      expand(held[i], w);
    else
      expand(load_weights<T, FORM>(from, row, a.C, lane.l[i]), w);
  };
  const bool flush = a.gate != nullptr && a.share.per_group == 0;
  int64_t group = a.gate != nullptr ? row / a.gate_rows : 0;
  int64_t group_end = flush ? (group + 1) * a.gate_rows : a.M;
  if (kHold && rows > 0) {
    fetch(0);
#pragma unroll
    for (int i = 0; i < (kHold ? NV : 0); ++i) {
      w_pre[i] = load_weights<T, FORM>(a.w_pre, 0, a.C, lane.l[i]);
      w_post[i] = load_weights<T, FORM>(a.w_post, 0, a.C, lane.l[i]);
      gate[i] = load_weights<T, FORM>(a.gate, group, a.C, lane.l[i]);
    }
#pragma unroll
    for (int i = 0; i < (kHold ? NV : 0); ++i) settle(w_pre[i]), settle(w_post[i]), settle(gate[i]);
  }
  for (uint32_t k = 0; k < rows; ++k) {
    float v[NV][8], y[NV][8], w[8], g[8];
    if (!kHold) fetch(k);
    const RowIn<T, K, NV> now = in;
    if (kHold && k + 1 < rows) fetch(k + 1);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      decode<K>(now.z[i], now.sz[i], y[i]);
      unpack(now.dn[i], lane.l[i], v[i]);
      weights(w_pre, a.w_pre, 0, i, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        pre[i][j] = __builtin_fmaf(v[i][j], y[i][j], pre[i][j]);
        v[i][j] *= w[j];
      }
    }
    norm_gradient<TEAM, NV>(v, y, now.rstd_n, a, sum, [&](int i, float (&t)[8]) __attribute__((always_inline)) { unpack(now.dr[i], lane.l[i], t); });
#pragma unroll
    for (int i = 0; i < NV; ++i) {   // v is D
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = a.alpha * v[i][j];
      to_r.store(k, lane.l[i], w);
      decode<K>(now.y[i], now.sy[i], y[i]);   // (zeros where nothing is kept of b)
      weights(w_post, a.w_post, 0, i, w);
      weights(gate, a.gate, group, i, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        both[i][j] = __builtin_fmaf(v[i][j], y[i][j], both[i][j]);
        v[i][j] *= g[j] * w[j];
      }
    }
    if (a.w_post != nullptr) {
      norm_gradient<TEAM, NV>(v, y, a.beta * now.rstd_b, a, sum, [&](int, float (&t)[8]) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = 0.0f;
      });
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] *= a.beta;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) to_b.store(k, lane.l[i], v[i]);
    if (flush && (first + k + 1 == group_end || k + 1 == rows)) {   // (a team's last row ends a group)
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const uint32_t c = (t + TEAM * i) * 8;
        weights(w_post, a.w_post, 0, i, w);
        weights(gate, a.gate, group, i, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float e = a.beta * both[i][j];
          post[i][j] = __builtin_fmaf(e, g[j], post[i][j]);
          w[j] *= e;
          both[i][j] = 0.0f;
        }
        store_piece(a.dgate + group * a.C + c, left(a.C, c), w);
      }
      ++group;
      group_end += a.gate_rows;
      if (kHold && k + 1 < rows) {
#pragma unroll
        for (int i = 0; i < (kHold ? NV : 0); ++i) gate[i] = load_weights<T, FORM>(a.gate, group, a.C, lane.l[i]);
#pragma unroll
        for (int i = 0; i < (kHold ? NV : 0); ++i) settle(gate[i]);
      }
    }
  }
  if (!flush) {   // one row of the gate, or none: both sums are multiples of one
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float w[8] = {}, g[8] = {};
      if (rows > 0) {
        weights(w_post, a.w_post, 0, i, w);
        weights(gate, a.gate, group, i, g);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float e = a.beta * both[i][j];
        post[i][j] = e * g[j];
        both[i][j] = e * w[j];
      }
    }
  }
  // The shares' sums, one for a block: the four teams of a wave each are added in LDS, one plane after the other.
  const int64_t width = (int64_t)a.pieces * 8, plane = (int64_t)gridDim.x * width;
  if constexpr (TEAM == 64) {
    static_assert(NV == 1, "teams of a wave have a piece a lane");
    __shared__ float parts[3][64][8];
    const int wave = threadIdx.x / 64;
    auto add = [&](float (&v)[8], int which) __attribute__((always_inline)) {
      if (wave > 0) store_piece(parts[wave - 1][t], 8, v);
      __syncthreads();
      if (wave == 0 && t < (uint32_t)a.pieces) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (v[j] + parts[0][t][j]) + (parts[1][t][j] + parts[2][t][j]);
        store_piece(a.part + which * plane + (int64_t)blockIdx.x * width + t * 8, 8, v);
      }
      __syncthreads();
    };
    add(pre[0], 0);
    if (a.w_post != nullptr) add(post[0], 1);
    if (a.share.per_group > 0) add(both[0], 2);
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t q = t + TEAM * i;
      if (q >= (uint32_t)a.pieces) continue;
      float* to = a.part + team * width + q * 8;
      store_piece(to, 8, pre[i]);
      if (a.w_post != nullptr) store_piece(to + plane, 8, post[i]);
      if (a.share.per_group > 0) store_piece(to + 2 * plane, 8, both[i]);
    }
  }
}

// The teams' sums: blockIdx.y = 0 dw_pre, 1 dw_post, 2 + g row g of dgate.  32 channels a block; thread (s, l) adds every 64th share
// of four channels, eight of them on their way at a time, then the 64 sums are added in turn.
constexpr int kSumRows = 64;
__global__ __launch_bounds__(8 * kSumRows) void resnorm_sum_kernel(const float* part, int64_t shares, int64_t per_group, int pieces, int C, float* dw_pre,
                                                                   float* dw_post, float* dgate) {
  __shared__ float4 sums[kSumRows][8];
  const int job = blockIdx.y, l = threadIdx.x & 7, s = threadIdx.x >> 3;
  float* out = job == 0 ? dw_pre : job == 1 ? dw_post : dgate + (int64_t)(job - 2) * C;
  if (out == nullptr) return;
  const int64_t width = (int64_t)pieces * 8, plane = shares * width;
  const int64_t first = job < 2 ? 0 : (job - 2) * per_group, last = job < 2 ? shares : first + per_group;
  const float* from = part + (job < 2 ? job : 2) * plane + (int64_t)blockIdx.x * 32 + l * 4;
  float4 a{0.0f, 0.0f, 0.0f, 0.0f};
  for (int64_t i = first + s; i < last; i += 8 * kSumRows) {
    float4 v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      v[k] = i + k * kSumRows < last ? *reinterpret_cast<const float4*>(from + (i + k * kSumRows) * width) : float4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < 8; ++k) a.x += v[k].x, a.y += v[k].y, a.z += v[k].z, a.w += v[k].w;
  }
  sums[s][l] = a;
  __syncthreads();
  if (threadIdx.x >= 32) return;
  const float* at = reinterpret_cast<const float*>(sums) + threadIdx.x;
  float total = 0.0f;
#pragma unroll 16
  for (int i = 0; i < kSumRows; ++i) total += at[32 * i];
  const int c = blockIdx.x * 32 + threadIdx.x;
  if (c < C) out[c] = total;
}

// (plain stores, not a memset: the call may be captured into a graph)
__global__ __launch_bounds__(256) void zero_kernel(float* p, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) p[i] = 0.0f;
}

// Threads of a team for rows of so many pieces: a piece for each up to 512 threads, then two and four (a block of 1024 threads has too few
// registers for the backward: 4096 x 8192 bf16 took 162 us).  Between 128 and 256 also 192, against 256 (13 shapes of 1032 to 1536 channels, both
// types): forward 0.88 to 1.05 of the time, 0.94 in the mean (1500 x 1111 fp32 10.1 instead of 11.4 us, 4096 x 1500 bf16 14.3 instead
// of 16.2); backward 0.91 to 1.10, 1.00 in the mean (1500 x 1111 fp32 15.1 instead of 16.1, 4096 x 1280 fp32 28.4 instead of 25.9).
// 384 and 768 threads, launched by the rules above (330 and 170 blocks for 256 units in the backward), lost to 512 with idle threads or two
// pieces: 8192 x 2560 bf16 50 and 60 us instead of 45 and 54, 4096 x 5120 51 and 66 instead of 46 and 56; launches of a whole number of
// blocks a unit were not tried with them.
int team_of(int pieces) {
  for (int t : {64, 128, 192, 256})
    if (pieces <= t) return t;
  return 512;
}

// f(TEAM, NV, FORM) as constants.
template <typename F>
void by_team(int C, int64_t bytes, F&& f) {
  const int pieces = (int)store_blocks(C) * 4;
  auto form = [&](auto team, auto nv) {
    if constexpr (decltype(team)::value >= 256) {
      if (C % 8 == 0 && bytes > kStreamBytes) return f(team, nv, std::integral_constant<Form, kStream>{});
    }
    if (C % 8 == 0) return f(team, nv, std::integral_constant<Form, kWhole>{});
    return f(team, nv, std::integral_constant<Form, kRagged>{});
  };
  const std::integral_constant<int, 1> one;
  if (C < 8) return f(std::integral_constant<int, 64>{}, one, std::integral_constant<Form, kShort>{});
  switch (team_of(pieces)) {
    case 64: return form(std::integral_constant<int, 64>{}, one);
    case 128: return form(std::integral_constant<int, 128>{}, one);
    case 192: return form(std::integral_constant<int, 192>{}, one);
    case 256: return form(std::integral_constant<int, 256>{}, one);
    default: {
      const std::integral_constant<int, 512> team;
      if (pieces <= 512) return form(team, one);
      if (pieces <= 1024) return form(team, std::integral_constant<int, 2>{});
      return form(team, std::integral_constant<int, 4>{});
    }
  }
}

}  // namespace

int launch_resnorm_forward(hipStream_t st, const abl_resnorm& s, const void* r, const void* b, const void* gate, const void* w_post,
                           const void* w_pre, void* r_out, void* n, void* ckpt_b, float* rstd_b, void* ckpt_n, float* rstd_n) {
  FwdArgs a;
  a.M = s.M, a.gate_rows = s.gate_rows < s.M ? s.gate_rows : s.M, a.r = r, a.b = b, a.gate = gate, a.w_post = w_post, a.w_pre = w_pre;
  a.r_out = r_out, a.n = n, a.ckpt_b = (unsigned char*)ckpt_b, a.ckpt_n = (unsigned char*)ckpt_n;
  a.rstd_b = rstd_b, a.rstd_n = rstd_n, a.C = s.C, a.pieces = (int)store_blocks(s.C) * 4;
  a.center = (s.flags & ABL_NORM_CENTER) != 0, a.alpha = s.alpha, a.beta = s.beta, a.eps = s.eps, a.inv_c = 1.0 / s.C;
  const int64_t bytes = s.M * s.C * (4 * size_of(s.dtype) + 2 * s.K / 8);
  by_team(s.C, bytes, [&](auto t, auto nv, auto form) {
    constexpr int TEAM = decltype(t)::value, NV = decltype(nv)::value;
    constexpr Form FORM = decltype(form)::value;
    const int64_t most = fwd_threads(NV) / TEAM;
    a.rows = (s.M + most - 1) / most;
    const int64_t teams = (s.M + a.rows - 1) / a.rows;
    const unsigned grid = (unsigned)(TEAM == 64 ? (teams + 3) / 4 : teams);
    auto pick = [&](auto e) {
      using T = decltype(e);
      return s.K == 0   ? resnorm_fwd_kernel<T, 0, FORM, TEAM, NV>
             : s.K == 8 ? resnorm_fwd_kernel<T, 8, FORM, TEAM, NV>
                        : resnorm_fwd_kernel<T, 4, FORM, TEAM, NV>;
    };
    auto kern = s.dtype == ABL_F32 ? pick(float{}) : pick(bf16_t{});
    kern<<<grid, kBlock<TEAM>, 0, st>>>(a);
  });
  return hip_status();
}

size_t resnorm_scratch_bytes(int64_t M, int C) {
  const int pieces = (int)store_blocks(C) * 4;
  // The blocks without a gate, and where groups of rows are cut: a group of g rows takes at most g / rows + 1 teams, or a block more where a block
  // has four, and there are M / g + 1 groups of more than `rows` rows, so at most M / rows + M / g + g / rows + ... <= 2 M / rows + 2 blocks' worth.
  const int team = team_of(pieces);
  const Shares s = shares_of(M > 0 ? M : 1, 0, team, false);   // (no rows: a size that is never 0 for valid arguments)
  const int64_t blocks = 2 * s.teams + 2;
  return (size_t)blocks * 3 * pieces * 8 * sizeof(float);
}

int launch_resnorm_backward(hipStream_t st, const abl_resnorm& s, const void* dn, const void* dr_out, const void* gate, const void* w_post,
                            const void* w_pre, const void* ckpt_b, const float* rstd_b, const void* ckpt_n, const float* rstd_n,
                            void* scratch, void* dr, void* db, float* dgate, float* dw_post, float* dw_pre) {
  const int64_t groups = gate != nullptr && s.M > 0 ? (s.M - 1) / s.gate_rows + 1 : 0;
  if (s.M == 0) {
    for (float* p : {dw_pre, dw_post})
      if (p != nullptr) zero_kernel<<<(unsigned)((s.C + 255) / 256), 256, 0, st>>>(p, s.C);
    return hip_status();
  }
  BwdArgs a;
  a.M = s.M, a.gate_rows = s.gate_rows < s.M ? s.gate_rows : s.M, a.dn = dn, a.dr_out = dr_out, a.gate = gate, a.w_post = w_post, a.w_pre = w_pre;
  a.ckpt_b = (const unsigned char*)ckpt_b, a.ckpt_n = (const unsigned char*)ckpt_n, a.rstd_b = rstd_b, a.rstd_n = rstd_n;
  a.dr = dr, a.db = db, a.dgate = dgate, a.part = (float*)scratch;
  a.C = s.C, a.pieces = (int)store_blocks(s.C) * 4, a.center = (s.flags & ABL_NORM_CENTER) != 0;
  a.alpha = s.alpha, a.beta = s.beta, a.inv_c = 1.0f / (float)s.C;
  a.share = shares_of(s.M, s.gate_rows, team_of(a.pieces), gate != nullptr);
  const int64_t bytes = s.M * s.C * (4 * size_of(s.dtype) + 2 * s.K / 8);
  by_team(s.C, bytes, [&](auto t, auto nv, auto form) {
    constexpr int TEAM = decltype(t)::value, NV = decltype(nv)::value;
    constexpr Form FORM = decltype(form)::value;
    const unsigned grid = (unsigned)(TEAM == 64 ? (a.share.teams + 3) / 4 : a.share.teams);
    auto pick = [&](auto e) {
      using T = decltype(e);
      return s.K == 8 ? resnorm_bwd_kernel<T, 8, FORM, TEAM, NV> : resnorm_bwd_kernel<T, 4, FORM, TEAM, NV>;
    };
    auto kern = s.dtype == ABL_F32 ? pick(float{}) : pick(bf16_t{});
    kern<<<grid, kBlock<TEAM>, 0, st>>>(a);
  });
  if (int e = hip_status()) return e;
  const int64_t a_block = team_of(a.pieces) == 64 ? 4 : 1, blocks = (a.share.teams + a_block - 1) / a_block;   // teams of a block
  const unsigned jobs = 2 + (gate != nullptr && a.share.per_group > 0 ? (unsigned)groups : 0);
  resnorm_sum_kernel<<<dim3((unsigned)((s.C + 31) / 32), jobs), 8 * kSumRows, 0, st>>>(a.part, blocks, a.share.per_group / a_block, a.pieces, s.C, dw_pre, dw_post, dgate);
  return hip_status();
}

}  // namespace abl
