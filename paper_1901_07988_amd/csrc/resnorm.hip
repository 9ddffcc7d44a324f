// The step between two blocks of a residual network (abl_resnorm_forward / abl_resnorm_backward):
//
//   y = N(b),  p = gate (w_post y),  r' = alpha r + beta p,  z = N(r'),  n = w_pre z          stores of y and z
//
//   D  = dr' + rstd_r (v - z mean(v z)),   v = dn w_pre           (ABL_NORM_CENTER: less the mean of v too)
//   dr = alpha D,   e = beta D,   dgate = sum e w_post y,   dw_post = sum e gate y,   dw_pre = sum dn z
//   db = rstd_b (v - y mean(v y)),   v = e gate w_post
//
// Both are bound by memory: an element of bf16 costs 8 bytes and its two stores (10.1 at K = 8).  A team of threads holds a row in registers,
// so that every tensor is read once; the sums over a row go through the waves' registers and, between waves, LDS.  In the
// backward a team takes consecutive rows and keeps its share of the sums over rows in registers as well; the teams' sums are added
// in a fixed order by a second launch.

#include "block_store.h"

namespace abl {
namespace {

// Channels that exist from channel c on (none or fewer for a thread beyond the row's end).
__device__ inline int left(int C, uint32_t c) { return C - (int)c; }

// ---- a team's rows in memory ----
// A team has consecutive rows, and accesses go through buffer descriptors of them: a lane beyond the row's end has an offset beyond
// the descriptor, and a tensor that is not there has a descriptor of no bytes; both read zero and store nothing.  Without branches
// around them the compiler can count the accesses on their way, so waiting for the next row's loads does not wait for
// this row's stores, and from row to row only three scalar offsets change.  (A store takes the sum of its offsets in a vector register:
// with the row's in the instruction's scalar operand the compiler lets the next instruction overwrite the store's data, and wrong
// words have been written here.)
// Rows of T from `first` on; WHOLE: of a multiple of eight channels.  Others take their last piece in parts (load_raw, store_piece).
// Piece q of the k-th row; `at`: this lane's byte offset of it in a row (kNowhere beyond the end).
template <typename T, bool WHOLE>
struct TeamRows {
  const T* p;
  int C;
  __amdgpu_buffer_rsrc_t d;
  __device__ inline TeamRows(const void* base, int64_t first, int64_t rows, int c)
      : p(base != nullptr ? (const T*)base + first * c : nullptr), C(c), d(descriptor(p, rows * c * (int64_t)sizeof(T))) {}
  static __device__ inline uint32_t offset(uint32_t q, int c) {
    return q * 8 < (uint32_t)c ? q * 8 * (uint32_t)sizeof(T) : kNowhere;
  }
  __device__ inline Raw<T> load(uint32_t k, uint32_t q, uint32_t at) const {
    if constexpr (!WHOLE) {
      return p != nullptr ? load_raw(p + (int64_t)k * C + q * 8, left(C, q * 8)) : Raw<T>{};
    } else {
      const uint32_t row = k * (uint32_t)C * (uint32_t)sizeof(T);
      if constexpr (std::is_same_v<T, float>) {
        Raw<float> r;
        r.a = __builtin_bit_cast(f32x4_any4, __builtin_amdgcn_raw_buffer_load_b128(d, at, row, 0));
        r.b = __builtin_bit_cast(f32x4_any4, __builtin_amdgcn_raw_buffer_load_b128(d, at, row + 16, 0));
        return r;
      } else {
        return Raw<bf16_t>{__builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(d, at, row, 0))};
      }
    }
  }
  __device__ inline void store(uint32_t k, uint32_t q, uint32_t at, const float (&v)[8]) const {
    if constexpr (!WHOLE) {
      if (p != nullptr) store_piece(const_cast<T*>(p) + (int64_t)k * C + q * 8, left(C, q * 8), v);
    } else {
      const uint32_t row = k * (uint32_t)C * (uint32_t)sizeof(T);
      if constexpr (std::is_same_v<T, float>) {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4_any4{v[0], v[1], v[2], v[3]}), d, at + row, 0, 0);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4_any4{v[4], v[5], v[6], v[7]}), d, at + row + 16, 0, 0);
      } else {
        __builtin_amdgcn_raw_buffer_store_b128(u32x4{two_bf16(v[0], v[1]), two_bf16(v[2], v[3]), two_bf16(v[4], v[5]), two_bf16(v[6], v[7])}, d,
                                               at + row, 0, 0);
      }
    }
  }
};

// The rows of a store: `pieces` = 4 B of each.
template <int K>
struct StoreRows {
  __amdgpu_buffer_rsrc_t codes, scales;
  uint32_t pieces;
  __device__ inline StoreRows(const unsigned char* store, int64_t M, int n, int64_t first, int64_t rows)
      : codes(descriptor(store != nullptr ? store + first * n * K : nullptr, rows * n * K)),
        scales(descriptor(store != nullptr ? store + M * n * K + (first * n >> 2) : nullptr, rows * n >> 2)),
        pieces((uint32_t)n) {}
  __device__ inline void load(uint32_t k, uint32_t q, Codes<K>& c, uint32_t& byte) const {
    const bool in = q < pieces;
    if constexpr (K == 8)
      c.w = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(codes, in ? q * 8 : kNowhere, k * pieces * 8, 0));
    else
      c.w = __builtin_amdgcn_raw_buffer_load_b32(codes, in ? q * 4 : kNowhere, k * pieces * 4, 0);
    byte = __builtin_amdgcn_raw_buffer_load_b8(scales, in ? q >> 2 : kNowhere, k * (pieces >> 2), 0);
  }
  __device__ inline void keep(uint32_t k, uint32_t q, const float (&v)[8]) const {
    const bool in = q < pieces;
    const uint32_t byte = scale_byte<K>(v);
    const Codes<K> c = encode<K>(v, byte);
    if constexpr (K == 8)
      __builtin_amdgcn_raw_buffer_store_b64(c.w, codes, (in ? q * 8 : kNowhere) + k * pieces * 8, 0, 0);
    else
      __builtin_amdgcn_raw_buffer_store_b32(c.w, codes, (in ? q * 4 : kNowhere) + k * pieces * 4, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b8((unsigned char)byte, scales, (in && (q & 3u) == 0 ? q >> 2 : kNowhere) + k * (pieces >> 2), 0, 0);
  }
};

// A vector over the channels, for all rows: ones where there is none.
template <typename T, bool WHOLE>
__device__ inline Raw<T> load_weights(const void* w, int64_t row, int C, uint32_t q) {
  if (w != nullptr) return TeamRows<T, WHOLE>(w, row, 1, C).load(0, q, TeamRows<T, WHOLE>::offset(q, C));
  Raw<T> r;
  if constexpr (std::is_same_v<T, float>)
    r.a = r.b = f32x4_any4{1.0f, 1.0f, 1.0f, 1.0f};
  else
    r.a = u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
  return r;
}

// ---- a team's sums over a row ----
template <int TEAM>
struct TeamSum {
  float* slots;   // [2][TEAM / 64], used in turn: the barrier of one sum keeps the next from overwriting what is still read
  int turn = 0;
  __device__ explicit TeamSum(float* s) : slots(s) {}
  __device__ inline float operator()(float v) {
    v = wave_sum(v);
    if constexpr (TEAM > 64) {
      float* s = slots + turn * (TEAM / 64);
      turn ^= 1;
      if ((threadIdx.x & 63u) == 0) s[threadIdx.x >> 6] = v;
      __syncthreads();
      v = 0.0f;
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
  float alpha, beta, eps, inv_c;
};

__device__ inline void zero_tail(unsigned char* store, int64_t pieces, int K) {
  const int64_t used = pieces * K + (pieces >> 2);
  const int64_t all = (used + 127) / 128 * 128;
  for (int64_t i = used + threadIdx.x; i < all; i += blockDim.x) store[i] = 0;
}

// v <- N(v); returns 1 / sqrt(mean square + eps).  Channels that do not exist hold zeros and stay zero.
template <int TEAM, int NV>
__device__ inline float normalize(float (&v)[NV][8], const FwdArgs& a, TeamSum<TEAM>& sum, uint32_t t) {
  if (a.center) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) m += v[i][j];
    m = sum(m) * a.inv_c;
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
  const float rstd = 1.0f / sqrtf(__builtin_fmaf(sum(s), a.inv_c, a.eps));
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] *= rstd;
  return rstd;
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
template <typename T, int K, bool WHOLE, int TEAM, int NV>
__global__ __launch_bounds__(kBlock<TEAM>) void resnorm_fwd_kernel(FwdArgs a) {
  __shared__ float slots[2 * (TEAM / 64)];
  TeamSum<TEAM> sum(slots);
  const uint32_t t = threadIdx.x % TEAM;
  if (K != 0 && blockIdx.x == 0) {
    zero_tail(a.ckpt_n, a.M * a.pieces, K);
    if (a.ckpt_b != nullptr) zero_tail(a.ckpt_b, a.M * a.pieces, K);
  }
  const int64_t first = team_index<TEAM>() * a.rows;
  if (first >= a.M) return;   // (a whole wave; blocks of larger teams are as many as teams)
  const uint32_t rows = (uint32_t)(first + a.rows < a.M ? a.rows : a.M - first);
  using In = TeamRows<T, WHOLE>;
  const In from_r(a.r, first, rows, a.C), from_b(a.b, first, rows, a.C), to_r(a.r_out, first, rows, a.C), to_n(a.n, first, rows, a.C);
  const StoreRows<K == 0 ? 8 : K> keep_b(K != 0 ? a.ckpt_b : nullptr, a.M, a.pieces, first, rows);
  const StoreRows<K == 0 ? 8 : K> keep_n(K != 0 ? a.ckpt_n : nullptr, a.M, a.pieces, first, rows);
  uint32_t at[NV];
  Raw<T> r[NV], b[NV], w_post[NV], w_pre[NV], gate[NV];
  auto fetch = [&](uint32_t k) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      r[i] = from_r.load(k, t + TEAM * i, at[i]);
      b[i] = from_b.load(k, t + TEAM * i, at[i]);
    }
  };
  int64_t group = a.gate != nullptr ? first / a.gate_rows : 0;
  int64_t group_end = a.gate != nullptr ? (group + 1) * a.gate_rows : a.M;
#pragma unroll
  for (int i = 0; i < NV; ++i) at[i] = In::offset(t + TEAM * i, a.C);
  fetch(0);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    w_pre[i] = load_weights<T, WHOLE>(a.w_pre, 0, a.C, t + TEAM * i);
    w_post[i] = load_weights<T, WHOLE>(a.w_post, 0, a.C, t + TEAM * i);
    gate[i] = load_weights<T, WHOLE>(a.gate, group, a.C, t + TEAM * i);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) settle(w_pre[i]), settle(w_post[i]), settle(gate[i]);
  for (uint32_t k = 0; k < rows; ++k) {
    float v[NV][8], x[NV][8], w[8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      expand(r[i], x[i]);
      expand(b[i], v[i]);
    }
    if (k + 1 < rows) fetch(k + 1);
    if (a.w_post != nullptr) {
      const float rstd = normalize<TEAM, NV>(v, a, sum, t);
      if (K != 0 && t == 0) a.rstd_b[first + k] = rstd;
    }
    if constexpr (K != 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i) keep_b.keep(k, t + TEAM * i, v[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      expand(w_post[i], w);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] *= w[j];
      expand(gate[i], w);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = a.alpha * x[i][j] + a.beta * (v[i][j] * w[j]);   // (v is zero where there is no b)
      to_r.store(k, t + TEAM * i, at[i], v[i]);
    }
    if (first + k + 1 == group_end && k + 1 < rows) {   // the next row has the next gate
      ++group;
      group_end += a.gate_rows;
#pragma unroll
      for (int i = 0; i < NV; ++i) gate[i] = load_weights<T, WHOLE>(a.gate, group, a.C, t + TEAM * i);
#pragma unroll
      for (int i = 0; i < NV; ++i) settle(gate[i]);
    }
    const float rstd = normalize<TEAM, NV>(v, a, sum, t);
    if constexpr (K != 0) {
      if (t == 0) a.rstd_n[first + k] = rstd;
#pragma unroll
      for (int i = 0; i < NV; ++i) keep_n.keep(k, t + TEAM * i, v[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      expand(w_pre[i], w);
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] *= v[i][j];
      to_n.store(k, t + TEAM * i, at[i], w);
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

constexpr int64_t kFwdThreads = 256 * 1024, kBwdThreads = 256 * 1024;   // of a launch at most (256 compute units)
Shares shares_of(int64_t M, int64_t gate_rows, int team, bool gate) {
  const int64_t most = kBwdThreads / team;   // up to twice as many where groups are cut
  Shares s;
  s.rows = (M + most - 1) / most;
  if (gate && gate_rows <= s.rows) {
    s.rows = (s.rows + gate_rows - 1) / gate_rows * gate_rows;
  } else if (gate && gate_rows < M) {
    s.per_group = (gate_rows + s.rows - 1) / s.rows;
    s.rows = (gate_rows + s.per_group - 1) / s.per_group;
    s.teams = (M + gate_rows - 1) / gate_rows * s.per_group;
    return s;
  } else if (gate) {   // one group
    s.per_group = (M + s.rows - 1) / s.rows;
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

// v <- rstd (v - y mean(v y)) (less the mean of v where the norm took the mean out)
template <int TEAM, int NV>
__device__ inline void norm_gradient(float (&v)[NV][8], const float (&y)[NV][8], float rstd, const BwdArgs& a, TeamSum<TEAM>& sum) {
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
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = rstd * (v[i][j] - m - y[i][j] * s);
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
template <typename T, int K, bool WHOLE, int TEAM, int NV>
__global__ __launch_bounds__(kBlock<TEAM>, 4) void resnorm_bwd_kernel(BwdArgs a) {
  __shared__ float slots[2 * (TEAM / 64)];
  TeamSum<TEAM> sum(slots);
  const uint32_t t = threadIdx.x % TEAM;
  const int64_t team = team_index<TEAM>();
  if (team >= a.share.teams) return;
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

  const int64_t first = row;
  const uint32_t rows = row < end ? (uint32_t)(end - row) : 0;
  using In = TeamRows<T, WHOLE>;
  const In from_dn(a.dn, first, rows, a.C), from_dr(a.dr_out, first, rows, a.C), to_r(a.dr, first, rows, a.C), to_b(a.db, first, rows, a.C);
  const StoreRows<K> kept_n(a.ckpt_n, a.M, a.pieces, first, rows), kept_b(a.ckpt_b, a.M, a.pieces, first, rows);
  uint32_t at[NV];
  RowIn<T, K, NV> in;
  auto fetch = [&](uint32_t k) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t q = t + TEAM * i;
      in.dn[i] = from_dn.load(k, q, at[i]);
      in.dr[i] = from_dr.load(k, q, at[i]);
      kept_n.load(k, q, in.z[i], in.sz[i]);
      kept_b.load(k, q, in.y[i], in.sy[i]);
    }
    in.rstd_n = a.rstd_n[first + k];
    in.rstd_b = a.w_post != nullptr ? a.rstd_b[first + k] : 0.0f;
  };
  float pre[NV][8] = {}, post[NV][8] = {}, gsum[NV][8] = {};
  Raw<T> w_pre[NV], w_post[NV], gate[NV];
  const bool flush = a.gate != nullptr && a.share.per_group == 0;
  int64_t group = a.gate != nullptr ? row / a.gate_rows : 0;
  int64_t group_end = flush ? (group + 1) * a.gate_rows : a.M;
#pragma unroll
  for (int i = 0; i < NV; ++i) at[i] = In::offset(t + TEAM * i, a.C);
  if (rows > 0) {
    fetch(0);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      w_pre[i] = load_weights<T, WHOLE>(a.w_pre, 0, a.C, t + TEAM * i);
      w_post[i] = load_weights<T, WHOLE>(a.w_post, 0, a.C, t + TEAM * i);
      gate[i] = load_weights<T, WHOLE>(a.gate, group, a.C, t + TEAM * i);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) settle(w_pre[i]), settle(w_post[i]), settle(gate[i]);
  }
  for (uint32_t k = 0; k < rows; ++k) {
    float v[NV][8], y[NV][8], w[8], g[8];
    const RowIn<T, K, NV> now = in;
    if (k + 1 < rows) fetch(k + 1);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      decode<K>(now.z[i], now.sz[i], y[i]);
      expand(now.dn[i], v[i]);
      expand(w_pre[i], w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        pre[i][j] = __builtin_fmaf(v[i][j], y[i][j], pre[i][j]);
        v[i][j] *= w[j];
      }
    }
    norm_gradient<TEAM, NV>(v, y, now.rstd_n, a, sum);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      expand(now.dr[i], w);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] += w[j];
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = a.alpha * v[i][j];
      to_r.store(k, t + TEAM * i, at[i], w);
      decode<K>(now.y[i], now.sy[i], y[i]);   // (zeros where nothing is kept of b)
      expand(w_post[i], w);
      expand(gate[i], g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float e = a.beta * v[i][j], ey = e * y[i][j];
        gsum[i][j] = __builtin_fmaf(ey, w[j], gsum[i][j]);
        post[i][j] = __builtin_fmaf(ey, g[j], post[i][j]);
        v[i][j] = e * g[j] * w[j];
      }
    }
    if (a.w_post != nullptr) norm_gradient<TEAM, NV>(v, y, now.rstd_b, a, sum);
#pragma unroll
    for (int i = 0; i < NV; ++i) to_b.store(k, t + TEAM * i, at[i], v[i]);
    if (flush && (first + k + 1 == group_end || k + 1 == rows)) {   // (a team's last row ends a group)
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const uint32_t c = (t + TEAM * i) * 8;
        store_piece(a.dgate + group * a.C + c, left(a.C, c), gsum[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) gsum[i][j] = 0.0f;
      }
      ++group;
      group_end += a.gate_rows;
      if (k + 1 < rows) {
#pragma unroll
        for (int i = 0; i < NV; ++i) gate[i] = load_weights<T, WHOLE>(a.gate, group, a.C, t + TEAM * i);
#pragma unroll
        for (int i = 0; i < NV; ++i) settle(gate[i]);
      }
    }
  }
  const int64_t width = (int64_t)a.pieces * 8, plane = a.share.teams * width;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const uint32_t q = t + TEAM * i;
    if (q >= (uint32_t)a.pieces) continue;
    float* to = a.part + team * width + q * 8;
    store_piece(to, 8, pre[i]);
    if (a.w_post != nullptr) store_piece(to + plane, 8, post[i]);
    if (a.share.per_group > 0) store_piece(to + 2 * plane, 8, gsum[i]);
  }
}

// The teams' sums: blockIdx.y = 0 dw_pre, 1 dw_post, 2 + g row g of dgate.  32 channels a block; thread (s, l) adds every 64th share
// of four channels, eight of them on their way at a time, then the 64 sums are added in turn.
constexpr int kSumRows = 64;
__global__ __launch_bounds__(8 * kSumRows) void resnorm_sum_kernel(const float* part, Shares share, int pieces, int C, float* dw_pre,
                                                                   float* dw_post, float* dgate) {
  __shared__ float4 sums[kSumRows][8];
  const int job = blockIdx.y, l = threadIdx.x & 7, s = threadIdx.x >> 3;
  float* out = job == 0 ? dw_pre : job == 1 ? dw_post : dgate + (int64_t)(job - 2) * C;
  if (out == nullptr) return;
  const int64_t width = (int64_t)pieces * 8, plane = share.teams * width;
  const int64_t first = job < 2 ? 0 : (job - 2) * share.per_group, last = job < 2 ? share.teams : first + share.per_group;
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

// Threads of a team for rows of so many pieces: a piece for each; above 1024 two.
int team_of(int pieces) {
  int t = 64;
  while (t < pieces && t < 1024) t *= 2;
  return t;
}

// f(TEAM, NV) as constants.
template <typename F>
void by_team(int pieces, F&& f) {
  const std::integral_constant<int, 1> one;
  switch (team_of(pieces)) {
    case 64: return f(std::integral_constant<int, 64>{}, one);
    case 128: return f(std::integral_constant<int, 128>{}, one);
    case 256: return f(std::integral_constant<int, 256>{}, one);
    case 512: return f(std::integral_constant<int, 512>{}, one);
    default:
      if (pieces <= 1024) return f(std::integral_constant<int, 1024>{}, one);
      return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
  }
}

}  // namespace

int launch_resnorm_forward(hipStream_t st, const abl_resnorm& s, const void* r, const void* b, const void* gate, const void* w_post,
                           const void* w_pre, void* r_out, void* n, void* ckpt_b, float* rstd_b, void* ckpt_n, float* rstd_n) {
  FwdArgs a;
  a.M = s.M, a.gate_rows = s.gate_rows, a.r = r, a.b = b, a.gate = gate, a.w_post = w_post, a.w_pre = w_pre;
  a.r_out = r_out, a.n = n, a.ckpt_b = (unsigned char*)ckpt_b, a.ckpt_n = (unsigned char*)ckpt_n;
  a.rstd_b = rstd_b, a.rstd_n = rstd_n, a.C = s.C, a.pieces = (int)store_blocks(s.C) * 4;
  a.center = (s.flags & ABL_NORM_CENTER) != 0, a.alpha = s.alpha, a.beta = s.beta, a.eps = s.eps, a.inv_c = 1.0f / (float)s.C;
  by_team(a.pieces, [&](auto t, auto nv) {
    constexpr int TEAM = decltype(t)::value, NV = decltype(nv)::value;
    const int64_t most = kFwdThreads / TEAM;
    a.rows = (s.M + most - 1) / most;
    const int64_t teams = (s.M + a.rows - 1) / a.rows;
    const unsigned grid = (unsigned)(TEAM == 64 ? (teams + 3) / 4 : teams);
    auto pick = [&](auto e) {
      using T = decltype(e);
      if (s.C % 8 == 0)
        return s.K == 0   ? resnorm_fwd_kernel<T, 0, true, TEAM, NV>
               : s.K == 8 ? resnorm_fwd_kernel<T, 8, true, TEAM, NV>
                          : resnorm_fwd_kernel<T, 4, true, TEAM, NV>;
      return s.K == 0   ? resnorm_fwd_kernel<T, 0, false, TEAM, NV>
             : s.K == 8 ? resnorm_fwd_kernel<T, 8, false, TEAM, NV>
                        : resnorm_fwd_kernel<T, 4, false, TEAM, NV>;
    };
    auto kern = s.dtype == ABL_F32 ? pick(float{}) : pick(bf16_t{});
    kern<<<grid, kBlock<TEAM>, 0, st>>>(a);
  });
  return hip_status();
}

size_t resnorm_scratch_bytes(int64_t M, int C) {
  const int pieces = (int)store_blocks(C) * 4;
  // the shares of the smallest rows, and twice as many where groups of the gate are cut
  const Shares s = shares_of(M, 0, team_of(pieces), false);
  return (size_t)(2 * s.teams + 1) * 3 * pieces * 8 * sizeof(float);
}

int launch_resnorm_backward(hipStream_t st, const abl_resnorm& s, bool has_b, const void* dn, const void* dr_out, const void* gate,
                            const void* w_post, const void* w_pre, const void* ckpt_b, const float* rstd_b, const void* ckpt_n,
                            const float* rstd_n, void* scratch, void* dr, void* db, float* dgate, float* dw_post, float* dw_pre) {
  const int64_t groups = gate != nullptr ? (s.M + s.gate_rows - 1) / s.gate_rows : 0;
  if (s.M == 0) {
    for (float* p : {dw_pre, dw_post})
      if (p != nullptr) zero_kernel<<<(unsigned)((s.C + 255) / 256), 256, 0, st>>>(p, s.C);
    return hip_status();
  }
  BwdArgs a;
  a.M = s.M, a.gate_rows = s.gate_rows, a.dn = dn, a.dr_out = dr_out, a.gate = gate, a.w_post = w_post, a.w_pre = w_pre;
  a.ckpt_b = (const unsigned char*)ckpt_b, a.ckpt_n = (const unsigned char*)ckpt_n, a.rstd_b = rstd_b, a.rstd_n = rstd_n;
  a.dr = dr, a.db = db, a.dgate = dgate, a.part = (float*)scratch;
  a.C = s.C, a.pieces = (int)store_blocks(s.C) * 4, a.center = (s.flags & ABL_NORM_CENTER) != 0;
  a.alpha = s.alpha, a.beta = s.beta, a.inv_c = 1.0f / (float)s.C;
  a.share = shares_of(s.M, s.gate_rows, team_of(a.pieces), gate != nullptr);
  by_team(a.pieces, [&](auto t, auto nv) {
    constexpr int TEAM = decltype(t)::value, NV = decltype(nv)::value;
    const unsigned grid = (unsigned)(TEAM == 64 ? (a.share.teams + 3) / 4 : a.share.teams);
    auto pick = [&](auto e) {
      using T = decltype(e);
      if (s.C % 8 == 0) return s.K == 8 ? resnorm_bwd_kernel<T, 8, true, TEAM, NV> : resnorm_bwd_kernel<T, 4, true, TEAM, NV>;
      return s.K == 8 ? resnorm_bwd_kernel<T, 8, false, TEAM, NV> : resnorm_bwd_kernel<T, 4, false, TEAM, NV>;
    };
    auto kern = s.dtype == ABL_F32 ? pick(float{}) : pick(bf16_t{});
    kern<<<grid, kBlock<TEAM>, 0, st>>>(a);
  });
  if (int e = hip_status()) return e;
  const unsigned jobs = 2 + (gate != nullptr && a.share.per_group > 0 ? (unsigned)groups : 0);
  resnorm_sum_kernel<<<dim3((unsigned)((s.C + 31) / 32), jobs), 8 * kSumRows, 0, st>>>(a.part, a.share, a.pieces, s.C, dw_pre, dw_post, dgate);
  return hip_status();
}

}  // namespace abl
