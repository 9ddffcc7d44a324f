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
  int C, pieces;   // pieces of a row
  int K, center;
  float alpha, beta, eps, inv_c;
};

template <int K, int TEAM, int NV>
__device__ inline void keep_row(unsigned char* store, int64_t M, int pieces, int64_t row, int t, const float (&v)[NV][8]) {
  unsigned char* scales = store + M * pieces * K;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int q = t + TEAM * i;
    if (q < pieces) keep_piece<K>(store, scales, row * pieces + q, v[i]);
  }
}
__device__ inline void zero_tail(unsigned char* store, int64_t pieces, int K) {
  const int64_t used = pieces * K + (pieces >> 2);
  const int64_t all = (used + 127) / 128 * 128;
  for (int64_t i = used + threadIdx.x; i < all; i += blockDim.x) store[i] = 0;
}

// v <- N(v); returns 1 / sqrt(mean square + eps).  Channels that do not exist hold zeros and stay zero.
template <int TEAM, int NV>
__device__ inline float normalize(float (&v)[NV][8], const FwdArgs& a, TeamSum<TEAM>& sum, int t) {
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
        if ((t + TEAM * i) * 8 + j < a.C) v[i][j] -= m;
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

template <int TEAM>
constexpr int kBlockOf = TEAM < 256 ? 256 : TEAM;   // threads of a block; teams of more than a wave have it to themselves

template <typename T, int TEAM, int NV>
__global__ __launch_bounds__(TEAM == 64 ? 256 : TEAM) void resnorm_fwd_kernel(FwdArgs a) {
  __shared__ float slots[2 * (TEAM / 64)];
  TeamSum<TEAM> sum(slots);
  const int t = threadIdx.x % TEAM;
  const int64_t row = TEAM == 64 ? (int64_t)blockIdx.x * 4 + threadIdx.x / 64 : (int64_t)blockIdx.x;
  if (blockIdx.x == 0 && a.K != 0) {
    if (a.ckpt_n != nullptr) zero_tail(a.ckpt_n, a.M * a.pieces, a.K);
    if (a.ckpt_b != nullptr) zero_tail(a.ckpt_b, a.M * a.pieces, a.K);
  }
  if (row >= a.M) return;   // (a whole wave; blocks of larger teams have one row each)
  const T* r = (const T*)a.r + row * a.C;
  const T* b = (const T*)a.b + row * a.C;
  const T* gate = (const T*)a.gate + (a.gate != nullptr ? row / a.gate_rows * a.C : 0);
  Raw<T> rr[NV];
  float v[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + TEAM * i) * 8;
    rr[i] = load_raw(r + c, a.C - c);
    if (a.b != nullptr) load_piece(b + c, a.C - c, v[i]);
  }
  if (a.b != nullptr) {
    if (a.w_post != nullptr) {
      const float rstd = normalize<TEAM, NV>(v, a, sum, t);
      if (a.rstd_b != nullptr && t == 0) a.rstd_b[row] = rstd;
    }
    if (a.ckpt_b != nullptr) {
      if (a.K == 8)
        keep_row<8, TEAM, NV>(a.ckpt_b, a.M, a.pieces, row, t, v);
      else
        keep_row<4, TEAM, NV>(a.ckpt_b, a.M, a.pieces, row, t, v);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + TEAM * i) * 8;
      float w[8];
      if (a.w_post != nullptr) {
        load_piece((const T*)a.w_post + c, a.C - c, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] *= w[j];
      }
      if (a.gate != nullptr) {
        load_piece(gate + c, a.C - c, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] *= w[j];
      }
      expand(rr[i], w);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = a.alpha * w[j] + a.beta * v[i][j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      expand(rr[i], v[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] *= a.alpha;
    }
  }
  if (a.r_out != nullptr) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + TEAM * i) * 8;
      store_piece((T*)a.r_out + row * a.C + c, a.C - c, v[i]);
    }
  }
  const float rstd = normalize<TEAM, NV>(v, a, sum, t);
  if (a.rstd_n != nullptr && t == 0) a.rstd_n[row] = rstd;
  if (a.ckpt_n != nullptr) {
    if (a.K == 8)
      keep_row<8, TEAM, NV>(a.ckpt_n, a.M, a.pieces, row, t, v);
    else
      keep_row<4, TEAM, NV>(a.ckpt_n, a.M, a.pieces, row, t, v);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + TEAM * i) * 8;
    float w[8];
    load_piece((const T*)a.w_pre + c, a.C - c, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] *= v[i][j];
    store_piece((T*)a.n + row * a.C + c, a.C - c, w);
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

constexpr int64_t kTeams = 1024;   // asked for; up to twice as many where groups are cut
Shares shares_of(int64_t M, int64_t gate_rows, int team, bool gate) {
  const int64_t most = team == 64 ? 2 * kTeams : team <= 256 ? kTeams : team == 512 ? kTeams / 2 : kTeams / 4;
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
  int C, pieces, K, center, has_b;
  float alpha, beta, inv_c;
};

template <int K, int TEAM, int NV>
__device__ inline void read_row(const unsigned char* store, int64_t M, int pieces, int64_t row, int t, float (&v)[NV][8]) {
  const unsigned char* scales = store + M * pieces * K;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int q = t + TEAM * i;
    if (q < pieces) {
      const int64_t p = row * pieces + q;
      decode<K>(load_codes<K>(store, p), scales[p >> 2], v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
    }
  }
}

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

template <typename T, int TEAM, int NV>
__global__ __launch_bounds__(TEAM == 64 ? 256 : TEAM) void resnorm_bwd_kernel(BwdArgs a) {
  __shared__ float slots[2 * (TEAM / 64)];
  TeamSum<TEAM> sum(slots);
  const int t = threadIdx.x % TEAM;
  const int64_t team = TEAM == 64 ? (int64_t)blockIdx.x * 4 + threadIdx.x / 64 : (int64_t)blockIdx.x;
  if (team >= a.share.teams) return;
  int64_t row, end;
  if (a.share.per_group > 0 && a.gate != nullptr) {
    const int64_t group = team / a.share.per_group, last = (group + 1) * a.gate_rows;
    row = group * a.gate_rows + (team - group * a.share.per_group) * a.share.rows;
    end = row + a.share.rows < last ? row + a.share.rows : last;
  } else {
    row = team * a.share.rows;
    end = row + a.share.rows;
  }
  end = end < a.M ? end : a.M;
  float pre[NV][8] = {}, post[NV][8] = {}, gsum[NV][8] = {};
  int64_t group = a.gate != nullptr ? row / a.gate_rows : 0;
  int64_t group_end = (group + 1) * a.gate_rows;
  for (; row < end; ++row) {
    float v[NV][8], y[NV][8], w[8];
    Raw<T> raw[NV], res[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + TEAM * i) * 8;
      raw[i] = load_raw((const T*)a.dn + row * a.C + c, a.C - c);
      if (a.dr_out != nullptr) res[i] = load_raw((const T*)a.dr_out + row * a.C + c, a.C - c);
    }
    if (a.K == 8)
      read_row<8, TEAM, NV>(a.ckpt_n, a.M, a.pieces, row, t, y);
    else
      read_row<4, TEAM, NV>(a.ckpt_n, a.M, a.pieces, row, t, y);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + TEAM * i) * 8;
      load_piece((const T*)a.w_pre + c, a.C - c, w);
      expand(raw[i], v[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        pre[i][j] = __builtin_fmaf(v[i][j], y[i][j], pre[i][j]);
        v[i][j] *= w[j];
      }
    }
    norm_gradient<TEAM, NV>(v, y, a.rstd_n[row], a, sum);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + TEAM * i) * 8;
      if (a.dr_out != nullptr) {
        expand(res[i], w);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] += w[j];
      }
      if (a.dr != nullptr) {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = a.alpha * v[i][j];
        store_piece((T*)a.dr + row * a.C + c, a.C - c, w);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] *= a.beta;   // e
    }
    if (!a.has_b) continue;
    if (a.ckpt_b != nullptr) {
      if (a.K == 8)
        read_row<8, TEAM, NV>(a.ckpt_b, a.M, a.pieces, row, t, y);
      else
        read_row<4, TEAM, NV>(a.ckpt_b, a.M, a.pieces, row, t, y);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (t + TEAM * i) * 8;
        float k[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = 1.0f;
        if (a.w_post != nullptr) load_piece((const T*)a.w_post + c, a.C - c, w);
        if (a.gate != nullptr) {
          load_piece((const T*)a.gate + group * a.C + c, a.C - c, k);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            gsum[i][j] = __builtin_fmaf(v[i][j], w[j] * y[i][j], gsum[i][j]);
            v[i][j] *= k[j];
          }
        }
        if (a.w_post != nullptr) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            post[i][j] = __builtin_fmaf(v[i][j], y[i][j], post[i][j]);
            v[i][j] *= w[j];
          }
        }
      }
      if (a.w_post != nullptr) norm_gradient<TEAM, NV>(v, y, a.rstd_b[row], a, sum);
    }
    if (a.db != nullptr) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (t + TEAM * i) * 8;
        store_piece((T*)a.db + row * a.C + c, a.C - c, v[i]);
      }
    }
    if (a.gate != nullptr && a.share.per_group == 0 && (row + 1 == group_end || row + 1 == a.M)) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (t + TEAM * i) * 8;
        store_piece(a.dgate + group * a.C + c, a.C - c, gsum[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) gsum[i][j] = 0.0f;
      }
      ++group;
      group_end += a.gate_rows;
    }
  }
  const int64_t width = (int64_t)a.pieces * 8, plane = a.share.teams * width;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int q = t + TEAM * i;
    if (q >= a.pieces) continue;
    float* to = a.part + team * width + q * 8;
    store_piece(to, 8, pre[i]);
    if (a.w_post != nullptr) store_piece(to + plane, 8, post[i]);
    if (a.gate != nullptr && a.share.per_group > 0) store_piece(to + 2 * plane, 8, gsum[i]);
  }
}

// The teams' sums: blockIdx.y = 0 dw_pre, 1 dw_post, 2 + g row g of dgate.  32 channels a block; thread (s, l) adds every 32nd share
// of four channels, then the 32 sums are added in turn.
__global__ __launch_bounds__(256) void resnorm_sum_kernel(const float* part, Shares share, int pieces, int C, float* dw_pre, float* dw_post,
                                                          float* dgate) {
  __shared__ float4 sums[32][8];
  const int job = blockIdx.y, l = threadIdx.x & 7, s = threadIdx.x >> 3;
  float* out = job == 0 ? dw_pre : job == 1 ? dw_post : dgate + (int64_t)(job - 2) * C;
  if (out == nullptr) return;
  const int64_t width = (int64_t)pieces * 8, plane = share.teams * width;
  const int64_t first = job < 2 ? 0 : (job - 2) * share.per_group, last = job < 2 ? share.teams : first + share.per_group;
  const float* from = part + (job < 2 ? job : 2) * plane + (int64_t)blockIdx.x * 32 + l * 4;
  float4 a{0.0f, 0.0f, 0.0f, 0.0f};
  for (int64_t i = first + s; i < last; i += 32) {
    const float4 v = *reinterpret_cast<const float4*>(from + i * width);
    a.x += v.x, a.y += v.y, a.z += v.z, a.w += v.w;
  }
  sums[s][l] = a;
  __syncthreads();
  if (threadIdx.x >= 32) return;
  const float* at = reinterpret_cast<const float*>(sums) + threadIdx.x;
  float total = 0.0f;
  for (int i = 0; i < 32; ++i) total += at[32 * i];
  const int c = blockIdx.x * 32 + threadIdx.x;
  if (c < C) out[c] = total;
}

// (plain stores, not a memset: the call may be captured into a graph)
__global__ __launch_bounds__(256) void zero_kernel(float* p, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) p[i] = 0.0f;
}

// Threads of a team for rows of so many pieces: two pieces a thread at most.
int team_of(int pieces) {
  for (int t = 64; t < 1024; t *= 2)
    if (pieces <= 2 * t) return t;
  return 1024;
}

// f(TEAM, NV) as constants.
template <typename F>
void by_team(int pieces, F&& f) {
  const int team = team_of(pieces);
  auto nv = [&](auto t) {
    if (pieces <= decltype(t)::value)
      f(t, std::integral_constant<int, 1>{});
    else
      f(t, std::integral_constant<int, 2>{});
  };
  if (team == 64) nv(std::integral_constant<int, 64>{});
  else if (team == 128) f(std::integral_constant<int, 128>{}, std::integral_constant<int, 2>{});
  else if (team == 256) f(std::integral_constant<int, 256>{}, std::integral_constant<int, 2>{});
  else if (team == 512) f(std::integral_constant<int, 512>{}, std::integral_constant<int, 2>{});
  else f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
}

}  // namespace

int launch_resnorm_forward(hipStream_t st, const abl_resnorm& s, const void* r, const void* b, const void* gate, const void* w_post,
                           const void* w_pre, void* r_out, void* n, void* ckpt_b, float* rstd_b, void* ckpt_n, float* rstd_n) {
  FwdArgs a;
  a.M = s.M, a.gate_rows = s.gate_rows, a.r = r, a.b = b, a.gate = gate, a.w_post = w_post, a.w_pre = w_pre;
  a.r_out = r_out, a.n = n, a.ckpt_b = (unsigned char*)ckpt_b, a.ckpt_n = (unsigned char*)ckpt_n;
  a.rstd_b = rstd_b, a.rstd_n = rstd_n, a.C = s.C, a.pieces = (int)store_blocks(s.C) * 4, a.K = s.K;
  a.center = (s.flags & ABL_NORM_CENTER) != 0, a.alpha = s.alpha, a.beta = s.beta, a.eps = s.eps, a.inv_c = 1.0f / (float)s.C;
  by_team(a.pieces, [&](auto t, auto nv) {
    constexpr int TEAM = decltype(t)::value, NV = decltype(nv)::value;
    const unsigned grid = (unsigned)(TEAM == 64 ? (s.M + 3) / 4 : s.M), threads = TEAM == 64 ? 256 : TEAM;
    if (s.dtype == ABL_F32)
      resnorm_fwd_kernel<float, TEAM, NV><<<grid, threads, 0, st>>>(a);
    else
      resnorm_fwd_kernel<bf16_t, TEAM, NV><<<grid, threads, 0, st>>>(a);
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
  a.C = s.C, a.pieces = (int)store_blocks(s.C) * 4, a.K = s.K, a.center = (s.flags & ABL_NORM_CENTER) != 0, a.has_b = has_b;
  a.alpha = s.alpha, a.beta = s.beta, a.inv_c = 1.0f / (float)s.C;
  a.share = shares_of(s.M, s.gate_rows, team_of(a.pieces), gate != nullptr);
  by_team(a.pieces, [&](auto t, auto nv) {
    constexpr int TEAM = decltype(t)::value, NV = decltype(nv)::value;
    const unsigned grid = (unsigned)(TEAM == 64 ? (a.share.teams + 3) / 4 : a.share.teams), threads = TEAM == 64 ? 256 : TEAM;
    if (s.dtype == ABL_F32)
      resnorm_bwd_kernel<float, TEAM, NV><<<grid, threads, 0, st>>>(a);
    else
      resnorm_bwd_kernel<bf16_t, TEAM, NV><<<grid, threads, 0, st>>>(a);
  });
  if (int e = hip_status()) return e;
  const unsigned jobs = 2 + (gate != nullptr && a.share.per_group > 0 ? (unsigned)groups : 0);
  resnorm_sum_kernel<<<dim3((unsigned)((s.C + 31) / 32), jobs), 256, 0, st>>>(a.part, a.share, a.pieces, s.C, dw_pre, dw_post, dgate);
  return hip_status();
}

}  // namespace abl
