// Losses over a vocabulary (abl_xent_*, abl_distill_*): rows h [M][C] against a table W [V][C] without the logits z = scale h W^T in memory.
//
//   forward    a tile of logits at a time: its rows' maximum m and sum_v exp(z - m) (and at the teacher's temperature, and sum_v z) go to memory,
//              16 bytes for a row of a tile; a second launch joins the tiles and writes the losses
//   backward   the logits again, a piece of the vocabulary at a time: a row's gradient
//                  d_v = a exp(z_v - L) + at exp(z_v / tau - Lt) + a0 + ay [v = label] - at sum_k p_k [v = id_k]
//              goes to a workspace that holds the piece, and dh += d W, dW = d^T h are products from there
//
// Rows that count are taken together first: a list of them, made by one block, and copies of their h, filled up with zero rows and
// channels to what the tiles need.  So the products see no masks, ragged ends or strange strides on that side, and rows
// that do not count (prompts, padding) cost nothing.  fp32 operands are copied as three bf16 parts whose sum they are; a product of such operands is six
// products of parts, one after the other in the same sums, the small ones first.

#include <utility>

#include "head.h"

namespace abl {
namespace {

constexpr int kRowTile = 256;        // copies of rows are filled up to a multiple of it
constexpr int kChannelTile = 64;     // channels of a step of the products
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ inline float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
__device__ inline float log_of(float x) { return __builtin_amdgcn_logf(x) * kLn2; }
__device__ inline float nan_value() { return __uint_as_float(0x7FC00000u); }

__device__ inline float wave_max(float v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}

// ---- which rows count -----------------------------------------------------------------------------------
enum { kLabel = 1, kTeacher = 2, kBad = 4 };   // of a row

__device__ inline bool entry_there(int64_t id, float t) { return id >= 0 && !(t == -__builtin_inff()); }

// Of a row with a teacher, by a wave.
__device__ inline int row_flags(int64_t row, const int64_t* labels, const int64_t* ids, const float* logits, int T, int V) {
  const int lane = threadIdx.x & 63;
  int f = 0;
  if (labels != nullptr) {
    const int64_t y = labels[row];
    f = y < 0 ? 0 : y < V ? kLabel : kLabel | kBad;
  }
  if (ids != nullptr) {
    int any = 0;
    for (int k = lane; k < T; k += 64) {
      const int64_t id = ids[row * T + k];
      if (entry_there(id, logits[row * T + k])) any |= id < V ? kTeacher : kTeacher | kBad;
    }
    f |= __any(any & kTeacher) ? kTeacher : 0;
    f |= __any(any & kBad) ? kBad : 0;
  }
  return f;
}

__global__ __launch_bounds__(256) void head_flags_kernel(int64_t M, const int64_t* __restrict__ labels, const int64_t* __restrict__ ids,
                                                         const float* __restrict__ logits, int T, int V, unsigned char* __restrict__ flags) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= M) return;
  const int f = row_flags(row, labels, ids, logits, T, V);
  if ((threadIdx.x & 63) == 0) flags[row] = (unsigned char)f;
}

// What the backward pass divides the gradient of the logits by where that is rounded to bf16, and multiplies its products with: the largest weight that a row's
// label has (without labels: its entries have).  Undivided, the labels' entries of rows of one weight - the mean over a batch - are all but the same
// number, w (q - 1), and share one rounding of up to 2^-9 of them, which no sum over rows averages out; divided they are q - 1, whose roundings have nothing to do with each
// other and vanish with q.
struct UnitOf {
  const float* dloss;      // nullptr: no unit is wanted
  float scale, first, second;
};

// The list of the rows that count, in their order, filled up with -1 to a multiple of kRowTile, their number, and the unit: one block (8192 rows: 7 us, 9 with the unit; places
// by atomics would change from call to call, and with them the order of the sums).
__global__ __launch_bounds__(1024) void head_rows_kernel(int64_t M, const int64_t* __restrict__ labels, const unsigned char* __restrict__ flags,
                                                         int* __restrict__ rows, int* __restrict__ count, UnitOf of, float* __restrict__ unit) {
  __shared__ int sums[17];
  __shared__ float largest[16];
  float large = 0.0f;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int base = 0;
  for (int64_t m0 = 0; m0 < M; m0 += 4096) {
    const int64_t m = m0 + threadIdx.x * 4;
    int on = 0;
    float w[4] = {};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (of.dloss != nullptr && m + e < M) w[e] = of.dloss[m + e];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (m + e < M && (flags != nullptr ? (flags[m + e] & (kLabel | kTeacher)) != 0 : labels[m + e] >= 0)) on |= 1 << e;
    const int n = __popc(on);
    int s = n;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int t = __shfl_up(s, d);
      if (lane >= d) s += t;
    }
    if (lane == 63) sums[wave] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
      int total = 0;
      for (int w = 0; w < 16; ++w) {
        const int v = sums[w];
        sums[w] = total;
        total += v;
      }
      sums[16] = total;
    }
    __syncthreads();
    int at = base + sums[wave] + s - n;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (on >> e & 1) {
        rows[at++] = (int)(m + e);
        large = finite(w[e]) ? fmaxf(large, fabsf(w[e])) : large;
      }
    base += sums[16];
    __syncthreads();
  }
  const int end = (base + kRowTile - 1) / kRowTile * kRowTile;
  for (int i = base + threadIdx.x; i < end; i += 1024) rows[i] = -1;
  if (of.dloss != nullptr) {
    large = wave_max(large);
    if (lane == 0) largest[wave] = large;
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    *count = base;
    if (of.dloss != nullptr) {
      for (int w = 0; w < 16; ++w) large = fmaxf(large, largest[w]);
      const float u = fabsf(large * of.scale * of.first * of.second);   // (in the order of the weights themselves: a quotient is one exactly)
      *unit = u >= 1e-30f && u <= 1e30f ? u : 1.0f;
    }
  }
}

// ---- copies of rows in bf16 parts -----------------------------------------------------------------------
// fp32 as three bf16 parts whose sum it is: the nearest, the nearest to what is left, and the rest, which then fits (products of parts that are left out are
// below 2^-25 of the whole).  A value that is not finite is its first part, one that would round to infinity is cut off there.
__device__ inline void three_parts(float v, uint32_t& h, uint32_t& m, uint32_t& l) {   // each in the upper half of its word
  h = two_bf16(0.0f, v);
  const bool fine = finite(v);
  if (fine && !finite(__uint_as_float(h))) h = __float_as_uint(v) & 0xFFFF0000u;
  const float r = fine ? v - __uint_as_float(h) : 0.0f;
  m = two_bf16(0.0f, r);
  l = __float_as_uint(r - __uint_as_float(m));
}

// A value in one part or three.
__device__ inline void put_parts(char* to, int64_t plane, int parts, float v) {
  if (parts == 3) {
    uint32_t h, m, l;
    three_parts(v, h, m, l);
    *(uint16_t*)to = (uint16_t)(h >> 16);
    *(uint16_t*)(to + plane) = (uint16_t)(m >> 16);
    *(uint16_t*)(to + 2 * plane) = (uint16_t)(l >> 16);
  } else {
    *(uint16_t*)to = (uint16_t)two_bf16(v, 0.0f);
  }
}

// A row of C elements (nullptr: zeros) to its place in P planes, `plane` bytes apart, with zeros up to Cp channels: by a wave.  P = 0: as fp32.
template <typename T, int P>
__device__ inline void copy_row(const T* from, int C, int Cp, char* to, int64_t plane) {
  for (int c = (threadIdx.x & 63) * 8; c < Cp; c += 512) {
    float v[8] = {};
    if (from != nullptr) load_piece(from + c, C - c, v);
    if constexpr (P == 0) {
      *reinterpret_cast<floatx4*>(to + 4 * c) = floatx4{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<floatx4*>(to + 4 * c + 16) = floatx4{v[4], v[5], v[6], v[7]};
    } else if constexpr (P == 1) {
      *reinterpret_cast<u32x4*>(to + 2 * c) = u32x4{two_bf16(v[0], v[1]), two_bf16(v[2], v[3]), two_bf16(v[4], v[5]), two_bf16(v[6], v[7])};
    } else {
      uint32_t h[8], m[8], l[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) three_parts(v[e], h[e], m[e], l[e]);
      u32x4 a, b, d;
#pragma unroll
      for (int e = 0; e < 4; ++e) {   // the upper halves of two words
        a[e] = __builtin_amdgcn_perm(h[2 * e + 1], h[2 * e], 0x07060302u);
        b[e] = __builtin_amdgcn_perm(m[2 * e + 1], m[2 * e], 0x07060302u);
        d[e] = __builtin_amdgcn_perm(l[2 * e + 1], l[2 * e], 0x07060302u);
      }
      *reinterpret_cast<u32x4*>(to + 2 * c) = a;
      *reinterpret_cast<u32x4*>(to + plane + 2 * c) = b;
      *reinterpret_cast<u32x4*>(to + 2 * plane + 2 * c) = d;
    }
  }
}

// Rows 0..n-1 of a tensor, and zero rows up to n_to.
template <typename T, int P>
__global__ __launch_bounds__(256) void head_copy_kernel(const T* __restrict__ from, int64_t ld, int64_t n, int64_t n_to, int C, int Cp,
                                                        char* __restrict__ to, int64_t pitch, int64_t plane) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row < n_to) copy_row<T, P>(row < n ? from + row * ld : nullptr, C, Cp, to + row * pitch, plane);
}

// What the backward pass knows of a row that counts (the formula above; all times the row's dloss and the logits' scale, over the unit).  At temperature one a
// holds at too.
struct RowGrad {
  float L, a, Lt, at, a0, ay;
  int label, counts;
};

struct Gather {
  int64_t M, slots;   // rows; places for those that count
  int C, Cp, T, V;
  const int* rows;
  const int* count;
  const unsigned char* flags;   // nullptr: by the labels
  const int64_t* labels;
  char* to;                     // planes of the rows that count
  int64_t pitch, plane, ldh;
  // forward: of the rows that do not count, written as zeros
  float *loss, *lse, *lse_t, *z_top;
  int* row_label;               // and the labels of those that do
  // backward
  void* dh;
  int64_t lddh;
  RowGrad* grad;
  const float *in_lse, *in_lse_t, *dloss;
  const float* unit;            // nullptr: one
  float scale, smoothing, z_weight, tau, label_weight, teacher_weight;
};

// The rows that count to their places, with their coefficients (backward), then - blocks of their own - zeros for the rows that do not.  Bound by memory
// (8192 x 4096 bf16: 25 us, 5.4 TB/s); a wave a row.
template <typename T, int P>
__global__ __launch_bounds__(256) void head_gather_kernel(Gather g, const T* __restrict__ h) {
  const int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int count = *g.count;
  if (n < g.slots) {
    if (n >= ((count > 1 ? count : 1) + kRowTile - 1) / kRowTile * kRowTile) return;
    const int64_t row = n < count ? g.rows[n] : -1;
    copy_row<T, P>(row >= 0 ? h + row * g.ldh : nullptr, g.C, g.Cp, g.to + n * g.pitch, g.plane);
    if (g.row_label != nullptr && lane == 0) {
      const int64_t y = row >= 0 ? g.labels[row] : -1;
      g.row_label[n] = y >= 0 && y < g.V ? (int)y : -1;
    }
    if (g.grad != nullptr && lane == 0) {
      RowGrad r{0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, -1, 0};
      if (row >= 0) {
        const int64_t y = g.labels != nullptr ? g.labels[row] : -1;
        const int f = g.flags != nullptr ? g.flags[row] : y < g.V ? kLabel : kLabel | kBad;
        const float w = g.dloss[row] * g.scale, l = f & kLabel ? w * g.label_weight : 0.0f;
        // (without a log-sum nothing is multiplied with its exponentials, which must not overflow then)
        r.L = g.in_lse != nullptr ? g.in_lse[row] : g.tau == 1.0f ? g.in_lse_t[row] : 1e38f;
        r.a = g.z_weight != 0.0f ? __builtin_fmaf(2.0f * g.z_weight * w, r.L, l) : l;
        r.Lt = g.in_lse_t != nullptr ? g.in_lse_t[row] : 0.0f;
        r.at = f & kTeacher ? w * g.teacher_weight * g.tau : 0.0f;
        if (g.tau == 1.0f) r.a += r.at;   // (one exponential for both)
        r.a0 = -l * g.smoothing / (float)g.V;
        r.ay = -l * (1.0f - g.smoothing);
        r.label = f & kLabel && y < g.V ? (int)y : -1;
        if (g.unit != nullptr) {
          const float u = *g.unit;
          r.a /= u, r.at /= u, r.a0 /= u, r.ay /= u;
        }
        if (f & kBad) r.a0 = nan_value();
        r.counts = 1;
      }
      g.grad[n] = r;
    }
    return;
  }
  const int64_t row = n - g.slots;
  if (row >= g.M) return;
  if (g.flags != nullptr ? (g.flags[row] & (kLabel | kTeacher)) != 0 : g.labels[row] >= 0) return;
  if (g.loss != nullptr && lane == 0) {
    g.loss[row] = 0.0f;
    if (g.lse != nullptr) g.lse[row] = 0.0f;
    if (g.lse_t != nullptr) g.lse_t[row] = 0.0f;
  }
  if (g.z_top != nullptr)
    for (int k = lane; k < g.T; k += 64) g.z_top[row * g.T + k] = 0.0f;
  if (g.dh != nullptr) {
    const float zero[8] = {};
    for (int c = lane * 8; c < g.C; c += 512) store_piece((T*)g.dh + row * g.lddh + c, g.C - c, zero);
  }
}

// ---- the products ---------------------------------------------------------------------------------------
// out [x][y] = sum_k X Y, x rows and y columns, both operands bf16 in planes of parts.  An operand lies either with k along its rows ([x][k]) or
// outermost ([k][x]).
struct Operand {
  const char* p;        // first element of the first plane
  int64_t plane;        // bytes from plane to plane
  int64_t pitch;        // bytes from row to row, less than 2^22
  int rows, along;      // rows, and elements along a row, that exist (others read as zero); along: a multiple of 8
};
struct Partial {        // of some logits: maximum; sum of exp(z - max), less one (what a certain row's small loss is made of), and of exp((z - max) / tau); sum of z
  float top, rest, rest_t, z;
};
struct Split {            // at most so many shares; compute units' blocks; ns of a step, of the rest of a tile, of the second launch; elements a ns of its slabs
  int most, units, step, fixed, second, bytes;
};
struct Product {
  Operand x, y;
  int nx, ny, k;            // sizes as the host knows them
  const int* count;         // rows that count: instead of nx, or (count_k) of k
  int count_k;
  int parts;                // pairs of planes, in the order of their products: 4 bits each plane, x first
  uint64_t pairs;
  // logits
  float scale, inv_tau;
  int y0;                   // token of the first column
  Partial* partial;         // [tile of columns][partial_ld]
  int64_t partial_ld;
  int sum_z;                // whether the sum of z is wanted
  const int* row_label;     // the label of a row that counts
  const int64_t* labels;    // few rows: of each row, as they are given
  float* z_label;
  const RowGrad* grad;
  char* d;                  // planes of the gradient of the logits
  int64_t d_plane, d_pitch;
  int d_parts;
  // sums
  void* out;
  int64_t ld;
  int out_f32, accumulate;
  const int* map;           // row of out for each x (nullptr: x itself)
  const float* unit;        // what the sums are multiplied with (nullptr: nothing), before accumulate
  const float* add;         // [x][add_ld], added (nullptr: nothing)
  int64_t add_ld;
  // sums whose k's are cut into shares of blocks of their own: where there are several, or no out, each leaves its sums in a slab [nx][ny] and a second launch
  // takes them from there
  Split split;
  float* slabs;
};

// The number of shares with the least time, in ns by the estimates of Split: the same for the product and what adds its slabs.
__host__ __device__ inline int shares_of(const Split& s, int64_t tiles, int steps, int64_t size) {
  if (s.most <= 1 || tiles >= 4 * s.units) return 1;
  int best = 1;
  int64_t least = 0;
  for (int n = 1; n <= s.most && (n == 1 || steps >= 2 * n); ++n) {
    const int64_t time = (tiles * n + s.units - 1) / s.units * ((steps + n - 1) / n * (int64_t)s.step + s.fixed) + (n > 1 ? s.second + n * (size / s.bytes) : 0);
    if (n == 1 || time < least) best = n, least = time;
  }
  return best;
}
enum { kEpiPartial, kEpiGrad, kEpiSum };

// A 16-byte piece of a staged tile of 64 k's.  k along the rows: rows of eight pieces, the c-th of row r at place c xor (r / 2) % 8: the 16
// rows of a fragment's read take all banks once.  k outermost: rows (one k) of B channels; the even pieces come first, the c-th of each kind at place
// c xor a key of the row, the odd ones further by half of a row's pieces and in other places of it: half a wave's transposing read, 16 pieces of
// the eight rows 0..3 and 8..11 (or 4..7 and 12..15), takes all banks once.  Rows of 64 channels are half of the banks: their pieces stay in order, the c-th at
// place c xor a key of bits 1 and 3 of the row.
__device__ inline int key_along(int row) { return (row >> 1) & 7; }
__device__ inline int key_outer(int k) { return (k & 3) | ((k >> 1) & 4); }
__device__ inline int key_narrow(int k) { return (k & 2) | ((k >> 1) & 4); }
template <int B, bool OUTER>
__device__ inline int staged_piece(int row, int q) {
  if constexpr (OUTER && B == 64) {
    return row * 128 + ((q ^ key_narrow(row)) * 16);
  } else if constexpr (OUTER) {
    constexpr int kHalf = B / 16;
    return row * (B * 2) + (q & 1) * B + (((q >> 1) ^ key_outer(row) ^ ((q & 1) * (kHalf - 4))) * 16);
  } else {
    return row * 128 + ((q ^ key_along(row)) * 16);
  }
}

// Two loads: each lane's 16 bytes at `at` + `step` go to LDS, one lane's behind the other's from byte `to` + TO on (zeros where they lie beyond the
// descriptor).  In assembly: the compiler takes every later read of LDS for one that needs the data and waits for all loads there.  Nothing comes back in
// registers.  What the compiler would otherwise see to: a load needs five states from a vector instruction's write of a scalar register that it
// reads, and one from m0's.
template <int TO, int TO2>
__device__ inline void load_two(u32x4 from, uint32_t to, uint32_t at, uint32_t at2, uint32_t step, uint32_t step2) {
  asm volatile(
      "s_add_u32 m0, %0, %6\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %3, %4 offen lds\n\t"
      "s_add_u32 m0, %0, %7\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, %5 offen lds" ::"s"(to),
      "v"(at), "v"(at2), "s"(from), "s"(step), "s"(step2), "i"(TO), "i"(TO2)
      : "scc");
}
template <int TO>
__device__ inline void load_one(u32x4 from, uint32_t to, uint32_t at, uint32_t step) {
  asm volatile("s_add_u32 m0, %0, %4\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(at), "s"(from), "s"(step), "i"(TO) : "scc");
}

__device__ inline uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }   // the same in all lanes, in a scalar register

// A thread's share of the tiles of an operand, from step to step.  The loads go to LDS in the order of the threads, so the places' order is undone
// here; the rows of a thread's loads are a constant apart that no key sees.  MASK: elements beyond `along` may lie in a step (k along the rows).
template <int B, bool OUTER, bool MASK, int THREADS>
struct Source {
  static constexpr int kLoads = B * 8 / THREADS, kPieces = OUTER ? B / 8 : 8, kRows = THREADS / kPieces;   // rows of a load
  static_assert(kRows % 16 == 0, "the keys' period");
  static constexpr int kPlaces = OUTER ? 1 : kLoads;   // (k outermost: the loads' distance goes with the scalar offset, to save registers)
  uint32_t at[kPlaces];
  int first;              // element along the row
  uint64_t base;
  uint32_t pitch, bytes;  // of the rows that a step may read
  int k, left;            // k outermost: rows that are left
  u32x4 from;
  uint32_t step;

  __device__ inline void init(const Operand& o, int w0) {
    pitch = (uint32_t)o.pitch;
    base = 0, k = 0, left = 0, bytes = 0;   // (next() combines old and new values by their bits: both have to have one)
    const int row = (int)threadIdx.x / kPieces, in = (int)threadIdx.x % kPieces;
    int q;
    if constexpr (OUTER && B == 64) {
      q = in ^ key_narrow(row);
    } else if constexpr (OUTER) {
      constexpr int kHalf = B / 16;
      const int odd = in / kHalf;
      q = 2 * ((in % kHalf) ^ key_outer(row) ^ (odd * (kHalf - 4))) + odd;
    } else {
      q = in ^ key_along(row);
    }
    first = q * 8;
#pragma unroll
    for (int n = 0; n < kPlaces; ++n)
      at[n] = OUTER && w0 + first >= o.along ? kNowhere : (uint32_t)(row + n * kRows) * pitch + (uint32_t)q * 16u;
  }
  // On by a step, or to the first step of a plane, or (not more) zeros from here on.  Without branches: a loop of one block keeps the sums in their registers.
  // first, more: all bits set, or none.
  __device__ inline void next(const Operand& o, int w0, int first_step, int plane, int more) {
    const uint64_t begin = (uint64_t)(o.p + plane * o.plane + (OUTER ? w0 * 2 : w0 * o.pitch)) & 0xFFFFFFFFFFFFull;
    const uint64_t after = base + (OUTER ? (uint64_t)pitch * 64u : 0u);
    base = after ^ ((after ^ begin) & (uint64_t)(int64_t)first_step);
    k = (k + 64) & ~first_step;
    if constexpr (OUTER) {
      const int rest = left - 64 > 0 ? left - 64 : 0;
      left = (rest ^ ((rest ^ o.rows) & first_step)) & more;
    } else {
      bytes = (uint32_t)(o.rows - w0 < B ? o.rows - w0 : B) * pitch & (uint32_t)more;
    }
    describe(more);
  }
  __device__ inline void describe(int more) {
    from = u32x4{uniform((uint32_t)base), uniform((uint32_t)(base >> 32)), uniform(OUTER ? (uint32_t)(left < 64 ? left : 64) * pitch : bytes), 0x00027000u};
    step = OUTER ? 0u : uniform((uint32_t)(2 * k & more));   // (an access is out of range where its own offset is not below the bytes less the scalar one)
  }
  // On by so many steps of a plane, from its first one.
  __device__ inline void skip(int steps) {
    k = 64 * steps;
    if constexpr (OUTER) base += (uint64_t)pitch * (uint64_t)k, left = left > k ? left - k : 0;
    describe(-1);
  }
  // The n-th load of a step, and the one after it where there is one: to byte TO and TO + THREADS * 16.
  template <int N, int TO>
  __device__ inline void load(const Operand& o, uint32_t to) const {
    constexpr int M = N + 1 < kLoads ? N + 1 : N;
    uint32_t a[2], by[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      if constexpr (OUTER) {
        a[n] = at[0], by[n] = (uint32_t)((n == 0 ? N : M) * kRows) * pitch;
        by[n] = uniform(by[n] < from[2] ? by[n] : from[2]);
      } else {
        a[n] = !MASK || first + k < o.along ? at[n == 0 ? N : M] : kNowhere, by[n] = step;
      }
    }
    if constexpr (M > N)
      load_two<TO, TO + THREADS * 16>(from, to, a[0], a[1], by[0], by[1]);
    else
      load_one<TO>(from, to, a[0], by[0]);
  }
};

// Where a wave's fragments of 16 rows or columns from w on lie in a tile: all addresses are the first one's with bits of the place changed and constants added.
template <int B, bool OUTER>
struct Fragments {
  uint32_t base;
  __device__ inline void init(uint32_t tile, int w) {
    const int lane = threadIdx.x & 63;
    if constexpr (OUTER)
      base = tile + staged_piece<B, true>((lane >> 4) * 8 + ((lane & 15) >> 2), w / 8 + ((lane >> 1) & 1)) + (lane & 1) * 8;
    else
      base = tile + staged_piece<B, false>(w + (lane & 15), lane >> 4);
  }
  // (keeps the compiler from holding all addresses in registers)
  __device__ inline void again() {
    if constexpr (OUTER) asm volatile("" : "+v"(base));
  }
  // The n-th one's 32 k's: the first or second of the tile in place `at`.
  __device__ inline bf16x8_t get(int n, int half, int at) const {
    constexpr int kTileBytes = B * 128;
    if constexpr (OUTER) {
      lds_short4* p = (lds_short4*)(uintptr_t)((base ^ (n * (B == 64 ? 32 : 16))) + at * kTileBytes + half * (kTileBytes / 2));
      struct two { short4_t a, b; };
      return __builtin_bit_cast(bf16x8_t, two{__builtin_amdgcn_ds_read_tr16_b64_v4i16(p), __builtin_amdgcn_ds_read_tr16_b64_v4i16(p + 4 * (B * 2) / 8)});
    } else {
      typedef __attribute__((address_space(3))) bf16x8_t lds_bf16x8;
      return *(lds_bf16x8*)(uintptr_t)((base ^ (half * 64)) + at * kTileBytes + n * (16 * 128));
    }
  }
};

template <int N, typename F, int... I>
__device__ inline void for_each(F f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ inline void for_each(F f) {
  for_each<N>(f, std::make_integer_sequence<int, N>{});
}

// The second and fourth 16 lanes of a change places with the first and third of b.
__device__ inline u32x2 lanes16_swap(uint32_t a, uint32_t b) {
#ifdef __HIP_DEVICE_COMPILE__
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  return u32x2{r[0], r[1]};
#else
  return u32x2{a, b};
#endif
}
// Over the four lanes 16 apart: rows of 16 lanes, then halves of the wave, change places with those of a copy.
template <typename F>
__device__ inline float lanes16(float v, F f) {
#ifdef __HIP_DEVICE_COMPILE__
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
#else
  return v;
#endif
}
__device__ inline float lanes16_max(float v) {
  return lanes16(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ inline float lanes16_sum(float v) {
  return lanes16(v, [](float a, float b) { return a + b; });
}

// Joins the sums of two sets of logits.
__device__ inline Partial join(const Partial& a, const Partial& b, float inv_tau) {
  const bool first = a.top >= b.top;
  const Partial &big = first ? a : b, &small = first ? b : a;
  const float d = a.top == b.top ? 0.0f : small.top - big.top;   // (there may be none on both sides)
  Partial r;
  r.top = fmaxf(a.top, b.top);
  r.rest = __builtin_fmaf(small.rest + 1.0f, exp_of(d), big.rest);
  r.rest_t = inv_tau != 1.0f ? __builtin_fmaf(small.rest_t + 1.0f, exp_of(d * inv_tau), big.rest_t) : 0.0f;
  r.z = a.z + b.z;
  return r;
}

template <int LANES = 64>
__device__ inline Partial lanes_joined(Partial p, float inv_tau) {   // of the wave's 64 lanes (or each 16 of them), the same for all of these
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < LANES; d *= 2) {
    const Partial o{__shfl_xor(p.top, d), __shfl_xor(p.rest, d), __shfl_xor(p.rest_t, d), __shfl_xor(p.z, d)};
    p = lane & d ? join(o, p, inv_tau) : join(p, o, inv_tau);   // (in the same order in both lanes)
  }
  return p;
}

// Bound by the matrix cores: 8192 x 4096 x 65536 logits take 3.3 ms, 1.3 PFLOP/s (the library's plain product of this size 3.26 ms), the matrix cores busy in 60 to
// 66 % of the cycles at 1.9 GHz; a step of 256 x 256 x 64 takes 1.47 us, a tile 7 to 10 us beside its steps.  LDS reads meet no bank twice (counted).
// A block has a tile of BX x BY, WX x WY waves a part of it each.  Steps of 64 k's: their operands go from memory straight to one of PLACES in
// LDS, PLACES - 1/2 steps ahead, and from there to registers half a step ahead, all between matrix instructions.  FEW: x may be a user's rows as they are.
template <int BX, int BY, int WX, int WY, int PLACES, bool XO, bool YO, int EPI, bool FEW>
__global__ __launch_bounds__(WX * WY * 64) void head_product_kernel(Product a) {
  constexpr int kThreads = WX * WY * 64, FX = BX / WX / 16, FY = BY / WY / 16;
  constexpr int kXBytes = BX * 128, kYBytes = BY * 128;
  extern __shared__ __align__(16) char lds[];   // [PLACES][BX][128], [PLACES][BY][128]
  const int count = a.count != nullptr ? (int)uniform((uint32_t)*a.count) : 0;
  const int nx = a.count != nullptr && !a.count_k ? count : a.nx, nk = a.count != nullptr && a.count_k ? count : a.k;
  // Blocks 8 apart share an XCD and its L2.  Each XCD takes consecutive items, in bands of eight tiles of rows.
  constexpr int kBand = 8;
  const int tiles_x = (nx + BX - 1) / BX, tiles_y = (a.ny + BY - 1) / BY, tiles = tiles_x * tiles_y;
  const int steps_k = (nk + 63) / 64, all_steps = steps_k * a.parts;
  const int shares = EPI == kEpiSum ? shares_of(a.split, tiles, all_steps, (int64_t)nx * a.ny) : 1, items = tiles * shares;
  const int xcd = blockIdx.x & 7, slot = blockIdx.x >> 3, per = items >> 3, more = items & 7;
  if (slot >= per + (xcd < more ? 1 : 0)) return;
  const int item = xcd * per + (xcd < more ? xcd : more) + slot, share = item / tiles, tile = item - share * tiles;
  const int band = tile / (kBand * tiles_y), rest = tile - band * kBand * tiles_y;
  const int high = tiles_x - band * kBand < kBand ? tiles_x - band * kBand : kBand;
  const int x0 = (band * kBand + rest % high) * BX, tile_y = rest / high, y0 = tile_y * BY;
  const int each = (all_steps + shares - 1) / shares, begin = share * each, end = begin + each < all_steps ? begin + each : all_steps;
  const int steps = end > begin ? end - begin : 0;

  Source<BX, XO, FEW, kThreads> sx;
  Source<BY, YO, !YO, kThreads> sy;
  sx.init(a.x, x0);
  sy.init(a.y, y0);
  constexpr int kLoads = sx.kLoads + sy.kLoads;   // of a step
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  int load_part = steps > 0 ? begin / steps_k - 1 : -1, load_k = steps_k - 1, load_s = -1;
  auto next_load = [&]() __attribute__((always_inline)) {   // (beyond the last step: zeros)
    ++load_k, ++load_s;
    const int first = ~((load_k - steps_k) >> 31);
    load_k &= ~first;
    load_part -= first;
    const int pair = (int)(a.pairs >> (8 * load_part & 63)), more = (load_s - steps) >> 31;
    sx.next(a.x, x0, first, pair & 15, more);
    sy.next(a.y, y0, first, (pair >> 4) & 15, more);
  };
  const uint32_t load_to = uniform(lds0 + (threadIdx.x >> 6) * 1024);
  auto load = [&](auto n, auto to) __attribute__((always_inline)) {   // the n-th load of a step, to place `to`; the second of a pair goes with the first
    constexpr int kN = n.value, kY = kN - sx.kLoads;
    if constexpr (kN < sx.kLoads) {
      if constexpr (kN % 2 == 0) sx.template load<kN, to.value * kXBytes + kN * kThreads * 16>(a.x, load_to);
    } else if constexpr (kY % 2 == 0) {
      sy.template load<kY, PLACES * kXBytes + to.value * kYBytes + kY * kThreads * 16>(a.y, load_to);
    }
  };

  floatx4 acc[FX][FY];
#pragma unroll
  for (int i = 0; i < FX; ++i)
#pragma unroll
    for (int j = 0; j < FY; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wx = wave / WY * (FX * 16), wy = wave % WY * (FY * 16);

  // Fragments: of x, which a wave has more of, each is read for the next half as soon as its products of this one are issued (the last one aside); of y, which
  // all products take, two sets.
  bf16x8_t x[FX - 1], x_last[2], y[2][FY];
  Fragments<BX, XO> fx;
  Fragments<BY, YO> fy;
  fx.init(lds0, wx);
  fy.init(lds0 + PLACES * kXBytes, wy);
  auto loads = [&](int i, auto place) __attribute__((always_inline)) {   // the i-th of FX shares
    for_each<kLoads>([&](auto n) {
      if (n.value * FX / kLoads == i) load(n, place);
    });
  };
  // All loads but the last `left` have come, and what was read of LDS, of all waves.  (No fence: it would wait for all loads.)
  auto arrived = [&](auto left) __attribute__((always_inline)) {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"i"(left.value) : "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  auto step = [&](auto place_of) __attribute__((always_inline)) {
    constexpr int place = place_of.value;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (half == 1) {
        arrived(std::integral_constant<int, (PLACES - 2) * kLoads>{});
        next_load();
      }
      const int from = half == 0 ? place : (place + 1) % PLACES;
      fx.again();
      fy.again();
#pragma unroll
      for (int i = 0; i < FX; ++i) {
        if (half == 1) loads(i, place_of);   // of PLACES steps later
        if (i == 0)
          x_last[half ^ 1] = fx.get(FX - 1, half ^ 1, from);
        else
          x[i - 1] = fx.get(i - 1, half ^ 1, from);
#pragma unroll
        for (int n = i * FY / FX; n < (i + 1) * FY / FX; ++n) y[half ^ 1][n] = fy.get(n, half ^ 1, from);
#pragma unroll
        for (int j = 0; j < FY; ++j) acc[i][j] = mfma32(y[half][j], i == FX - 1 ? x_last[half] : x[i], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);   // (left to itself the compiler puts reads where it then waits for them)
      }
    }
  };
  if (steps > 0) {
    for_each<PLACES>([&](auto place) {
      next_load();
      if (place.value == 0 && begin % steps_k != 0) {   // (a share that begins inside a plane)
        load_k = begin % steps_k;
        sx.skip(load_k);
        sy.skip(load_k);
      }
      for_each<kLoads>([&](auto n) { load(n, place); });
    });
    arrived(std::integral_constant<int, (PLACES - 1) * kLoads>{});
#pragma unroll
    for (int n = 0; n < FY; ++n) y[0][n] = fy.get(n, 0, 0);
#pragma unroll
    for (int n = 0; n < FX - 1; ++n) x[n] = fx.get(n, 0, 0);
    x_last[0] = fx.get(FX - 1, 0, 0);
    for (int s = 0; s < steps; s += PLACES)   // (beyond the last step: of zeros)
      for_each<PLACES>([&](auto place) { step(place); });
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (nothing may come to LDS any more)

  // lane: row lane % 16 of a 16 x 16 tile, columns 4 (lane / 16) + 0..3
  if constexpr (EPI == kEpiPartial) {
    __syncthreads();
    Partial* joined = reinterpret_cast<Partial*>(lds);   // [WY][BX]
    const bool ragged = y0 + BY > a.ny, soft = a.inv_tau != 1.0f;
#pragma unroll
    for (int i = 0; i < FX; ++i) {
      const int x = wx + 16 * i + (lane & 15);
      const int col0 = y0 + wy + (lane >> 4) * 4;
      int label = -1;
      if constexpr (FEW) {
        const int64_t l = a.labels != nullptr && x0 + x < nx ? a.labels[x0 + x] : -1;
        if (l >= 0 && l < a.ny) label = (int)l;
      } else if (a.row_label != nullptr && x0 + x < nx) {
        label = a.row_label[x0 + x] - a.y0;
      }
      float top = -__builtin_inff(), all = 0.0f;
#pragma unroll
      for (int j = 0; j < FY; ++j) acc[i][j] *= a.scale;
      if (__any((uint32_t)(label - col0) < 16u * FY)) {
#pragma unroll
        for (int j = 0; j < FY; ++j) {
          const int at = label - col0 - 16 * j;
          if ((uint32_t)at < 4u) a.z_label[x0 + x] = at & 2 ? (at & 1 ? acc[i][j][3] : acc[i][j][2]) : (at & 1 ? acc[i][j][1] : acc[i][j][0]);
        }
      }
      if (a.sum_z) {
#pragma unroll
        for (int j = 0; j < FY; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) all += col0 + 16 * j + e < a.ny ? acc[i][j][e] : 0.0f;
      }
      if (ragged) {
#pragma unroll
        for (int j = 0; j < FY; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][e] = col0 + 16 * j + e < a.ny ? acc[i][j][e] : -__builtin_inff();
      }
#pragma unroll
      for (int j = 0; j < FY; ++j) top = fmaxf(fmaxf(top, fmaxf(acc[i][j][0], acc[i][j][1])), fmaxf(acc[i][j][2], acc[i][j][3]));
      top = lanes16_max(top);
      const float ref = top == -__builtin_inff() ? 0.0f : top;
      float sum, sum_t, tops;
      auto add_up = [&](float ref, auto aside) __attribute__((always_inline)) {   // aside: the maximum is counted beside the sum, so that nothing of a small one is lost
        sum = sum_t = tops = 0.0f;
#pragma unroll
        for (int j = 0; j < FY; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float z = (acc[i][j][e] - ref) * kLog2e;   // (the difference first: it is exact next to the maximum)
            const bool hit = aside.value && acc[i][j][e] == ref;
            sum += hit ? 0.0f : __builtin_amdgcn_exp2f(z);
            if (soft) sum_t += hit ? 0.0f : __builtin_amdgcn_exp2f(z * a.inv_tau);
            if (aside.value) tops += hit ? 1.0f : 0.0f;
          }
        sum = lanes16_sum(sum);
        if (soft) sum_t = lanes16_sum(sum_t);
        if (aside.value) tops = lanes16_sum(tops);
      };
      // FEW waits for memory anyway.  The others count the maximum aside only where a row is all but certain of it: the sum of the rest, an eighth or more, is off by 2^-17 of
      // itself otherwise (16 + 2 roundings of up to 2^-24 next to one).
      add_up(ref, std::integral_constant<bool, FEW>{});
      if (!FEW && __builtin_expect(__any(sum < 1.125f || (soft && sum_t < 1.125f)), 0)) {
        float again = ref;
        asm volatile("" : "+v"(again));   // (else the terms that both ways have in common are kept, and made where none of them is wanted: 2 %)
        add_up(again, std::true_type{});
      }
      if (a.sum_z) all = lanes16_sum(all);
      if (lane < 16) joined[wave % WY * BX + x] = Partial{top, sum + (tops - 1.0f), sum_t + (tops - 1.0f), all};
    }
    __syncthreads();
    for (int x = threadIdx.x; x < BX; x += kThreads) {
      if (x0 + x >= nx) break;
      Partial p = joined[x];
#pragma unroll
      for (int w = 1; w < WY; ++w) p = join(p, joined[w * BX + x], a.inv_tau);
      a.partial[(int64_t)tile_y * a.partial_ld + x0 + x] = p;
    }
  } else if constexpr (EPI == kEpiGrad) {
    const bool ragged = x0 + BX > nx || y0 + BY > a.ny, soft = a.inv_tau != 1.0f;
    // Two neighbouring tiles' columns at a time: lanes 16 apart change places, so that each has eight columns of one of them and a row's 64 bytes go to
    // memory together.
    auto store = [&](char* row, int j, u32x2 even, u32x2 odd) __attribute__((always_inline)) {
      const int g = lane >> 4;
      const u32x2 lo = lanes16_swap(even[0], odd[0]), hi = lanes16_swap(even[1], odd[1]);
      *reinterpret_cast<u32x4*>(row + (y0 + wy + 16 * (j + (g & 1)) + (g >> 1) * 8) * 2) = u32x4{lo[0], hi[0], lo[1], hi[1]};
    };
#pragma unroll
    for (int i = 0; i < FX; ++i) {
      const int x = x0 + wx + 16 * i + (lane & 15);
      const RowGrad g = a.grad[x];   // (the rows up to a whole tile are there)
      const int label = g.label >= 0 ? g.label - a.y0 : -1;
      char* row = a.d + x * a.d_pitch;
#pragma unroll
      for (int j = 0; j < FY; j += 2) {
        float d[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int col = y0 + wy + 16 * (j + h) + (lane >> 4) * 4;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float s = acc[i][j + h][e];
            d[h][e] = __builtin_fmaf(g.a, exp_of(__builtin_fmaf(s, a.scale, -g.L)), g.a0);
            if (soft) d[h][e] = __builtin_fmaf(g.at, exp_of(__builtin_fmaf(s * a.scale, a.inv_tau, -g.Lt)), d[h][e]);
          }
          if ((uint32_t)(label - col) < 4u) {
#pragma unroll
            for (int e = 0; e < 4; ++e) d[h][e] += col + e == label ? g.ay : 0.0f;
          }
          if (ragged) {
#pragma unroll
            for (int e = 0; e < 4; ++e) d[h][e] = x < nx && col + e < a.ny ? d[h][e] : 0.0f;
          }
        }
        if (a.d_parts == 3) {
          uint32_t p[2][3][4];
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) three_parts(d[h][e], p[h][0][e], p[h][1][e], p[h][2][e]);
          auto upper = [](const uint32_t(&v)[4]) {
            return u32x2{__builtin_amdgcn_perm(v[1], v[0], 0x07060302u), __builtin_amdgcn_perm(v[3], v[2], 0x07060302u)};
          };
#pragma unroll
          for (int n = 0; n < 3; ++n) store(row + n * a.d_plane, j, upper(p[0][n]), upper(p[1][n]));
        } else {
          store(row, j, u32x2{two_bf16(d[0][0], d[0][1]), two_bf16(d[0][2], d[0][3])}, u32x2{two_bf16(d[1][0], d[1][1]), two_bf16(d[1][2], d[1][3])});
        }
      }
    }
  } else if (shares > 1 || a.out == nullptr) {
    float* slab = a.slabs + (int64_t)share * nx * a.ny;
#pragma unroll
    for (int i = 0; i < FX; ++i) {
      const int x = x0 + wx + 16 * i + (lane & 15);
      if (x >= nx) continue;
#pragma unroll
      for (int j = 0; j < FY; ++j) {
        const int col = y0 + wy + 16 * j + (lane >> 4) * 4;
        float* to = slab + (int64_t)x * a.ny + col;
        if (col + 4 <= a.ny) {
          *reinterpret_cast<f32x4_any4*>(to) = acc[i][j];
        } else {
#pragma unroll
          for (int e = 0; e < 3; ++e)
            if (col + e < a.ny) to[e] = acc[i][j][e];
        }
      }
    }
  } else {
    const float unit = a.unit != nullptr ? *a.unit : 1.0f;
#pragma unroll
    for (int i = 0; i < FX; ++i) {
      const int x = x0 + wx + 16 * i + (lane & 15);
      if (x >= nx) continue;
      const int64_t row = a.map != nullptr ? a.map[x] : x;
#pragma unroll
      for (int j = 0; j < FY; ++j) {
        const int col = y0 + wy + 16 * j + (lane >> 4) * 4;
        if (col >= a.ny) continue;
        f32x4_any4 v = acc[i][j];
        const int n = a.ny - col;
        const float* add = a.add != nullptr ? a.add + x * a.add_ld + col : nullptr;
        if (a.out_f32) {
          float* to = (float*)a.out + row * a.ld + col;
          if (n >= 4) {
            if (add != nullptr) v += *reinterpret_cast<const f32x4_any4*>(add);
            v *= unit;
            if (a.accumulate) v += *reinterpret_cast<const f32x4_any4*>(to);
            *reinterpret_cast<f32x4_any4*>(to) = v;
          } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
              if (e < n) to[e] = (v[e] + (add != nullptr ? add[e] : 0.0f)) * unit + (a.accumulate ? to[e] : 0.0f);
          }
        } else {
          bf16_t* to = (bf16_t*)a.out + row * a.ld + col;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e < n) v[e] = (v[e] + (add != nullptr ? add[e] : 0.0f)) * unit + (a.accumulate ? (float)to[e] : 0.0f);
          if (n >= 4) {
            *reinterpret_cast<u32x2_any2*>(to) = u32x2_any2{two_bf16(v[0], v[1]), two_bf16(v[2], v[3])};
          } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
              if (e < n) to[e] = (bf16_t)v[e];
          }
        }
      }
    }
  }
}

// The shares' slabs of a product, added in turn: a wave takes 256 columns of a row.  Bound by memory (2867 x 2048, two slabs and what earlier pieces left: 30 us).
__global__ __launch_bounds__(256) void head_sum_kernel(Product a, int bx, int by) {
  const int count = a.count != nullptr ? *a.count : 0;
  const int nx = a.count != nullptr && !a.count_k ? count : a.nx, nk = a.count != nullptr && a.count_k ? count : a.k;
  const int64_t tiles = (int64_t)((nx + bx - 1) / bx) * ((a.ny + by - 1) / by), size = (int64_t)nx * a.ny;
  const int shares = shares_of(a.split, tiles, (nk + 63) / 64 * a.parts, size);
  if (shares == 1) return;   // (the product wrote the result)
  const int across = (a.ny + 255) / 256;
  const int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), x = n / across;
  const int col = (int)(n - x * across) * 256 + (threadIdx.x & 63) * 4, left = a.ny - col;
  if (x >= nx || left <= 0) return;
  auto four = [&](const float* p) __attribute__((always_inline)) {
    f32x4_any4 v{};
    if (left >= 4) {
      v = *reinterpret_cast<const f32x4_any4*>(p);
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (e < left) v[e] = p[e];
    }
    return v;
  };
  f32x4_any4 v{}, slab[8];   // (their loads on the way together)
#pragma unroll
  for (int i = 0; i < 8; ++i) slab[i] = i < shares ? four(a.slabs + i * size + x * a.ny + col) : f32x4_any4{};
#pragma unroll
  for (int i = 0; i < 8; ++i) v += slab[i];
  if (a.add != nullptr) v += four(a.add + x * a.add_ld + col);
  if (a.unit != nullptr) v *= *a.unit;
  const int64_t row = a.map != nullptr ? a.map[x] : x;
  if (a.out_f32) {
    float* to = (float*)a.out + row * a.ld + col;
    if (a.accumulate) v += four(to);
    if (left >= 4) {
      *reinterpret_cast<f32x4_any4*>(to) = v;
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (e < left) to[e] = v[e];
    }
  } else {
    bf16_t* to = (bf16_t*)a.out + row * a.ld + col;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) to[e] = (bf16_t)(a.accumulate ? v[e] + (float)to[e] : v[e]);
  }
}

// ---- few tiles of logits --------------------------------------------------------------------------------
// Where the logits are few tiles of many k's, their product, too, is cut into shares, and these launches take the place of its epilogues.  Taken where the fit says a quarter
// of the time, and 5 us, at least: closer calls went either way.
constexpr int kSlabColumns = 1024;   // of a block: four a thread, 256 apart, all shares' loads on the way together
struct Slabs {
  const float* p;
  int shares, nx, ny;
  __device__ inline void get(int x, int col, float (&z)[4]) const {   // (zeros beyond the last column)
    float v[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i][e] = i < shares && col + 256 * e < ny ? p[((int64_t)i * nx + x) * ny + col + 256 * e] : 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      z[e] = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) z[e] += v[i][e];
    }
  }
};
__device__ inline Slabs slabs_of(const Product& a, int bx, int by) {
  const int nx = a.count != nullptr ? *a.count : a.nx;
  const int64_t tiles = (int64_t)((nx + bx - 1) / bx) * ((a.ny + by - 1) / by);
  return {a.slabs, shares_of(a.split, tiles, (a.k + 63) / 64 * a.parts, (int64_t)nx * a.ny), nx, a.ny};
}
// The sums of a row's kSlabColumns logits: a block each.
__global__ __launch_bounds__(256) void head_slab_partial_kernel(Product a, int bx, int by) {
  __shared__ Partial joined[4];
  const Slabs s = slabs_of(a, bx, by);
  const int x = blockIdx.x, col = blockIdx.y * kSlabColumns + threadIdx.x;
  if (x >= s.nx) return;
  const int label = a.row_label != nullptr ? a.row_label[x] - a.y0 : -1;
  Partial p{-__builtin_inff(), -1.0f, -1.0f, 0.0f};
  float z[4];
  s.get(x, col, z);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (col + 256 * e >= s.ny) continue;
    z[e] *= a.scale;
    if (col + 256 * e == label) a.z_label[x] = z[e];
    p = join(p, Partial{z[e], 0.0f, 0.0f, z[e]}, a.inv_tau);
  }
  p = lanes_joined(p, a.inv_tau);
  if ((threadIdx.x & 63) == 0) joined[threadIdx.x >> 6] = p;
  __syncthreads();
  if (threadIdx.x == 0)
    a.partial[(int64_t)blockIdx.y * a.partial_ld + x] = join(join(joined[0], joined[1], a.inv_tau), join(joined[2], joined[3], a.inv_tau), a.inv_tau);
}
// The gradient of a row's logits, with the zeros behind it that the products take: likewise.
__global__ __launch_bounds__(256) void head_slab_grad_kernel(Product a, int bx, int by) {
  const Slabs s = slabs_of(a, bx, by);
  const int x = blockIdx.x, col = blockIdx.y * kSlabColumns + threadIdx.x;
  if (x >= (s.nx + kRowTile - 1) / kRowTile * kRowTile) return;
  const RowGrad g = a.grad[x];
  const int label = g.label >= 0 ? g.label - a.y0 : -1;
  float z[4] = {};
  if (x < s.nx) s.get(x, col, z);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int c = col + 256 * e;
    if (c >= (s.ny + 63) / 64 * 64) continue;
    float d = __builtin_fmaf(g.a, exp_of(__builtin_fmaf(z[e], a.scale, -g.L)), g.a0);
    if (a.inv_tau != 1.0f) d = __builtin_fmaf(g.at, exp_of(__builtin_fmaf(z[e] * a.scale, a.inv_tau, -g.Lt)), d);
    if (c == label) d += g.ay;
    put_parts(a.d + x * a.d_pitch + c * 2, a.d_plane, a.d_parts, x < s.nx && c < s.ny ? d : 0.0f);
  }
}

// ---- the teacher's entries ------------------------------------------------------------------------------
// z at a row's entries.  rounded: operands as bf16 (fp32 with ABL_MATH_BF16).
struct EntryLogits {
  const void *h, *W;
  int64_t ldh, ldw;
  int C, V, T, dtype, rounded;
  const int64_t* ids;
  const float* logits;
  float scale;
  float* z_top;
};
// At the k-th one, by a wave: of few rows, whose operands are never rounded.
template <typename T>
__device__ inline void entry_logit(const EntryLogits& a, int64_t row, int k) {
  const int lane = threadIdx.x & 63;
  const int64_t at = row * a.T + k, id = a.ids[at];
  if (!entry_there(id, a.logits[at]) || id >= a.V) {
    if (lane == 0) a.z_top[at] = id >= a.V ? nan_value() : 0.0f;
    return;
  }
  const T *h = (const T*)a.h + row * a.ldh, *w = (const T*)a.W + id * a.ldw;
  float s = 0.0f;
  auto add = [&](int c, int n) __attribute__((always_inline)) {
    float x[8], y[8];
    load_piece(h + c, n, x);
    load_piece(w + c, n, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) s = __builtin_fmaf(x[e], y[e], s);
  };
  const int whole = a.C / 512 * 512;
#pragma unroll 4
  for (int c = 0; c < whole; c += 512) add(c + lane * 8, 8);
  if (whole < a.C) add(whole + lane * 8, a.C - whole - lane * 8);
  s = wave_sum(s);
  if (lane == 0) a.z_top[at] = s * a.scale;
}
// Four waves a row that counts.  A wave takes two entries at a time, their rows of the table on the way together: rows from anywhere in a table that
// no cache holds (2867 rows, 32 entries of 4 KB each: 59 us, 6.4 TB/s).
template <typename T>
__global__ __launch_bounds__(256) void head_entries_kernel(EntryLogits a, const int* __restrict__ rows, const int* __restrict__ count) {
  if ((int)blockIdx.x >= *count) return;
  const int64_t row = rows[blockIdx.x];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const T* h = (const T*)a.h + row * a.ldh;
  for (int k0 = 0; k0 < a.T; k0 += 64) {
    // the tokens of 64 entries, one a lane: -1: absent, V: beyond the vocabulary
    const int64_t at = row * a.T + k0 + lane, wide = k0 + lane < a.T ? a.ids[at] : -1;
    const bool there = k0 + lane < a.T && entry_there(wide, a.logits[at]);
    const int id = !there ? -1 : wide < a.V ? (int)wide : a.V, n = a.T - k0 < 64 ? a.T - k0 : 64;
    float mine = there ? nan_value() : 0.0f;
    uint64_t left = __ballot(there && id < a.V) & (0x1111111111111111ull << wave);   // of this wave
    while (left != 0) {
      const int i = __builtin_ctzll(left);
      left &= left - 1;
      const int j = left != 0 ? __builtin_ctzll(left) : i;
      left &= left - 1;
      const T *wi = (const T*)a.W + (int64_t)__builtin_amdgcn_readlane(id, i) * a.ldw, *wj = (const T*)a.W + (int64_t)__builtin_amdgcn_readlane(id, j) * a.ldw;
      float si = 0.0f, sj = 0.0f;
      auto add = [&](int c, int m) __attribute__((always_inline)) {
        float x[8], y[8], z[8];
        load_piece(wi + c, m, y);
        load_piece(wj + c, m, z);
        load_piece(h + c, m, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float u = a.rounded ? (float)(bf16_t)x[e] : x[e];
          si = __builtin_fmaf(u, a.rounded ? (float)(bf16_t)y[e] : y[e], si);
          sj = __builtin_fmaf(u, a.rounded ? (float)(bf16_t)z[e] : z[e], sj);
        }
      };
      const int whole = a.C / 512 * 512;
#pragma unroll 4
      for (int c = 0; c < whole; c += 512) add(c + lane * 8, 8);
      if (whole < a.C) add(whole + lane * 8, a.C - whole - lane * 8);
      si = wave_sum(si), sj = wave_sum(sj);
      if (lane == i) mine = si * a.scale;
      if (lane == j) mine = sj * a.scale;
    }
    if (lane < n && (lane & 3) == wave) a.z_top[at] = mine;
  }
}

// ---- few rows -------------------------------------------------------------------------------------------
// Logits of up to 64 rows: bound by the table, which is read once, straight into registers.  A block takes 16 YT tokens at a time, its WAVES waves a share
// of the channels each (eight up to 16 rows, four beyond), so that a small table, too, is many waves' work; rows come from the caches again and again.  A lane's 32 bytes of a row are
// its operands of two matrix instructions (bf16) or eight (fp32, exact): which k they stand for does not matter as long as both sides agree.  fp32 2 x 2688 x 116480:
// 240 us with the second launch, 5.2 TB/s; 48 x 2048 x 32768: 101 (as 64 rows 118); 64 x 4096 x 65536: 450, the fp32 instructions' rate.
struct Thin {
  const void *h, *W;
  int64_t ldh, ldw;
  int M, C, V, groups;    // groups: blocks that share the tokens
  const int64_t* labels;
  float scale, inv_tau;
  float* z_label;
  Partial* partial;       // [groups][M]
  // backward: the rows that count, with zero rows up to the tiles', and the gradient of their logits
  const RowGrad* grad;
  float* d;
  int64_t d_ld;
  int v0;                 // the table's first row, in the vocabulary
};
template <typename T>
struct Run {   // 32 bytes of a row: 16, and 16 of 64 bytes further
  static constexpr int kElements = 32 / sizeof(T);
  u32x4_any2 a, b;
};
template <typename T>
__device__ inline Run<T> load_run(const T* p) {
  return {*reinterpret_cast<const u32x4_any2*>(p), *reinterpret_cast<const u32x4_any2*>(p + 64 / sizeof(T))};
}
template <typename T>
__device__ inline Run<T> load_run_end(const T* p, int n) {   // n elements exist from p on
  constexpr int kFar = 64 / sizeof(T);
  Run<T> r;
  if constexpr (std::is_same_v<T, float>) {
    r.a = u32x4{}, r.b = u32x4{};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (e < n) r.a[e] = __float_as_uint(p[e]);
      if (e + kFar < n) r.b[e] = __float_as_uint(p[e + kFar]);
    }
  } else {
    r.a = load_raw(p, n).a, r.b = load_raw(p + kFar, n - kFar).a;
  }
  return r;
}
__device__ inline floatx4 multiply(const Run<bf16_t>& y, const Run<bf16_t>& x, floatx4 c) {
  c = mfma32(__builtin_bit_cast(bf16x8_t, (u32x4)y.a), __builtin_bit_cast(bf16x8_t, (u32x4)x.a), c);
  return mfma32(__builtin_bit_cast(bf16x8_t, (u32x4)y.b), __builtin_bit_cast(bf16x8_t, (u32x4)x.b), c);
}
__device__ inline floatx4 multiply(const Run<float>& y, const Run<float>& x, floatx4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(y.a[e]), __uint_as_float(x.a[e]), c, 0, 0, 0);
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(y.b[e]), __uint_as_float(x.b[e]), c, 0, 0, 0);
  return c;
}

template <typename T, int XT, int YT, int WAVES, int AHEAD, bool GRAD>
__global__ __launch_bounds__(WAVES * 64) void head_thin_kernel(Thin a) {
  constexpr int kRun = Run<T>::kElements, kStep = 4 * kRun;
  __shared__ floatx4 sums[WAVES][XT * YT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int tiles = (a.V + 16 * YT - 1) / (16 * YT), whole = a.C / kStep;
  const T* h[XT];
#pragma unroll
  for (int i = 0; i < XT; ++i) h[i] = (const T*)a.h + (int64_t)(16 * i + r < a.M ? 16 * i + r : a.M - 1) * a.ldh + g * (kRun / 2);
  Partial all{-__builtin_inff(), -1.0f, -1.0f, 0.0f};   // of this lane's row of the tile that its wave sums up
  for (int tile = blockIdx.x; tile < tiles; tile += a.groups) {
    const int v0 = tile * (16 * YT);
    const T* w[YT];
#pragma unroll
    for (int j = 0; j < YT; ++j) w[j] = (const T*)a.W + (int64_t)(v0 + 16 * j + r < a.V ? v0 + 16 * j + r : a.V - 1) * a.ldw + g * (kRun / 2);
    floatx4 acc[XT][YT];
#pragma unroll
    for (int i = 0; i < XT; ++i)
#pragma unroll
      for (int j = 0; j < YT; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    auto steps = [&](int s, auto n) __attribute__((always_inline)) {   // n steps, all their loads on the way together
      Run<T> y[n.value][YT], x[n.value][XT];
#pragma unroll
      for (int u = 0; u < n.value; ++u) {
#pragma unroll
        for (int j = 0; j < YT; ++j) y[u][j] = load_run(w[j] + (int64_t)(s + WAVES * u) * kStep);
#pragma unroll
        for (int i = 0; i < XT; ++i) x[u][i] = load_run(h[i] + (int64_t)(s + WAVES * u) * kStep);
      }
#pragma unroll
      for (int u = 0; u < n.value; ++u)
#pragma unroll
        for (int j = 0; j < YT; ++j)
#pragma unroll
          for (int i = 0; i < XT; ++i) acc[i][j] = multiply(y[u][j], x[u][i], acc[i][j]);
    };
    int s = wave;
    for (; s + WAVES * (AHEAD - 1) < whole; s += WAVES * AHEAD) steps(s, std::integral_constant<int, AHEAD>{});
    for (; s < whole; s += WAVES) steps(s, std::integral_constant<int, 1>{});
    if (wave == 0 && whole * kStep < a.C) {   // the ragged end
      const int n = a.C - whole * kStep - g * (kRun / 2);
#pragma unroll
      for (int j = 0; j < YT; ++j) {
        const Run<T> y = load_run_end(w[j] + (int64_t)whole * kStep, n);
#pragma unroll
        for (int i = 0; i < XT; ++i) acc[i][j] = multiply(y, load_run_end(h[i] + (int64_t)whole * kStep, n), acc[i][j]);
      }
    }
#pragma unroll
    for (int i = 0; i < XT; ++i)
#pragma unroll
      for (int j = 0; j < YT; ++j) sums[wave][i * YT + j][lane] = acc[i][j];
    __syncthreads();
    if (GRAD && wave < XT) {   // (the lanes' rows and tokens: see below)
      const int row = 16 * wave + r;
      const RowGrad k = a.grad[row];
#pragma unroll
      for (int j = 0; j < YT; ++j) {
        const int at = wave * YT + j, col = v0 + 16 * j + 4 * g;
        floatx4 v = sums[0][at][lane], d;
#pragma unroll
        for (int n = 1; n < WAVES; ++n) v += sums[n][at][lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float z = v[e] * a.scale;
          d[e] = __builtin_fmaf(k.a, exp_of(z - k.L), k.a0);
          if (a.inv_tau != 1.0f) d[e] = __builtin_fmaf(k.at, exp_of(__builtin_fmaf(z, a.inv_tau, -k.Lt)), d[e]);
          if (k.label >= 0 && col + e == k.label - a.v0) d[e] += k.ay;
          if (!k.counts || col + e >= a.V) d[e] = 0.0f;   // (whatever the table holds)
        }
        *reinterpret_cast<floatx4*>(a.d + row * a.d_ld + col) = d;
      }
    }
    if (!GRAD && wave < XT) {   // the wave's tile of rows: lane's row lane % 16, tokens 4 (lane / 16) + 0..3 of each tile of tokens
      const int row = 16 * wave + r;
      const int64_t label = a.labels != nullptr && row < a.M ? a.labels[row] : -1;
      float z[YT][4];
      Partial p{-__builtin_inff(), -1.0f, -1.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < YT; ++j) {
        const int at = wave * YT + j;
        floatx4 v = sums[0][at][lane];
#pragma unroll
        for (int n = 1; n < WAVES; ++n) v += sums[n][at][lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int col = v0 + 16 * j + 4 * g + e;
          z[j][e] = v[e] * a.scale;
          if (col == label) a.z_label[row] = z[j][e];
          p.z += col < a.V ? z[j][e] : 0.0f;
          z[j][e] = col < a.V ? z[j][e] : -__builtin_inff();
          p.top = fmaxf(p.top, z[j][e]);
        }
      }
      p.top = lanes16_max(p.top);
      float tops = 0.0f;
      p.rest = p.rest_t = 0.0f;
      const float ref = p.top == -__builtin_inff() ? 0.0f : p.top;
#pragma unroll
      for (int j = 0; j < YT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool hit = z[j][e] == ref;
          p.rest += hit ? 0.0f : exp_of(z[j][e] - ref);
          if (a.inv_tau != 1.0f) p.rest_t += hit ? 0.0f : exp_of((z[j][e] - ref) * a.inv_tau);
          tops += hit ? 1.0f : 0.0f;
        }
      tops = lanes16_sum(tops);
      p.rest = lanes16_sum(p.rest) + (tops - 1.0f), p.rest_t = lanes16_sum(p.rest_t) + (tops - 1.0f), p.z = lanes16_sum(p.z);
      all = join(all, p, a.inv_tau);
    }
    __syncthreads();
  }
  if (!GRAD && wave < XT && g == 0 && 16 * wave + r < a.M) a.partial[(int)blockIdx.x * a.M + 16 * wave + r] = all;
}

// Both gradients of up to 64 rows, from the gradient of their logits in fp32 and in fp32 throughout (matrix instructions of 16 x 16 x 4): bound by the table, which is
// read, and its gradient, which is written.  A wave keeps 64 channels of h and of dh in its registers (128: 10 to 30 % slower, fewer waves fit) and goes along a share
// of the tokens, 16 at a time: four neighbours of the channels are a lane's, in all its loads and stores.  The shares' sums of dh are joined by a launch of their own.
// 2 x 2688 x 116480 fp32: 829 us with the logits' launch, 4.5 TB/s (three bf16 parts padded to 64 rows: 3437); 64 x 4096 x 65536: 1228 (2993); bf16, 7 x 5632 x 11705:
// 121 us (156), 8 x 4096 x 131072: 1012 (1059).  With 17 to 64 rows of bf16 the products in bf16 are faster (32 x 2048 x 32768: 138 us, here 186; 64: 137, 324).
struct ThinGrad {
  const void *h, *W;          // h: the copy, with zeros up to the tiles' rows and whole 64 channels
  int64_t ldh, ldw;
  int M, C, n;                // n: tokens
  const float* d;             // [rows][d_ld]: zeros behind the tokens up to a multiple of 16
  int64_t d_ld;
  int shares, per, more;      // per: tokens of a share, a multiple of 16; more: the slabs hold sums of earlier pieces
  float* slabs;               // [shares][M][C]; nullptr: no dh
  void* dW;                   // nullptr: none
  int out_f32, accumulate;
};
// Four elements, n of which exist.
__device__ inline floatx4 load_four(const float* p, int n) {
  if (n >= 4) return *reinterpret_cast<const f32x4_any4*>(p);
  floatx4 v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < n) v[e] = p[e];
  return v;
}
__device__ inline floatx4 load_four(const bf16_t* p, int n) {
  if (n >= 4) {
    const u32x2_any2 w = *reinterpret_cast<const u32x2_any2*>(p);
    return floatx4{low_bf16(w[0]), high_bf16(w[0]), low_bf16(w[1]), high_bf16(w[1])};
  }
  floatx4 v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < n) v[e] = (float)p[e];
  return v;
}
__device__ inline void store_four(float* p, int n, floatx4 v) {
  if (n >= 4) {
    *reinterpret_cast<f32x4_any4*>(p) = v;
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < n) p[e] = v[e];
  }
}
__device__ inline void store_four(bf16_t* p, int n, floatx4 v) {
  if (n >= 4) {
    *reinterpret_cast<u32x2_any2*>(p) = u32x2_any2{two_bf16(v[0], v[1]), two_bf16(v[2], v[3])};
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < n) p[e] = (bf16_t)v[e];
  }
}
template <typename T, int XT>
__global__ __launch_bounds__(256, XT == 4 ? 1 : 2) void head_thin_grad_kernel(ThinGrad a) {
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int across = (a.C + 63) / 64;
  const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int share = (int)(id / across), c = (int)(id - (int64_t)share * across) * 64 + 4 * r;
  if (share >= a.shares) return;
  const int t0 = share * a.per, t1 = a.n - t0 < a.per ? a.n : t0 + a.per;
  const T* W = (const T*)a.W + c;
  floatx4 h[XT][4], dh[XT][4];   // h of row 16 x + 4 k + g; dh of rows 16 x + 4 g + 0..3 and channel c + e
#pragma unroll
  for (int x = 0; x < XT; ++x)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      h[x][k] = load_four((const T*)a.h + (16 * x + 4 * k + g) * a.ldh + c, 4);
      dh[x][k] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    }
  if (a.more && a.slabs != nullptr) {
#pragma unroll
    for (int x = 0; x < XT; ++x)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int row = 16 * x + 4 * g + q;
        const floatx4 v = load_four(a.slabs + ((int64_t)share * a.M + row) * a.C + c, row < a.M ? a.C - c : 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) dh[x][e][q] = v[e];
      }
  }
  floatx4 w[4], by_token[XT];
  float by_row[XT][4];
  auto load = [&](int t) __attribute__((always_inline)) {
    if (a.slabs != nullptr) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int v = t + 4 * g + u < a.n ? t + 4 * g + u : a.n - 1;   // (d is zero behind the last token)
        w[u] = load_four(W + v * a.ldw, a.C - c);
      }
#pragma unroll
      for (int x = 0; x < XT; ++x) by_token[x] = *reinterpret_cast<const floatx4*>(a.d + (16 * x + r) * a.d_ld + t + 4 * g);
    }
    if (a.dW != nullptr) {
#pragma unroll
      for (int x = 0; x < XT; ++x)
#pragma unroll
        for (int k = 0; k < 4; ++k) by_row[x][k] = a.d[(16 * x + 4 * k + g) * a.d_ld + t + r];
    }
  };
  if (t0 < t1) load(t0);
  for (int t = t0; t < t1; t += 16) {
    floatx4 v[4], bt[XT];
    float br[XT][4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = w[u];
#pragma unroll
    for (int x = 0; x < XT; ++x) {
      bt[x] = by_token[x];
#pragma unroll
      for (int k = 0; k < 4; ++k) br[x][k] = by_row[x][k];
    }
    if (t + 16 < t1) load(t + 16);   // on the way while these are multiplied
    if (a.slabs != nullptr) {
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int x = 0; x < XT; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) dh[x][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(bt[x][u], v[u][e], dh[x][e], 0, 0, 0);
    }
    if (a.dW == nullptr) continue;
    floatx4 dw[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) dw[e] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int x = 0; x < XT; ++x)
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) dw[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(br[x][k], h[x][k][e], dw[e], 0, 0, 0);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int token = t + 4 * g + q, n = token < a.n ? a.C - c : 0;
      floatx4 o{dw[0][q], dw[1][q], dw[2][q], dw[3][q]};
      auto put = [&](auto* to) __attribute__((always_inline)) {
        if (a.accumulate) o += load_four(to, n);
        store_four(to, n, o);
      };
      if (a.out_f32)
        put((float*)a.dW + (int64_t)token * a.C + c);
      else
        put((bf16_t*)a.dW + (int64_t)token * a.C + c);
    }
  }
  if (a.slabs == nullptr) return;
#pragma unroll
  for (int x = 0; x < XT; ++x)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int row = 16 * x + 4 * g + q;
      store_four(a.slabs + ((int64_t)share * a.M + row) * a.C + c, row < a.M ? a.C - c : 0, floatx4{dh[x][0][q], dh[x][1][q], dh[x][2][q], dh[x][3][q]});
    }
}
// dh of a row: the shares' sums, 64 channels a block, a quarter of the shares a wave.
__global__ __launch_bounds__(256) void head_thin_sum_kernel(ThinGrad a, const int* __restrict__ rows, const int* __restrict__ count, void* dh, int64_t ld, int f32) {
  __shared__ float joined[4][64];
  const int x = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.y * 64 + lane;
  if (x >= *count) return;
  float v = 0.0f;
  if (c < a.C)
#pragma unroll 8
    for (int i = wave; i < a.shares; i += 4) v += a.slabs[((int64_t)i * a.M + x) * a.C + c];
  joined[wave][lane] = v;
  __syncthreads();
  if (wave != 0 || c >= a.C) return;
  v = (joined[0][lane] + joined[1][lane]) + (joined[2][lane] + joined[3][lane]);
  const int64_t at = rows[x] * ld + c;
  if (f32)
    ((float*)dh)[at] = v;
  else
    ((bf16_t*)dh)[at] = (bf16_t)v;
}

// Maximum and sum of a row's softmax over its entries at temperature tau, by a wave: p_k = exp((t_k - top) / tau) / sum (the difference first: a t of the type's largest values
// may not be divided by a small tau).
__device__ inline void teacher_sums(const int64_t* ids, const float* logits, int T, float inv_tau, float& top, float& sum) {
  const int lane = threadIdx.x & 63;
  top = -__builtin_inff();
  for (int k = lane; k < T; k += 64)
    if (entry_there(ids[k], logits[k])) top = fmaxf(top, logits[k]);
  top = wave_max(top);
  sum = 0.0f;
  for (int k = lane; k < T; k += 64)
    if (entry_there(ids[k], logits[k])) sum += exp_of((logits[k] - top) * inv_tau);
  sum = wave_sum(sum);
}

// The tiles' sums of each row, joined, and its loss: a block of 1024 threads takes ROWS of them (16, or one where there are few), a wave each at the end.
// Without a list of rows (rows = nullptr) all M of them are there, and those that do not count get zeros here.  16 rows read whole 256 bytes of a tile's sums (8192 rows, 256 tiles: 14 us); for few rows the time is the
// chain of loads, sums and logarithms of a launch (one row: 4 us), and with a teacher its entries' rows of the table (16 rows of 8: 9 us).
struct Loss {
  int M;
  const Partial* partial;
  int64_t partial_ld;
  int tiles;
  const Partial* before;   // of the pieces of the vocabulary before this one (nullptr: none)
  Partial* after;          // where more pieces follow (nullptr: this is the last one)
  const int *rows, *count;
  const unsigned char* flags;
  const int64_t *labels, *ids;
  const float *logits, *z_label;
  int T, V;
  float smoothing, z_weight, tau, label_weight, teacher_weight;
  float *loss, *lse, *lse_t;
  const float* z_top;
  EntryLogits entries;   // few rows, T > 0: made here
};
template <int ROWS>
__global__ __launch_bounds__(1024) void head_loss_kernel(Loss a) {
  constexpr int kGroups = 1024 / ROWS;
  __shared__ Partial joined[ROWS == 1 ? 16 : 64][ROWS == 1 ? 1 : ROWS + 1];
  const int n0 = blockIdx.x * ROWS, count = a.rows != nullptr ? *a.count : a.M;
  if (n0 >= count) return;
  const float inv_tau = 1.0f / a.tau;
  if constexpr (ROWS == 1) {
    // (by the last waves first, which have no sums to join where there are few; read below by the wave of the row, behind the barrier)
    for (int k = 15 - (int)(threadIdx.x >> 6); k < a.entries.T; k += 16) {
      if (a.entries.dtype == ABL_F32)
        entry_logit<float>(a.entries, n0, k);
      else
        entry_logit<bf16_t>(a.entries, n0, k);
    }
  }
  // What a wave will need of its row, on the way while the sums are joined.
  const int r = threadIdx.x >> 6, lane = threadIdx.x & 63, n = n0 + r;
  const bool mine = r < ROWS && n < count;
  int64_t row = n;
  int f = 0;
  float z_label = 0.0f;
  if (mine && a.after == nullptr) {
    if (a.rows != nullptr) row = a.rows[n];
    f = a.flags != nullptr ? a.flags[row] : row_flags(row, a.labels, a.ids, a.logits, a.T, a.V);
    if (f & kLabel) z_label = a.z_label[n];
  }
  const Partial none{-__builtin_inff(), -1.0f, -1.0f, 0.0f};
  Partial p = none;
  {
    const int r = threadIdx.x % ROWS, group = threadIdx.x / ROWS;
    if (n0 + r < count) {
      if (group == 0 && a.before != nullptr) p = a.before[n0 + r];
      const Partial* from = a.partial + n0 + r;
      int t = group;
      for (; t + 3 * kGroups < a.tiles; t += 4 * kGroups) {   // (four loads on the way together)
        Partial q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = from[(t + i * kGroups) * a.partial_ld];
#pragma unroll
        for (int i = 0; i < 4; ++i) p = join(p, q[i], inv_tau);
      }
      for (; t < a.tiles; t += kGroups) p = join(p, from[t * a.partial_ld], inv_tau);
    }
    if constexpr (ROWS == 1) {
      p = lanes_joined(p, inv_tau);
      if ((threadIdx.x & 63) == 0) joined[threadIdx.x >> 6][0] = p;
    } else {
      joined[group][r] = p;
    }
  }
  __syncthreads();
  if (!mine) return;
  if constexpr (ROWS == 1)
    p = lanes_joined<16>(joined[lane & 15][0], inv_tau);
  else
    p = lanes_joined(joined[lane][r], inv_tau);
  if (a.after != nullptr) {
    if (lane == 0) a.after[n] = p;
    return;
  }
  if ((f & (kLabel | kTeacher)) == 0) {
    if (lane == 0) {
      a.loss[row] = 0.0f;
      if (a.lse != nullptr) a.lse[row] = 0.0f;
      if (a.lse_t != nullptr) a.lse_t[row] = 0.0f;
    }
    return;   // (its entries are absent: z_top has zeros there)
  }
  const float ln = log1pf(p.rest), L = p.top + ln;
  const float ln_t = a.tau != 1.0f ? log1pf(p.rest_t) : ln, top_t = p.top * inv_tau;
  float loss = a.z_weight != 0.0f ? a.z_weight * L * L : 0.0f;
  if (f & kLabel) {   // (differences to the maximum first: L and z are large where the loss is small)
    float ce = ln + (p.top - z_label);
    if (a.smoothing != 0.0f) ce = (1.0f - a.smoothing) * ce + a.smoothing * (ln + (p.top - p.z / (float)a.V));
    loss += a.label_weight * ce;
  }
  if (f & kTeacher) {
    const int64_t* ids = a.ids + row * a.T;
    const float *t = a.logits + row * a.T, *z = a.z_top + row * a.T;
    float top, sum, kd = 0.0f;
    teacher_sums(ids, t, a.T, inv_tau, top, sum);
    const float norm = 1.0f / sum, ln_sum = log_of(sum);
    for (int k = lane; k < a.T; k += 64)
      if (entry_there(ids[k], t[k])) {
        const float u = (t[k] - top) * inv_tau, q = exp_of(u) * norm;
        if (q != 0.0f) kd += q * ((u - ln_sum) + (p.top - z[k]) * inv_tau);   // (NaN goes in)
      }
    loss += a.teacher_weight * a.tau * a.tau * (wave_sum(kd) + ln_t);
  }
  if (f & kBad) loss = nan_value();
  if (lane == 0) {
    a.loss[row] = loss;
    if (a.lse != nullptr) a.lse[row] = L;
    if (a.lse_t != nullptr) a.lse_t[row] = top_t + ln_t;
  }
}

// The gradient of the logits at a row's entries, over what the product wrote there: from the row's z_top, before any rounding; of entries with the
// same id the first one takes the sum of their probabilities.  A wave a row.
struct Entries {
  const int *rows, *count;
  const int64_t* ids;
  const float *logits, *z_top;
  const RowGrad* grad;
  int T, v0, v1;   // tokens of this piece
  float inv_tau;
  char* d;
  int64_t d_plane, d_pitch;
  int d_parts;
};
__device__ inline void put_entry_grad(const Entries& a, const RowGrad& g, int n, int id, float z, float p) {
  float v = __builtin_fmaf(g.a, exp_of(z - g.L), g.a0);
  v = __builtin_fmaf(g.at, (a.inv_tau != 1.0f ? exp_of(__builtin_fmaf(z, a.inv_tau, -g.Lt)) : 0.0f) - p, v);
  if (id == g.label) v += g.ay;
  if (a.d_parts == 0)   // (fp32)
    ((float*)(a.d + n * a.d_pitch))[id - a.v0] = v;
  else
    put_parts(a.d + n * a.d_pitch + (id - a.v0) * 2, a.d_plane, a.d_parts, v);
}
__global__ __launch_bounds__(256) void head_entry_grad_kernel(Entries a) {
  const int n = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (n >= *a.count) return;
  const int64_t row = a.rows[n];
  const int64_t* ids = a.ids + row * a.T;
  const float* t = a.logits + row * a.T;
  if (a.T <= 64) {   // an entry a lane; tokens fit 32 bits
    const int64_t wide = lane < a.T ? ids[lane] : -1;
    const float u = lane < a.T ? t[lane] : 0.0f;
    const bool there = lane < a.T && entry_there(wide, t[lane]);
    const int id = there && wide < a.v1 ? (int)wide : -1;
    if (!__any(id >= a.v0)) return;
    const float top = wave_max(there ? u : -__builtin_inff());
    const float e = there ? exp_of((u - top) * a.inv_tau) : 0.0f, mine = e / wave_sum(e);
    bool first = true;
    float p = 0.0f;
    for (int i = 0; i < a.T; ++i) {
      const bool same = __builtin_amdgcn_readlane(id, i) == id;
      first = first && !(same && i < lane);
      p += same ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine), i)) : 0.0f;
    }
    if (first && id >= a.v0) put_entry_grad(a, a.grad[n], n, id, a.z_top[row * a.T + lane], p);
    return;
  }
  float top, sum;
  teacher_sums(ids, t, a.T, a.inv_tau, top, sum);
  if (sum == 0.0f) return;   // (no entries)
  const RowGrad g = a.grad[n];
  const float norm = 1.0f / sum;
  for (int k = lane; k < a.T; k += 64) {
    const int64_t id = ids[k];
    if (id < a.v0 || id >= a.v1 || !entry_there(id, t[k])) continue;
    bool first = true;
    for (int i = 0; i < k; ++i) first = first && !(ids[i] == id && entry_there(id, t[i]));
    if (!first) continue;
    float p = 0.0f;
    for (int i = k; i < a.T; ++i)
      if (ids[i] == id && entry_there(id, t[i])) p += exp_of((t[i] - top) * a.inv_tau) * norm;
    put_entry_grad(a, g, n, (int)id, a.z_top[row * a.T + k], p);
  }
}

__global__ __launch_bounds__(256) void head_zero_kernel(uint16_t* p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = 0;
}

// ---- how a call is cut ----------------------------------------------------------------------------------
inline int64_t up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }

constexpr int64_t kSlabBytes = (int64_t)128 << 20, kFewLogits = (int64_t)16 << 20;
// Columns of the narrowest tile that leaves its rows' sums of the logits: 64 up to kNarrowRows rows.
constexpr int kNarrowRows = 1024;
inline int narrowest(int64_t rows) { return rows <= kNarrowRows ? 64 : 128; }
constexpr int kThinRows = 64, kThinGroups = 1024, kThinTile = 64, kThinWaves = 4096, kThinShares = 256;
constexpr int64_t kPad = 128;   // bytes behind a row of a copy: rows a power of two apart meet in few channels of the L2
// Bytes of the workspace's parts.  A piece's gradient of the logits, a part: what stays in the last-level cache (256 MB) beside the piece's rows of the table until the
// products have read it, or twice that where it is all there is (8192 x 4096 x 65536: 10.2 ms with 128 MB, 10.5 with 256, 10.3 with 512; 3277 x 2048 x
// 32768, one piece: 1.28 ms, two: 1.35).
constexpr int64_t kPartialBytes = (int64_t)64 << 20, kTableBytes = (int64_t)64 << 20, kGradBytes = (int64_t)128 << 20;

struct Plan {
  int parts, d_parts;       // bf16 parts of h and W; of the gradient of the logits
  int64_t Mp, Cp;           // rows and channels of the copies
  int64_t c_pitch, d_pitch; // bytes from row to row of the copies, of the gradient of the logits
  int64_t piece, table;     // tokens of a piece; of a piece's copied part of the table (0: in place)
  int pieces;
  // places in the workspace
  size_t count, unit, rows, flags, labels, z_label, h, W, partial, carry, grad, d, acc, slabs, bytes;
  int64_t slab_bytes;
};

// copied: whether the table's rows have to be copied.
Plan plan_of(const abl_head& p, bool backward, bool copied) {
  Plan q{};
  const bool one = (p.flags & ABL_MATH_BF16) != 0;
  q.parts = p.dtype == ABL_F32 && !one ? 3 : 1;
  // One part of 8 bits is half a step of bf16 off, as the results are; of a gradient in fp32 three are asked for (8192 x 2048 x 32768, four rows of ten count: 2.25 ms;
  // with two parts 1.81, and errors of 2^-18 instead of 2^-24).
  q.d_parts = q.parts == 3 ? 3 : p.dtype == ABL_BF16 && p.dw_dtype == ABL_F32 && !one ? 3 : 1;
  q.Mp = up(p.M > 0 ? p.M : 1, kRowTile), q.Cp = up(p.C, kChannelTile);
  const int64_t all = up(p.V, 256);
  auto within = [&](int64_t budget, int64_t bytes) {   // of a token
    const int64_t n = budget / bytes / 256 * 256;
    return n < 256 ? 256 : n < all ? n : all;
  };
  const int64_t grad_token = q.Mp * 2 * q.d_parts;
  const int64_t once = 2 * kGradBytes * q.d_parts;
  int64_t piece = backward ? within(all * grad_token <= once ? once : once / 2, grad_token)
                           : within(kPartialBytes, q.Mp * (int64_t)sizeof(Partial) / narrowest(q.Mp));
  if (piece > 1 << 20) piece = 1 << 20;
  const int64_t table = within(kTableBytes, q.Cp * 2 * q.parts);
  if (copied && table < piece) piece = table;
  q.pieces = (int)((p.V + piece - 1) / piece);
  q.piece = up((p.V + q.pieces - 1) / q.pieces, 256);
  q.pieces = (int)((p.V + q.piece - 1) / q.piece);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  q.count = take(16);
  q.unit = q.count + 8;
  q.rows = take(q.Mp * 4);
  q.flags = take(p.T != 0 ? p.M : 0);
  q.labels = take(backward ? 0 : q.Mp * 4);
  q.z_label = take(backward ? 0 : q.Mp * 4);
  q.grad = take(backward ? q.Mp * sizeof(RowGrad) : 0);
  q.c_pitch = q.Cp * 2 + kPad, q.d_pitch = q.piece * 2 + kPad;
  q.h = take(q.Mp * q.c_pitch * q.parts);
  q.table = copied ? q.piece : 0;
  q.W = take(q.table * q.c_pitch * q.parts);
  int64_t sums = q.piece / narrowest(q.Mp) * q.Mp;
  if (p.M <= kThinRows) {
    const int64_t few = (int64_t)((p.V + kThinTile - 1) / kThinTile > kThinGroups ? (p.V + kThinTile - 1) / kThinTile : kThinGroups) * kThinRows;
    sums = sums > few ? sums : few;
  }
  q.partial = take(backward ? 0 : sums * sizeof(Partial));
  q.carry = take(!backward && q.pieces > 1 ? q.Mp * sizeof(Partial) : 0);
  q.d = take(backward ? q.Mp * q.d_pitch * q.d_parts : 0);
  q.acc = take(backward && q.pieces > 1 ? q.Mp * p.C * 4 : 0);
  // shares' sums: as many slabs as fit, of dh or of a piece of dW or of the logits (where these are few tiles: more have no use for shares)
  const int64_t logits = q.Mp * q.piece * 4, few = logits <= kFewLogits ? 8 * logits : 0;
  const int64_t widest_sum = 8 * (q.Mp > q.piece ? q.Mp : q.piece) * p.C * 4;
  q.slab_bytes = backward ? (widest_sum > few ? widest_sum : few) : few < 2 * kFewLogits ? few : 2 * kFewLogits;
  if (q.slab_bytes > kSlabBytes) q.slab_bytes = kSlabBytes;
  q.slabs = take(q.slab_bytes);
  q.bytes = at;
  return q;
}

constexpr uint64_t kPairs1 = 0x00, kPairs3 = 0x000102;               // (x plane in the low four bits; the first product in the low byte)
constexpr uint64_t kPairs6 = 0x000110110220ull;                      // (0,2) (2,0) (1,1) (0,1) (1,0) (0,0)

constexpr int kUnits = 256;   // compute units
template <int BX, int BY, int WX, int WY, int PLACES, bool XO, bool YO, int EPI, bool FEW = false>
int launch_tiles(hipStream_t st, const Product& a) {
  auto kern = head_product_kernel<BX, BY, WX, WY, PLACES, XO, YO, EPI, FEW>;
  constexpr int kBytes = PLACES * (BX + BY) * 128;
  if (kBytes > 64 * 1024)
    if (int e = allow_full_lds((const void*)kern)) return e;
  const int64_t tiles = (int64_t)((a.nx + BX - 1) / BX) * ((a.ny + BY - 1) / BY);
  kern<<<(unsigned)up(tiles * (EPI == kEpiSum && a.split.most > 1 ? a.split.most : 1), 8), WX * WY * 64, kBytes, st>>>(a);
  if (EPI == kEpiSum && a.split.most > 1 && a.out != nullptr) {
    if (int e = hip_status()) return e;
    head_sum_kernel<<<(unsigned)(((int64_t)a.nx * ((a.ny + 255) / 256) + 3) / 4), 256, 0, st>>>(a, BX, BY);
  }
  return hip_status();
}

// Tiles of 256 x 256, 256 x 128, 128 x 128 or 64 x 64, whichever takes the least time for the rows that a call has, by a fit of measured times.  Large tiles read their operands
// less often, small ones fill the units of a small call: bf16 logits of 2048 x 1024 x 8192 in tiles of 256 x 256 50 us, 128 x 128 71, 64 x 64 95; of 100 x 1024 x 3000
// 128 x 128 25.1 us, 64 x 64 20.6; gradients of 130 x 2048 x 1000 47 and 37, of 1000 x 2048 x 2000 75 and 80.
// The constants come from few of these sizes.  Over 139 others (M 100 to 4000, C 512 to 4096, V 1000 to 50000, both types) a call that goes by them takes as long as one with the
// best of the four in the median, and in nine of ten at most 1.4 % longer, bf16 gradients 6 % (their three products in one kind of tiles); at worst 15 % forward (100 x 4096 x 50000
// bf16: 136 us, 128 x 128: 118) and 25 % backward (2000 x 2048 x 1000 bf16: 121 us, 64 x 64: 97).
struct Tiling {
  int bx, by;
  Split split;
};
constexpr Tiling kTilings[4] = {{256, 256, {8, 256, 1600, 8000, 4000, 800}}, {256, 128, {8, 256, 950, 6000, 4000, 800}},
                                {128, 128, {8, 256, 800, 5000, 4000, 800}}, {64, 64, {8, 512, 500, 4500, 4000, 800}}};
// The first so many of them have columns enough for the room that a workspace has for the sums.
inline int tilings_for_sums(int64_t rows) { return narrowest(rows) == 64 ? 4 : 3; }
static_assert(kTilings[0].by >= 128 && kTilings[1].by >= 128 && kTilings[2].by >= 128 && kTilings[3].by >= 64 && kSlabColumns >= 128 && kNarrowRows % kRowTile == 0);
int64_t tiles_of(const Tiling& t, int64_t nx, int64_t ny) { return (nx + t.bx - 1) / t.bx * ((ny + t.by - 1) / t.by); }
int64_t time_of(const Split& s, int64_t tiles, int steps, int64_t size) {
  const int n = shares_of(s, tiles, steps, size);
  return (tiles * n + s.units - 1) / s.units * ((steps + n - 1) / n * (int64_t)s.step + s.fixed) + (n > 1 ? s.second + n * (size / s.bytes) : 0);
}
struct Choice {
  int tiling;
  Split split;
  int64_t time;
};
// The rows that count, of which there may be fewer, are k (count_k) or nx.
Choice choice_of(int64_t nx, int64_t ny, int64_t k, int parts, bool sums, int64_t slab_bytes, bool count_k, int tilings = 4) {
  const int64_t size = nx * ny, fit = slab_bytes / (size * 4);
  const int steps = (int)((k + 63) / 64 * parts);
  Choice c{};
  int64_t least = 0;
  for (int i = 0; i < tilings; ++i) {
    Split s = kTilings[i].split;
    s.most = !sums || fit < 2 ? 1 : fit < 8 ? (int)fit : 8;
    const int64_t time = time_of(s, tiles_of(kTilings[i], nx, ny), steps, size);
    if (i == 0 || time < least) c = {i, s, time}, least = time;
  }
  int most = 1;   // shares that any number of rows may want
  for (int64_t d = 1; d <= 16 && c.split.most > 1; d *= 2) {
    const int64_t x = count_k ? nx : (nx + d - 1) / d, kk = count_k ? (k + d - 1) / d : k;
    const int n = shares_of(c.split, tiles_of(kTilings[c.tiling], x, ny), (int)((kk + 63) / 64 * parts), x * ny);
    if (n > most) most = n;
  }
  c.split.most = most;
  return c;
}
// Whether few tiles of logits are cut into shares (the launch that takes their slabs costs what one that adds them does).
bool cut_logits(const Product& a, int64_t slab_bytes, Choice& c) {
  const Choice whole = choice_of(a.nx, a.ny, a.k, a.parts, false, 0, false);
  c = choice_of(a.nx, a.ny, a.k, a.parts, true, slab_bytes, false);
  return c.split.most > 1 && c.time + 5000 < whole.time * 3 / 4;
}
template <bool XO, bool YO, int EPI>
int launch_tiling(hipStream_t st, const Product& a, int tiling) {
  if (tiling == 3) return launch_tiles<64, 64, 2, 2, 4, XO, YO, EPI>(st, a);
  if (tiling == 0) return launch_tiles<256, 256, 2, 4, 2, XO, YO, EPI>(st, a);
  return tiling == 1 ? launch_tiles<256, 128, 4, 2, 3, XO, YO, EPI>(st, a) : launch_tiles<128, 128, 2, 4, 4, XO, YO, EPI>(st, a);
}
int launch_slabs(hipStream_t st, Product& a, const Choice& c, float* slabs) {
  a.split = c.split, a.slabs = slabs, a.out = nullptr;
  return launch_tiling<false, false, kEpiSum>(st, a, c.tiling);
}
// (slab_bytes: of the workspace for shares' sums; whether shares are worth it, the kernel decides by the rows that count.  columns: of the tiles that it took)
template <bool XO, bool YO, int EPI>
int launch_product(hipStream_t st, Product a, float* slabs = nullptr, int64_t slab_bytes = 0, int* columns = nullptr) {
  const Choice c = choice_of(a.nx, a.ny, a.k, a.parts, EPI == kEpiSum, slab_bytes, a.count_k != 0, EPI == kEpiPartial ? tilings_for_sums(a.nx) : 4);
  a.split = c.split, a.slabs = slabs;
  if (columns != nullptr) *columns = kTilings[c.tiling].by;
  return launch_tiling<XO, YO, EPI>(st, a, c.tiling);
}

template <typename T, int P>
int copy_table(hipStream_t st, const HeadCall& c, const Plan& q, int64_t v0, int64_t n, int64_t n_to, char* to) {
  head_copy_kernel<T, P><<<(unsigned)((n_to + 3) / 4), 256, 0, st>>>((const T*)c.W.p + v0 * c.W.ld, c.W.ld, n, n_to, c.p.C, (int)q.Cp, to,
                                                                    q.c_pitch, q.table * q.c_pitch);
  return hip_status();
}
template <typename T, int P>
int gather(hipStream_t st, const Gather& g, const void* h, bool zeros) {
  head_gather_kernel<T, P><<<(unsigned)((g.slots + (zeros ? g.M : 0) + 3) / 4), 256, 0, st>>>(g, (const T*)h);
  return hip_status();
}

// The table's rows from v0 on as an operand: in place, or copied into the workspace.
struct Call {
  const HeadCall& c;
  const Plan& q;
  hipStream_t st;
  char* ws;
  bool copied, few = false;   // few: rows as they are, up to kThinRows

  int prepare(bool backward, Operand& h) const {
    const abl_head& p = c.p;
    int* rows = (int*)(ws + q.rows);
    int* count = (int*)(ws + q.count);
    unsigned char* flags = p.T != 0 ? (unsigned char*)(ws + q.flags) : nullptr;
    if (flags != nullptr) head_flags_kernel<<<(unsigned)((p.M + 3) / 4), 256, 0, st>>>(p.M, c.labels, c.ids, c.logits, p.T, p.V, flags);
    // (the gradient of the logits of few rows, and of operands in fp32, is not rounded to bf16)
    float* unit = (float*)(ws + q.unit);
    UnitOf of{backward && !few && q.parts == 1 ? c.dloss : nullptr, p.scale, p.teacher_weight, p.temperature};
    if (c.labels != nullptr && p.label_weight != 0.0f) of.first = p.label_weight, of.second = 1.0f - p.smoothing;
    head_rows_kernel<<<1, 1024, 0, st>>>(p.M, c.labels, flags, rows, count, of, unit);
    Gather g{};
    g.M = p.M, g.slots = q.Mp, g.C = p.C, g.Cp = (int)q.Cp, g.T = p.T, g.V = p.V, g.rows = rows, g.count = count, g.flags = flags;
    g.labels = c.labels, g.to = ws + q.h, g.pitch = q.c_pitch, g.plane = q.Mp * q.c_pitch, g.ldh = c.h.ld;
    g.loss = c.loss, g.lse = c.lse, g.lse_t = c.lse_t, g.z_top = c.z_top, g.dh = c.dh.p, g.lddh = c.dh.ld;
    g.row_label = !backward && c.labels != nullptr ? (int*)(ws + q.labels) : nullptr;
    g.grad = backward ? (RowGrad*)(ws + q.grad) : nullptr;
    g.in_lse = c.in_lse, g.in_lse_t = c.in_lse_t, g.dloss = c.dloss, g.unit = of.dloss != nullptr ? unit : nullptr;
    g.scale = p.scale, g.smoothing = p.smoothing, g.z_weight = p.z_weight, g.tau = p.temperature, g.label_weight = p.label_weight;
    g.teacher_weight = p.teacher_weight;
    if (int e = hip_status()) return e;
    if (few) {
      g.slots = kThinRows;
      if (p.dtype == ABL_BF16) return gather<bf16_t, 1>(st, g, c.h.p, true);
      g.pitch = q.Cp * 4 + kPad;
      return gather<float, 0>(st, g, c.h.p, true);
    }
    h = {g.to, g.plane, q.c_pitch, (int)q.Mp, (int)q.Cp};
    if (p.dtype == ABL_BF16) return gather<bf16_t, 1>(st, g, c.h.p, true);
    return q.parts == 3 ? gather<float, 3>(st, g, c.h.p, true) : gather<float, 1>(st, g, c.h.p, true);
  }

  int table(int64_t v0, int64_t n, Operand& w) const {
    if (!copied) {
      w = {(const char*)c.W.p + v0 * c.W.ld * 2, 0, c.W.ld * 2, (int)n, c.p.C};
      return ABL_OK;
    }
    char* to = ws + q.W;
    w = {to, q.table * q.c_pitch, q.c_pitch, (int)q.table, (int)q.Cp};
    const int64_t n_to = up(n, 256);
    if (c.p.dtype == ABL_BF16) return copy_table<bf16_t, 1>(st, c, q, v0, n, n_to, to);
    return q.parts == 3 ? copy_table<float, 3>(st, c, q, v0, n, n_to, to) : copy_table<float, 1>(st, c, q, v0, n, n_to, to);
  }
};

}  // namespace

size_t head_layout_bytes(const abl_head& p, bool backward, bool copied) { return plan_of(p, backward, copied).bytes; }
// (whether the table is copied goes by its address and pitch, which are not known here; copied pieces are smaller, but what lies beside them need not be)
size_t head_scratch_bytes(const abl_head& p, bool backward) {
  const size_t in_place = plan_of(p, backward, false).bytes, copied = plan_of(p, backward, true).bytes;
  return in_place > copied ? in_place : copied;
}

namespace {

// Whether the products can read the table where it is: bf16, 16-byte pieces within rows that lie close enough for 31-bit offsets.
bool in_place(const HeadCall& c) {
  return c.p.dtype == ABL_BF16 && c.p.C % 8 == 0 && c.W.ld % 8 == 0 && c.W.ld < 1 << 21 && (reinterpret_cast<uintptr_t>(c.W.p) & 15u) == 0;
}

EntryLogits entry_logits(const HeadCall& c, const Plan& q) {
  return {c.h.p, c.W.p, c.h.ld, c.W.ld, c.p.C, c.p.V, c.p.T, c.p.dtype, c.p.dtype == ABL_F32 && q.parts == 1, c.ids, c.logits, c.p.scale, c.z_top};
}

Loss loss_of(const HeadCall& c, const Plan& q, char* ws) {
  const abl_head& p = c.p;
  Loss l{};
  l.M = (int)p.M, l.partial = (const Partial*)(ws + q.partial), l.partial_ld = q.Mp, l.labels = c.labels, l.ids = c.ids;
  l.logits = c.logits, l.z_label = (const float*)(ws + q.z_label), l.T = p.T, l.V = p.V, l.smoothing = p.smoothing, l.z_weight = p.z_weight;
  l.tau = p.temperature, l.label_weight = p.label_weight, l.teacher_weight = p.teacher_weight, l.loss = c.loss, l.lse = c.lse, l.lse_t = c.lse_t;
  l.z_top = c.z_top;
  return l;
}

// Few rows: two launches.
template <typename T, int XT, int YT, int WAVES, int AHEAD>
int launch_thin(hipStream_t st, const HeadCall& c, const Plan& q, char* ws) {
  const abl_head& p = c.p;
  const int tiles = (p.V + 16 * YT - 1) / (16 * YT);
  Thin a{c.h.p, c.W.p, c.h.ld, c.W.ld, (int)p.M, p.C, p.V, tiles < kThinGroups ? tiles : kThinGroups, c.labels, p.scale, 1.0f / p.temperature,
         (float*)(ws + q.z_label), (Partial*)(ws + q.partial)};
  head_thin_kernel<T, XT, YT, WAVES, AHEAD, false><<<(unsigned)a.groups, WAVES * 64, 0, st>>>(a);
  Loss l = loss_of(c, q, ws);
  l.tiles = a.groups, l.partial_ld = p.M, l.entries = entry_logits(c, q);
  head_loss_kernel<1><<<(unsigned)p.M, 1024, 0, st>>>(l);
  return hip_status();
}
// The same for a table that the products can read where it is, and rows likewise.
bool thin_in_place(const HeadCall& c) {
  return in_place(c) && c.h.ld % 8 == 0 && c.h.ld < 1 << 21 && (reinterpret_cast<uintptr_t>(c.h.p) & 15u) == 0;
}
int launch_thin_product(hipStream_t st, const HeadCall& c, const Plan& q, char* ws) {
  const abl_head& p = c.p;
  Product a{};
  a.x = {(const char*)c.h.p, 0, c.h.ld * 2, (int)p.M, p.C}, a.y = {(const char*)c.W.p, 0, c.W.ld * 2, p.V, p.C};
  a.nx = (int)p.M, a.ny = p.V, a.k = p.C, a.parts = 1, a.pairs = kPairs1, a.scale = p.scale, a.inv_tau = 1.0f / p.temperature;
  a.partial = (Partial*)(ws + q.partial), a.partial_ld = kThinRows, a.sum_z = p.smoothing != 0.0f, a.labels = c.labels, a.z_label = (float*)(ws + q.z_label);
  // Tiles of 64 tokens where those of 128 are two a compute unit or fewer (16 x 2048 x 32768: 37.6 us instead of 39.2; 8 x 1024 x 131072: 57.6 instead of 53.3).
  const bool narrow = (p.V + 127) / 128 <= 2 * kUnits;
  const int columns = narrow ? 64 : 128;
  int e;
  if (p.M <= 32)
    e = narrow ? launch_tiles<32, 64, 1, 4, 4, false, false, kEpiPartial, true>(st, a) : launch_tiles<32, 128, 1, 4, 4, false, false, kEpiPartial, true>(st, a);
  else
    e = narrow ? launch_tiles<64, 64, 1, 4, 4, false, false, kEpiPartial, true>(st, a) : launch_tiles<64, 128, 1, 4, 4, false, false, kEpiPartial, true>(st, a);
  if (e != ABL_OK) return e;
  Loss l = loss_of(c, q, ws);
  l.tiles = (p.V + columns - 1) / columns, l.partial_ld = kThinRows, l.entries = entry_logits(c, q);
  head_loss_kernel<1><<<(unsigned)p.M, 1024, 0, st>>>(l);
  return hip_status();
}
template <typename T>
int launch_thin(hipStream_t st, const HeadCall& c, const Plan& q, char* ws) {
  if (std::is_same_v<T, bf16_t> && thin_in_place(c)) return launch_thin_product(st, c, q, ws);
  if (c.p.M <= 16) return launch_thin<T, 1, 1, 8, 4>(st, c, q, ws);
  if (c.p.M <= 32) return launch_thin<T, 2, 2, 4, 2>(st, c, q, ws);
  return c.p.M <= 48 ? launch_thin<T, 3, 2, 4, 2>(st, c, q, ws) : launch_thin<T, 4, 2, 4, 2>(st, c, q, ws);
}

}  // namespace

int launch_head_forward(hipStream_t st, const HeadCall& c, void* scratch, size_t scratch_bytes) {
  const abl_head& p = c.p;
  if (p.M <= kThinRows && !(p.dtype == ABL_F32 && (p.flags & ABL_MATH_BF16))) {
    const Plan q = plan_of(p, false, false);
    if (q.bytes > scratch_bytes) return ABL_ERR_SCRATCH;
    return p.dtype == ABL_F32 ? launch_thin<float>(st, c, q, (char*)scratch) : launch_thin<bf16_t>(st, c, q, (char*)scratch);
  }
  const bool copied = !in_place(c);
  const Plan q = plan_of(p, false, copied);
  if (q.bytes > scratch_bytes) return ABL_ERR_SCRATCH;
  const Call call{c, q, st, (char*)scratch, copied};
  char* ws = call.ws;
  const int* rows = (const int*)(ws + q.rows);
  const int* count = (const int*)(ws + q.count);
  const unsigned char* flags = p.T != 0 ? (const unsigned char*)(ws + q.flags) : nullptr;
  Product a{};
  if (int e = call.prepare(false, a.x)) return e;
  if (c.ids != nullptr) {
    const EntryLogits e = entry_logits(c, q);
    if (p.dtype == ABL_F32)
      head_entries_kernel<float><<<(unsigned)p.M, 256, 0, st>>>(e, rows, count);
    else
      head_entries_kernel<bf16_t><<<(unsigned)p.M, 256, 0, st>>>(e, rows, count);
  }
  if (int e = hip_status()) return e;
  Partial* carry = (Partial*)(ws + q.carry);
  for (int i = 0; i < q.pieces; ++i) {
    const int64_t v0 = i * q.piece, n = v0 + q.piece < p.V ? q.piece : p.V - v0;
    if (int e = call.table(v0, n, a.y)) return e;
    a.nx = (int)p.M, a.ny = (int)n, a.k = (int)q.Cp, a.count = count, a.count_k = 0;
    a.parts = q.parts == 3 ? 6 : 1, a.pairs = q.parts == 3 ? kPairs6 : kPairs1;
    a.scale = p.scale, a.inv_tau = 1.0f / p.temperature, a.y0 = (int)v0;
    a.partial = (Partial*)(ws + q.partial), a.partial_ld = q.Mp, a.sum_z = p.smoothing != 0.0f;
    a.row_label = c.labels != nullptr ? (const int*)(ws + q.labels) : nullptr, a.z_label = (float*)(ws + q.z_label);
    Choice how;
    int columns;   // of a tile that the loss finds sums of
    if (cut_logits(a, q.slab_bytes, how)) {
      const Tiling& t = kTilings[how.tiling];
      if (int e = launch_slabs(st, a, how, (float*)(ws + q.slabs))) return e;
      head_slab_partial_kernel<<<dim3((unsigned)p.M, (unsigned)((n + kSlabColumns - 1) / kSlabColumns)), 256, 0, st>>>(a, t.bx, t.by);
      columns = kSlabColumns;
    } else if (int e = launch_product<false, false, kEpiPartial>(st, a, nullptr, 0, &columns)) {
      return e;
    }
    Loss l = loss_of(c, q, ws);
    l.tiles = (int)((n + columns - 1) / columns);
    l.before = i > 0 ? carry : nullptr, l.after = i + 1 < q.pieces ? carry : nullptr, l.rows = rows, l.count = count, l.flags = flags;
    head_loss_kernel<16><<<(unsigned)((p.M + 15) / 16), 1024, 0, st>>>(l);
    if (int e = hip_status()) return e;
  }
  return ABL_OK;
}

namespace {

void launch_entry_grad(hipStream_t st, const HeadCall& c, const Plan& q, char* ws, int64_t v0, int64_t n, const Operand& d, int d_parts) {
  const abl_head& p = c.p;
  Entries a{};
  a.rows = (const int*)(ws + q.rows), a.count = (const int*)(ws + q.count), a.ids = c.ids, a.logits = c.logits, a.z_top = c.in_z_top;
  a.grad = (const RowGrad*)(ws + q.grad), a.T = p.T;
  a.v0 = (int)v0, a.v1 = (int)(v0 + n), a.inv_tau = 1.0f / p.temperature, a.d = ws + q.d, a.d_plane = d.plane, a.d_pitch = d.pitch;
  a.d_parts = d_parts;
  head_entry_grad_kernel<<<(unsigned)((p.M + 3) / 4), 256, 0, st>>>(a);
}

// Few rows: the gradient of a piece's logits in fp32, then both products of it.
template <typename T, int XT, int YT, int WAVES, int AHEAD>
int launch_thin_backward(hipStream_t st, const HeadCall& c, char* ws, size_t ws_bytes) {
  const abl_head& p = c.p;
  const Plan q = plan_of(p, true, false);
  if (q.bytes > ws_bytes) return ABL_ERR_SCRATCH;
  const Call call{c, q, st, ws, false, true};
  Operand none;
  if (int e = call.prepare(true, none)) return e;
  const int64_t pitch = sizeof(T) == 4 ? q.Cp * 4 + kPad : q.c_pitch, d_ld = q.piece;
  const int across = (p.C + 63) / 64;
  ThinGrad a{};
  a.h = ws + q.h, a.ldh = pitch / (int64_t)sizeof(T), a.ldw = c.W.ld, a.M = (int)p.M, a.C = p.C, a.d = (const float*)(ws + q.d), a.d_ld = d_ld;
  a.slabs = c.dh.p != nullptr ? (float*)(ws + q.slabs) : nullptr, a.out_f32 = p.dw_dtype == ABL_F32, a.accumulate = (p.flags & ABL_ACCUM_DW) != 0;
  // Shares: as many as make enough waves (of 16 rows 2048 in all: 140 us instead of 121 for 7 x 5632 x 11705 bf16; 8192: 124).
  int64_t shares = kThinWaves / XT / across;   // (of 64 rows one wave fits a SIMD: not one more than there are)
  const int64_t fit = q.slab_bytes / ((int64_t)p.M * p.C * 4), of_tokens = (q.piece + 31) / 32;
  shares = shares < kThinShares ? shares : kThinShares;
  shares = shares < fit ? shares : fit;
  shares = shares < of_tokens ? shares : of_tokens;
  if (shares < 1) shares = 1;
  a.per = (int)up((q.piece + shares - 1) / shares, 16);
  a.shares = (int)((q.piece + a.per - 1) / a.per);
  for (int i = 0; i < q.pieces; ++i) {
    const int64_t v0 = i * q.piece, n = v0 + q.piece < p.V ? q.piece : p.V - v0;
    const int tiles = (int)((n + 16 * YT - 1) / (16 * YT));
    Thin t{};
    t.h = a.h, t.W = (const T*)c.W.p + v0 * c.W.ld, t.ldh = a.ldh, t.ldw = c.W.ld, t.M = 16 * XT, t.C = p.C, t.V = (int)n;
    t.groups = tiles < kThinGroups ? tiles : kThinGroups, t.scale = p.scale, t.inv_tau = 1.0f / p.temperature;
    t.grad = (const RowGrad*)(ws + q.grad), t.d = (float*)(ws + q.d), t.d_ld = d_ld, t.v0 = (int)v0;
    head_thin_kernel<T, XT, YT, WAVES, AHEAD, true><<<(unsigned)t.groups, WAVES * 64, 0, st>>>(t);
    if (c.ids != nullptr) launch_entry_grad(st, c, q, ws, v0, n, Operand{nullptr, 0, d_ld * 4, 0, 0}, 0);
    a.W = t.W, a.n = (int)n, a.more = i > 0, a.dW = c.dW != nullptr ? (char*)c.dW + v0 * p.C * size_of(p.dw_dtype) : nullptr;
    head_thin_grad_kernel<T, XT><<<(unsigned)(((int64_t)a.shares * across + 3) / 4), 256, 0, st>>>(a);
    if (int e = hip_status()) return e;
  }
  if (c.dh.p != nullptr)
    head_thin_sum_kernel<<<dim3((unsigned)p.M, (unsigned)((p.C + 63) / 64)), 256, 0, st>>>(a, (const int*)(ws + q.rows), (const int*)(ws + q.count), c.dh.p, c.dh.ld,
                                                                                      p.dtype == ABL_F32);
  return hip_status();
}
// (fp32 with ABL_MATH_BF16 rounds its operands: not here.)
bool thin_backward(const abl_head& p) { return p.dtype == ABL_F32 ? p.M <= kThinRows && !(p.flags & ABL_MATH_BF16) : p.M <= 16; }

}  // namespace

int launch_head_backward(hipStream_t st, const HeadCall& c, void* scratch, size_t scratch_bytes) {
  const abl_head& p = c.p;
  const bool accumulate = (p.flags & ABL_ACCUM_DW) != 0;
  if (p.M == 0) {
    if (c.dW == nullptr || accumulate) return ABL_OK;
    const int64_t n = (int64_t)p.V * p.C * (size_of(p.dw_dtype) / 2);
    head_zero_kernel<<<(unsigned)(n < 1 << 20 ? (n + 255) / 256 : 4096), 256, 0, st>>>((uint16_t*)c.dW, n);
    return hip_status();
  }
  if (thin_backward(p)) {
    char* ws = (char*)scratch;
    if (p.dtype == ABL_BF16) return launch_thin_backward<bf16_t, 1, 1, 8, 4>(st, c, ws, scratch_bytes);
    if (p.M <= 16) return launch_thin_backward<float, 1, 1, 8, 4>(st, c, ws, scratch_bytes);
    return p.M <= 32 ? launch_thin_backward<float, 2, 2, 4, 2>(st, c, ws, scratch_bytes) : launch_thin_backward<float, 4, 2, 4, 2>(st, c, ws, scratch_bytes);
  }
  const bool copied = !in_place(c);
  const Plan q = plan_of(p, true, copied);
  if (q.bytes > scratch_bytes) return ABL_ERR_SCRATCH;
  const Call call{c, q, st, (char*)scratch, copied};
  char* ws = call.ws;
  const int* rows = (const int*)(ws + q.rows);
  const int* count = (const int*)(ws + q.count);
  const float* unit = q.parts == 1 ? (const float*)(ws + q.unit) : nullptr;
  Operand h, w;
  if (int e = call.prepare(true, h)) return e;
  for (int i = 0; i < q.pieces; ++i) {
    const int64_t v0 = i * q.piece, n = v0 + q.piece < p.V ? q.piece : p.V - v0;
    if (int e = call.table(v0, n, w)) return e;
    const Operand d{ws + q.d, q.Mp * q.d_pitch, q.d_pitch, (int)q.Mp, (int)q.piece};
    {
      Product a{};
      a.x = h, a.y = w, a.nx = (int)p.M, a.ny = (int)n, a.k = (int)q.Cp, a.count = count;
      a.parts = q.parts == 3 ? 6 : 1, a.pairs = q.parts == 3 ? kPairs6 : kPairs1;
      a.scale = p.scale, a.inv_tau = 1.0f / p.temperature, a.y0 = (int)v0, a.grad = (const RowGrad*)(ws + q.grad);
      a.d = ws + q.d, a.d_plane = d.plane, a.d_pitch = d.pitch, a.d_parts = q.d_parts;
      Choice how;
      if (cut_logits(a, q.slab_bytes, how)) {
        const Tiling& t = kTilings[how.tiling];
        if (int e = launch_slabs(st, a, how, (float*)(ws + q.slabs))) return e;
        head_slab_grad_kernel<<<dim3((unsigned)q.Mp, (unsigned)((n + 63 + kSlabColumns - 1) / kSlabColumns)), 256, 0, st>>>(a, t.bx, t.by);
        if (int e = hip_status()) return e;
      } else if (int e = launch_product<false, false, kEpiGrad>(st, a)) {
        return e;
      }
    }
    if (c.ids != nullptr) {
      launch_entry_grad(st, c, q, ws, v0, n, d, q.d_parts);
      if (int e = hip_status()) return e;
    }
    if (c.dh.p != nullptr) {
      Product a{};
      const bool last = i + 1 == q.pieces;
      float* acc = (float*)(ws + q.acc);
      a.x = d, a.y = w, a.nx = (int)p.M, a.ny = p.C, a.k = (int)up(n, 64), a.count = count;
      a.parts = q.parts == 3 ? 6 : 1, a.pairs = q.parts == 3 ? kPairs6 : kPairs1;
      a.out = last ? c.dh.p : acc, a.ld = last ? c.dh.ld : p.C, a.out_f32 = !last || p.dtype == ABL_F32, a.map = last ? rows : nullptr;
      a.unit = last ? unit : nullptr;
      a.add = i > 0 ? acc : nullptr, a.add_ld = p.C;
      if (int e = launch_product<false, true, kEpiSum>(st, a, (float*)(ws + q.slabs), q.slab_bytes)) return e;
    }
    if (c.dW != nullptr) {
      Product a{};
      a.x = d, a.y = h, a.nx = (int)n, a.ny = p.C, a.k = (int)p.M, a.count = count, a.count_k = 1;
      a.parts = q.parts == 3 ? 6 : q.d_parts, a.pairs = q.parts == 3 ? kPairs6 : q.d_parts == 3 ? kPairs3 : kPairs1;
      a.out = (char*)c.dW + v0 * p.C * size_of(p.dw_dtype), a.ld = p.C, a.out_f32 = p.dw_dtype == ABL_F32, a.accumulate = accumulate;
      a.unit = unit;
      if (int e = launch_product<true, true, kEpiSum>(st, a, (float*)(ws + q.slabs), q.slab_bytes)) return e;
    }
  }
  return ABL_OK;
}

}  // namespace abl
