// Weight gradient of a product from the block store of its input (abl_ckpt_wgrad): dW [Cin][Cout] = (scale * x~)^T dy, a contraction
// over the M rows.
//
// Bound by the matrix cores and the card's power: 8192 x 4096 x 8192 (rows, Cin, Cout) in bf16 takes 415 to 430 us at best and 450 to
// 465 in the mean of many, by the card (1330 and 1200 TFLOP/s).  The matrix cores are busy in 62 % of the cycles, at 1.75 GHz; a loop of these instructions
// reaches 2420 TFLOP/s on zeros and 2050 on normal data.  Without decoding it would take 374, without loads 368, without staging
// 294, with a quarter of the matrix instructions 292: the two halves of a step overlap, not perfectly.  dy straight from memory to
// LDS, past the registers, measured the same.  4096 x 4096 x 4096: 114 us (1210 TFLOP/s); fp32 at 8192 x 1024 x 4096, three
// products: 178 us.
//
// A stored value is a code of at most eight bits times a power of two, so it is exact in bf16: the codes become the bf16 operand of the
// matrix cores while a tile is staged and nothing is rounded.  dy in bf16 goes in as it is, dy in fp32 as
// three bf16 parts of eight bits each (three products), or rounded to one.
//
// Both operands lie with the contraction index outermost.  They are staged that way, [m][channels] in bf16, and the fragments are
// read with ds_read_b64_tr_b16: 16 lanes fetch four rows' 16 channels and receive one channel's four rows each.  The order of the
// rows within a step of 32 is 4 (lane / 16) + 0..3 and 16 more, for both operands alike.  In a staged row the even 16-byte pieces
// come first and then the odd ones, the c-th of each at place c xor row % 8, the odd ones moved by four places more (and by half
// of the even ones' range): half a wave's read, 16 pieces of eight rows, takes all 64 banks once, and eight lanes' writes, of
// neighbouring pieces or of every other one, 128 different bytes modulo 128 (both counted: no conflicts; with 32-byte chunks at c
// xor row % 8 an eighth of the LDS cycles were conflicts).

#include "block_store.h"

namespace abl {
namespace {

struct WgArgs {
  const unsigned char *codes, *scales;
  const void* dy;
  const void* scale;   // of dW's rows, with the dtype of dy (nullptr: ones)
  float* out;          // dW, or the copies of the shares
  int64_t ldy;
  int64_t M, rows;     // rows of a share
  int64_t copy;        // elements from one share's copy to the next
  int Cin, Cout, blocks;   // blocks: of a stored row
  int tiles_i, tiles_j;
  int accum;
};

template <typename T>
__device__ inline float row_scale(const void* s, int i) {
  return s == nullptr ? 1.0f : (float)((const T*)s)[i];
}

// Byte of piece q of row r in a staged tile whose rows have `pitch` bytes (256 or 512), and of the eight bytes that a lane of a
// fragment's read asks for (chunk c of 16 channels, rows from r on).
__device__ inline int staged_at(int r, int q, int pitch) {
  return r * pitch + (q & 1) * (pitch / 2) + (((q >> 1) ^ (r & 7) ^ ((q & 1) * (pitch / 32 - 4))) * 16);
}
__device__ inline int fragment_at(int r, int c, int lane, int pitch) { return staged_at(r, 2 * c + ((lane >> 1) & 1), pitch) + (lane & 1) * 8; }

template <int K>
__device__ inline float stored_value(const WgArgs& a, int64_t row, int c) {
  const int64_t block = row * a.blocks + c / 32;
  const float s = scale_of(a.scales[block]);
  if constexpr (K == 8) {
    return (float)(int8_t)a.codes[block * 32 + c % 32] * s;
  } else {
    float v[8];
    decode<4>(Codes<4>{(uint32_t)(a.codes[block * 16 + c % 32 / 2] >> (4 * (c & 1))) & 15u}, a.scales[block], v);
    return v[0];
  }
}

// fp32 as three bf16 parts whose sum it is: the upper 16 bits of what is left, twice (nothing is rounded); a value that is not
// finite is its first part.
__device__ inline void parts_of(const float (&v)[8], u32x4 (&part)[3]) {
  uint32_t h[8], m[8], l[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t b = __float_as_uint(v[e]);
    const bool fine = finite(v[e]), nan = (b & 0x7FFFFFFFu) > 0x7F800000u;
    h[e] = nan ? 0x7FC00000u : b & 0xFFFF0000u;
    const float r = fine ? v[e] - __uint_as_float(h[e]) : 0.0f;
    m[e] = __float_as_uint(r);
    l[e] = __float_as_uint(r - __uint_as_float(m[e] & 0xFFFF0000u));
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {   // the upper halves of two words
    part[0][e] = __builtin_amdgcn_perm(h[2 * e + 1], h[2 * e], 0x07060302u);
    part[1][e] = __builtin_amdgcn_perm(m[2 * e + 1], m[2 * e], 0x07060302u);
    part[2][e] = __builtin_amdgcn_perm(l[2 * e + 1], l[2 * e], 0x07060302u);
  }
}

// ---- rows far apart ----
// The plain form of the kernel below, with 64-bit addresses: for a dy whose rows lie so far apart that a step of 32 of them does not fit a buffer
// descriptor.  NP: bf16 parts of an element of dy.
template <typename T, int K, int NP>
__global__ __launch_bounds__(256) void store_wgrad_far_kernel(WgArgs a) {
  constexpr int BI = 128, BJ = 128, WI = 2, WJ = 2, BK = 32, kThreads = WI * WJ * 64;
  constexpr int FI = BI / WI / 16, FJ = BJ / WJ / 16;   // 16 x 16 tiles of a wave
  constexpr int PX = BK * BI / 8 / kThreads, PY = BK * BJ / 8 / kThreads;   // pieces of a thread
  constexpr int kXBytes = BK * BI * 2, kYBytes = BK * BJ * 2, kStage = kXBytes + NP * kYBytes;
  __shared__ __align__(16) char lds[2 * kStage];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int tile = blockIdx.x % (a.tiles_i * a.tiles_j), share = blockIdx.x / (a.tiles_i * a.tiles_j);
  const int i0 = tile / a.tiles_j * BI, j0 = tile % a.tiles_j * BJ;
  const int64_t m0 = share * a.rows, m1 = m0 + a.rows < a.M ? m0 + a.rows : a.M;

  Codes<K> cx[PX];
  uint32_t sx[PX];
  Raw<T> ry[PY];
  auto fetch = [&](int64_t m) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < PX; ++p) {
      const int at = p * kThreads + tid, r = at / (BI / 8), q = at % (BI / 8);
      const int64_t row = m + r;
      const int block = i0 / 32 + q / 4;
      if (row < m1 && block < a.blocks) {
        const int64_t n = row * a.blocks + block;
        cx[p] = load_codes<K>(a.codes, n * 4 + (q & 3));
        sx[p] = a.scales[n];
      } else {
        cx[p] = Codes<K>{};
        sx[p] = 127;
      }
    }
#pragma unroll
    for (int p = 0; p < PY; ++p) {
      const int at = p * kThreads + tid, r = at / (BJ / 8), q = at % (BJ / 8);
      const int64_t row = m + r;
      const int c = j0 + q * 8;
      ry[p] = load_raw((const T*)a.dy + row * a.ldy + c, row < m1 ? a.Cout - c : 0);
    }
  };
  auto stage = [&](char* to) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < PX; ++p) {
      const int at = p * kThreads + tid, r = at / (BI / 8), q = at % (BI / 8);
      float v[8];
      decode<K>(cx[p], sx[p], v);
      put(to + staged_at(r, q, BI * 2), to_bf16x8(v));
    }
#pragma unroll
    for (int p = 0; p < PY; ++p) {
      const int at = p * kThreads + tid, r = at / (BJ / 8), q = at % (BJ / 8);
      char* y = to + kXBytes + staged_at(r, q, BJ * 2);
      if constexpr (std::is_same_v<T, bf16_t>) {
        put(y, __builtin_bit_cast(bf16x8_t, ry[p]));
      } else {
        float v[8];
        expand(ry[p], v);
        if constexpr (NP == 1) {
          put(y, to_bf16x8(v));
        } else {
          u32x4 part[3];
          parts_of(v, part);
#pragma unroll
          for (int n = 0; n < 3; ++n) *reinterpret_cast<u32x4*>(y + n * kYBytes) = part[n];
        }
      }
    }
  };

  floatx4 acc[FI][FJ];
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < FJ; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};

  const int wi = wave / WJ * (FI * 16), wj = wave % WJ * (FJ * 16);
  const int r = (lane >> 4) * 4 + ((lane & 15) >> 2);   // row of this lane's first address; 16 more for the second
  auto fragment = [&](const char* plane, int pitch, int c) __attribute__((always_inline)) {
    const char* p = plane + fragment_at(r, c >> 4, lane, pitch);
    return transposed(p, p + 16 * pitch);
  };

  fetch(m0);
  stage(lds);
  __syncthreads();
  int turn = 0;
  for (int64_t m = m0; m < m1; m += BK) {
    const bool more = m + BK < m1;
    if (more) fetch(m + BK);
    const char* now = lds + turn * kStage;
    bf16x8_t x[FI];
#pragma unroll
    for (int i = 0; i < FI; ++i) x[i] = fragment(now, BI * 2, wi + 16 * i);
#pragma unroll
    for (int n = 0; n < NP; ++n)
#pragma unroll
      for (int j = 0; j < FJ; ++j) {
        const bf16x8_t y = fragment(now + kXBytes + n * kYBytes, BJ * 2, wj + 16 * j);
#pragma unroll
        for (int i = 0; i < FI; ++i) acc[i][j] = mfma32(y, x[i], acc[i][j]);
      }
    if (more) stage(lds + (turn ^ 1) * kStage);
    __syncthreads();
    turn ^= 1;
  }

  // lane: channel lane % 16 of x, channels 4 (lane / 16) + 0..3 of dy
  const bool whole = a.copy == 0;
  float* out = a.out + share * a.copy;
#pragma unroll
  for (int i = 0; i < FI; ++i) {
    const int ci = i0 + wi + 16 * i + (lane & 15);
    if (ci >= a.Cin) continue;
    const float s = whole ? row_scale<T>(a.scale, ci) : 1.0f;
#pragma unroll
    for (int j = 0; j < FJ; ++j) {
      const int cj = j0 + wj + 16 * j + (lane >> 4) * 4;
      float* to = out + (int64_t)ci * a.Cout + cj;
      floatx4 v = acc[i][j];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (cj + e >= a.Cout) continue;
        v[e] *= s;
        to[e] = whole && a.accum ? to[e] + v[e] : v[e];
      }
    }
  }
}

// ---- the product ----
// A block of eight waves has a tile of BI channels of x and BJ of dy, a wave an eighth of it.  Waves w and w + 4 share a SIMD and take turns:
// while one issues the matrix instructions of a step of 32 rows, the other reads its next fragments from LDS and writes its share of the next
// tile there; a barrier changes the roles, and waves 4 to 7 are one barrier behind.  A wave issues an instruction about every four cycles, so what
// needs registers only - codes to bf16, the loads of later tiles - goes between its matrix instructions, which leave three such places each.
//   phase 2 s      waves 0-3 read step s and write their share of tile s + 1       waves 4-7 multiply step s - 1
//   phase 2 s + 1  waves 0-3 multiply step s                                       waves 4-7 read step s, write tile s + 1
// Two tiles in LDS are enough: tile s + 1 replaces tile s - 1, which waves 4-7 read in phase 2 s - 1.
// Blocks that a compute unit holds (ragged tiles of three parts lack a few registers; with them spilled they take 1 us more).
template <int BI, int NP, bool RAGGED>
constexpr int kPerUnit = BI > 128 || (NP == 3 && RAGGED) ? 1 : 2;
template <typename T, int K, int NP, int BI, int BJ, bool RAGGED>
__global__ __launch_bounds__(512, (kPerUnit<BI, NP, RAGGED> * 2)) void store_wgrad_kernel(WgArgs a) {
  constexpr int BK = 32, WI = NP == 3 ? 2 : 4, WJ = 8 / WI;   // (three parts: fewer columns of dy a wave)
  constexpr int FI = BI / WI / 16, FJ = BJ / WJ / 16;
  constexpr int XP = BI / 128;                       // pieces of x of a thread
  constexpr int PY = BK * BJ / 8 / 512;              // pieces of dy of a thread
  constexpr int kXBytes = BK * BI * 2, kYBytes = BK * BJ * 2, kStage = kXBytes + NP * kYBytes;
  extern __shared__ __align__(16) char lds[];        // [2][kStage]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool late = wave >= 4;

  // Blocks 8 apart share an XCD and its L2.  Each XCD takes consecutive items, in the order of columns of four tiles of x: what runs there at one
  // time shares four tiles of x and a few of dy.
  const int tiles = a.tiles_i * a.tiles_j, items = gridDim.x;
  const int xcd = blockIdx.x & 7, slot = blockIdx.x >> 3, per = items >> 3, more = items & 7;
  const int item = xcd * per + (xcd < more ? xcd : more) + slot;
  const int share = item / tiles, tile = item - share * tiles;
  const int band = tile / (4 * a.tiles_j), rest = tile - band * 4 * a.tiles_j;
  const int high = a.tiles_i - band * 4 < 4 ? a.tiles_i - band * 4 : 4;
  const int i0 = (band * 4 + rest % high) * BI, j0 = rest / high * BJ;
  const int64_t m0 = share * a.rows, m1 = m0 + a.rows < a.M ? m0 + a.rows : a.M;
  const int steps = (int)((m1 - m0 + BK - 1) / BK);

  // This thread's share of a tile: XP pieces of x next to each other in a row, PY pieces of dy.  Loads go through descriptors of the share's rows; rows beyond them
  // and channels that do not exist read zero.
  const int xr = tid >> 4, xq = (tid & 15) * XP;
  const int block = i0 / 32 + (xq >> 2);
  const int rows = (int)(m1 - m0);
  const auto codes = descriptor(a.codes + m0 * a.blocks * 4 * K, (int64_t)rows * a.blocks * 4 * K);
  const auto scales = descriptor(a.scales + m0 * a.blocks, (int64_t)rows * a.blocks);
  // (RAGGED, where another share follows: a piece may reach beyond the channels, which adds to columns that are not written)
  const bool ends = m1 == a.M;
  const int64_t last = rows == 0 ? 0 : ends ? (rows - 1) * a.ldy + a.Cout : rows * a.ldy + (RAGGED ? 8 : 0);
  const auto dy = descriptor((const T*)a.dy + m0 * a.ldy, last * (int64_t)sizeof(T));
  // Steps beyond the last one are asked for too.  An access is out of range, and reads zero, where its own offset is not below the descriptor's
  // bytes less the scalar offset, so that one stays within the bytes.
  const uint32_t c_end = (uint32_t)rows * (uint32_t)a.blocks * (4u * K), s_end = (uint32_t)rows * (uint32_t)a.blocks, y_end = (uint32_t)(last * (int64_t)sizeof(T));
  auto within = [](uint32_t at, uint32_t end) __attribute__((always_inline)) { return at < end ? at : end; };
  const uint32_t s_at = block < a.blocks ? (uint32_t)xr * (uint32_t)a.blocks + (uint32_t)block : kNowhere;
  const uint32_t c_at = block < a.blocks ? s_at * (4u * K) + (uint32_t)(xq & 3) * K : kNowhere;
  uint32_t y_at[PY];
  int y_row[PY];   // RAGGED: its row in a tile, one more for a piece that is not whole: that of the last row is left out here and added at the end
#pragma unroll
  for (int p = 0; p < PY; ++p) {
    const int c = j0 + (p * 512 + tid) % (BJ / 8) * 8;
    y_row[p] = (p * 512 + tid) / (BJ / 8);
    y_at[p] = c < a.Cout ? ((uint32_t)y_row[p] * (uint32_t)a.ldy + (uint32_t)c) * (uint32_t)sizeof(T) : kNowhere;
    if (RAGGED && ends && c < a.Cout && c + 8 > a.Cout) ++y_row[p];
  }
  const uint32_t c_step = (uint32_t)a.blocks * (4u * K * BK), s_step = (uint32_t)a.blocks * BK, y_step = (uint32_t)a.ldy * (uint32_t)(sizeof(T) * BK);

  struct XCodes {
    Codes<K> c[XP];
    uint32_t s;
  };
  struct YPieces {
    Raw<T> r[PY];
  };
  auto fetch_x = [&](int step, XCodes& t) __attribute__((always_inline)) {
    const uint32_t at = within((uint32_t)step * c_step, c_end);
    if constexpr (K * XP == 16) {
      const u32x4 w = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(codes, c_at, at, 0));
      t.c[0].w = u32x2{w[0], w[1]}, t.c[1].w = u32x2{w[2], w[3]};
    } else if constexpr (K * XP == 8) {
      const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(codes, c_at, at, 0));
      if constexpr (K == 8)
        t.c[0].w = w;
      else
        t.c[0].w = w[0], t.c[1].w = w[1];
    } else {
      t.c[0].w = __builtin_amdgcn_raw_buffer_load_b32(codes, c_at, at, 0);
    }
    t.s = __builtin_amdgcn_raw_buffer_load_b8(scales, s_at, within((uint32_t)step * s_step, s_end), 0);
  };
  auto fetch_y = [&](int step, YPieces& t) __attribute__((always_inline)) {
    const uint32_t at = within((uint32_t)step * y_step, y_end);
    const int left = rows - step * BK;
#pragma unroll
    for (int p = 0; p < PY; ++p) {
      uint32_t of = y_at[p];
      if constexpr (RAGGED) of = y_row[p] < left ? of : kNowhere;
      if constexpr (std::is_same_v<T, float>) {
        t.r[p].a = __builtin_bit_cast(f32x4_any4, __builtin_amdgcn_raw_buffer_load_b128(dy, of, at, 0));
        t.r[p].b = __builtin_bit_cast(f32x4_any4, __builtin_amdgcn_raw_buffer_load_b128(dy, of + 16, at, 0));
      } else {
        t.r[p].a = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(dy, of, at, 0));
      }
    }
  };
  u32x4 xw[XP];   // of the next tile, in bf16
  auto decode_x = [&](const XCodes& t) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < XP; ++p) {
      if constexpr (K == 4) {   // (the conversion makes pairs of bf16 with the scale applied)
        const float scale = scale_of(t.s);
        auto two = [&](auto b) {
          xw[p][b.value] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(t.c[p].w, scale, b.value));
        };
        two(std::integral_constant<int, 0>{}), two(std::integral_constant<int, 1>{});
        two(std::integral_constant<int, 2>{}), two(std::integral_constant<int, 3>{});
#pragma unroll
        for (int e = 0; e < 4; ++e) xw[p][e] = t.s == 255u ? 0x7FC07FC0u : xw[p][e];
      } else {
        float v[8];
        decode<K>(t.c[p], t.s, v);
#pragma unroll   // (the upper halves: nothing is below them)
        for (int e = 0; e < 4; ++e) xw[p][e] = __builtin_amdgcn_perm(__float_as_uint(v[2 * e + 1]), __float_as_uint(v[2 * e]), 0x07060302u);
      }
    }
  };
  constexpr bool kSplit = NP == 3;   // dy's parts, too, are made between the matrix instructions
  u32x4 yw[PY][NP];
  auto split_y = [&](const YPieces& t) __attribute__((always_inline)) {
    if constexpr (kSplit) {
#pragma unroll
      for (int p = 0; p < PY; ++p) {
        float v[8];
        expand(t.r[p], v);
        parts_of(v, yw[p]);
      }
    }
  };
  auto stage = [&](const YPieces& t, char* to) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < XP; ++p) *reinterpret_cast<u32x4*>(to + staged_at(xr, xq + p, BI * 2)) = xw[p];
#pragma unroll
    for (int p = 0; p < PY; ++p) {
      const int at = p * 512 + tid, r = at / (BJ / 8), q = at % (BJ / 8);
      char* y = to + kXBytes + staged_at(r, q, BJ * 2);
      if constexpr (kSplit) {
#pragma unroll
        for (int n = 0; n < NP; ++n) *reinterpret_cast<u32x4*>(y + n * kYBytes) = yw[p][n];
      } else if constexpr (std::is_same_v<T, bf16_t>) {
        *reinterpret_cast<u32x4*>(y) = t.r[p].a;
      } else {
        float v[8];
        expand(t.r[p], v);
        put(y, to_bf16x8(v));
      }
    }
  };

  floatx4 acc[FI][FJ];
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < FJ; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  const int wi = wave / WJ * (FI * 16), wj = wave % WJ * (FJ * 16);
  const int fr = (lane >> 4) * 4 + ((lane & 15) >> 2);
  auto fragment = [&](const char* plane, int pitch, int c) __attribute__((always_inline)) {
    const char* p = plane + fragment_at(fr, c >> 4, lane, pitch);
    return transposed(p, p + 16 * pitch);
  };
  auto phase_end = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    __builtin_amdgcn_sched_barrier(0);
  };

  // tile t waits in registers of set t % 2
  XCodes xs[2];
  YPieces ys[2];
  fetch_x(0, xs[0]);
  fetch_x(1, xs[1]);
  fetch_y(0, ys[0]);
  fetch_y(1, ys[1]);
  decode_x(xs[0]);
  split_y(ys[0]);
  stage(ys[0], lds);
  fetch_x(2, xs[0]);
  fetch_y(2, ys[0]);
  decode_x(xs[1]);
  fetch_x(3, xs[1]);
  if constexpr (kSplit) {
    split_y(ys[1]);
    fetch_y(3, ys[1]);
  }
  phase_end();
  if (late) phase_end();
  bf16x8_t x[FI], y[NP][FJ];
  auto step = [&](int s, XCodes& xset, YPieces& ynow, YPieces& ynext, char* now, char* then) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < FI; ++i) x[i] = fragment(now, BI * 2, wi + 16 * i);
#pragma unroll
    for (int n = 0; n < NP; ++n)
#pragma unroll
      for (int j = 0; j < FJ; ++j) y[n][j] = fragment(now + kXBytes + n * kYBytes, BJ * 2, wj + 16 * j);
    stage(ynext, then);                      // tile s + 1
    phase_end();
    decode_x(xset);                          // tile s + 2
    fetch_x(s + 4, xset);
    if constexpr (kSplit) {
      split_y(ynow);                         // tile s + 2
      fetch_y(s + 4, ynow);
    } else {
      fetch_y(s + 3, ynext);
    }
#pragma unroll
    for (int n = 0; n < NP; ++n)
#pragma unroll
      for (int j = 0; j < FJ; ++j)
#pragma unroll
        for (int i = 0; i < FI; ++i) acc[i][j] = mfma32(y[n][j], x[i], acc[i][j]);
#pragma unroll
    for (int k = 0; k < NP * FI * FJ; ++k) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);   // a matrix instruction
      __builtin_amdgcn_sched_group_barrier(0x002, kSplit ? 3 : 2, 0);   // two or three vector ones
      __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);   // a load
    }
    phase_end();
  };
  for (int s = 0; s < steps; s += 2) {
    step(s, xs[0], ys[0], ys[1], lds, lds + kStage);
    step(s + 1, xs[1], ys[1], ys[0], lds + kStage, lds);   // (beyond the last step of an odd number: of zeros)
  }
  if (!late) phase_end();

  const bool whole = a.copy == 0;
  float* out = a.out + share * a.copy;
  // The piece of the last row that was left out: its loads on their way together, from places that exist.
  float last_x[FI] = {}, last_y[FJ][4] = {};
  if constexpr (RAGGED) {
    const int part = a.Cout / 8 * 8;   // its first column
    if (ends && a.M > 0 && j0 + BJ > part && j0 < a.Cout) {
      const T* row = (const T*)a.dy + (a.M - 1) * a.ldy;
#pragma unroll
      for (int i = 0; i < FI; ++i) {
        const int ci = i0 + wi + 16 * i + (lane & 15);
        last_x[i] = stored_value<K>(a, a.M - 1, ci < a.Cin ? ci : a.Cin - 1);
      }
#pragma unroll
      for (int j = 0; j < FJ; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int cj = j0 + wj + 16 * j + (lane >> 4) * 4 + e;
          const float yv = (float)row[cj < a.Cout ? cj : a.Cout - 1];
          last_y[j][e] = NP == 1 ? (float)(__bf16)yv : yv;
        }
    }
  }
#pragma unroll
  for (int i = 0; i < FI; ++i) {
    const int ci = i0 + wi + 16 * i + (lane & 15);
    if (ci >= a.Cin) continue;
    const float s = whole ? row_scale<T>(a.scale, ci) : 1.0f;
#pragma unroll
    for (int j = 0; j < FJ; ++j) {
      const int cj = j0 + wj + 16 * j + (lane >> 4) * 4;
      float* to = out + (int64_t)ci * a.Cout + cj;
      f32x4_any4 v = acc[i][j];
      if (RAGGED && cj >= a.Cout / 8 * 8) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(last_x[i], last_y[j][e], v[e]);
      }
      v *= s;
      if (cj + 4 <= a.Cout) {
        if (whole && a.accum) v += *reinterpret_cast<const f32x4_any4*>(to);
        *reinterpret_cast<f32x4_any4*>(to) = v;
      } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
          if (cj + e < a.Cout) to[e] = whole && a.accum ? to[e] + v[e] : v[e];
      }
    }
  }
}

// The shares' copies, added in turn: four neighbouring elements a thread, the copies' loads on their way together.
template <typename T>
__global__ __launch_bounds__(256) void wgrad_sum_kernel(const float* copies, int n, int64_t size, const void* scale, Divisor by_cout, int accum,
                                                        float* dW) {
  const int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (e >= size) return;
  const bool whole = e + 4 <= size;
  f32x4_any4 s{};
  for (int i = 0; i < n; i += 8) {
    f32x4_any4 v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float* from = copies + (int64_t)(i + k) * size + e;
      v[k] = f32x4_any4{};
      if (i + k < n) {
        if (whole) {
          v[k] = *reinterpret_cast<const f32x4_any4*>(from);
        } else {
#pragma unroll
          for (int j = 0; j < 3; ++j)
            if (e + j < size) v[k][j] = from[j];
        }
      }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) s += v[k];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (e + j >= size) continue;
    const float v = s[j] * row_scale<T>(scale, by_cout.of((int)(e + j)));
    s[j] = accum ? dW[e + j] + v : v;
  }
  if (whole) {
    *reinterpret_cast<f32x4_any4*>(dW + e) = s;
  } else {
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (e + j < size) dW[e + j] = s[j];
  }
}

// How a product is cut: tiles of bi x bj channels, and the rows into shares whose sums go to copies of dW that a second launch adds.
struct Plan {
  int bi = 128, bj = 128, tiles_i = 0, tiles_j = 0, shares = 1;
  int64_t rows = 0;
};

// The choice with the least time by these estimates, in us, fitted to 20 products of either type (128 to 16384 rows, 256 to 4096 channels, K = 8),
// each timed with both tilings and 1 to 64 shares.  On these and 12 others the choices are within 9 % of the fastest, most within 3 %.
// A step of 32 rows: `one` with a block on a compute unit and `load` more where all units have one, `two` with two blocks on a unit.
// `second`, `eight`: the launch that adds the shares' copies, and more for each eight; `bytes_per_us`: of the copies, written and read.
struct Cost {
  double one, load, two, start, second, eight, bytes_per_us;
};
constexpr Cost kCost[2][2] = {   // dy in one part: tiles of 128 x 128, 256 x 256; in three: 128 x 128, 256 x 128
    {{0.28, 0.068, 0.579, 5.8, 3.3, 0.38, 8.5e6}, {0.542, 0.127, 0.0, 11.4, 3.3, 0.38, 8.5e6}},
    {{0.551, 0.19, 1.23, 7.7, 3.4, 0.73, 11.3e6}, {0.837, 0.246, 0.0, 9.1, 3.4, 0.73, 11.3e6}}};
constexpr int kShares[] = {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 16, 24, 32, 48, 64};
constexpr int64_t kUnits = 256, kFewestRows = 192;   // of a share, if there are several
// most: shares at most.
Plan plan_of(int64_t M, int Cin, int Cout, bool parts, int64_t most) {
  Plan best;
  best.tiles_i = (Cin + 127) / 128, best.tiles_j = (Cout + 127) / 128, best.rows = M;
  double time = 1e30;
  for (int large = 0; large < 2; ++large) {
    const Cost& c = kCost[parts][large];
    const int bi = large ? 256 : 128, bj = large && !parts ? 256 : 128;
    const int64_t ti = (Cin + bi - 1) / bi, tj = (Cout + bj - 1) / bj, tiles = ti * tj;
    const int64_t held = large || (parts && Cout % 8 != 0) ? kUnits : 2 * kUnits;    // blocks
    for (int n : kShares) {
      if (n > 1 && n * kFewestRows > M) break;
      const int64_t rows = ((M + n - 1) / n + 63) / 64 * 64;
      const int64_t shares = M > 0 ? (M + rows - 1) / rows : 1, items = tiles * shares;
      if (shares > most || (n > 1 && shares * Cin * Cout > (int64_t)24 << 20)) break;   // (96 MB of copies)
      const double steps = (double)(rows < M ? rows : M) / 32;
      const int64_t rounds = items / held, rest = items % held;
      double t = (double)rounds * (steps * (held == kUnits ? c.one + c.load : c.two) + c.start);
      if (rest > 0) t += steps * (rest <= kUnits ? c.one + c.load * (double)rest / kUnits : c.two) + c.start;
      if (shares > 1) t += c.second + c.eight * (double)((shares + 7) / 8) + (double)(shares * Cin * Cout * 8) / c.bytes_per_us;
      if (t < time) {
        time = t;
        best.bi = bi, best.bj = bj, best.tiles_i = (int)ti, best.tiles_j = (int)tj, best.shares = (int)shares, best.rows = rows;
      }
    }
  }
  return best;
}

// How M rows are cut into products, one after the other, of which all but the first add to dW: into as few as there can be (a power of two, up to
// the last) for the offsets of a share, some steps beyond its end included, to fit 31 bits.  Where not even kFewest rows fit, and for fewer
// than eight channels, whose pieces would reach beyond the tensor's end, the far kernel takes all rows.  8192 rows 2 MB apart, 4096 x 4096:
// products 510 us, far kernel 700.
struct Cut {
  Plan plan;
  int64_t rows;   // of a product
  bool far;
};
constexpr int64_t kFewest = 256;
bool offsets_fit(const Plan& p, int64_t row_bytes, int Cin) {
  const int64_t x_bytes = store_blocks(Cin) * 32, wide = row_bytes > x_bytes ? row_bytes : x_bytes;
  return (p.rows + 256) * wide < (int64_t)0x7FFFFF00;
}
Cut cut_of(int64_t M, int64_t row_bytes, int Cin, int Cout, bool parts, int64_t most) {
  Cut c{plan_of(M, Cin, Cout, parts, most), M, Cout < 8};
  if (c.far || offsets_fit(c.plan, row_bytes, Cin)) return c;
  for (int64_t n = 2; c.rows > kFewest; n *= 2) {
    c.rows = ((M + n - 1) / n + 63) / 64 * 64;
    c.plan = plan_of(c.rows, Cin, Cout, parts, most);
    if (offsets_fit(c.plan, row_bytes, Cin)) return c;
  }
  return Cut{plan_of(M, Cin, Cout, parts, most), M, true};
}

template <typename T, int NP, int BI, int BJ>
int launch_tiles(hipStream_t st, int K, bool ragged, unsigned grid, const WgArgs& a) {
  auto kern = K == 8 ? (ragged ? store_wgrad_kernel<T, 8, NP, BI, BJ, true> : store_wgrad_kernel<T, 8, NP, BI, BJ, false>)
                     : (ragged ? store_wgrad_kernel<T, 4, NP, BI, BJ, true> : store_wgrad_kernel<T, 4, NP, BI, BJ, false>);
  constexpr int kBytes = 2 * 32 * 2 * (BI + NP * BJ);
  if (kBytes > 64 * 1024)
    if (int e = allow_full_lds((const void*)kern)) return e;
  kern<<<grid, 512, kBytes, st>>>(a);
  return hip_status();
}

}  // namespace

// (For either way of fp32 and any distance of dy's rows: rows that are farther apart take no more shares.)
size_t store_wgrad_scratch_bytes(int64_t M, int Cin, int Cout, int dtype) {
  size_t most = 16;
  for (int parts = 0; parts < (dtype == ABL_F32 ? 2 : 1); ++parts) {
    const int shares = cut_of(M, (int64_t)Cout * size_of(dtype), Cin, Cout, parts != 0, 64).plan.shares;
    const size_t need = shares > 1 ? (size_t)shares * Cin * Cout * sizeof(float) : 16;
    if (need > most) most = need;
  }
  return most;
}

static int launch_product(hipStream_t st, const Plan& p, bool far, bool f32, bool parts, int K, WgArgs a, float* copies, float* dW) {
  a.rows = p.rows, a.tiles_i = p.tiles_i, a.tiles_j = p.tiles_j;
  a.copy = p.shares > 1 ? (int64_t)a.Cin * a.Cout : 0;
  a.out = p.shares > 1 ? copies : dW;
  const unsigned grid = (unsigned)(p.tiles_i * p.tiles_j * p.shares);
  const bool ragged = a.Cout % 8 != 0;
  int e;
  if (far) {
    auto kern = f32 ? (parts ? (K == 8 ? store_wgrad_far_kernel<float, 8, 3> : store_wgrad_far_kernel<float, 4, 3>)
                             : (K == 8 ? store_wgrad_far_kernel<float, 8, 1> : store_wgrad_far_kernel<float, 4, 1>))
                    : (K == 8 ? store_wgrad_far_kernel<bf16_t, 8, 1> : store_wgrad_far_kernel<bf16_t, 4, 1>);
    kern<<<grid, 256, 0, st>>>(a);
    e = hip_status();
  } else if (!f32) {
    e = p.bi == 256 ? launch_tiles<bf16_t, 1, 256, 256>(st, K, ragged, grid, a) : launch_tiles<bf16_t, 1, 128, 128>(st, K, ragged, grid, a);
  } else if (!parts) {
    e = p.bi == 256 ? launch_tiles<float, 1, 256, 256>(st, K, ragged, grid, a) : launch_tiles<float, 1, 128, 128>(st, K, ragged, grid, a);
  } else {
    e = p.bi == 256 ? launch_tiles<float, 3, 256, 128>(st, K, ragged, grid, a) : launch_tiles<float, 3, 128, 128>(st, K, ragged, grid, a);
  }
  if (e != ABL_OK || p.shares == 1) return e;
  const int64_t size = (int64_t)a.Cin * a.Cout;
  auto sum = f32 ? wgrad_sum_kernel<float> : wgrad_sum_kernel<bf16_t>;
  sum<<<(unsigned)((size + 1023) / 1024), 256, 0, st>>>(copies, p.shares, size, a.scale, Divisor(a.Cout), a.accum, dW);
  return hip_status();
}

int launch_store_wgrad(hipStream_t st, int dtype, uint32_t flags, const void* ckpt, int64_t M, int Cin, int K, const void* scale,
                       Rows dy, int Cout, void* scratch, float* dW) {
  const bool parts = dtype == ABL_F32 && !(flags & ABL_MATH_BF16), f32 = dtype == ABL_F32;
  const int64_t size = size_of(dtype), blocks = store_blocks(Cin);
  const int64_t ld = M > 1 ? dy.ld : Cout;
  Cut c = cut_of(M, Cout * size, Cin, Cout, parts, 64);
  if (!c.far && !offsets_fit(c.plan, ld * size, Cin)) c = cut_of(M, ld * size, Cin, Cout, parts, c.plan.shares);
  if (c.far) c.plan.bi = c.plan.bj = 128, c.plan.tiles_i = (Cin + 127) / 128, c.plan.tiles_j = (Cout + 127) / 128;
  WgArgs a{};
  a.ldy = ld, a.scale = scale, a.Cin = Cin, a.Cout = Cout, a.blocks = (int)blocks, a.accum = (flags & ABL_ACCUM_DW) != 0;
  int64_t m = 0;
  do {
    a.M = m + c.rows < M ? c.rows : M - m;
    a.codes = (const unsigned char*)ckpt + m * blocks * 4 * K;
    a.scales = (const unsigned char*)ckpt + store_code_bytes(M, Cin, K) + m * blocks;
    a.dy = (const char*)dy.p + m * ld * size;
    Plan p = c.plan;
    if (a.M < c.rows) p.shares = (int)((a.M + p.rows - 1) / p.rows);
    if (int e = launch_product(st, p, c.far, f32, parts, K, a, (float*)scratch, dW)) return e;
    a.accum = 1;
    m += c.rows;   // (a multiple of 64 where more follow: pieces stay aligned)
  } while (m < M);
  return ABL_OK;
}

}  // namespace abl
