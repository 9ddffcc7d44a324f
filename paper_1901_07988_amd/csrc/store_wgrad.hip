// Weight gradient of a product from the block store of its input (abl_ckpt_wgrad): dW [Cin][Cout] = (scale * x~)^T dy, a contraction
// over the M rows.
//
// A stored value is a code of at most eight bits times a power of two, so it is exact in bf16: the codes become the bf16 operand of the
// matrix cores while a tile is staged and nothing is rounded.  dy in bf16 goes in as it is, dy in fp32 as
// three bf16 parts of eight bits each (three products), or rounded to one.
//
// Both operands lie with the contraction index outermost.  They are staged that way, [m][channels] in bf16, and the fragments
// are read with ds_read_b64_tr_b16: 16 lanes fetch four rows' 16 channels and receive one channel's four rows each.  The order
// of the rows within a step of 32 is 4 (lane / 16) + 0..3 and 16 more, for both operands alike.  A row's 32-byte chunks (16
// channels) are stored at their number xor row % 8, which puts the 8 rows that half a wave reads at once on different banks.

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

// NP: bf16 parts of an element of dy.
template <typename T, int K, int NP, int BI, int BJ, int WI, int WJ>
__global__ __launch_bounds__(WI * WJ * 64) void store_wgrad_kernel(WgArgs a) {
  constexpr int BK = 32, kThreads = WI * WJ * 64;
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
      put(to + r * (BI * 2) + (((q >> 1) ^ (r & 7)) * 32) + (q & 1) * 16, to_bf16x8(v));
    }
#pragma unroll
    for (int p = 0; p < PY; ++p) {
      const int at = p * kThreads + tid, r = at / (BJ / 8), q = at % (BJ / 8);
      char* y = to + kXBytes + r * (BJ * 2) + (((q >> 1) ^ (r & 7)) * 32) + (q & 1) * 16;
      if constexpr (std::is_same_v<T, bf16_t>) {
        put(y, __builtin_bit_cast(bf16x8_t, ry[p]));
      } else {
        float v[8];
        expand(ry[p], v);
#pragma unroll
        for (int n = 0; n < NP; ++n) {
          const bf16x8_t h = to_bf16x8(v);
          put(y + n * kYBytes, h);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = finite(v[e]) ? v[e] - (float)h[e] : 0.0f;
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
    const char* p = plane + r * pitch + (((c >> 4) ^ (r & 7)) * 32) + (lane & 3) * 8;
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

// The shares' copies, added in turn.
template <typename T>
__global__ __launch_bounds__(256) void wgrad_sum_kernel(const float* copies, int n, int64_t size, const void* scale, Divisor by_cout, int accum,
                                                        float* dW) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= size) return;
  float s = 0.0f;
  for (int i = 0; i < n; ++i) s += copies[i * size + e];
  s *= row_scale<T>(scale, by_cout.of((int)e));
  dW[e] = accum ? dW[e] + s : s;
}

template <int TILE>
struct Plan {
  int tiles_i, tiles_j, shares;
  int64_t rows;
  Plan(int64_t M, int Cin, int Cout) {
    tiles_i = (Cin + TILE - 1) / TILE, tiles_j = (Cout + TILE - 1) / TILE;
    const int64_t tiles = (int64_t)tiles_i * tiles_j;
    int64_t n = tiles >= 256 ? 1 : 512 / tiles;
    const int64_t most = (M + 255) / 256;
    if (n > most) n = most;
    if (n < 1) n = 1;
    rows = ((M + n - 1) / n + 31) / 32 * 32;
    shares = M > 0 ? (int)((M + rows - 1) / rows) : 1;
  }
};

template <typename T>
void sum_copies(hipStream_t st, const float* copies, int n, int Cin, int Cout, const void* scale, bool accum, float* dW) {
  const int64_t size = (int64_t)Cin * Cout;
  wgrad_sum_kernel<T><<<(unsigned)((size + 255) / 256), 256, 0, st>>>(copies, n, size, scale, Divisor(Cout), accum, dW);
}

}  // namespace

size_t store_wgrad_scratch_bytes(int64_t M, int Cin, int Cout, int dtype) {
  const Plan<128> p(M, Cin, Cout);
  return p.shares > 1 ? (size_t)p.shares * Cin * Cout * sizeof(float) : 16;
}

int launch_store_wgrad(hipStream_t st, int dtype, uint32_t flags, const void* ckpt, int64_t M, int Cin, int K, const void* scale,
                       Rows dy, int Cout, void* scratch, float* dW) {
  const Plan<128> p(M, Cin, Cout);
  WgArgs a;
  a.codes = (const unsigned char*)ckpt, a.scales = a.codes + store_code_bytes(M, Cin, K);
  a.dy = dy.p, a.ldy = dy.ld, a.scale = scale, a.M = M, a.rows = p.rows, a.Cin = Cin, a.Cout = Cout, a.blocks = (int)store_blocks(Cin);
  a.tiles_i = p.tiles_i, a.tiles_j = p.tiles_j, a.accum = (flags & ABL_ACCUM_DW) != 0;
  a.copy = p.shares > 1 ? (int64_t)Cin * Cout : 0;
  a.out = p.shares > 1 ? (float*)scratch : dW;
  const unsigned grid = (unsigned)(p.tiles_i * p.tiles_j * p.shares);
  if (dtype == ABL_BF16) {
    auto kern = K == 8 ? store_wgrad_kernel<bf16_t, 8, 1, 128, 128, 2, 2> : store_wgrad_kernel<bf16_t, 4, 1, 128, 128, 2, 2>;
    kern<<<grid, 256, 0, st>>>(a);
  } else if (flags & ABL_MATH_BF16) {
    auto kern = K == 8 ? store_wgrad_kernel<float, 8, 1, 128, 128, 2, 2> : store_wgrad_kernel<float, 4, 1, 128, 128, 2, 2>;
    kern<<<grid, 256, 0, st>>>(a);
  } else {
    auto kern = K == 8 ? store_wgrad_kernel<float, 8, 3, 128, 128, 2, 2> : store_wgrad_kernel<float, 4, 3, 128, 128, 2, 2>;
    kern<<<grid, 256, 0, st>>>(a);
  }
  if (int e = hip_status()) return e;
  if (p.shares > 1) {
    if (dtype == ABL_BF16)
      sum_copies<bf16_t>(st, (const float*)scratch, p.shares, Cin, Cout, scale, a.accum, dW);
    else
      sum_copies<float>(st, (const float*)scratch, p.shares, Cin, Cout, scale, a.accum, dW);
    return hip_status();
  }
  return ABL_OK;
}

}  // namespace abl
