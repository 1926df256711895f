// LayerNorm of rows on its own, forward and backward: the one between the last state and the head of a network, where
// the layers' own are parts of their steps (rowwise.hip).
//   mu = mean x,  rstd = (mean (x - mu)^2 + eps)^-1/2,  xhat = (x - mu) rstd,  y = xhat gamma + beta
//   g = dy gamma,  dx = rstd (g - mean g - xhat mean(g xhat)),  dgamma = sum_rows dy xhat,  dbeta = sum_rows dy
// A row lies in the registers of LPR lanes, NV vectors of 4 in each; all arithmetic is fp32.  Bound by moving its rows.
#include "kernels.h"
#include "lds_limit.h"
#include "prof.h"
#include "q8.h"

namespace mg {
namespace {

__device__ __forceinline__ float sum4(f32x4 v) { return (v[0] + v[1]) + (v[2] + v[3]); }
__device__ __forceinline__ float dot4(f32x4 a, f32x4 b) { return (a[0] * b[0] + a[1] * b[1]) + (a[2] * b[2] + a[3] * b[3]); }

template <int CTRL> __device__ __forceinline__ float add_lane(float v) { return v + bits_f(lane_move<CTRL>(f_bits(v))); }
// Sums of two values over the LPR lanes of a row, the same bits in each of them.  red: 2 floats per wavefront for rows that
// span several (one block per row then).
template <int LPR> __device__ __forceinline__ void row_sums(float& a, float& b, float* red) {
  auto step = [&](auto f) { a = f(a); b = f(b); };
  step([](float v) { return add_lane<LANE_XOR1>(v); });
  step([](float v) { return add_lane<LANE_XOR2>(v); });
  step([](float v) { return add_lane<LANE_MIRROR8>(v); });
  step([](float v) { return add_lane<LANE_MIRROR16>(v); });
  if constexpr (LPR >= 32) step([](float v) { return v + __shfl_xor(v, 16, 64); });
  if constexpr (LPR >= 64) step([](float v) { return v + __shfl_xor(v, 32, 64); });
  if constexpr (LPR > 64) {
    constexpr int NW = LPR / 64;
    const int wave = threadIdx.x >> 6;
    __syncthreads();                                     // the previous sums have been read
    if ((threadIdx.x & 63) == 0) { red[2 * wave] = a; red[2 * wave + 1] = b; }
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) { a += red[2 * w]; b += red[2 * w + 1]; }
  }
}

__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}

template <int LPR> constexpr int block_threads() { return LPR > 256 ? LPR : 256; }

// zeros where the vector lies past the end of a row (uniform test first: only the last vectors of a row can)
template <int LPR> __device__ __forceinline__ f32x4 inside(f32x4 v, int i, int c, int cols) {
  if ((i + 1) * LPR * 4 > cols) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = c + j < cols ? v[j] : 0.f;
  }
  return v;
}

template <typename T, int LPR, int NV>
__device__ __forceinline__ void load_row(f32x4 (&v)[NV], const T* row, int lane, int cols) {
#pragma unroll
  for (int i = 0; i < NV; ++i) v[i] = load4_row<T>(row, (i * LPR + lane) * 4, cols);
}
template <int LPR, int NV> __device__ __forceinline__ void settle_row(f32x4 (&v)[NV], int lane, int cols) {
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if ((i + 1) * LPR * 4 > cols) v[i] = settle4(v[i], (i * LPR + lane) * 4, cols);
}

// gamma (or beta) of the lane's columns; ones (zeros) without
template <int LPR, int NV> __device__ __forceinline__ void load_vector(f32x4 (&v)[NV], const float* p, float missing, int lane, int cols) {
  if (p) {
    load_row<float, LPR, NV>(v, p, lane, cols);
    settle_row<LPR, NV>(v, lane, cols);
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = f32x4{missing, missing, missing, missing};
  }
}

// the 8-bit copy of a row that lies in registers, zeros in its last block past the end
template <int LPR, int NV>
__device__ __forceinline__ void keep_row(const f32x4 (&v)[NV], unsigned char* q, unsigned char* scale, int lane, int cols, int blocks, bool live) {
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * LPR + lane) * 4;
    unsigned s;
    const unsigned w = q8_quantise(v[i], s);             // (all lanes)
    if (live && c < blocks * Q8_BLOCK) {
      reinterpret_cast<unsigned*>(q)[c >> 2] = w;
      if ((lane & 7) == 0) scale[c / Q8_BLOCK] = (unsigned char)s;
    }
  }
}

template <typename T, int LPR, int NV>
__global__ void __launch_bounds__(block_threads<LPR>()) norm_forward_kernel(const NormFwdArgs a, long first_row) {
  constexpr int RPB = block_threads<LPR>() / LPR;
  __shared__ float red[2 * (LPR > 64 ? LPR / 64 : 1)];
  const int lane = threadIdx.x % LPR, cols = a.cols;
  const long slot = first_row + (long)blockIdx.x * RPB + threadIdx.x / LPR;
  const bool live = slot < a.rows;
  const long row = live ? slot : a.rows - 1;             // (no lane leaves: sums go over lanes)
  f32x4 v[NV], gm[NV], bt[NV];
  load_row<T, LPR, NV>(v, static_cast<const T*>(a.x) + row * a.ldx, lane, cols);
  load_vector<LPR, NV>(gm, a.gamma, 1.f, lane, cols);
  load_vector<LPR, NV>(bt, a.beta, 0.f, lane, cols);
  settle_row<LPR, NV>(v, lane, cols);
  if (a.xq)
    keep_row<LPR, NV>(v, a.xq + row * a.blocks * Q8_BLOCK, a.xs + row * a.blocks, lane, cols, a.blocks, live);
  const float n = 1.0f / cols;
  float s = 0.f, none = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) s += sum4(v[i]);
  row_sums<LPR>(s, none, red);
  // The mean of the differences to this mean is what rounding left of it; with it both are right to the last bit or two
  // also where the values nearly cancel.  (Every difference has to be to the same number: one that the compiler fuses with
  // the product is not.)
  const float mu0 = rounded_product(s, n);
  float d = 0.f, d2 = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    v[i] = inside<LPR>(v[i] - mu0, i, (i * LPR + lane) * 4, cols);
    d += sum4(v[i]);
    d2 += dot4(v[i], v[i]);
  }
  row_sums<LPR>(d, d2, red);
  const float rest = rounded_product(d, n), mu = mu0 + rest;
  const float var = fmaxf(d2 * n - rest * rest, 0.f);
  // (fmaxf drops a NaN: a row with one, or with an infinity, has NaN throughout)
  const float rstd = d2 == d2 ? 1.0f / sqrtf(var + a.eps) : d2;
  if (live && lane == 0) {
    if (a.mean) a.mean[row] = mu;
    if (a.rstd) a.rstd[row] = rstd;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) v[i] = (v[i] - rest) * rstd * gm[i] + bt[i];
  if (a.y_bf16) {
    bf16* y = static_cast<bf16*>(a.y) + row * a.ldy;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      // rounded here, so that the kept copy is that of the values the caller sees
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i][j] = (float)(bf16)v[i][j];
      if (live) store4_row<bf16>(y, (i * LPR + lane) * 4, cols, v[i]);
    }
  } else {
    float* y = static_cast<float*>(a.y) + row * a.ldy;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (live) store4_row<float>(y, (i * LPR + lane) * 4, cols, v[i]);
  }
  if (a.yq) {
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = inside<LPR>(v[i], i, (i * LPR + lane) * 4, cols);
    keep_row<LPR, NV>(v, a.yq + row * a.blocks * Q8_BLOCK, a.ys + row * a.blocks, lane, cols, a.blocks, live);
  }
}

// Where x is kept in 8 bits: tag of the third form of the backward kernel's x.
struct Kept {};

// Backward.  Every row slot of the grid walks rows with the grid's stride and adds up its columns' dy xhat and dy in
// registers; a block adds up its slots' and leaves one row of [dgamma | dbeta] partial sums (part_cols columns each), which
// norm_join_kernel adds up in order.  With one block the sums are final (partial = null).
template <typename TX, typename TY, int LPR, int NV>
__global__ void __launch_bounds__(block_threads<LPR>()) norm_backward_kernel(const NormBwdArgs a, float* partial, int part_cols) {
  constexpr int RPB = block_threads<LPR>() / LPR;
  constexpr bool KEPT = std::is_same<TX, Kept>::value;
  __shared__ float red[2 * (LPR > 64 ? LPR / 64 : 1)];
  __shared__ __attribute__((aligned(16))) float join[RPB > 1 ? (RPB - 1) * NV * LPR * 4 : 4];
  const int lane = threadIdx.x % LPR, cols = a.cols, r = threadIdx.x / LPR;
  const long first = (long)blockIdx.x * RPB + r, stride = (long)gridDim.x * RPB;
  const float n = 1.0f / cols;
  f32x4 gm[NV], ag[NV], ab[NV];
  load_vector<LPR, NV>(gm, a.gamma, 1.f, lane, cols);
#pragma unroll
  for (int i = 0; i < NV; ++i) ag[i] = ab[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const long trips = (a.rows + stride - 1) / stride;     // the same for all slots: a row's sums may span the block
  for (long t = 0; t < trips; ++t) {
    const bool live = first + t * stride < a.rows;
    const long row = live ? first + t * stride : a.rows - 1;
    f32x4 x[NV], dy[NV];
    if constexpr (KEPT) {
      const unsigned* q = reinterpret_cast<const unsigned*>(a.xq + row * a.blocks * Q8_BLOCK);
      const unsigned char* s = a.xs + row * a.blocks;
      unsigned w[NV], sc[NV];
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * LPR + lane) * 4, cc = c < a.blocks * Q8_BLOCK ? c : 0;
        w[i] = q[cc >> 2];
        sc[i] = s[cc / Q8_BLOCK];
      }
      load_row<TY, LPR, NV>(dy, static_cast<const TY*>(a.dy) + row * a.ldy, lane, cols);
#pragma unroll
      for (int i = 0; i < NV; ++i) x[i] = q8_values(w[i], q8_step(sc[i]));
    } else {
      load_row<TX, LPR, NV>(x, static_cast<const TX*>(a.x) + row * a.ldx, lane, cols);
      load_row<TY, LPR, NV>(dy, static_cast<const TY*>(a.dy) + row * a.ldy, lane, cols);
      settle_row<LPR, NV>(x, lane, cols);
    }
    const float mu = a.mean[row], rstd = a.rstd[row];
    settle_row<LPR, NV>(dy, lane, cols);
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * LPR + lane) * 4;
      x[i] = inside<LPR>((x[i] - mu) * rstd, i, c, cols);
      if (live) {
        ag[i] += dy[i] * x[i];
        ab[i] += dy[i];
      }
      dy[i] = dy[i] * gm[i];
      s1 += sum4(dy[i]);
      s2 += dot4(dy[i], x[i]);
    }
    if (!a.dx) continue;
    row_sums<LPR>(s1, s2, red);
    s1 *= n;
    s2 *= n;
#pragma unroll
    for (int i = 0; i < NV; ++i) x[i] = ((dy[i] - s1) - x[i] * s2) * rstd;
    if (!live) continue;
    if (a.x_bf16) {
      bf16* dx = static_cast<bf16*>(a.dx) + row * a.lddx;
#pragma unroll
      for (int i = 0; i < NV; ++i) store4_row<bf16>(dx, (i * LPR + lane) * 4, cols, x[i]);
    } else {
      float* dx = static_cast<float*>(a.dx) + row * a.lddx;
#pragma unroll
      for (int i = 0; i < NV; ++i) store4_row<float>(dx, (i * LPR + lane) * 4, cols, x[i]);
    }
  }
  if (!a.dgamma && !a.dbeta) return;
  float* out_g = partial ? partial + (long)blockIdx.x * 2 * part_cols : a.dgamma;
  float* out_b = partial ? out_g + part_cols : a.dbeta;
  auto leave = [&](f32x4 (&v)[NV], float* out) {
    if constexpr (RPB > 1) {
      __syncthreads();
      if (r > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) *reinterpret_cast<f32x4*>(&join[((r - 1) * NV + i) * LPR * 4 + lane * 4]) = v[i];
      }
      __syncthreads();
      if (r > 0) return;
#pragma unroll
      for (int k = 0; k < RPB - 1; ++k)
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] += *reinterpret_cast<const f32x4*>(&join[(k * NV + i) * LPR * 4 + lane * 4]);
    }
    if (!out) return;
#pragma unroll
    for (int i = 0; i < NV; ++i) store4_row<float>(out, (i * LPR + lane) * 4, cols, v[i]);
  };
  leave(ag, out_g);
  leave(ab, out_b);
}

// dgamma, dbeta from the blocks' partial sums: 64 columns and 16 runs of blocks per thread block
__global__ void __launch_bounds__(1024) norm_join_kernel(const float* partial, int n, int part_cols, int cols, float* dgamma, float* dbeta) {
  __shared__ float red[16][64];
  float* out = blockIdx.y ? dbeta : dgamma;
  if (!out) return;
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), run = threadIdx.x >> 6;
  float s = 0.f;
  if (c < cols) {
    const float* p = partial + blockIdx.y * part_cols + c;
#pragma unroll 8
    for (int b = run; b < n; b += 16) s += p[(long)b * 2 * part_cols];
  }
  red[run][threadIdx.x & 63] = s;
  __syncthreads();
  if (run || c >= cols) return;
#pragma unroll
  for (int k = 1; k < 16; ++k) s += red[k][threadIdx.x];
  out[c] = s;
}

// without rows
__global__ void __launch_bounds__(256) norm_zero_kernel(int cols, float* dgamma, float* dbeta) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= cols) return;
  if (dgamma) dgamma[c] = 0.f;
  if (dbeta) dbeta[c] = 0.f;
}

// Lanes per row and vectors per lane, by the row's length.  f(LPR, NV) is called with the pair as types.
template <int V> using Int = std::integral_constant<int, V>;
template <typename F> hipError_t by_width(int cols, F f) {
  if (cols <= 64) return f(Int<16>{}, Int<1>{});
  if (cols <= 128) return f(Int<32>{}, Int<1>{});
  if (cols <= 256) return f(Int<64>{}, Int<1>{});
  if (cols <= 512) return f(Int<64>{}, Int<2>{});
  if (cols <= 768) return f(Int<64>{}, Int<3>{});
  if (cols <= 1024) return f(Int<64>{}, Int<4>{});
  if (cols <= 2048) return f(Int<256>{}, Int<2>{});
  if (cols <= 4096) return f(Int<256>{}, Int<4>{});
  if (cols <= 8192) return f(Int<256>{}, Int<8>{});
  return f(Int<1024>{}, Int<4>{});
}

// Blocks of the backward pass: enough to fill the chip (4 wavefronts each), and no more partial rows than that.
constexpr int BWD_BLOCKS = 768;
int backward_blocks(long rows, int rows_per_block) {
  const long want = (rows + rows_per_block - 1) / rows_per_block;
  return (int)(want < BWD_BLOCKS ? want : BWD_BLOCKS);
}
int part_cols(int cols) { return (cols + 3) & ~3; }

template <typename TX, typename TY> hipError_t backward(const NormBwdArgs& a, float* partial, hipStream_t st) {
  return by_width(a.cols, [&](auto lpr, auto nv) {
    constexpr int LPR = decltype(lpr)::value, NV = decltype(nv)::value, RPB = block_threads<LPR>() / LPR;
    const int blocks = backward_blocks(a.rows, RPB), pc = part_cols(a.cols);
    const bool sums = a.dgamma || a.dbeta;
    hipLaunchKernelGGL((norm_backward_kernel<TX, TY, LPR, NV>), dim3(blocks), dim3(block_threads<LPR>()), 0, st, a,
                       blocks > 1 ? partial : nullptr, pc);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (!sums || blocks == 1) return hipSuccess;
    hipLaunchKernelGGL(norm_join_kernel, dim3((a.cols + 63) / 64, 2), dim3(1024), 0, st, partial, blocks, pc, a.cols, a.dgamma, a.dbeta);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t launch_norm_forward(const NormFwdArgs& a, bool x_bf16, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  const double n = (double)a.rows * a.cols;
  ProfScope ps(PC_NORM_FWD, 8.0 * n, n * ((x_bf16 ? 2 : 4) + (a.y_bf16 ? 2 : 4)) + 33.0 * a.rows * a.blocks * ((a.xq != nullptr) + (a.yq != nullptr)), st);
  return by_width(a.cols, [&](auto lpr, auto nv) {
    constexpr int LPR = decltype(lpr)::value, NV = decltype(nv)::value, RPB = block_threads<LPR>() / LPR;
    constexpr long MOST = (1l << 30) / block_threads<LPR>() * RPB;         // rows of a launch: its threads have a 32-bit count
    for (long first = 0; first < a.rows; first += MOST) {
      const long rows = a.rows - first < MOST ? a.rows - first : MOST;
      const dim3 grid((unsigned)((rows + RPB - 1) / RPB)), block(block_threads<LPR>());
      if (x_bf16) hipLaunchKernelGGL((norm_forward_kernel<bf16, LPR, NV>), grid, block, 0, st, a, first);
      else hipLaunchKernelGGL((norm_forward_kernel<float, LPR, NV>), grid, block, 0, st, a, first);
      if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
  });
}

size_t norm_backward_partial_floats(long rows, int cols) {
  if (rows <= 0) return 0;
  size_t blocks = 0;
  (void)by_width(cols, [&](auto lpr, auto) {
    blocks = backward_blocks(rows, block_threads<decltype(lpr)::value>() / decltype(lpr)::value);
    return hipSuccess;
  });
  return blocks > 1 ? blocks * 2 * part_cols(cols) : 0;
}

hipError_t launch_norm_backward(const NormBwdArgs& a, bool dy_bf16, float* partial, hipStream_t st) {
  if (a.rows <= 0) {
    if (!a.dgamma && !a.dbeta) return hipSuccess;
    hipLaunchKernelGGL(norm_zero_kernel, dim3((a.cols + 255) / 256), dim3(256), 0, st, a.cols, a.dgamma, a.dbeta);
    return hipGetLastError();
  }
  const double n = (double)a.rows * a.cols;
  ProfScope ps(PC_NORM_BWD, 14.0 * n,
               n * ((a.x_bf16 ? 2 : 4) + (dy_bf16 ? 2 : 4)) + (a.xq ? 33.0 * a.rows * a.blocks : n * (a.x_bf16 ? 2 : 4)), st);
  if (a.xq) return dy_bf16 ? backward<Kept, bf16>(a, partial, st) : backward<Kept, float>(a, partial, st);
  if (a.x_bf16) return dy_bf16 ? backward<bf16, bf16>(a, partial, st) : backward<bf16, float>(a, partial, st);
  return dy_bf16 ? backward<float, bf16>(a, partial, st) : backward<float, float>(a, partial, st);
}

}  // namespace mg
