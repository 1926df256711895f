// Gradients of a linear map y = x W^T + b whose input rows were kept in 8 bits:
//   dW[m,n] = scale * sum_t dY[t,m] x~[t,n],   db[m] = scale * sum_t dY[t,m]
// A kept value is 7 bits and a sign times a power of two, so it is a bf16 number as it is; a bf16 dY is one as well, and an
// fp32 dY is exactly the sum of three of 8 bits each (cut, not rounded: hi = its upper 16 bits, then the same of the rest,
// then what is left).  So the products run on the bf16 matrix cores, one or three of them, without any rounding of an
// operand, and the sums are fp32 either way: what differs from an fp32 product is only the order of the additions.
// Bound by the matrix cores (2 T M N flops, or three times that).
//
// Both operands are token-major and the reduction runs over the tokens, so the tiles are staged as they lie in memory
// ([token][feature], bf16) and the fragments come out of LDS through the transposing read; rows of a tile keep their
// 16-byte chunks XOR-swizzled by the row.  Global loads go to registers a tile and a half ahead; between there and LDS the
// kept rows become bf16 and an fp32 dY its three parts.
#include "kernels.h"
#include "lds_limit.h"
#include "prof.h"
#include "q8.h"

namespace mg {
namespace {

constexpr int BK = 32;                                   // tokens per tile

// upper halves of two words: the two as bf16, cut
__device__ __forceinline__ unsigned upper(float lo, float hi) { return __builtin_amdgcn_perm(f_bits(hi), f_bits(lo), 0x07060302u); }
__device__ __forceinline__ float cut(float v) { return bits_f(f_bits(v) & 0xffff0000u); }

// 8 consecutive elements of a row of dY, as they are loaded
template <typename T> struct Chunk;
template <> struct Chunk<bf16> {
  u32x4 v;
  __device__ void clear() { v = u32x4{0, 0, 0, 0}; }
  __device__ void load(const bf16* p) {
    typedef const __attribute__((address_space(1))) u32x4_u* gptr;
    const u32x4_u u = *(gptr)p;
    v = u32x4{u[0], u[1], u[2], u[3]};
  }
  __device__ void load_some(const bf16* p, int n) {      // the first n, zeros behind them
    clear();
    const unsigned short* s = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) v[j >> 1] |= (unsigned)s[j] << (16 * (j & 1));
  }
  __device__ float at(int j) const { return bits_f(j & 1 ? v[j >> 1] & 0xffff0000u : v[j >> 1] << 16); }
  __device__ void parts(u32x4 (&out)[1]) const { out[0] = v; }
};
template <> struct Chunk<float> {
  f32x4 v[2];
  __device__ void clear() { v[0] = v[1] = f32x4{0.f, 0.f, 0.f, 0.f}; }
  __device__ void load(const float* p) { v[0] = load4u<float>(p); v[1] = load4u<float>(p + 4); }
  __device__ void load_some(const float* p, int n) {
    clear();
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) v[j >> 2][j & 3] = p[j];
  }
  __device__ float at(int j) const { return v[j >> 2][j & 3]; }
  __device__ void parts(u32x4 (&out)[3]) const {
    float hi[8], mid[8], lo[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float x = at(j);
      hi[j] = x;
      const float r = __builtin_isinf(x) ? 0.f : x - cut(x);       // an infinity has no rest; a NaN stays one
      mid[j] = r;
      lo[j] = r - cut(r);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      out[0][j] = upper(hi[2 * j], hi[2 * j + 1]);
      out[1][j] = upper(mid[2 * j], mid[2 * j + 1]);
      out[2][j] = upper(lo[2 * j], lo[2 * j + 1]);
    }
  }
};

template <typename T, int BM, int BN, int WM, int WN, int OCC>
__global__ void __launch_bounds__(64 * WM * WN, OCC * WM * WN / 4)
q8_grad_kernel(const Q8GradArgs a, int tiles_n, int per_slice, int splits, int total, int per_xcd, float* partial) {
  constexpr int NT = 64 * WM * WN, PARTS = std::is_same<T, float>::value ? 3 : 1;
  constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 32, TN = WTN / 32;
  constexpr int RA = BM * 2, RB = BN * 2;                // bytes per LDS row
  constexpr int A_BYTES = BK * RA, B_BYTES = BK * RB, STAGE = PARTS * A_BYTES + B_BYTES;
  constexpr int A_CH = BK * BM / 8 / NT, B_CH = BK * BN / 8 / NT;
  static_assert(A_CH * NT * 8 == BK * BM && B_CH * NT * 8 == BK * BN && NT % (BM / 8) == 0, "tile / thread split");
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  // an XCD takes a contiguous range of tiles, which share panels of the operands in its L2
  const int tile = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  if (tile >= total) return;
  const int sp = __builtin_amdgcn_readfirstlane(tile / per_slice), tg = tile - sp * per_slice;
  const int tm = __builtin_amdgcn_readfirstlane(tg / tiles_n), tn = tg - tm * tiles_n;
  const int m0 = tm * BM, n0 = tn * BN, M = a.M, N = a.N, NP = a.blocks * Q8_BLOCK;
  const long all_tiles = (a.rows + BK - 1) / BK;
  const long kt0 = all_tiles * sp / splits, kt1 = all_tiles * (sp + 1) / splits;
  const long K = (kt1 * BK < a.rows ? kt1 * BK : a.rows) - kt0 * BK;
  const T* A = static_cast<const T*>(a.dy) + kt0 * BK * a.ldy + m0;
  const unsigned char* Q = a.xq + kt0 * BK * NP + n0;
  const unsigned char* S = a.xs + kt0 * BK * a.blocks + n0 / Q8_BLOCK;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wm0 = (wave / WN) * WTM, wn0 = (wave % WN) * WTN;
  auto swz_of = [](int row_bytes, int r) { return row_bytes >= 256 ? (r & 3) << 2 : ((r >> 1) & 1) << 2; };

  // this thread's chunks of a tile: token and feature
  int arow[A_CH], brow[B_CH], adst[A_CH], bdst[B_CH];
  const int ac = (threadIdx.x % (BM / 8)) * 8;
  int bc[B_CH];
#pragma unroll
  for (int j = 0; j < A_CH; ++j) {
    arow[j] = (threadIdx.x + j * NT) / (BM / 8);
    adst[j] = arow[j] * RA + (((ac >> 3) ^ swz_of(RA, arow[j])) << 4);
  }
#pragma unroll
  for (int j = 0; j < B_CH; ++j) {
    const int id = threadIdx.x + j * NT;
    brow[j] = id / (BN / 8);
    bc[j] = id % (BN / 8) * 8;
    bdst[j] = PARTS * A_BYTES + brow[j] * RB + (((bc[j] >> 3) ^ swz_of(RB, brow[j])) << 4);
  }
  Chunk<T> ra[A_CH];
  u32x2 rq[B_CH];
  unsigned rs[B_CH];
  const bool inner = m0 + BM <= M && n0 + BN <= NP;
  auto load = [&](long k0) {
    if (k0 >= K) return;
    const T* at = A + k0 * a.ldy;
    const unsigned char *q = Q + k0 * NP, *s = S + k0 * a.blocks;
    if (inner && k0 + BK <= K) {
#pragma unroll
      for (int j = 0; j < A_CH; ++j) ra[j].load(at + arow[j] * a.ldy + ac);
#pragma unroll
      for (int j = 0; j < B_CH; ++j) {
        rq[j] = *reinterpret_cast<const u32x2*>(q + (long)brow[j] * NP + bc[j]);
        rs[j] = s[brow[j] * a.blocks + bc[j] / Q8_BLOCK];
      }
      return;
    }
#pragma unroll
    for (int j = 0; j < A_CH; ++j) {                      // zeros past the last token and the last feature
      const int n = k0 + arow[j] < K ? M - m0 - ac : 0;
      if (n >= 8) ra[j].load(at + arow[j] * a.ldy + ac);
      else if (n > 0) ra[j].load_some(at + arow[j] * a.ldy + ac, n);
      else ra[j].clear();
    }
#pragma unroll
    for (int j = 0; j < B_CH; ++j) {
      rq[j] = u32x2{0, 0};
      rs[j] = 127;
      if (k0 + brow[j] < K && n0 + bc[j] < NP) {
        rq[j] = *reinterpret_cast<const u32x2*>(q + (long)brow[j] * NP + bc[j]);
        rs[j] = s[brow[j] * a.blocks + bc[j] / Q8_BLOCK];
      }
    }
  };
  const bool sums = tn == 0 && a.db;                      // the first column of tiles adds up dY as well
  CarrySum bias[8];
  auto store = [&](int stage) {
    unsigned char* base = smem + stage * STAGE;
#pragma unroll
    for (int j = 0; j < A_CH; ++j) {
      u32x4 p[PARTS];
      ra[j].parts(p);
#pragma unroll
      for (int i = 0; i < PARTS; ++i) *reinterpret_cast<u32x4*>(base + i * A_BYTES + adst[j]) = p[i];
    }
#pragma unroll
    for (int j = 0; j < B_CH; ++j) {
      const float step = q8_step(rs[j]);
      const f32x4 lo = q8_values(rq[j][0], step), hi = q8_values(rq[j][1], step);
      *reinterpret_cast<u32x4*>(base + bdst[j]) = u32x4{upper(lo[0], lo[1]), upper(lo[2], lo[3]), upper(hi[0], hi[1]), upper(hi[2], hi[3])};
    }
    if (sums) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float t = ra[0].at(e);
#pragma unroll
        for (int j = 1; j < A_CH; ++j) t += ra[j].at(e);
        bias[e].add(t);
      }
    }
  };

  // fragments: tokens 8*(lane/32).., one column per lane
  const int lh = lane >> 5, trow = 8 * lh + ((lane & 15) >> 2), low = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  int offa[TM], offb[TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
    offa[i] = trow * RA + (((((wm0 + 32 * i) >> 3) + low) ^ swz_of(RA, trow)) << 4) + (lane & 1) * 8;
#pragma unroll
  for (int j = 0; j < TN; ++j)
    offb[j] = PARTS * A_BYTES + trow * RB + (((((wn0 + 32 * j) >> 3) + low) ^ swz_of(RB, trow)) << 4) + (lane & 1) * 8;
  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  const lds_byte* lds0 = (const lds_byte*)smem;

  const long KT = kt1 - kt0;
  load(0);
  if (KT > 0) store(0);
  load(BK);
  wait_lgkm();
  bare_barrier();
  for (long kt = 0; kt < KT; ++kt) {
    const int cur = (int)(kt & 1);
    if (kt + 1 < KT) store(cur ^ 1);
    load((kt + 2) * BK);
    const lds_byte* base = lds0 + cur * STAGE;
#pragma unroll
    for (int ks = 0; ks < BK / 16; ++ks) {
      bf16x8 xb[TN];
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        TrFrag f;
        f.lo = tr_read4(base + offb[j] + 16 * ks * RB);
        f.hi = tr_read4(base + offb[j] + (16 * ks + 4) * RB);
        xb[j] = tr_value(f);
      }
#pragma unroll
      for (int p = PARTS - 1; p >= 0; --p) {
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          TrFrag f;
          f.lo = tr_read4(base + p * A_BYTES + offa[i] + 16 * ks * RA);
          f.hi = tr_read4(base + p * A_BYTES + offa[i] + (16 * ks + 4) * RA);
          const bf16x8 xa = tr_value(f);
#pragma unroll
          for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xb[j], xa, acc[i][j], 0, 0, 0);
        }
      }
    }
    wait_lgkm();
    bare_barrier();
  }
  float *dW = a.dW, *db = a.db, scale = a.scale;
  if (splits > 1) {                                       // unscaled into the slice's [M x N | M] of the scratch
    dW = partial + (long)sp * ((long)M * N + M);
    db = dW + (long)M * N;
    scale = 1.f;
  }
  if (sums) {                                             // block-uniform
    float* red = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int e = 0; e < 8; ++e) red[threadIdx.x / (BM / 8) * BM + ac + e] = bias[e].sum;
    __syncthreads();
    for (int m = threadIdx.x; m < BM && m0 + m < M; m += NT) {
      CarrySum t;
      for (int g = 0; g < NT / (BM / 8); ++g) t.add(red[g * BM + m]);
      db[m0 + m] = scale * t.sum;
    }
  }
  // a lane holds 4 consecutive columns of one row at a time
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int m = m0 + wm0 + 32 * i + (lane & 31);
    if (m >= M) continue;
    float* out = dW + (long)m * N;
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int n = n0 + wn0 + 32 * j + 8 * q + 4 * lh;
        const f32x4 v = {scale * acc[i][j][4 * q], scale * acc[i][j][4 * q + 1], scale * acc[i][j][4 * q + 2], scale * acc[i][j][4 * q + 3]};
        if (n < N) store4_row<float>(out, n, N, v);
      }
  }
}

// sums of the slices, in order
__global__ void __launch_bounds__(256) q8_grad_join_kernel(const float* partial, int splits, long mn, int M, float* dW, float* db, float scale) {
  const long each = mn + M, i = ((long)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= each) return;
  CarrySum acc[4];
  const int n = each - i < 4 ? (int)(each - i) : 4;
  for (int s = 0; s < splits; ++s) {
    const float* p = partial + s * each + i;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (n == 4) v = load4u<float>(p);
    else
      for (int e = 0; e < n; ++e) v[e] = p[e];
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e].add(v[e]);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (i + e < mn) dW[i + e] = scale * acc[e].sum;
    else if (i + e < each && db) db[i + e - mn] = scale * acc[e].sum;
  }
}

__global__ void __launch_bounds__(256) q8_grad_zero_kernel(long mn, int M, float* dW, float* db) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  if (i < mn) dW[i] = 0.f;
  else if (i < mn + M && db) db[i - mn] = 0.f;
}

// Slices of the token sum: a launch with few tiles is cut along the tokens until the chip is full, which costs writing and
// adding up the slices' results.  The number follows from the sizes alone, not from the device, so that results do not
// depend on it either.
constexpr int CUS = 256;
struct Plan { int splits; };
Plan plan(long rows, int M, int N, bool dy_bf16) {
  const long tiles = (long)((M + 127) / 128) * ((N + 127) / 128), ktiles = (rows + BK - 1) / BK;
  Plan best = {1};
  double best_cost = 1e300;
  for (int s = 1; s <= 64 && (s == 1 || (ktiles / s >= 8 && tiles * s <= 1 << 20)); s *= 2) {
    const double rounds = (double)((tiles * s + 2 * CUS - 1) / (2 * CUS));
    double cost = rounds * (4.0 + (dy_bf16 ? 0.5 : 1.2) * ((ktiles + s - 1) / s));
    if (s > 1) cost += 4.0 + 2.0 * s * (double)M * N * 4.0 / 3e6;
    if (cost < best_cost) { best_cost = cost; best.splits = s; }
  }
  return best;
}

template <typename T, int BM, int BN, int WM, int WN, int OCC>
hipError_t launch_tile(const Q8GradArgs& a, int splits, float* partial, hipStream_t st) {
  constexpr int PARTS = std::is_same<T, float>::value ? 3 : 1;
  const long tiles_m = (a.M + BM - 1) / BM, tiles_n = (a.N + BN - 1) / BN, total = tiles_m * tiles_n * splits;
  const int per_xcd = (int)((total + 7) / 8);
  const size_t smem = 2 * (size_t)BK * 2 * (PARTS * BM + BN);
  static_assert(64 * WM * WN / (BM / 8) * BM * 4 <= 2 * BK * 2 * (PARTS * BM + BN), "the bias sums fit");
  auto kern = q8_grad_kernel<T, BM, BN, WM, WN, OCC>;
  static unsigned long raised = 0;
  if (const hipError_t e = raise_lds_limit(reinterpret_cast<const void*>(kern), (int)smem, raised); e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3(per_xcd * 8), dim3(64 * WM * WN), smem, st, a, (int)tiles_n, (int)(tiles_m * tiles_n), splits, (int)total, per_xcd, partial);
  return hipGetLastError();
}

}  // namespace

size_t q8_grad_partial_floats(long rows, int M, int N, bool dy_bf16) {
  if (rows <= 0) return 0;
  const int s = plan(rows, M, N, dy_bf16).splits;
  return s == 1 ? 0 : (size_t)s * ((size_t)M * N + M);
}

hipError_t launch_q8_grad(const Q8GradArgs& a, bool dy_bf16, float* partial, hipStream_t st) {
  const long mn = (long)a.M * a.N, each = mn + a.M;
  if (a.rows <= 0) {
    hipLaunchKernelGGL(q8_grad_zero_kernel, dim3((unsigned)((each + 255) / 256)), dim3(256), 0, st, mn, a.M, a.dW, a.db);
    return hipGetLastError();
  }
  ProfScope ps(PC_Q8_GRAD, 2.0 * a.rows * mn, (double)a.rows * (a.M * (dy_bf16 ? 2.0 : 4.0) + 33.0 * a.blocks) + 4.0 * each, st);
  const Plan p = plan(a.rows, a.M, a.N, dy_bf16);
  const hipError_t e = dy_bf16 ? launch_tile<bf16, 128, 128, 2, 2, 2>(a, p.splits, partial, st) : launch_tile<float, 128, 128, 2, 2, 2>(a, p.splits, partial, st);
  if (e != hipSuccess || p.splits == 1) return e;
  hipLaunchKernelGGL(q8_grad_join_kernel, dim3((unsigned)((each + 1023) / 1024)), dim3(256), 0, st, partial, p.splits, mn, a.M, a.dW, a.db, a.scale);
  return hipGetLastError();
}

}  // namespace mg
