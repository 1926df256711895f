// LayerNorm of rows on its own, forward and backward: the one between the last state and the head of a network, where
// the layers' own are parts of their steps (rowwise.hip).
//   mu = mean x,  rstd = (mean (x - mu)^2 + eps)^-1/2,  xhat = (x - mu) rstd,  y = xhat gamma + beta
//   g = dy gamma,  dx = rstd (g - mean g - xhat mean(g xhat)),  dgamma = sum_rows dy xhat,  dbeta = sum_rows dy
// A row lies in the registers of LPR lanes, NV vectors of 4 in each, so that it is read once; all arithmetic is fp32.  Bound
// by moving its rows: 16384 x 4096, bf16, forward 46.6 us, 5.8 TB/s; 32768 x 768, fp32 x and bf16 dy, backward 41.8 us and
// 4.2 for joining the partial sums, 5.5 TB/s together (a copy reaches 5.7); what goes to and comes from memory are the
// algorithm's bytes.  Few or short rows wait for one chain of load, sums and store: 1 x 768 3.2 us, 64 x 64 backward 4.2,
// 12608 x 384 from kept rows 11.2 where its bytes need 6.
// What paid: the next row's loads in flight while a row is reduced, and one exchange through LDS for a row of several
// wavefronts instead of two (forward, 16384 x 4096, bf16, 70 -> 54 us a call; backward, 32768 x 768, 59.6 -> 53).  What did not: blocks of
// 512 and 1024 lanes where 256 hold the row (equal); non-temporal stores of y (faster alone, slower with the kernel that
// reads y next).
// Rows past fp32's range are taken care of off that path, and their test costs up to 1.6 % (65536 x 64, bf16, 7.6 -> 7.7 us;
// 16384 x 4096 47.6 -> 47.9); mean and rstd of a row loaded before the row and not behind it: 8192 x 8192, bf16, 100 -> 83 us,
// other backward passes within 1 to 3 %.
#include <type_traits>

#include "kernels.h"
#include "prof.h"
#include "q8.h"

namespace mg {
namespace {

__device__ __forceinline__ float sum4(f32x4 v) { return (v[0] + v[1]) + (v[2] + v[3]); }
__device__ __forceinline__ float dot4(f32x4 a, f32x4 b) { return (a[0] * b[0] + a[1] * b[1]) + (a[2] * b[2] + a[3] * b[3]); }

template <int CTRL> __device__ __forceinline__ float add_lane(float v) { return v + bits_f(lane_move<CTRL>(f_bits(v))); }
// Sums of two values over a wavefront's lanes of a row, the same bits in each of them.
template <int LPR> __device__ __forceinline__ void wave_sums(float& a, float& b) {
  auto step = [&](auto f) { a = f(a); b = f(b); };
  step([](float v) { return add_lane<LANE_XOR1>(v); });
  step([](float v) { return add_lane<LANE_XOR2>(v); });
  step([](float v) { return add_lane<LANE_MIRROR8>(v); });
  step([](float v) { return add_lane<LANE_MIRROR16>(v); });
  if constexpr (LPR >= 32) step([](float v) { return v + __shfl_xor(v, 16, 64); });
  if constexpr (LPR >= 64) step([](float v) { return v + __shfl_xor(v, 32, 64); });
}
// Two values of every wavefront of a row, known to all of them (rows that span several wavefronts: one block per row).  Two
// halves of LDS are used in turn, so that one barrier is enough, and it waits for LDS alone: the next rows' loads stay in
// flight.
template <int LPR> struct Exchange {
  static constexpr int NW = LPR > 64 ? LPR / 64 : 1;
  f32x4 (*lds)[NW];
  int turn = 0;
  __device__ __forceinline__ const f32x4* operator()(f32x4 v) {
    f32x4* half = lds[turn];
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) half[threadIdx.x >> 6] = v;
    wait_lgkm();
    bare_barrier();
    return half;
  }
};
template <int LPR> __device__ __forceinline__ void row_sums(float& a, float& b, Exchange<LPR>& exchange) {
  wave_sums<LPR>(a, b);
  if constexpr (LPR > 64) {
    const f32x4* all = exchange(f32x4{a, b, 0.f, 0.f});
    a = b = 0.f;
#pragma unroll 4
    for (int w = 0; w < LPR / 64; ++w) { a += all[w][0]; b += all[w][1]; }
  }
}

__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}

template <int LPR> constexpr int block_threads() { return LPR > 256 ? LPR : 256; }

// A row's last vector, the only one that can lie past its end or across it (by_width): zeros there
__device__ __forceinline__ f32x4 inside(f32x4 v, int c, int cols) {
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = c + j < cols ? v[j] : 0.f;
  return v;
}

// A row's elements as they are loaded, 4 per vector, and what they stand for.  Rows of fewer than 4 elements (TINY) are loaded
// one by one; any others without a branch around the loads, which stay in flight until value() asks for them: a vector
// that reaches past the end starts at the last 4 elements, and value() moves what it found to its place.
struct Kept {};                                          // the tag of rows in 8 bits
template <typename T, int LPR, int NV, bool TINY> struct Row {
  static constexpr bool WIDE = std::is_same<T, float>::value;
  typedef typename std::conditional<WIDE, f32x4, u32x2>::type Raw;
  Raw v[NV];
  __device__ __forceinline__ void load(const T* row, int lane, int cols) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * LPR + lane) * 4;
      if constexpr (TINY) {
        f32x4 f = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 3; ++j)
          if (c + j < cols) f[j] = to_f(row[c + j]);
        if constexpr (WIDE) v[i] = f;
        else v[i] = u32x2{f_bits(f[0]) >> 16 | (f_bits(f[1]) & 0xffff0000u), f_bits(f[2]) >> 16};
      } else {
        const T* p = row + (i < NV - 1 || c < cols - 4 ? c : cols - 4);
        if constexpr (WIDE) {
          v[i] = load4u<float>(p);
        } else {
          typedef const __attribute__((address_space(1))) u32x2_u* gptr;
          const u32x2_u u = *(gptr)p;
          v[i] = u32x2{u[0], u[1]};
        }
      }
    }
  }
  __device__ __forceinline__ f32x4 value(int i, int lane, int cols) const {
    f32x4 f;
    if constexpr (WIDE) f = v[i];
    else f = f32x4{bits_f(v[i][0] << 16), bits_f(v[i][0] & 0xffff0000u), bits_f(v[i][1] << 16), bits_f(v[i][1] & 0xffff0000u)};
    if constexpr (TINY) return f;
    return i == NV - 1 ? settle4(f, (i * LPR + lane) * 4, cols) : f;
  }
};
template <int LPR, int NV, bool TINY> struct Row<Kept, LPR, NV, TINY> {
  unsigned q[NV], s[NV];
  __device__ __forceinline__ void load(const unsigned char* xq, const unsigned char* xs, int lane, int blocks) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * LPR + lane) * 4, in = i < NV - 1 || c < blocks * Q8_BLOCK ? c : 0;
      q[i] = reinterpret_cast<const unsigned*>(xq)[in >> 2];
      s[i] = xs[in / Q8_BLOCK];
    }
  }
  __device__ __forceinline__ f32x4 value(int i, int, int) const { return q8_values(q[i], q8_step(s[i])); }
};
// the row's vectors to memory; only the last ones can reach past the end
template <typename T, int LPR, int NV> __device__ __forceinline__ void store_row(T* row, const f32x4 (&v)[NV], int lane, int cols) {
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * LPR + lane) * 4;
    if (i < NV - 1) store4u<T>(row + c, v[i]);
    else store4_row<T>(row, c, cols, v[i]);
  }
}

// gamma (or beta) of the lane's columns; ones (zeros) without
template <int LPR, int NV, bool TINY> __device__ __forceinline__ void load_vector(f32x4 (&v)[NV], const float* p, float missing, int lane, int cols) {
  if (p) {
    Row<float, LPR, NV, TINY> r;
    r.load(p, lane, cols);
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = r.value(i, lane, cols);
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = f32x4{missing, missing, missing, missing};
  }
}

// index of a row, in a scalar register where all lanes of a wavefront share it
template <int LPR> __device__ __forceinline__ long row_index(long row) {
  if constexpr (LPR >= 64)
    return (long)__builtin_amdgcn_readfirstlane((int)(row >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)row);
  return row;
}

// the 8-bit copy of a row that lies in registers, zeros in its last block past the end
template <int LPR, int NV>
__device__ __forceinline__ void keep_row(const f32x4 (&v)[NV], unsigned char* q, unsigned char* scale, int lane, int cols, int blocks, bool live) {
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * LPR + lane) * 4;
    unsigned s;
    const unsigned w = q8_quantise(v[i], s);             // (all lanes)
    if (live && (i < NV - 1 || c < blocks * Q8_BLOCK)) {
      reinterpret_cast<unsigned*>(q)[c >> 2] = w;
      if ((lane & 7) == 0) scale[c / Q8_BLOCK] = (unsigned char)s;
    }
  }
}

// Rows whose loads are in flight while a row is reduced and written.  The loop is unrolled over them, each in registers of
// its own: a copy of registers would wait for the loads that fill them.
// (Blocks of 1024 lanes have 128 registers each, which hold one row.)
template <int LPR> constexpr int rows_ahead() { return LPR < 1024 ? 1 : 0; }

// Forward.  Every row slot of the grid walks rows with the grid's stride; gamma and beta stay in registers.
template <typename TX, typename TY, int LPR, int NV, bool TINY>
__global__ void __launch_bounds__(block_threads<LPR>()) norm_forward_kernel(const NormFwdArgs a) {
  constexpr int RPB = block_threads<LPR>() / LPR, AHEAD = rows_ahead<LPR>();
  __shared__ f32x4 red[2][LPR > 64 ? LPR / 64 : 1];
  Exchange<LPR> exchange{red};
  const int lane = threadIdx.x % LPR, cols = a.cols;
  const long first = (long)blockIdx.x * RPB + threadIdx.x / LPR, stride = (long)gridDim.x * RPB;
  const long trips = (a.rows - (long)blockIdx.x * RPB + stride - 1) / stride;             // the block's
  auto at = [&](long t) { return row_index<LPR>(first + t * stride < a.rows ? first + t * stride : a.rows - 1); };
  const TX* x = static_cast<const TX*>(a.x);
  const float n = 1.0f / cols;
  // a wavefront's share of a row, and the inverse (none: 0)
  int share = cols;
  if constexpr (LPR > 64) {
    share = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = cols - (i * LPR + (lane & ~63)) * 4;
      share += c < 0 ? 0 : c < 256 ? c : 256;
    }
  }
  const float n_share = share ? 1.0f / share : 0.f;
  f32x4 gm[NV], bt[NV];
  Row<TX, LPR, NV, TINY> ring[AHEAD + 1];
#pragma unroll
  for (int k = 0; k < AHEAD; ++k) ring[k].load(x + at(k) * a.ldx, lane, cols);
  load_vector<LPR, NV, TINY>(gm, a.gamma, 1.f, lane, cols);
  load_vector<LPR, NV, TINY>(bt, a.beta, 0.f, lane, cols);
  auto one_row = [&](const Row<TX, LPR, NV, TINY>& r, long t) {
    const bool live = first + t * stride < a.rows;       // (no lane leaves: sums go over lanes)
    const long row = at(t);
    f32x4 v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = r.value(i, lane, cols);
    if (a.xq)
      keep_row<LPR, NV>(v, a.xq + row * a.blocks * Q8_BLOCK, a.xs + row * a.blocks, lane, cols, a.blocks, live);
    float s = 0.f, none = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) s += sum4(v[i]);
    wave_sums<LPR>(s, none);
    // The mean of the differences to this mean is what rounding left of it; with it both are right to the last bit or two
    // also where the values nearly cancel.  (Every difference has to be to the same number: one that the compiler fuses with
    // the product is not.)
    const float mu0 = rounded_product(s, n_share);
    float d = 0.f, d2 = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      v[i] = v[i] - mu0;
      if (i == NV - 1) v[i] = inside(v[i], (i * LPR + lane) * 4, cols);
      d += sum4(v[i]);
      d2 += dot4(v[i], v[i]);
    }
    wave_sums<LPR>(d, d2);
    float rest = rounded_product(d, n_share), mu = mu0 + rest;
    // sum of (x - mu)^2; fmaxf drops a NaN, d2 keeps it (an infinite d2 has nothing to be corrected)
    float m2 = d2 < __builtin_inff() ? fmaxf(d2 - d * rest, 0.f) : d2;
    if constexpr (LPR > 64) {
      // the wavefronts' shares: mean of the means, and sum (x - mu)^2 = sum over shares of theirs + their number * (difference
      // of the means)^2
      const f32x4* all = exchange(f32x4{mu, m2, (float)share, 0.f});
      const float own = mu, base = all[0][0];
      float mean = 0.f, sq = 0.f;
#pragma unroll 4
      for (int w = 0; w < LPR / 64; ++w) {
        mean += all[w][2] * (all[w][0] - base);
        sq += all[w][1];
      }
      mu = base + mean * n;
#pragma unroll 4
      for (int w = 0; w < LPR / 64; ++w) sq += all[w][2] * ((all[w][0] - mu) * (all[w][0] - mu));
      rest += mu - own;
      m2 = sq;
    }
    float rstd = 1.0f / sqrtf(m2 * n + a.eps);
    if (__builtin_expect(__any(!(rstd > 0.f)), 0)) {
      // A row with a NaN or an infinity, which has NaN throughout; or a finite one whose sums pass fp32's range.  Of such a
      // row a 2^16th is summed up again: 2^14 differences of a 2^16th of any two numbers stay inside.  Its mean is right
      // then; where the sum of squares itself is past the range, rstd is 0 and y is beta.  (Rows of one wavefront go
      // through it together; of a row of several wavefronts all know the same rstd.)
      const bool past = !(rstd > 0.f);
      Row<TX, LPR, NV, TINY> again;
      again.load(x + row * a.ldx, lane, cols);           // (in place as well: it is stored further down)
      f32x4 w[NV];
      float all = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        w[i] = again.value(i, lane, cols) * 0x1p-16f;
        all += sum4(w[i]);
      }
      row_sums<LPR>(all, none, exchange);
      const float base = rounded_product(all, n);
      float left = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        w[i] = w[i] - base;
        if (i == NV - 1) w[i] = inside(w[i], (i * LPR + lane) * 4, cols);
        left += sum4(w[i]);
      }
      row_sums<LPR>(left, none, exchange);
      const float shift = left / (float)cols;            // (exact for a row of one value, a product may not be)
      float sq = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        w[i] = (w[i] - shift) * 0x1p16f;
        if (i == NV - 1) w[i] = inside(w[i], (i * LPR + lane) * 4, cols);
        sq += dot4(w[i], w[i]);
      }
      row_sums<LPR>(sq, none, exchange);
      const bool mend = past && __builtin_isfinite(all);
      mu = mend ? (base + shift) * 0x1p16f : mu;
      rest = mend ? 0.f : rest;
      rstd = mend ? 1.0f / sqrtf(sq * n + a.eps) : rstd;
#pragma unroll
      for (int i = 0; i < NV; ++i)                       // (with a wavefront to itself, a NaN's row needs no values: registers)
        if (LPR >= 64 || mend) v[i] = sq < __builtin_inff() ? w[i] : f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (live && lane == 0) {
      if (a.mean) a.mean[row] = mu;
      if (a.rstd) a.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = (v[i] - rest) * rstd * gm[i] + bt[i];
    if constexpr (std::is_same<TY, bf16>::value) {
      // rounded here, so that the kept copy is that of the values the caller sees
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i][j] = (float)(bf16)v[i][j];
    }
    if (live) store_row<TY, LPR, NV>(static_cast<TY*>(a.y) + row * a.ldy, v, lane, cols);
    if (a.yq) {
      v[NV - 1] = inside(v[NV - 1], ((NV - 1) * LPR + lane) * 4, cols);
      keep_row<LPR, NV>(v, a.yq + row * a.blocks * Q8_BLOCK, a.ys + row * a.blocks, lane, cols, a.blocks, live);
    }
  };
  for (long t = 0; t < trips; t += AHEAD + 1) {
#pragma unroll
    for (int k = 0; k <= AHEAD; ++k) {
      ring[(k + AHEAD) % (AHEAD + 1)].load(x + at(t + k + AHEAD) * a.ldx, lane, cols);
      if (k == 0 || t + k < trips) one_row(ring[k], t + k);
    }
  }
}

// Backward.  Every row slot of the grid walks rows with the grid's stride, as forward, and adds up its columns' dy xhat and
// dy in registers; a block adds up its slots' and leaves one row of [dgamma | dbeta] partial sums (part_cols columns each),
// which norm_join_kernel adds up in order.  With one block the sums are final (partial = null).
template <typename TX, typename TY, typename TD, int LPR, int NV, bool TINY>
__global__ void __launch_bounds__(block_threads<LPR>()) norm_backward_kernel(const NormBwdArgs a, float* partial, int part_cols) {
  constexpr int RPB = block_threads<LPR>() / LPR;
  constexpr int AHEAD = rows_ahead<LPR>();
  __shared__ f32x4 red[2][LPR > 64 ? LPR / 64 : 1];
  __shared__ __attribute__((aligned(16))) float join[RPB > 1 ? (RPB - 1) * NV * LPR * 4 : 4];
  Exchange<LPR> exchange{red};
  const int lane = threadIdx.x % LPR, cols = a.cols, r = threadIdx.x / LPR;
  const long first = (long)blockIdx.x * RPB + r, stride = (long)gridDim.x * RPB;
  const long trips = (a.rows - (long)blockIdx.x * RPB + stride - 1) / stride;
  const float n = 1.0f / cols;
  auto at = [&](long t) { return row_index<LPR>(first + t * stride < a.rows ? first + t * stride : a.rows - 1); };
  f32x4 gm[NV], ag[NV], ab[NV];
  struct Rows2 {
    Row<TX, LPR, NV, TINY> x;
    Row<TY, LPR, NV, TINY> dy;
    float mu, rstd;
  } ring[AHEAD + 1];
  auto load = [&](Rows2& f, long row) {
    f.mu = a.mean[row];                                  // (first: both are needed for the row's first element)
    f.rstd = a.rstd[row];
    if constexpr (std::is_same<TX, Kept>::value) f.x.load(a.xq + row * a.blocks * Q8_BLOCK, a.xs + row * a.blocks, lane, a.blocks);
    else f.x.load(static_cast<const TX*>(a.x) + row * a.ldx, lane, cols);
    f.dy.load(static_cast<const TY*>(a.dy) + row * a.ldy, lane, cols);
  };
#pragma unroll
  for (int k = 0; k < AHEAD; ++k) load(ring[k], at(k));
  load_vector<LPR, NV, TINY>(gm, a.gamma, 1.f, lane, cols);
#pragma unroll
  for (int i = 0; i < NV; ++i) ag[i] = ab[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto one_row = [&](const Rows2& f, long t) {
    const bool live = first + t * stride < a.rows;
    const long row = at(t);
    f32x4 x[NV], dy[NV];
    float s1 = 0.f, s2 = 0.f;
    const float mu = f.rstd == 0.f ? 0.f : f.mu;         // (past fp32's range x - mu may be infinite, and 0 times it NaN)
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * LPR + lane) * 4;
      x[i] = (f.x.value(i, lane, cols) - mu) * f.rstd;
      if (i == NV - 1) x[i] = inside(x[i], c, cols);
      dy[i] = f.dy.value(i, lane, cols);
      if (live) {
        ag[i] += dy[i] * x[i];
        ab[i] += dy[i];
      }
      dy[i] = dy[i] * gm[i];
      s1 += sum4(dy[i]);
      s2 += dot4(dy[i], x[i]);
    }
    if (!a.dx) return;
    row_sums<LPR>(s1, s2, exchange);
    s1 *= n;
    s2 *= n;
#pragma unroll
    for (int i = 0; i < NV; ++i) x[i] = ((dy[i] - s1) - x[i] * s2) * f.rstd;
    if (live) store_row<TD, LPR, NV>(static_cast<TD*>(a.dx) + row * a.lddx, x, lane, cols);
  };
  for (long t = 0; t < trips; t += AHEAD + 1) {
#pragma unroll
    for (int k = 0; k <= AHEAD; ++k) {
      load(ring[(k + AHEAD) % (AHEAD + 1)], at(t + k + AHEAD));
      if (k == 0 || t + k < trips) one_row(ring[k], t + k);
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

// dgamma, dbeta from the blocks' partial sums: 16 columns and 64 runs of blocks per thread block
__global__ void __launch_bounds__(1024) norm_join_kernel(const float* partial, int n, int part_cols, int cols, float* dgamma, float* dbeta) {
  __shared__ float red[16][16];
  float* out = blockIdx.y ? dbeta : dgamma;
  if (!out) return;
  const int k = threadIdx.x & 15, c = blockIdx.x * 16 + k;
  float s = 0.f;
  if (c < cols) {
    const float* p = partial + blockIdx.y * part_cols + c;
#pragma unroll 8
    for (int b = threadIdx.x >> 4; b < n; b += 64) s += p[(long)b * 2 * part_cols];
  }
  s += __shfl_xor(s, 16, 64);
  s += __shfl_xor(s, 32, 64);
  if ((threadIdx.x & 63) < 16) red[threadIdx.x >> 6][k] = s;
  __syncthreads();
  if (threadIdx.x >= 16 || c >= cols) return;
#pragma unroll
  for (int w = 1; w < 16; ++w) s += red[w][k];
  out[c] = s;
}

// without rows
__global__ void __launch_bounds__(256) norm_zero_kernel(int cols, float* dgamma, float* dbeta) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= cols) return;
  if (dgamma) dgamma[c] = 0.f;
  if (dbeta) dbeta[c] = 0.f;
}

// Lanes per row and vectors per lane, by the row's length.  f(LPR, NV, TINY) is called with the three as types.
template <int V> using Int = std::integral_constant<int, V>;
template <int LPR, int LEAST, int MOST, typename F> hipError_t by_vectors(int cols, F f) {
  const int nv = (cols + 4 * LPR - 1) / (4 * LPR);         // no fewer than the row needs: only the last vector is ever cut off
  if constexpr (MOST > LEAST) if (nv < MOST) return by_vectors<LPR, LEAST, MOST - 1>(cols, f);
  return f(Int<LPR>{}, Int<MOST>{}, std::false_type{});
}
template <typename F> hipError_t by_width(int cols, F f) {
  if (cols < 4) return f(Int<16>{}, Int<1>{}, std::true_type{});
  if (cols <= 64) return by_vectors<16, 1, 1>(cols, f);
  if (cols <= 128) return by_vectors<32, 1, 1>(cols, f);
  if (cols <= 1024) return by_vectors<64, 1, 4>(cols, f);
  if (cols <= 4096) return by_vectors<256, 2, 4>(cols, f);
  if (cols <= 8192) return by_vectors<512, 3, 4>(cols, f);
  return by_vectors<1024, 3, 4>(cols, f);
}

// Blocks of a launch.  Forward 4 per CU (32768 x 1024, bf16: 23.3 us, with 6 24.7, with 16 26.1; 16384 x 4096 46.7, 47.1, 44.3).
// Backward 2 per CU, of more than 4 wavefronts 1 (2 and 3 of them, us: 32768 x 768, fp32 and bf16, 43.1, 44.0; 16384 x
// 4096, bf16, 83.9, 88.5; 1 and 2: 8192 x 8192 81.7, 89.5; 4096 x 16384 100, 113): each leaves a row of partial sums.
// Few rows, up to 8 trips, take one block, whose sums are final, and no second launch and workspace, for which the host takes
// longer than the block's trips: calls back to back, one block and as many as rows allow with a join, us, fp32: 64 x 64
// 12.6, 16.5; 32 x 1024 12.8, 16.8; 8 x 4096 12.6, 16.7; 4 x 16384 13.5, 16.7.  The other way round it is where 8 rows are
// as wide as they can be, 8 x 16384 24.1, 16.7, and in captured graphs, which hold the kernels' time alone: 64 x 64 4.8, 6.0;
// 128 x 64 6.1, 6.0; 2 x 16384 8.7, 11.1; 32 x 1024 9.9, 6.9; 8 x 4096 11.6, 6.9; 8 x 16384 24.6, 11.7.
constexpr int CUS = 256, FWD_BLOCKS = 4 * CUS, ONE_BLOCK_TRIPS = 8;
int backward_blocks(long rows, int threads, int rows_per_block) {
  const long want = (rows + rows_per_block - 1) / rows_per_block, most = threads > 256 ? CUS : 2 * CUS;
  if (want <= ONE_BLOCK_TRIPS) return 1;
  return (int)(want < most ? want : most);
}
int part_cols(int cols) { return (cols + 3) & ~3; }

template <typename TX, typename TY, typename TD> hipError_t backward(const NormBwdArgs& a, float* partial, hipStream_t st) {
  return by_width(a.cols, [&](auto lpr, auto nv, auto tiny) {
    constexpr int LPR = decltype(lpr)::value, NV = decltype(nv)::value, RPB = block_threads<LPR>() / LPR;
    const int blocks = backward_blocks(a.rows, block_threads<LPR>(), RPB), pc = part_cols(a.cols);
    hipLaunchKernelGGL((norm_backward_kernel<TX, TY, TD, LPR, NV, decltype(tiny)::value>), dim3(blocks), dim3(block_threads<LPR>()), 0, st, a,
                       blocks > 1 ? partial : nullptr, pc);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (blocks == 1 || (!a.dgamma && !a.dbeta)) return hipSuccess;
    hipLaunchKernelGGL(norm_join_kernel, dim3((a.cols + 15) / 16, 2), dim3(1024), 0, st, partial, blocks, pc, a.cols, a.dgamma, a.dbeta);
    return hipGetLastError();
  });
}

template <typename TX, typename TY> hipError_t forward(const NormFwdArgs& a, hipStream_t st) {
  return by_width(a.cols, [&](auto lpr, auto nv, auto tiny) {
    constexpr int LPR = decltype(lpr)::value, NV = decltype(nv)::value, RPB = block_threads<LPR>() / LPR;
    const long want = (a.rows + RPB - 1) / RPB;
    hipLaunchKernelGGL((norm_forward_kernel<TX, TY, LPR, NV, decltype(tiny)::value>), dim3((unsigned)(want < FWD_BLOCKS ? want : FWD_BLOCKS)),
                       dim3(block_threads<LPR>()), 0, st, a);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t launch_norm_forward(const NormFwdArgs& a, bool x_bf16, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  const double n = (double)a.rows * a.cols;
  ProfScope ps(PC_NORM_FWD, 8.0 * n, n * ((x_bf16 ? 2 : 4) + (a.y_bf16 ? 2 : 4)) + 33.0 * a.rows * a.blocks * ((a.xq != nullptr) + (a.yq != nullptr)), st);
  if (x_bf16) return a.y_bf16 ? forward<bf16, bf16>(a, st) : forward<bf16, float>(a, st);
  return a.y_bf16 ? forward<float, bf16>(a, st) : forward<float, float>(a, st);
}

size_t norm_backward_partial_floats(long rows, int cols) {
  if (rows <= 0) return 0;
  size_t blocks = 0;
  (void)by_width(cols, [&](auto lpr, auto, auto) {
    constexpr int LPR = decltype(lpr)::value;
    blocks = backward_blocks(rows, block_threads<LPR>(), block_threads<LPR>() / LPR);
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
  const double n = (double)a.rows * a.cols, ex = a.x_bf16 ? 2 : 4;
  ProfScope ps(PC_NORM_BWD, 14.0 * n, n * ((a.dx ? ex : 0) + (dy_bf16 ? 2 : 4)) + (a.xq ? 33.0 * a.rows * a.blocks : n * ex), st);
  if (a.xq && a.x_bf16) return dy_bf16 ? backward<Kept, bf16, bf16>(a, partial, st) : backward<Kept, float, bf16>(a, partial, st);
  if (a.xq) return dy_bf16 ? backward<Kept, bf16, float>(a, partial, st) : backward<Kept, float, float>(a, partial, st);
  if (a.x_bf16) return dy_bf16 ? backward<bf16, bf16, bf16>(a, partial, st) : backward<bf16, float, bf16>(a, partial, st);
  return dy_bf16 ? backward<float, bf16, float>(a, partial, st) : backward<float, float, float>(a, partial, st);
}

}  // namespace mg
