// Rows to 8 bits and back (q8.h has the format).  Both kernels move their bytes and wait for them: per element 4 or 2
// bytes on the wide side, 33/32 on the narrow one.  528384 x 768, fp32: to 8 bits 387 us, 5.3 TB/s, and back 332 us, 6.2 TB/s
// (a copy reaches 5.7); 1088 x 64: 2.7 and 2.9 us.
#include "kernels.h"
#include "prof.h"
#include "q8.h"

namespace mg {
namespace {

// Threads take 4 elements each, 8 lanes a block of 32, so that a wavefront's accesses are contiguous on both sides.  A thread
// block takes TILE blocks, ITER loads in flight per thread.  (Rows are not walked: nothing of one is needed by the next.)
constexpr int ITER = 4, TILE = 32 * ITER;

// The rows are one run of whole blocks (FLAT: whole rows of a multiple of 32 elements, one behind the other), or a block's
// row is found by a division.
template <bool FLAT> struct Place {
  long row; int c;                                       // FLAT: row 0, c unused
  __device__ Place(unsigned b, const Divisor& per_row) {
    row = FLAT ? 0 : per_row.quotient(b);
    c = FLAT ? 0 : (int)(b - (unsigned)row * per_row.d) * Q8_BLOCK;
  }
};

template <typename T, bool FLAT>
__global__ void __launch_bounds__(256) q8_pack_kernel(const T* __restrict__ x, long ldx, int cols, Divisor per_row,
                                                      unsigned blocks, unsigned* __restrict__ q,
                                                      unsigned char* __restrict__ scale) {
  const unsigned b0 = blockIdx.x * TILE + (threadIdx.x >> 3);
  const int sub = (threadIdx.x & 7) * 4;
  f32x4 v[ITER];
  int c[ITER];
#pragma unroll
  for (int i = 0; i < ITER; ++i) {
    const unsigned b = b0 + 32 * i < blocks ? b0 + 32 * i : blocks - 1;
    const Place<FLAT> p(b, per_row);
    c[i] = p.c + sub;
    v[i] = FLAT ? load4u<T>(x + (long)b * Q8_BLOCK + sub) : load4_row<T>(x + p.row * ldx, c[i], cols);
  }
#pragma unroll
  for (int i = 0; i < ITER; ++i) {
    if constexpr (!FLAT) v[i] = settle4(v[i], c[i], cols);
    unsigned s;
    const unsigned w = q8_quantise(v[i], s);
    const long b = (long)b0 + 32 * i;
    if (b < blocks) {
      q[b * 8 + (threadIdx.x & 7)] = w;
      if ((threadIdx.x & 7) == 0) scale[b] = (unsigned char)s;
    }
  }
}

template <typename T, bool FLAT>
__global__ void __launch_bounds__(256) q8_unpack_kernel(const unsigned* __restrict__ q,
                                                        const unsigned char* __restrict__ scale, int cols,
                                                        Divisor per_row, unsigned blocks, T* __restrict__ x, long ldx,
                                                        long src_group, long dst_group) {
  const unsigned b0 = blockIdx.x * TILE + (threadIdx.x >> 3);
  const int sub = (threadIdx.x & 7) * 4;
  q += blockIdx.y * src_group * 8;                       // (signed: groups may go backwards)
  scale += blockIdx.y * src_group;
  x += blockIdx.y * dst_group;
  unsigned w[ITER], s[ITER];
#pragma unroll
  for (int i = 0; i < ITER; ++i) {
    const unsigned b = b0 + 32 * i < blocks ? b0 + 32 * i : blocks - 1;
    w[i] = q[(long)b * 8 + (threadIdx.x & 7)];
    s[i] = scale[b];
  }
#pragma unroll
  for (int i = 0; i < ITER; ++i) {
    const unsigned b = b0 + 32 * i;
    if (b >= blocks) return;
    const f32x4 v = q8_values(w[i], q8_step(s[i]));
    if constexpr (FLAT) {
      store4u<T>(x + (long)b * Q8_BLOCK + sub, v);
    } else {
      const Place<FLAT> p(b, per_row);
      store4_row<T>(x + p.row * ldx, p.c + sub, cols, v);
    }
  }
}

// a launch takes at most this many blocks: their index has 32 bits, and so has the division's numerator
constexpr long MOST_BLOCKS = 1l << 30;

template <typename T>
hipError_t pack(const Q8Rows& r, const T* x, long ldx, hipStream_t st) {
  const long per_row = q8_blocks(r.cols), chunk = MOST_BLOCKS / per_row;
  const bool flat = r.cols % Q8_BLOCK == 0 && (ldx == r.cols || r.rows == 1);
  for (long row = 0; row < r.rows; row += chunk) {
    const long n = r.rows - row < chunk ? r.rows - row : chunk;
    const unsigned blocks = (unsigned)(n * per_row), grid = (blocks + TILE - 1) / TILE;
    unsigned* q = reinterpret_cast<unsigned*>(r.q) + row * per_row * 8;
    unsigned char* s = r.scale + row * per_row;
    const Divisor div((unsigned)per_row);
    if (flat) hipLaunchKernelGGL((q8_pack_kernel<T, true>), dim3(grid), dim3(256), 0, st, x + row * ldx, ldx, r.cols, div, blocks, q, s);
    else hipLaunchKernelGGL((q8_pack_kernel<T, false>), dim3(grid), dim3(256), 0, st, x + row * ldx, ldx, r.cols, div, blocks, q, s);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T>
hipError_t unpack(const Q8Rows& r, T* x, long ldx, int groups, long src_rows, long dst_rows, hipStream_t st) {
  const long per_row = q8_blocks(r.cols), chunk = MOST_BLOCKS / per_row;
  const bool flat = r.cols % Q8_BLOCK == 0 && (ldx == r.cols || r.rows == 1);
  for (long row = 0; row < r.rows; row += chunk) {
    const long n = r.rows - row < chunk ? r.rows - row : chunk;
    const unsigned blocks = (unsigned)(n * per_row);
    const dim3 grid((blocks + TILE - 1) / TILE, groups);
    const unsigned* q = reinterpret_cast<const unsigned*>(r.q) + row * per_row * 8;
    const unsigned char* s = r.scale + row * per_row;
    const Divisor div((unsigned)per_row);
    if (flat) hipLaunchKernelGGL((q8_unpack_kernel<T, true>), grid, dim3(256), 0, st, q, s, r.cols, div, blocks, x + row * ldx, ldx, src_rows * per_row, dst_rows * ldx);
    else hipLaunchKernelGGL((q8_unpack_kernel<T, false>), grid, dim3(256), 0, st, q, s, r.cols, div, blocks, x + row * ldx, ldx, src_rows * per_row, dst_rows * ldx);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_q8_pack(const Q8Rows& r, const void* x, long ldx, bool is_bf16, hipStream_t st) {
  if (r.rows <= 0) return hipSuccess;
  const double n = (double)r.rows * r.cols;
  ProfScope ps(PC_Q8, 0.0, n * (is_bf16 ? 2 : 4) + 33.0 * r.rows * q8_blocks(r.cols), st);
  return is_bf16 ? pack<bf16>(r, static_cast<const bf16*>(x), ldx, st) : pack<float>(r, static_cast<const float*>(x), ldx, st);
}

hipError_t launch_q8_unpack(const Q8Rows& r, void* x, long ldx, bool is_bf16, int groups, long src_rows, long dst_rows,
                            hipStream_t st) {
  if (r.rows <= 0 || groups <= 0) return hipSuccess;
  const double n = (double)r.rows * r.cols;
  ProfScope ps(PC_Q8, 0.0, groups * (n * (is_bf16 ? 2 : 4) + 33.0 * r.rows * q8_blocks(r.cols)), st);
  return is_bf16 ? unpack<bf16>(r, static_cast<bf16*>(x), ldx, groups, src_rows, dst_rows, st)
                 : unpack<float>(r, static_cast<float*>(x), ldx, groups, src_rows, dst_rows, st);
}

}  // namespace mg
