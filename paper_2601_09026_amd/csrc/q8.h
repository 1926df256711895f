// Rows kept in 8 bits.  A row is cut into blocks of 32 consecutive elements (the last one filled up with zeros); a block
// has one power of two 2^e, the smallest with max|x| < 127.5 * 2^e and e >= -126, and its elements are
// q = round_half_even(x * 2^-e), -127 <= q <= 127; they stand for q * 2^e.  Kept are q as int8, [rows, 32 * blocks], and
// e + 127 as a byte, [rows, blocks].  A block that holds a NaN, an infinity or the last half percent below it (127.5 * 2^121
// and more, which could round to 2^128) has the byte 255 (and q = 0) and stands for 32 NaNs.
// Why a power of two and not max / 127: x * 2^-e is exact, so that the rounding to q is the only one and every
// implementation finds the same q; and q * 2^e, 7 bits and a sign, is a bf16 number as it is, so that the matrix cores
// take kept rows without a further rounding.  It costs 0.4 bits on average.  The error is at most 2^(e-1), between
// max / 255 and max / 127 over the block.
#pragma once
#include "common.h"

namespace mg {

constexpr int Q8_BLOCK = 32;
__host__ __device__ inline long q8_blocks(long cols) { return (cols + Q8_BLOCK - 1) / Q8_BLOCK; }

// Vectors at addresses that are aligned to their elements only (rows of odd lengths, slices of wider rows); global
// memory takes such accesses in one instruction on this target.
typedef float f32x4_u __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned u32x2_u __attribute__((ext_vector_type(2), aligned(2)));
typedef unsigned u32x4_u __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bits_f(unsigned v) { return __builtin_bit_cast(float, v); }
__device__ __forceinline__ unsigned f_bits(float v) { return __builtin_bit_cast(unsigned, v); }

// 4 elements at any element address
template <typename T> __device__ __forceinline__ f32x4 load4u(const T* p);
template <> __device__ __forceinline__ f32x4 load4u<float>(const float* p) {
  typedef const __attribute__((address_space(1))) f32x4_u* gptr;
  const f32x4_u v = *(gptr)p;
  return f32x4{v[0], v[1], v[2], v[3]};
}
template <> __device__ __forceinline__ f32x4 load4u<bf16>(const bf16* p) {
  typedef const __attribute__((address_space(1))) u32x2_u* gptr;
  const u32x2_u v = *(gptr)p;
  return f32x4{bits_f(v[0] << 16), bits_f(v[0] & 0xffff0000u), bits_f(v[1] << 16), bits_f(v[1] & 0xffff0000u)};
}
template <typename T> __device__ __forceinline__ void store4u(T* p, f32x4 v);
template <> __device__ __forceinline__ void store4u<float>(float* p, f32x4 v) {
  typedef __attribute__((address_space(1))) f32x4_u* gptr;
  *(gptr)p = f32x4_u{v[0], v[1], v[2], v[3]};
}
template <> __device__ __forceinline__ void store4u<bf16>(bf16* p, f32x4 v) {
  typedef __attribute__((address_space(1))) u32x2_u* gptr;
  const bf16x4 b = {(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
  const u32x2 u = __builtin_bit_cast(u32x2, b);
  *(gptr)p = u32x2_u{u[0], u[1]};
}

// The 4 elements of a row from column c on, zeros past its `cols` elements.  Without a branch around the load: it starts at
// the last 4 elements at the latest and what it found is moved to its place.  (cols < 4: one by one.)
template <typename T> __device__ __forceinline__ f32x4 load4_row(const T* row, int c, int cols) {
  if (cols < 4) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < 3; ++j)
      if (c + j < cols) v[j] = to_f(row[c + j]);
    return v;
  }
  return load4u<T>(row + (c < cols - 4 ? c : cols - 4));
}
// (after load4_row, where the 4 elements may reach past the row's end)
__device__ __forceinline__ f32x4 settle4(f32x4 v, int c, int cols) {
  if (cols < 4) return v;
  const int past = 4 - (cols - c);                        // elements past the end (c + 4 can pass 32 bits)
  f32x4 r = v;
  r = past & 1 ? f32x4{r[1], r[2], r[3], 0.f} : r;
  r = past & 2 ? f32x4{r[2], r[3], 0.f, 0.f} : r;
  r = past >= 4 ? f32x4{0.f, 0.f, 0.f, 0.f} : r;
  return past > 0 ? r : v;
}
// stores those of the 4 elements that lie inside the row (its length is at most 2^31 - 1, so c + 4 can pass 32 bits; c + 3
// cannot, and neither can the difference)
template <typename T> __device__ __forceinline__ void store4_row(T* row, int c, int cols, f32x4 v) {
  if (cols - c >= 4) {
    store4u<T>(row + c, v);
  } else {
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (c + j < cols) row[c + j] = from_f<T>(v[j]);
  }
}

// a value from another lane of the row of 16 (DPP control), all lanes of the 16 being active
template <int CTRL> __device__ __forceinline__ unsigned lane_move(unsigned v) {
  return (unsigned)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true);
}
constexpr int LANE_XOR1 = 0xB1, LANE_XOR2 = 0x4E, LANE_MIRROR8 = 0x141, LANE_MIRROR16 = 0x140;

// Quantisation of a block of 32 elements that lie in 8 consecutive lanes, 4 in each.  Returns the lane's 4 bytes; `scale`
// is the block's byte, the same in its 8 lanes.
// The order of magnitudes is that of their bits (0x7f7f0000: 127.5 * 2^121), NaN above infinity.  Adding 0x10000 carries into the exponent from
// 127.5 / 64 = 1.9921875 on.  x * 2^-e + 1.5 * 2^23 rounds to an integer, ties to even, and has it in its lowest byte.
__device__ __forceinline__ unsigned q8_quantise(f32x4 v, unsigned& scale) {
  unsigned top = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const unsigned b = f_bits(v[j]) & 0x7fffffffu;
    top = b > top ? b : top;
  }
  auto most = [&](unsigned o) { top = o > top ? o : top; };
  most(lane_move<LANE_XOR1>(top));
  most(lane_move<LANE_XOR2>(top));
  most(lane_move<LANE_MIRROR8>(top));
  const bool finite = top < 0x7f7f0000u;
  int e = (int)((top + 0x10000u) >> 23) - 6;
  e = e > 1 ? e : 1;
  scale = finite ? (unsigned)e : 255u;
  const float inv = bits_f((unsigned)(254 - e) << 23);   // (not used where the block is not finite)
  unsigned w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = f_bits(fmaf(v[j], inv, 12582912.0f));
  const unsigned lo = __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(w[3], w[2], 0x04000c0cu);
  return finite ? lo | hi : 0u;
}

// 2^e of a block's byte; infinity for 255, so that 0 * 2^e is NaN
__device__ __forceinline__ float q8_step(unsigned scale) { return bits_f(scale << 23); }
// the 4 values that 4 bytes stand for
__device__ __forceinline__ f32x4 q8_values(unsigned q, float step) {
  return f32x4{(float)(signed char)(q & 0xff) * step, (float)(signed char)(q >> 8 & 0xff) * step,
               (float)(signed char)(q >> 16 & 0xff) * step, (float)(signed char)(q >> 24) * step};
}

// n / d for 0 <= n < 2^31 by a multiplication
struct Divisor {
  unsigned d, mul, shift;
  explicit Divisor(unsigned div) : d(div) {
    shift = 0;
    while (shift < 31 && (1u << shift) < div) ++shift;
    mul = (unsigned)(((1ull << 32) * ((1ull << shift) - div)) / div + 1);
  }
  __device__ __forceinline__ unsigned quotient(unsigned n) const { return (__umulhi(mul, n) + n) >> shift; }
};

}  // namespace mg
