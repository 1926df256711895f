// Gradients of a linear map y = x W^T + b whose input rows were kept in 8 bits:
//   dW[m,n] = scale * sum_t dY[t,m] x~[t,n],   db[m] = scale * sum_t dY[t,m]
// A kept value is 7 bits and a sign times a power of two, so it is a bf16 number as it is; a bf16 dY is one as well, and an
// fp32 dY is exactly the sum of three of 8 bits each (cut, not rounded: hi = its upper 16 bits, then the same of the rest,
// then what is left; bits below 2^-133, bf16's last, are lost).  So the products run on the bf16 matrix cores, one or three of
// them, without any rounding of an operand, and the sums are fp32 either way: what differs from an fp32 product is only the
// order of the additions.
// Bound by the matrix cores (2 T M N flops, or three times that).  16384 tokens, 4096 x 4096, bf16: 482 us, 1140 TFLOP/s, where
// the library's product of bf16 operands in this order reaches 1150; 8192 tokens, 4096 x 2048, fp32: 346 us, 397 TFLOP/s (1190
// of bf16 products; the fp32 matrix cores' own limit is 157).
//
// Both operands are token-major and the reduction runs over the tokens, so the tiles are staged as they lie in memory
// ([token][feature], bf16) and the fragments come out of LDS through the transposing read; rows of a tile keep their
// 16-byte chunks XOR-swizzled by the row.  Global loads go to registers two tiles ahead; between there and LDS the kept rows
// become bf16 (2.5 instructions per element, once per tile and not per fragment) and an fp32 dY its three parts.  What
// paid, at 16384 x 4096 x 4096 in bf16: one tile of LDS stored before another is multiplied 721 us; stores, loads and
// fragment reads between the products 731 (spilling); conversions and addresses of fewer instructions 508; wavefronts of
// 64 x 128 instead of 128 x 64 in the block 495; db from the registers on their way to LDS and not from the fragments, shared
// out over the columns of tiles, 503 -> 484 on another card.  What is left: 910 k cycles of an XCD, whatever the card's clock
// under this load (506 us at 1.80 GHz with the counters on, 539 at 1.69 on another card; 482 us are 1.89), of which the matrix
// cores are busy for 58 %, LDS for 43 %; wavefronts wait for a slot to issue in for 40 % of theirs and
// for data or the barrier for 25 %.  Loads that are waited for one by one and not at a tile's start gained nothing, nor did a swizzle that spreads the kept
// rows' stores over all banks, a sixth of the LDS cycles less.  The conversions cost 511 -> 491 us for the kept rows (values wrong
// without), and with fp32, 8192 x 4096 x 2048, 370 -> 346, and 313 without the parts of dY; a pass that did them beforehand would
// take 36 us for its bytes in the one case, 58 in the other.  Rows of dY at odd addresses cost 3 to 12 % (16384 x 4095 x 4096;
// 4096 x 50257 x 768, aligned to 2, 4, 8 and 16 bytes, on a slow card: 398, 385, 362, 355 us; on others the first takes 343 to 358).
#include <climits>
#include <type_traits>

#include "kernels.h"
#include "lds_limit.h"
#include "prof.h"
#include "q8.h"

namespace mg {
namespace {

template <int V> using Int = std::integral_constant<int, V>;

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
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 8; j += 2) top = fmaxf(top, fmaxf(fabsf(at(j)), fabsf(at(j + 1))));
    float mid[8], lo[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) mid[j] = at(j) - cut(at(j));
    if (__builtin_expect(__builtin_isinf(top), 0)) {      // an infinity has no rest (a NaN's is one)
#pragma unroll
      for (int j = 0; j < 8; ++j) mid[j] = __builtin_isinf(at(j)) ? 0.f : mid[j];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) lo[j] = mid[j] - cut(mid[j]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      out[0][j] = upper(at(2 * j), at(2 * j + 1));
      out[1][j] = upper(mid[2 * j], mid[2 * j + 1]);
      out[2][j] = upper(lo[2 * j], lo[2 * j + 1]);
    }
  }
};

// byte I of a word, signed, as a float (the compiler takes two instructions for it)
template <int I> __device__ __forceinline__ float signed_byte(unsigned v) {
  float f;
  if constexpr (I == 0) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(f) : "v"(v));
  if constexpr (I == 1) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(f) : "v"(v));
  if constexpr (I == 2) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(f) : "v"(v));
  if constexpr (I == 3) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(f) : "v"(v));
  return f;
}
// 4 kept elements as bf16
__device__ __forceinline__ u32x2 kept_bf16(unsigned q, float step) {
  return u32x2{upper(signed_byte<0>(q) * step, signed_byte<1>(q) * step), upper(signed_byte<2>(q) * step, signed_byte<3>(q) * step)};
}

// A thread's sums of db carry their errors, but for the largest bf16 tile, which has no 8 registers left for them.  Values of 8
// bits lose little: 16384 tokens, 4096 x 4096, 3.7e-8 of db's size (chains of 16 tiles of 64 tokens), 131072 tokens 4.8e-8 (128),
// and with one column of tiles, 65536 tokens, 65536 x 200, 6.4e-8 (1024), at worst 1.7e-7 of an element whose terms have one
// sign.  Half a step of fp32 is 6e-8.
struct PlainSum {
  float sum = 0.f;
  __device__ __forceinline__ void add(float x) { sum += x; }
};

// The work of a launch: `whole` tiles in one piece, then `rest` tiles of `slices` slices each.  Blocks go to the 8 XCDs in
// turn; each XCD takes a contiguous run of either kind, so that what it works on at a time shares panels of the operands in
// its L2.
struct Items {
  int whole, rest, slices, whole_xcd, rest_xcd;
  Items(int tiles, int w, int s) : whole(w), rest(tiles - w), slices(s), whole_xcd((w + 7) / 8), rest_xcd((int)(((long)rest * s + 7) / 8)) {}
  int blocks() const { return 8 * (whole_xcd + rest_xcd); }
  __device__ bool item(int block, int& tile, int& slice) const {
    const int xcd = block & 7, i = block >> 3;
    slice = 0;
    if (i < whole_xcd) {
      tile = xcd * whole_xcd + i;
      return tile < whole;
    }
    const int k = xcd * rest_xcd + i - whole_xcd;
    tile = __builtin_amdgcn_readfirstlane(k / slices);
    slice = k - tile * slices;
    tile += whole;
    return k < rest * slices;
  }
};

template <typename T, int BM, int BN, int BK, int WM, int WN, int OCC>
__global__ void __launch_bounds__(64 * WM * WN, OCC * WM * WN / 4)
q8_grad_kernel(const Q8GradArgs a, int tiles_n, Items it, float* partial, float* column) {
  constexpr int NT = 64 * WM * WN, PARTS = std::is_same<T, float>::value ? 3 : 1;
  constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 32, TN = WTN / 32;
  constexpr int RA = BM * 2, RB = BN * 2;                // bytes per LDS row
  constexpr int A_BYTES = BK * RA, B_BYTES = BK * RB, STAGE = PARTS * A_BYTES + B_BYTES;
  constexpr int BE = BK * BN >= 16 * NT ? 16 : 8;          // kept elements per chunk
  constexpr int A_CH = BK * BM / 8 / NT, B_CH = BK * BN / BE / NT, JOBS = A_CH + B_CH;
  static_assert(A_CH * NT * 8 == BK * BM && B_CH * NT * BE == BK * BN && NT % (BM / 8) == 0, "tile / thread split");
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  int tile, sp;
  if (!it.item(blockIdx.x, tile, sp)) return;
  const int splits = tile < it.whole ? 1 : it.slices;
  const int tm = __builtin_amdgcn_readfirstlane(tile / tiles_n), tn = tile - tm * tiles_n;
  const int m0 = tm * BM, n0 = tn * BN, M = a.M, N = a.N, NP = a.blocks * Q8_BLOCK;
  const int all_tiles = (int)((a.rows + BK - 1) / BK);
  const int kt0 = (int)((long)all_tiles * sp / splits), KT = (int)((long)all_tiles * (sp + 1) / splits) - kt0;
  const long first = (long)kt0 * BK;
  const int K = (int)(first + (long)KT * BK < a.rows ? (long)KT * BK : a.rows - first);     // tokens of the slice
  const T* A = static_cast<const T*>(a.dy) + first * a.ldy + m0;
  const unsigned char* Q = a.xq + first * NP + n0;
  const unsigned char* S = a.xs + first * a.blocks + n0 / Q8_BLOCK;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wm0 = (wave / WN) * WTM, wn0 = (wave % WN) * WTN;
  auto swz_of = [](int row_bytes, int r) { return row_bytes >= 256 ? (r & 3) << 2 : ((r >> 1) & 1) << 2; };

  // This thread's chunks of a tile: chunk j lies j * (rows of a pass) tokens below chunk 0.  A tile's base is uniform, a
  // thread's place in it has 32 bits.
  constexpr int A_ROWS = NT / (BM / 8), B_ROWS = NT / (BN / BE);
  const int ar = threadIdx.x / (BM / 8), ac = threadIdx.x % (BM / 8) * 8;
  const int br = threadIdx.x / (BN / BE), bc = threadIdx.x % (BN / BE) * BE;
  Chunk<T> ra[A_CH];
  unsigned rq[B_CH][BE / 4], rs[B_CH];
  // (chunks past the last feature read the tile's first one instead: their columns are never stored)
  const int ac_in = m0 + ac < M ? ac : 0, bc_in = n0 + bc < NP ? bc : 0;
  const unsigned va = (unsigned)(ar * a.ldy + ac_in), vq = (unsigned)(br * NP + bc_in), vs = (unsigned)(br * a.blocks + bc_in / Q8_BLOCK);
  auto load = [&](auto whole, int j, int kt) {            // job j of tile kt
    const int k0 = kt * BK;
    if (j < A_CH) {
      const T* p = A + (long)(k0 + j * A_ROWS) * a.ldy;
      if constexpr (decltype(whole)::value) {
        ra[j < A_CH ? j : 0].load(p + va);
      } else {                                            // zeros past the last token
        Chunk<T>& c = ra[j < A_CH ? j : 0];
        const int n = k0 + ar + j * A_ROWS < K ? M - m0 - ac_in : 0;
        if (n >= 8) c.load(p + va);
        else c.load_some(p + va, n);
      }
    } else {
      const int i = j - A_CH < 0 ? 0 : j - A_CH;
      const unsigned char *q = Q + (long)(k0 + i * B_ROWS) * NP, *s = S + (long)(k0 + i * B_ROWS) * a.blocks;
      bool there = true;
      if constexpr (!decltype(whole)::value) there = k0 + br + i * B_ROWS < K;
#pragma unroll
      for (int e = 0; e < BE / 4; ++e) rq[i][e] = 0;
      rs[i] = 127;
      if (there) {
        if constexpr (BE == 16) {
          const u32x4 v = *reinterpret_cast<const u32x4*>(q + vq);
#pragma unroll
          for (int e = 0; e < 4; ++e) rq[i][e] = v[e];
        } else {
          const u32x2 v = *reinterpret_cast<const u32x2*>(q + vq);
          rq[i][0] = v[0]; rq[i][1] = v[1];
        }
        rs[i] = s[vs];
      }
    }
  };
  auto store = [&](int j, int stage) {
    unsigned char* base = smem + stage * STAGE;
    if (j < A_CH) {
      const int row = ar + j * A_ROWS, at = row * RA + (((ac >> 3) ^ swz_of(RA, row)) << 4);
      u32x4 p[PARTS];
      ra[j < A_CH ? j : 0].parts(p);
#pragma unroll
      for (int i = 0; i < PARTS; ++i) *reinterpret_cast<u32x4*>(base + i * A_BYTES + at) = p[i];
    } else {
      const int i = j - A_CH < 0 ? 0 : j - A_CH;
      const int row = br + i * B_ROWS;
      const float step = q8_step(rs[i]);
#pragma unroll
      for (int e = 0; e < BE / 8; ++e) {
        const int at = PARTS * A_BYTES + row * RB + ((((bc >> 3) + e) ^ swz_of(RB, row)) << 4);
        const u32x2 lo = kept_bf16(rq[i][2 * e], step), hi = kept_bf16(rq[i][2 * e + 1], step);
        *reinterpret_cast<u32x4*>(base + at) = u32x4{lo[0], lo[1], hi[0], hi[1]};
      }
    }
  };
  // dY is added up as well, as it lies in the registers between memory and LDS: all of a thread's chunks have the same 8
  // features.  With `column`, every column of tiles takes its share of the token tiles and leaves its sums there; else the first
  // one takes them all.
  const bool sums = a.db && (column || tn == 0);
  const int share = column ? tiles_n : 1;
  int due = !sums ? INT_MIN : column ? tn : 0;            // the next token tile of the share, counted from the slice's first
  if (sums && kt0) {                                      // (a row of tiles may have whole ones and slices: shares are of all tokens)
    const int at = __builtin_amdgcn_readfirstlane(kt0 % share);
    due += due < at ? share - at : -at;
  }
  typename std::conditional<(BM < 256), CarrySum, PlainSum>::type total[8];
  auto add_tile = [&] {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float t = ra[0].at(e);
#pragma unroll
      for (int j = 1; j < A_CH; ++j) t += ra[j].at(e);
      total[e].add(t);
    }
    due += share;
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

  // A tile is STEPS steps of NM products each: 16 tokens and one part of dY.  During a step the next one's fragments are
  // read.  The next tile's chunks go to the other stage during all steps but the last, the registers that held them are
  // loaded again (for the tile after that) right behind; the last step begins with the block's barrier and reads the next
  // tile's first fragments.
  constexpr int KS = BK / 16, STEPS = KS * PARTS, NM = TM * TN, SLOTS = (STEPS - 1) * NM;
  static_assert(STEPS >= 2, "a step to hand over in");
  TrFrag fa[2][TM], fb[2][TN];
  auto read_a = [&](auto step, unsigned stage_off, int i) {
    constexpr int s = decltype(step)::value, ks = s / PARTS, part = PARTS - 1 - s % PARTS;
    tr_read<part * A_BYTES + 16 * ks * RA, part * A_BYTES + (16 * ks + 4) * RA>(fa[s & 1][i], lds0 + stage_off + offa[i]);
  };
  auto read_b = [&](auto step, unsigned stage_off, int j) {
    constexpr int s = decltype(step)::value, ks = s / PARTS;
    tr_read<16 * ks * RB, (16 * ks + 4) * RB>(fb[ks & 1][j], lds0 + stage_off + offb[j]);
  };
  auto run_step = [&](auto step, auto jobs, auto whole, unsigned read_off, int nxt, int kt) {
    constexpr int s = decltype(step)::value, ks = s / PARTS, r = (s + 1) % STEPS;
    constexpr int RD = TM + (r % PARTS == 0 ? TN : 0);
    bf16x8 xa[TM], xb[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) xa[i] = tr_value(fa[s & 1][i]);
#pragma unroll
    for (int j = 0; j < TN; ++j) xb[j] = tr_value(fb[ks & 1][j]);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 0; q < NM; ++q) {
      const int i = q / TN, j = q % TN;
      acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xb[j], xa[i], acc[i][j], 0, 0, 0);
      const int r0 = (q * RD * 4 / 3 + NM - 1) / NM, r1 = ((q + 1) * RD * 4 / 3 + NM - 1) / NM;
#pragma unroll
      for (int u = 0; u < RD; ++u)
        if (u >= r0 && (u < r1 || q == NM - 1)) {
          if (u < TM) read_a(Int<r>{}, read_off, u < TM ? u : 0);
          else read_b(Int<r>{}, read_off, u < TM ? 0 : u - TM);
        }
      if constexpr (decltype(jobs)::value) {
        if (s == 0 && q == 0 && kt + 1 == due) add_tile();
        const int slot = s * NM + q;
#pragma unroll
        for (int u = 0; u < JOBS; ++u)
          if (u * SLOTS / JOBS == slot) {
            store(u, nxt);
            if (decltype(whole)::value || kt + 2 < KT) load(whole, u, kt + 2);
          }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  int cur = 0;
  auto tile_step = [&](auto jobs, auto whole, int kt) {
    const unsigned so = cur * STAGE, sn = (cur ^ 1) * STAGE;
    auto go = [&](auto self, auto step) {
      constexpr int s = decltype(step)::value;
      if constexpr (s < STEPS - 1) {
        run_step(step, jobs, whole, so, cur ^ 1, kt);
        self(self, Int<s + 1>{});
      } else {
        wait_lgkm();
        bare_barrier();
        run_step(step, std::false_type{}, whole, sn, cur ^ 1, kt);
      }
    };
    go(go, Int<0>{});
    cur ^= 1;
  };
  auto every_load = [&](int kt) {
#pragma unroll
    for (int j = 0; j < JOBS; ++j) load(std::false_type{}, j, kt);
  };
  every_load(0);
  if (due == 0) add_tile();
#pragma unroll
  for (int j = 0; j < JOBS; ++j) store(j, 0);
  if (KT > 1) every_load(1);
  wait_lgkm();
  bare_barrier();
#pragma unroll
  for (int i = 0; i < TM; ++i) read_a(Int<0>{}, 0, i);
#pragma unroll
  for (int j = 0; j < TN; ++j) read_b(Int<0>{}, 0, j);
  // Whole tiles are loaded without a test: those that end before the last token, and, where a chunk reaches past the last
  // feature into the next token's row, before the tokens behind which there are not 7 more elements.
  const long safe = m0 + BM <= M || M % 8 == 0 ? a.rows : a.rows - (7 + a.ldy - 1) / a.ldy;
  const int whole_tiles = (int)((safe - first < K ? safe - first : K) / BK);
  int kt = 0;
  for (; kt + 2 < whole_tiles; ++kt) tile_step(std::true_type{}, std::true_type{}, kt);
  for (; kt + 1 < KT; ++kt) tile_step(std::true_type{}, std::false_type{}, kt);
  if (KT > 0) tile_step(std::false_type{}, std::false_type{}, kt);
  wait_lgkm();
  bare_barrier();
  // a slice's sums go unscaled to the scratch, [BM x BN | BM] per slice of a tile
  float scale = a.scale, *part = nullptr;
  if (splits > 1) {
    part = partial + (long)((tile - it.whole) * splits + sp) * (BM * BN + BM);
    scale = 1.f;
  }
  if (sums) {                                             // block-uniform
    float* red = reinterpret_cast<float*>(smem);          // [A_ROWS][BM]
#pragma unroll
    for (int e = 0; e < 8; ++e) red[ar * BM + ac + e] = total[e].sum;
    __syncthreads();
    for (int m = threadIdx.x; m < BM && m0 + m < M; m += NT) {
      CarrySum t;
#pragma unroll
      for (int g = 0; g < A_ROWS; ++g) t.add(red[g * BM + m]);
      if (part) part[BM * BN + m] = t.sum;
      else if (column) column[(long)tile * BM + m] = t.sum;
      else a.db[m0 + m] = scale * t.sum;
    }
  }
  // a lane holds 4 consecutive columns of one row at a time
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int m = wm0 + 32 * i + (lane & 31);
    if (m0 + m >= M) continue;
    float* out = part ? part + m * BN - n0 : a.dW + (long)(m0 + m) * N;
    const int stop = part ? n0 + BN : N;
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int n = n0 + wn0 + 32 * j + 8 * q + 4 * lh;
        const f32x4 v = {scale * acc[i][j][4 * q], scale * acc[i][j][4 * q + 1], scale * acc[i][j][4 * q + 2], scale * acc[i][j][4 * q + 3]};
        if (n < N) store4_row<float>(out, n, stop, v);
      }
  }
}

// The tiles that were cut into slices: the slices' sums, in order, 1024 elements of a tile per block.  Blocks behind those add
// up db: 16 features each, their columns of tiles and slices in 16 runs.
__global__ void __launch_bounds__(256) q8_grad_join_kernel(const Q8GradArgs a, const float* partial, const float* column, int whole, int rest, int slices, int BM, int BN, int tiles_n) {
  const long each = (long)BM * BN + BM;
  if ((int)blockIdx.y >= rest) {
    __shared__ float red[16][16];
    const int k = threadIdx.x & 15, run = threadIdx.x >> 4;
    const long blocks = (long)(gridDim.y - rest) * gridDim.x;
    for (long b = ((long)blockIdx.y - rest) * gridDim.x + blockIdx.x; b * 16 < a.M; b += blocks) {
      const long m = b * 16 + k;
      CarrySum t;
      if (m < a.M) {
        const int tm = (int)(m / BM), r = (int)(m - (long)tm * BM);
#pragma unroll 4
        for (int p = run; p < tiles_n * slices; p += 16) {
          const int tn = p / slices, s = p - tn * slices, tile = tm * tiles_n + tn;
          if (tile >= whole) t.add(partial[((long)(tile - whole) * slices + s) * each + BM * BN + r]);
          else if (s == 0) t.add(column[(long)tile * BM + r]);
        }
      }
      __syncthreads();
      red[run][k] = t.sum;
      __syncthreads();
      if (run == 0 && m < a.M) {
#pragma unroll
        for (int i = 1; i < 16; ++i) t.add(red[i][k]);
        a.db[m] = a.scale * t.sum;
      }
    }
    return;
  }
  const int tile = whole + blockIdx.y, tm = tile / tiles_n, tn = tile - tm * tiles_n;
  const float* p = partial + (long)blockIdx.y * slices * each;
  const int e = (blockIdx.x * 256 + threadIdx.x) * 4, r = e / BN, m = tm * BM + r, n = tn * BN + e - r * BN;
  if (m >= a.M || n >= a.N) return;
  CarrySum acc[4];
#pragma unroll 4
  for (int s = 0; s < slices; ++s) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(p + s * each + e);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i].add(v[i]);
  }
  store4_row<float>(a.dW + (long)m * a.N, n, a.N, a.scale * f32x4{acc[0].sum, acc[1].sum, acc[2].sum, acc[3].sum});
}

__global__ void __launch_bounds__(256) q8_grad_zero_kernel(long mn, int M, float* dW, float* db) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  if (i < mn) dW[i] = 0.f;
  else if (i < mn + M && db) db[i - mn] = 0.f;
}

// Tile and slices of a launch.  Tiles that fill whole rounds of the chip are computed in one piece; those of the last
// round, which would leave part of it idle, are cut along the tokens into slices that fill it, which costs writing and
// adding up the slices' sums.  The time of a round is fixed + tokens * per_token[blocks on a CU], that of joining slices
// J0 + J1 * slices and their bytes, fitted to 1232 launches (64 to 70001 tokens, 64 x 64 to 50257 x 768 weights, both
// types) and within 7-10 % of them; the pick is 0.7 % slower than the best of all tiles and slices on average, 15 % at worst
// (3000 tokens, 9000 x 130).  One piece or slices of the last round: 16384 tokens, 4096 x 1024, bf16, 372 against 151 us.  Large
// tiles or small ones, in one run: 16384 tokens, 4096 x 4096, 470, 630, 1510 us; 2048, 384 x 384, each with its best slices, 22, 15, 11.7.
// CUS is a constant: the plan, and with it the order of the sums, follows from the sizes alone.
constexpr int CUS = 256;
struct Tile { int bm, bn, bk, per_cu; double fixed, per_token[4]; };       // us, us per 1000 tokens
constexpr Tile TILES_BF16[] = {{256, 256, 64, 1, 6.6, {24.6}}, {128, 128, 64, 2, 6.35, {13.6, 18.8}},
                               {64, 64, 64, 4, 5.4, {7.8, 9.6, 14.0, 18.3}}};
constexpr Tile TILES_F32[] = {{128, 256, 64, 1, 6.5, {33.7}}, {128, 128, 32, 2, 5.75, {32.9, 45.3}},
                              {64, 64, 32, 4, 5.15, {18.5, 22.2, 30.9, 39.6}}};
constexpr double J0 = 2.1, J1 = 0.07, J_BYTES = 5.1e6;                     // us, us a slice, bytes per us
constexpr int MOST_SLICES = 64;
// db: the first column of tiles takes all of it, or the columns share it out and the join adds up theirs.  The first column's
// blocks take up to 1.3 us per 1000 tokens more than the others, and a launch of few rounds waits for them; a join that would not
// run otherwise takes 3 to 7 us.  One column and all of them, us, bf16: joined anyway, 12608 tokens, 384 x 384, 23.0, 21.2; 4096,
// 50257 x 768, 354, 349; 8192, 20000 x 1024, 353, 344; fp32 12608, 2048 x 1000, 150.7, 147.2; not joined otherwise, 16384, 4096 x 4096, 500, 484;
// 8192, 8192 x 4096, 505, 501; 4096, 4096 x 4096, 134, 131, but 4096, 32000 x 512, 141, 145 and 2048, 4096 x 4096, 73.8, 74.2.
constexpr long SPREAD_ROWS = 8192;
struct Plan {
  int cfg, tiles_m, tiles_n, whole, slices;
  int rest() const { return tiles_m * tiles_n - whole; }
  bool spread(long rows) const { return rest() || (tiles_n > 1 && rows >= SPREAD_ROWS); }
};
Plan plan(long rows, int M, int N, bool dy_bf16) {
  Plan best = {};
  double best_cost = 1e300;
  for (int c = 0; c < 3; ++c) {
    const Tile& t = dy_bf16 ? TILES_BF16[c] : TILES_F32[c];
    const long tm = (M + t.bm - 1) / t.bm, tn = (N + t.bn - 1) / t.bn, tiles = tm * tn, fill = CUS * t.per_cu;
    const long whole = tiles / fill * fill, rest = tiles - whole, ktiles = (rows + t.bk - 1) / t.bk;
    const double base = (double)(whole / fill) * (t.fixed + t.per_token[t.per_cu - 1] * rows / 1000.0);
    for (long s = 1; s == 1 || (rest && s <= MOST_SLICES && s <= ktiles && rest * s <= fill); ++s) {
      double cost = base;
      if (rest) cost += t.fixed + t.per_token[(rest * s - 1) / CUS] * ((ktiles + s - 1) / s * t.bk) / 1000.0;
      if (s > 1) cost += J0 + J1 * s + 2.0 * s * rest * t.bm * t.bn * 4.0 / J_BYTES;
      if (cost < best_cost) {
        best_cost = cost;
        best = {c, (int)tm, (int)tn, (int)(s > 1 ? whole : tiles), (int)s};
      }
    }
  }
  return best;
}

template <typename T, int BM, int BN, int BK, int WM, int WN, int OCC>
hipError_t launch_tile(const Q8GradArgs& a, const Plan& p, float* partial, hipStream_t st) {
  constexpr int PARTS = std::is_same<T, float>::value ? 3 : 1;
  const size_t smem = 2 * (size_t)BK * 2 * (PARTS * BM + BN);
  static_assert(64 * WM * WN * 8 * 4 <= 2 * BK * 2 * (PARTS * BM + BN), "the sums of db fit");
  auto kern = q8_grad_kernel<T, BM, BN, BK, WM, WN, OCC>;
  static unsigned long raised = 0;
  if (const hipError_t e = raise_lds_limit(reinterpret_cast<const void*>(kern), (int)smem, raised); e != hipSuccess) return e;
  const Items it(p.tiles_m * p.tiles_n, p.whole, p.slices);
  float* column = p.spread(a.rows) ? partial + (size_t)it.rest * p.slices * (BM * BN + BM) : nullptr;
  hipLaunchKernelGGL(kern, dim3(it.blocks()), dim3(64 * WM * WN), smem, st, a, p.tiles_n, it, partial, column);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  constexpr int X = BM * BN / 1024;
  const int sums = a.db && column ? (a.M + 16 * X - 1) / (16 * X) : 0, y = it.rest + (sums < 1024 ? sums : 1024);
  if (!y) return hipSuccess;
  hipLaunchKernelGGL(q8_grad_join_kernel, dim3(X, y), dim3(256), 0, st, a, partial, column, p.whole, it.rest, p.slices, BM, BN, p.tiles_n);
  return hipGetLastError();
}

}  // namespace

size_t q8_grad_partial_floats(long rows, int M, int N, bool dy_bf16) {
  if (rows <= 0) return 0;
  const Plan p = plan(rows, M, N, dy_bf16);
  const Tile& t = dy_bf16 ? TILES_BF16[p.cfg] : TILES_F32[p.cfg];
  return (size_t)p.rest() * p.slices * (t.bm * t.bn + t.bm) + (p.spread(rows) ? (size_t)p.whole * t.bm : 0);
}

hipError_t launch_q8_grad(const Q8GradArgs& a, bool dy_bf16, float* partial, hipStream_t st) {
  const long mn = (long)a.M * a.N, each = mn + a.M;
  if (a.rows <= 0) {
    hipLaunchKernelGGL(q8_grad_zero_kernel, dim3((unsigned)((each + 255) / 256)), dim3(256), 0, st, mn, a.M, a.dW, a.db);
    return hipGetLastError();
  }
  ProfScope ps(PC_Q8_GRAD, 2.0 * a.rows * mn, (double)a.rows * (a.M * (dy_bf16 ? 2.0 : 4.0) + 33.0 * a.blocks) + 4.0 * each, st);
  const Plan p = plan(a.rows, a.M, a.N, dy_bf16);
  if (dy_bf16) {
    if (p.cfg == 0) return launch_tile<bf16, 256, 256, 64, 4, 2, 1>(a, p, partial, st);
    if (p.cfg == 1) return launch_tile<bf16, 128, 128, 64, 2, 2, 2>(a, p, partial, st);
    return launch_tile<bf16, 64, 64, 64, 2, 2, 4>(a, p, partial, st);
  }
  if (p.cfg == 0) return launch_tile<float, 128, 256, 64, 2, 4, 1>(a, p, partial, st);
  if (p.cfg == 1) return launch_tile<float, 128, 128, 32, 2, 2, 2>(a, p, partial, st);
  return launch_tile<float, 64, 64, 32, 2, 2, 4>(a, p, partial, st);
}

}  // namespace mg
