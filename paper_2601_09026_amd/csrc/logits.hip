// Between a head's logits and the gradient that enters the network again: log probabilities of given tokens with entropy
// and the most likely alternatives, distillation from a teacher's top logits, and the gradients of both.  Over a row z:
//   p = softmax(z / tau),  lse = log sum exp(z / tau),  H = lse - sum p z / tau
//   log p_i = z_i / tau - lse,  dz_i = 1 / tau (g ([i = token] - p_i) - h p_i (log p_i + H))
//   L = sum_j q_j (log q_j - log p_id(j)),  dz_i = g / tau (Q p_i - sum_{j: id(j) = i} q_j),  Q = sum q
// A row is read in 16-byte vectors from its first 16-byte address on, the elements before and behind them one by one; all
// arithmetic is fp32, sums in a tree over a lane's vectors, lanes and wavefronts, the gradient is rounded once.
//
// What bounds it: moving the logits, and in bf16 next to that the vector unit: an element of the values takes 8 vector
// instructions of a lane (counted at 2048 x 131072 fp32, loop and sums included), and in bf16 twice as many elements come
// with the same bytes.  Hence the exponents of one instruction (Reader) and sums of which nothing is rescaled as a rule.
// Values, fp32, 2048 x 131072: 158 us, 6.8 TB/s; bf16, 4096 x 50257: 70 us, 5.9 TB/s, 81 with 5 alternatives.  Backward,
// 4096 x 50257 bf16 with entropies: 143 us, 5.8 TB/s (a large copy reaches 5.7).  Both in one call, 8192 x 50304 bf16: 312 us, 5.3
// TB/s over one reading and one writing; the two calls one after the other take 133 and 275.  One row of 50257 with 20
// alternatives: 12 us in two launches.
#include <math.h>

#include <type_traits>

#include "kernels.h"
#include "prof.h"
#include "q8.h"

namespace mg {
namespace {

constexpr float LOWEST = -3.402823466e38f, LOG2E = 1.44269504088896340736f;
constexpr int THREADS = 256, WAVES = THREADS / WAVE;
constexpr int STEP = 4;                                  // vectors of a lane that are loaded together
constexpr int LIST = 256;                                // candidates of a wavefront
constexpr int ROOM = LIST + 4 + 64;
constexpr int GROUPS = 8;                                // groups of a lane's elements whose maxima are kept
typedef unsigned long long u64;
typedef float f32x2 __attribute__((ext_vector_type(2)));

template <typename T> constexpr int vec() { return 16 / (int)sizeof(T); }

// ---- a run of elements in memory -------------------------------------------------
template <typename T> struct Run {
  T* p;
  int head, vecs, odd;                                   // odd: elements outside the vectors, head of them in front
  __device__ __forceinline__ Run(const void* base, long at, int n) {
    p = static_cast<T*>(const_cast<void*>(base)) + at;
    const int lead = (int)((16u - ((unsigned)reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) / (int)sizeof(T);
    head = lead < n ? lead : n;
    vecs = (n - head) / vec<T>();
    odd = n - vecs * vec<T>();
  }
  __device__ __forceinline__ int odd_at(int i) const { return i < head ? i : i + vecs * vec<T>(); }
  __device__ __forceinline__ int vec_at(int v) const { return head + v * vec<T>(); }
  // Chunks of STEP vectors per lane of a block; 2^fold of them are a group, at most GROUPS a run
  __device__ __forceinline__ int chunks() const { return vecs ? (vecs - 1) / (STEP * THREADS) + 1 : 1; }
  __device__ __forceinline__ int fold() const { return chunks() <= GROUPS ? 0 : 32 - __builtin_clz((chunks() - 1) / GROUPS); }
  __device__ __forceinline__ int groups() const { return ((chunks() - 1) >> fold()) + 1; }
};

template <typename T> __device__ __forceinline__ void decode(u32x4 r, float (&x)[vec<T>()]);
template <> __device__ __forceinline__ void decode<float>(u32x4 r, float (&x)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = bits_f(r[j]);
}
template <> __device__ __forceinline__ void decode<bf16>(u32x4 r, float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[2 * j] = bits_f(r[j] << 16);
    x[2 * j + 1] = bits_f(r[j] & 0xffff0000u);
  }
}
template <typename T> __device__ __forceinline__ u32x4 encode(const float (&x)[vec<T>()]);
template <> __device__ __forceinline__ u32x4 encode<float>(const float (&x)[4]) {
  return u32x4{f_bits(x[0]), f_bits(x[1]), f_bits(x[2]), f_bits(x[3])};
}
template <> __device__ __forceinline__ u32x4 encode<bf16>(const float (&x)[8]) {
  bf16x8 b;
#pragma unroll
  for (int j = 0; j < 8; ++j) b[j] = (bf16)x[j];
  return __builtin_bit_cast(u32x4, b);
}

__device__ __forceinline__ long block_index() { return (long)blockIdx.y * gridDim.x + blockIdx.x; }

__device__ __forceinline__ long id_of(const void* ids, long i, bool wide) {
  return wide ? static_cast<const int64_t*>(ids)[i] : (long)static_cast<const int32_t*>(ids)[i];
}

// ---- over the lanes of a wavefront: the first LANES of them, or groups of so many; the result in all ---------------
template <int LANES, typename F> __device__ __forceinline__ float over_lanes(float v, F f) {
  static_assert(LANES == 1 || LANES == 4 || LANES == 8 || LANES == 16 || LANES == 64, "in steps of rows of 16");
  auto step = [&](unsigned other) { v = f(v, bits_f(other)); };
  if constexpr (LANES >= 4) { step(lane_move<LANE_XOR1>(f_bits(v))); step(lane_move<LANE_XOR2>(f_bits(v))); }
  if constexpr (LANES >= 8) step(lane_move<LANE_MIRROR8>(f_bits(v)));
  if constexpr (LANES >= 16) step(lane_move<LANE_MIRROR16>(f_bits(v)));
  if constexpr (LANES == 64) {
    // (rows 1 and 3 against 0 and 2, then the upper 32 lanes against the lower: each of a swap's two results has one side in both places)
    const auto rows = __builtin_amdgcn_permlane16_swap(f_bits(v), f_bits(v), false, false);
    v = f(bits_f(rows[0]), bits_f(rows[1]));
    const auto halves = __builtin_amdgcn_permlane32_swap(f_bits(v), f_bits(v), false, false);
    v = f(bits_f(halves[0]), bits_f(halves[1]));
  }
  return v;
}
template <int LANES = 64> __device__ __forceinline__ float all_max(float v) { return over_lanes<LANES>(v, [](float a, float b) { return fmaxf(a, b); }); }
template <int LANES = 64> __device__ __forceinline__ float all_sum(float v) { return over_lanes<LANES>(v, [](float a, float b) { return a + b; }); }

// ---- sums of exponentials ----------------------------------------------------------
// s = sum 2^((x - m) c), t = sum (x - m) c 2^((x - m) c) over the values seen, m one of them, c = log2(e) / tau.  A NaN or
// +infinity makes s NaN.  Exponents of -160 and less, -infinity among them, have 2^a = 0, and 0 in t.
struct Sums { float m, s, t; };
__device__ __forceinline__ float bounded(float a) { return fmaxf(a, -160.f); }
__device__ __forceinline__ float exp2_of(float a) { return __builtin_amdgcn_exp2f(a); }

__device__ __forceinline__ void shift(float& s, float& t, float d) {     // every exponent d higher
  const float f = exp2_of(d);
  t = f * (t + d * s);
  s = f * s;
}
__device__ __forceinline__ void raise(Sums& a, float m, float c) {
  shift(a.s, a.t, bounded((a.m - m) * c));
  a.m = m;
}
__device__ __forceinline__ void merge(Sums& a, Sums b, float c) {
  const float m = fmaxf(a.m, b.m);
  raise(a, m, c);
  raise(b, m, c);
  a.s += b.s;
  a.t += b.t;
}
__device__ __forceinline__ Sums wave_merge(Sums a, float c) {
  raise(a, all_max(a.m), c);
  return Sums{a.m, all_sum(a.s), all_sum(a.t)};
}

// A wavefront's sums while it reads.  All lanes refer to one m, which lags behind the maximum: it is raised where a value has an
// exponent above 8, so that nothing is rescaled as a rule and the exponents of the largest terms keep 20 bits behind the point.
// An exponent is one instruction, x c - P with P = m c rounded; what was rounded off is the same for all, rest = m c - P,
// and taken out at the end.  Where |m c| is so large that the rest is no small number (FAR) the difference is taken before it is scaled.
template <bool T_SUM> struct Reader {
  float c, m, P, rest, s, t;                             // c to rest are the same in all lanes
  bool far;
  __device__ __forceinline__ void start(float scale) { c = scale; m = LOWEST; P = rest = s = t = 0.f; far = true; }
  __device__ __forceinline__ bool low(float most) const { return __any((most - m) * c > 8.f); }
  __device__ __forceinline__ void lift(float most) {
    const float top = fmaxf(all_max(most), m), product = top * c;
    const bool beyond = !(fabsf(product) < 0x1p20f);
    const float left = beyond ? 0.f : fmaf(top, c, -product);
    shift(s, t, bounded((m - top) * c - rest + left));
    m = top; P = product; rest = left; far = beyond;
  }
  template <bool FAR, int N> __device__ __forceinline__ void add(const float (&x)[N], float& s_, float& t_) const {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float a = FAR ? (x[j] - m) * c : fmaf(x[j], c, -P), e = exp2_of(a);
      s_ += e;
      if constexpr (T_SUM) t_ = fmaf(bounded(a), e, t_);
    }
  }
  __device__ __forceinline__ Sums finish() {             // the wavefront's, in all lanes
    shift(s, t, -rest);
    return Sums{m, all_sum(s), T_SUM ? all_sum(t) : 0.f};
  }
};

// What a row's sums come to.  lse: +-infinity where the row's largest quotient by tau is: no distribution (-infinity: zeros
// in place of p) or, as with a NaN among the logits, NaN.
struct RowSums {
  float top, lse, log_s, inv_tau;                        // log p = (z - top) inv_tau - log_s
  float entropy;
  bool bad, none;
  __device__ __forceinline__ RowSums(Sums a, float tau) {
    inv_tau = 1.0f / tau;
    top = a.m;
    log_s = logf(a.s);
    lse = a.m / tau + log_s;
    bad = !(a.s >= 0.f) || lse == __builtin_inff();
    none = !bad && !(lse > -__builtin_inff());
    entropy = none ? 0.f : fmaxf(log_s - 0.69314718055994530942f * a.t / a.s, 0.f);
    if (bad) lse = entropy = __builtin_nanf("");
  }
  __device__ __forceinline__ float logprob(float z, float tau) const {
    return bad ? __builtin_nanf("") : none ? -__builtin_inff() : (z - top) / tau - log_s;
  }
};

// ---- the largest elements ------------------------------------------------------------
// A candidate is one number: the value's order in the upper half, the complement of its index below, so that the greater
// of two comes first and equal values come by index.  While a row is read each lane keeps the largest of its elements, and of
// each group of them.  A value that k lanes' largest reach is a bar below which nothing can be among the k largest; the
// groups that reach it, little more than k, are read again.  What they hold goes to a list in LDS, one per wavefront, which
// is sorted down to k when it is full.
__device__ __forceinline__ u64 candidate(float x, int index) {
  const unsigned b = f_bits(x + 0.f);                    // (-0 and 0 are equal)
  return (u64)(b ^ ((unsigned)((int)b >> 31) | 0x80000000u)) << 32 | (unsigned)~index;
}
__device__ __forceinline__ float value_of(u64 key) {
  const unsigned b = (unsigned)(key >> 32);
  return bits_f(b ^ (b & 0x80000000u ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int index_of(u64 key) { return (int)~(unsigned)key; }
__device__ __forceinline__ u64 uniform(u64 v) {
  return (u64)(unsigned)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)v);
}
__device__ __forceinline__ void wave_sync() {            // LDS accesses of a wavefront keep their order
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

struct Top {
  u64* list;                                             // [ROOM] of this wavefront: candidates, zeros behind them, the sorted ones
  float* groups;                                         // [GROUPS][THREADS], an entry per group for this lane
  int k, n;                                              // n: candidates in the list
  u64 floor;                                             // only what is greater is taken
  float best, first;                                     // the lane's largest element; its odd element
  __device__ __forceinline__ void start(u64* lists, float* lds_groups, int want) {
    list = lists + threadIdx.x / WAVE * ROOM;
    groups = lds_groups + threadIdx.x;
    k = want; n = 0; floor = 0; best = first = -__builtin_inff();
  }
  // The largest number of 16 bits, in the order of candidates' upper halves, that `want` lanes' largest elements reach
  __device__ __forceinline__ unsigned reached(int want) const {
    const unsigned mine = (unsigned)(candidate(best, 0) >> 32);
    unsigned low = 0;
#pragma unroll
    for (unsigned bit = 1u << 31; bit >= 1u << 16; bit >>= 1)
      if (__popcll(__ballot(mine >= (low | bit))) >= want) low |= bit;
    return low;
  }
  static __device__ __forceinline__ float bar_of(unsigned low) { return low > 0x007fffffu ? value_of((u64)low << 32) : LOWEST; }    // (masked elements: fill())
  // sorts the list, the k first stay
  __device__ __forceinline__ void settle() {
    const int lane = threadIdx.x & 63;
    if (lane < 4) list[n + lane] = 0;                                   // (read four at a time)
    wave_sync();
    u64* sorted = list + LIST + 4;
    for (int i = lane; i - lane < n; i += WAVE) {
      const u64 own = i < n ? list[i] : 0;
      int rank = 0;
      for (int j = 0; j < n; j += 4) {
#pragma unroll
        for (int u = 0; u < 4; ++u) rank += list[j + u] > own;
      }
      if (i < n && rank < k) sorted[rank] = own;
    }
    wave_sync();
    const int kept = n < k ? n : k;
    if (lane < kept) list[lane] = sorted[lane];
    wave_sync();
    n = kept;
    if (n == k) floor = uniform(list[k - 1]);
  }
  // the lanes' keys, where one is given
  __device__ __forceinline__ void take(bool given, u64 key) {
    const u64 who = __ballot(given && key > floor);
    if (!who) return;
    const int lane = threadIdx.x & 63;
    if (who >> lane & 1) list[n + __popcll(who & ((1ull << lane) - 1))] = key;
    n += __popcll(who);
    if (n > LIST - WAVE) settle();
  }
  // the elements of the lane's vectors that reach the bar: those of vector u where inside(u), index(u) the first's
  template <typename T, int COUNT, typename F, typename G> __device__ __forceinline__ void take_high(const u32x4* raw, float bar, F inside, G index) {
    constexpr int N = vec<T>();
    static_assert(COUNT * N <= 32, "a bit each");
    unsigned high = 0;
#pragma unroll
    for (int u = COUNT - 1; u >= 0; --u) {
      const bool in = inside(u);
      float x[N];
      decode<T>(raw[u], x);
#pragma unroll
      for (int j = N - 1; j >= 0; --j) high = high << 1 | (unsigned)(in && x[j] >= bar);
    }
    while (__any(high != 0)) {
      const int e = high ? __builtin_ctz(high) : 0, u = e / N, j = e % N;
      unsigned w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[i] = raw[0][i];
#pragma unroll
        for (int o = 1; o < COUNT; ++o) w[i] = u == o ? raw[o][i] : w[i];
      }
      const int d = sizeof(T) == 2 ? j >> 1 : j;
      const unsigned lo = d & 1 ? w[1] : w[0], hi = d & 1 ? w[3] : w[2], word = d & 2 ? hi : lo;
      const float x = bits_f(sizeof(T) == 4 ? word : j & 1 ? word & 0xffff0000u : word << 16);
      take(high != 0, candidate(x, index(u) + j));
      high &= high - 1;
    }
  }
  // sorted; the rest of the list is empty
  __device__ __forceinline__ void finish() {
    settle();
    const int lane = threadIdx.x & 63;
    if (lane >= n && lane < k) list[lane] = 0;
    wave_sync();
  }
  // A list of fewer than k that holds all elements but the masked ones: of those, the first of the `count` from `from` on
  __device__ __forceinline__ void fill(int from, int count) {
    const int lane = threadIdx.x & 63;
    int have = n;
    for (int i0 = 0; have < k && i0 < count; i0 += WAVE) {
      bool masked = i0 + lane < count;
      for (int j = 0; j < n; ++j) masked = masked && index_of(list[j]) != from + i0 + lane;
      const u64 who = __ballot(masked);
      const int at = have + __popcll(who & ((1ull << lane) - 1));
      if (masked && at < k) list[at] = candidate(-__builtin_inff(), from + i0 + lane);
      have += __popcll(who);
    }
    wave_sync();
  }
};

// ---- a row's sums (and its largest elements), by a block --------------------------------
template <typename T> constexpr unsigned NOTHING = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;          // -infinity

// The block goes through the run's chunks of STEP vectors per lane.  What comes back is each wavefront's own.
template <typename T, bool T_SUM, bool TOP>
__device__ __forceinline__ Sums read_run(const Run<T>& r, int lane, float c, Top& top) {
  constexpr int N = vec<T>(), team = THREADS;
  const float none = -__builtin_inff();
  const int fold = TOP ? r.fold() : 0;
  Reader<T_SUM> sums;
  sums.start(c);
  const bool odd = lane < r.odd;                         // (odd < 2 N: lanes of the first wavefront)
  const float first[1] = {odd ? to_f(r.p[r.odd_at(lane)]) : none};
  float group = none;
  for (int v0 = 0, chunk = 0; v0 == 0 || v0 < r.vecs; v0 += STEP * team, ++chunk) {
    u32x4 raw[STEP];
    if (r.vecs) {
#pragma unroll
      for (int u = 0; u < STEP; ++u) {
        const int v = v0 + u * team + lane;
        raw[u] = ld_stream(reinterpret_cast<const u32x4*>(r.p + r.vec_at(v < r.vecs ? v : r.vecs - 1)));
      }
    }
    auto steps = [&](auto f) {                           // the chunk's vectors
#pragma unroll
      for (int u = 0; u < STEP; ++u)
        if (v0 + u * team < r.vecs) {
          float x[N];
          asm("" : "+v"(raw[u]));                        // (decoded anew in every pass: a chunk's 32 values are not kept)
          decode<T>(raw[u], x);
          f(x, u);
        }
    };
    if (v0 + STEP * team > r.vecs) {
#pragma unroll
      for (int u = 0; u < STEP; ++u)
        if (v0 + u * team + lane >= r.vecs) raw[u] = u32x4{NOTHING<T>, NOTHING<T>, NOTHING<T>, NOTHING<T>};
    }
    float most[STEP], all = none;
    auto maxima = [&](const float (&x)[N], int u) {
      most[u] = none;
#pragma unroll
      for (int j = 0; j < N; ++j) most[u] = fmaxf(most[u], x[j]);
    };
    auto overall = [&]() {
      all = first[0];
      if (v0) all = none;
#pragma unroll
      for (int u = 0; u < STEP; ++u) all = fmaxf(all, most[u]);
    };
#pragma unroll
    for (int u = 0; u < STEP; ++u) most[u] = none;
    if (v0 == 0) {
      steps(maxima);
      overall();
      sums.lift(all);
      if (r.odd) {
        if (sums.far) sums.template add<true>(first, sums.s, sums.t);
        else sums.template add<false>(first, sums.s, sums.t);
      }
    }
    for (;;) {
      float s = 0.f, t = 0.f;
      if (sums.far) {
        steps([&](const float (&x)[N], int u) { maxima(x, u); sums.template add<true>(x, s, t); });
      } else {
        steps([&](const float (&x)[N], int u) { maxima(x, u); sums.template add<false>(x, s, t); });
      }
      overall();
      if (!sums.low(all)) {
        sums.s += s;
        sums.t += t;
        break;
      }
      sums.lift(all);
    }
    if constexpr (TOP) {
      group = fmaxf(group, all);
      if (((chunk + 1) & ((1 << fold) - 1)) == 0 || v0 + STEP * team >= r.vecs) {
        top.groups[(chunk >> fold) * THREADS] = group;
        top.best = fmaxf(top.best, group);
        group = none;
      }
    }
  }
  if constexpr (TOP) top.first = first[0];
  return sums.finish();
}

// The candidates among a lane's elements: those of its groups that reach the bar are read again
template <typename T> __device__ __forceinline__ void pick(const Run<T>& r, int lane, int index, unsigned low, Top& top) {
  constexpr int team = THREADS;
  const float bar = Top::bar_of(low);
  const int fold = r.fold(), groups = r.groups();
  top.take(lane < r.odd && top.first >= bar, candidate(top.first, index + r.odd_at(lane)));
  unsigned hit = 0;
  for (int g = 0; g < groups; ++g) hit |= top.groups[g * THREADS] >= bar ? 1u << g : 0u;
  if (r.vecs == 0) hit = 0;
  while (__any(hit != 0)) {
    const int g = hit ? __builtin_ctz(hit) : 0;
    for (int i = 0; i < 1 << fold; ++i) {
      const int v0 = ((g << fold) + i) * (STEP * team) + lane;
      u32x4 raw[STEP];
#pragma unroll
      for (int u = 0; u < STEP; ++u) {
        const int v = v0 + u * team;
        raw[u] = ld_global(reinterpret_cast<const u32x4*>(r.p + r.vec_at(hit && v < r.vecs ? v : 0)));
      }
      top.template take_high<T, STEP>(raw, bar, [&](int u) { return hit && v0 + u * team < r.vecs; }, [&](int u) { return index + r.vec_at(v0 + u * team); });
    }
    hit &= hit - 1;
  }
  top.finish();
}

// What a block's wavefronts found: the sums in all of them, the list in the first.
template <typename T, bool TOP>
__device__ __forceinline__ void join_waves(const Run<T>& r, int index, Sums& sums, Top& top, f32x4* waves, u64* lists, float c) {
  const int wave = threadIdx.x / WAVE, lane = threadIdx.x & 63;
  unsigned low = 0;
  if constexpr (TOP) low = top.reached((top.k + WAVES - 1) / WAVES);
  if (lane == 0) waves[wave] = f32x4{sums.m, sums.s, sums.t, bits_f(low)};
  __syncthreads();
  sums = Sums{waves[0][0], waves[0][1], waves[0][2]};
  low = f_bits(waves[0][3]);
#pragma unroll
  for (int w = 1; w < WAVES; ++w) {
    merge(sums, Sums{waves[w][0], waves[w][1], waves[w][2]}, c);
    const unsigned other = f_bits(waves[w][3]);          // (a quarter of the k lanes in every wavefront reach the least of these)
    low = other < low ? other : low;
  }
  if constexpr (TOP) {
    pick<T>(r, threadIdx.x, index, low, top);
    __syncthreads();
    if (wave == 0) {
      for (int w = 1; w < WAVES; ++w) top.take(lane < top.k, lane < top.k ? lists[w * ROOM + lane] : 0);
      top.finish();
      if (top.n < top.k) top.fill(index, r.vecs * vec<T>() + r.odd);
    }
  }
}

// ---- what a row is measured by ----------------------------------------------------------
// Ids with weights w that sum to `mass`.  Log probabilities (MODE 0): the token, w = 1, in the first lane.  Distillation
// (MODE 1): the teacher's kept ids with w = q, id j in lane j % 64.  mass 0: the row has none; NaN: one is out of range (or a
// teacher's logit is no number, or the sum passes fp32's range).  Held by one wavefront.
constexpr int KEPT = 256;
template <int MODE> struct Points {
  static constexpr int N = MODE == 0 ? 1 : KEPT / WAVE, OUTSIDE = -2;
  int id[N];                                             // -1: none
  float w[N], z[N];                                      // z: the student's logits
  float mass;
  // fetch starts the loads, settle makes the weights of them
  __device__ __forceinline__ void fetch(const LogitsArgs& a, long row) {
    if constexpr (MODE == 0) {
      const long token = a.tokens ? id_of(a.tokens, row, a.wide_ids) : -1;
      const bool valid = token >= 0 && token < a.cols;
      id[0] = valid ? (int)token : -1;
      w[0] = 1.f;
      mass = valid ? 1.f : token < 0 ? 0.f : __builtin_nanf("");
    } else {
      const int lane = threadIdx.x & 63;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        id[i] = -1;
        w[i] = 0.f;
        if (i * WAVE < a.kept && i * WAVE + lane < a.kept) {
          const long at = row * a.kept + i * WAVE + lane, v = id_of(a.teacher_ids, at, a.wide_ids);
          id[i] = v < 0 ? -1 : v < a.cols ? (int)v : OUTSIDE;
          w[i] = a.teacher_bf16 ? to_f(static_cast<const bf16*>(a.teacher)[at]) : static_cast<const float*>(a.teacher)[at];
        }
      }
    }
  }
  __device__ __forceinline__ void settle(const LogitsArgs& a, long row) {
    if constexpr (MODE == 1) {
      float top = -__builtin_inff();
      bool out = false;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        out |= id[i] == OUTSIDE;
        if (id[i] == OUTSIDE) id[i] = -1;
        if (id[i] >= 0) top = fmaxf(top, w[i]);
      }
      const float l = a.teacher_lse ? a.teacher_lse[row] : 0.f;
      top = fmaxf(all_max(top), LOWEST);
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i * WAVE < a.kept) {
          w[i] = id[i] < 0 ? 0.f : expf(a.teacher_lse ? w[i] / a.tau - l : (w[i] - top) / a.tau);
          s += w[i];
        }
      s = all_sum(s);
      mass = s;
      if (!a.teacher_lse) {
        const float one = 1.f / s;
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          w[i] = s != 0.f ? w[i] * one : 0.f;            // (NaN stays)
          m += w[i];
        }
        mass = all_sum(m);
      }
      if (__any(out) || !(mass < __builtin_inff())) mass = __builtin_nanf("");         // (infinite: by a teacher's log-sum-exp alone)
    }
  }
  __device__ __forceinline__ void load(const LogitsArgs& a, long row) {
    fetch(a, row);
    settle(a, row);
  }
  // the logits of the ids among the n from `from` on
  template <typename T> __device__ __forceinline__ void gather(const T* row, int from, int n) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      z[i] = 0.f;
      if (id[i] >= from && id[i] - from < n) z[i] = to_f(row[id[i]]);
    }
  }
};

// A row's values, from its sums and points
template <int MODE> __device__ __forceinline__ void put_values(const LogitsArgs& a, long row, const RowSums& r, const Points<MODE>& pt) {
  const int lane = threadIdx.x & 63;
  if (lane == 0) {
    if (a.lse) a.lse[row] = r.lse;
    if (MODE == 0 && a.entropy) a.entropy[row] = r.entropy;
  }
  if constexpr (MODE == 0) {
    if (lane == 0 && a.logprob) a.logprob[row] = pt.mass == 1.f ? r.logprob(pt.z[0], a.tau) : pt.mass;
  } else {
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < Points<MODE>::N; ++i)
      if (pt.id[i] >= 0 && pt.w[i] != 0.f) l += pt.w[i] * (logf(pt.w[i]) - r.logprob(pt.z[i], a.tau));
    l = all_sum(l);
    if (lane == 0 && a.loss) a.loss[row] = pt.mass == 0.f || pt.mass != pt.mass ? pt.mass : l;
  }
}
__device__ __forceinline__ void put_alternatives(const LogitsArgs& a, long row, const RowSums& r, const u64* list) {
  const int lane = threadIdx.x & 63;
  if (lane >= a.top_k) return;
  const u64 key = list[lane];
  const long at = row * a.top_k + lane;
  const int id = r.bad ? -1 : index_of(key);
  if (a.wide_ids) static_cast<int64_t*>(a.top_ids)[at] = id;
  else static_cast<int32_t*>(a.top_ids)[at] = id;
  a.top_logprobs[at] = r.logprob(value_of(key), a.tau);
}

// ---- values of a row --------------------------------------------------------------------
// A block per row, or per part of it; with several parts a row's sums, lists and points go to the workspace.  A task to a block and
// no loop over them.  The alternatives were the most of it: with a list that every element is held against, 4096 x 50304 bf16
// took 142 us with 5 and 396 with 64 (89 without any); with the second look at the few groups that matter 78 and 98 (68 without any).
template <typename T, bool TOP, int MODE>
__global__ void __launch_bounds__(THREADS, 6) logits_values_kernel(const LogitsArgs a) {
  __shared__ u64 lists[TOP ? WAVES * ROOM : 1];
  __shared__ f32x4 waves[WAVES];
  __shared__ float groups[TOP ? GROUPS * THREADS : 1];
  const int wave = threadIdx.x / WAVE, lane = threadIdx.x & 63;
  const float c = LOG2E / a.tau;
  const long task = block_index();
  if (task >= a.rows * a.parts) return;
  const long row = task / a.parts;
  const int part = (int)(task - row * a.parts), from = part * a.part_cols;
  const int n = a.cols - from < a.part_cols ? a.cols - from : a.part_cols;
  const T* z = static_cast<const T*>(a.z) + row * a.ld;
  const bool asked = wave == 0 && part == 0 && (!a.part_sums || a.part_points);
  Points<MODE> pt;
  if (asked) {
    pt.load(a, row);
    pt.gather(z, 0, a.cols);
  }
  Top top;
  if constexpr (TOP) top.start(lists, groups, a.top_k);
  const Run<T> in(z, from, n);
  Sums sums = read_run<T, MODE == 0, TOP>(in, threadIdx.x, c, top);
  join_waves<T, TOP>(in, from, sums, top, waves, lists, c);
  if (wave != 0) return;
  if (!a.part_sums) {
    const RowSums r(sums, a.tau);
    put_values<MODE>(a, row, r, pt);
    if constexpr (TOP) put_alternatives(a, row, r, top.list);
    return;
  }
  if (lane == 0) a.part_sums[task] = f32x4{sums.m, sums.s, sums.t, 0.f};
  if constexpr (TOP)
    if (lane < a.top_k) a.part_lists[task * a.top_k + lane] = top.list[lane];
  if (asked) {
#pragma unroll
    for (int i = 0; i < Points<MODE>::N; ++i)
      if (i * WAVE + lane < a.points) a.part_points[row * a.points + i * WAVE + lane] = pt.z[i];
  }
}

// A row's sums from those of its parts, one per lane
__device__ __forceinline__ Sums joined(const LogitsArgs& a, long row, float c) {
  const int lane = threadIdx.x & 63;
  Sums own = {LOWEST, 0.f, 0.f};
  if (lane < a.parts) {
    const f32x4 s = a.part_sums[row * a.parts + lane];
    own = Sums{s[0], s[1], s[2]};
  }
  return wave_merge(own, c);
}

// The parts' results, a wavefront per row
template <typename T, bool TOP, int MODE>
__global__ void __launch_bounds__(THREADS) logits_join_kernel(const LogitsArgs a) {
  __shared__ u64 lists[TOP ? WAVES * ROOM : 1];
  const int wave = threadIdx.x / WAVE, lane = threadIdx.x & 63;
  const long row = block_index() * WAVES + wave;
  if (row >= a.rows) return;
  // (what is loaded comes first: each load's way there and back is as long as the rest)
  constexpr int FIRST = 4;
  const int all = a.parts * a.top_k;
  u64 low = ~0ull, keys[FIRST];
  if constexpr (TOP) {
    const u64* from = a.part_lists + row * all;
#pragma unroll
    for (int i = 0; i < FIRST; ++i) keys[i] = i * WAVE + lane < all ? from[i * WAVE + lane] : 0;
    // each of the parts has (k / parts, rounded up) candidates that reach the least of their last
    if (lane < a.parts) low = from[lane * a.top_k + (a.top_k + a.parts - 1) / a.parts - 1];
  }
  Points<MODE> pt;
  pt.load(a, row);
  pt.gather(static_cast<const T*>(a.z) + row * a.ld, 0, a.cols);
  const RowSums r(joined(a, row, LOG2E / a.tau), a.tau);
  if constexpr (TOP) {
    Top top;
    top.start(lists, nullptr, a.top_k);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) { const u64 other = __shfl_xor(low, o, 64); low = other < low ? other : low; }
    top.floor = low ? uniform(low) - 1 : 0;
#pragma unroll
    for (int i = 0; i < FIRST; ++i) top.take(true, keys[i]);
    const u64* from = a.part_lists + row * all;
    for (int i = FIRST * WAVE; i < all; i += WAVE) top.take(i + lane < all, i + lane < all ? from[i + lane] : 0);
    top.finish();
    put_alternatives(a, row, r, top.list);
  }
  put_values<MODE>(a, row, r, pt);
}

// ---- gradients of a row -------------------------------------------------------------------
// dz_i = slope (sum of the points' w at i) - p_i (A + B log p_i)
struct Slope {
  float top, off, inv_tau;                               // log p = (z - top) inv_tau - off
  float A, B, slope;
  bool zero;                                             // nothing but zeros
  // mass: of the row's points.  sign: 1 for log probabilities, -1 for losses.  What g holds for a row without points is not looked at.
  template <bool ENTROPY> __device__ __forceinline__ void set(const LogitsArgs& a, long row, float mass, float sign, float entropy) {
    inv_tau = 1.0f / a.tau;
    slope = mass == 0.f ? 0.f : sign * (a.g ? a.g[row] : 1.f) * inv_tau;
    A = slope * mass;
    B = 0.f;
    if constexpr (ENTROPY) {
      B = a.h[row] * inv_tau;
      A += B * entropy;
    }
    zero = !ENTROPY && mass == 0.f;
  }
  // A given lse, through the logit that has it for a quotient by tau: only differences to that are rounded, not the quotients, which
  // may be far larger.  off is what it, rounded, leaves of lse; left: 1 / tau - inv_tau.  (Figures past 2^100 leave nothing to tell apart.)
  __device__ __forceinline__ void from_lse(float lse, float tau) {
    top = lse * tau;
    const float left = fmaf(-tau, inv_tau, 1.f) * inv_tau;
    off = fmaf(-top, left, fmaf(-top, inv_tau, lse));
    if (!(fabsf(lse) < 0x1p100f)) { top = 0.f; off = lse; }
    zero |= lse == -__builtin_inff();
  }
  __device__ __forceinline__ void from_sums(const RowSums& r) {
    top = r.top;
    off = r.bad ? __builtin_nanf("") : r.log_s;
    zero |= r.none;
  }
  template <bool ENTROPY> __device__ __forceinline__ float at(float z) const {
    const float lp = fmaf(z - top, inv_tau, -off), p = exp2_of(lp * LOG2E);
    const float d = ENTROPY ? -p * fmaf(B, bounded(lp), A) : -p * A;
    return zero ? 0.f : d;
  }
};

template <typename T> __device__ __forceinline__ void put_vector(T* p, const float (&x)[vec<T>()], bool stream) {
  typedef __attribute__((address_space(1))) u32x4_u* gptr;
  const u32x4 w = encode<T>(x);
  const u32x4_u v = {w[0], w[1], w[2], w[3]};
  if (stream) {
    asm volatile("; past the caches");                   // (between two of these, or the compiler makes one ordinary store of both)
    __builtin_nontemporal_store(v, (gptr)p);
    asm volatile("; past the caches");
  } else {
    *(gptr)p = v;
  }
}
// the gradient of a vector's elements, in place of them; token: its place among them, if it is there
template <typename T, bool ENTROPY> __device__ __forceinline__ void slope_vector(float (&x)[vec<T>()], const Slope& s, int token) {
#pragma unroll
  for (int j = 0; j < vec<T>(); ++j) x[j] = s.template at<ENTROPY>(x[j]);
  if ((unsigned)token < (unsigned)vec<T>()) {
#pragma unroll
    for (int j = 0; j < vec<T>(); ++j) x[j] += token == j ? s.slope : 0.f;
  }
}

// A teacher's ids (MODE 1).  The vectors (and odd elements) that hold one are left out by the team as it writes a run, and written
// by the first wavefront, from memory: no other touches them, also where the gradient replaces the logits.
// left_out: a word per lane, bit u for its vector u of the run and the highest for its odd element.
constexpr int ODD_BIT = 31;
template <typename T> struct Place { int lane, bit; };
template <typename T> __device__ __forceinline__ Place<T> place_of(const Run<T>& r, int at, int team) {
  const int v = (at - r.head) / vec<T>();
  if (at < r.head) return {at, ODD_BIT};
  if (v >= r.vecs) return {at - r.vecs * vec<T>(), ODD_BIT};
  return {v % team, v / team};
}
// Marks the ids among the run's n elements from `from` on.  first: a bit per id of the lane that is the first of its vector;
// twice: two are the same.
struct Marked { unsigned first; bool twice; };
template <typename T> __device__ __forceinline__ Marked leave_out(const Run<T>& r, const Points<1>& pt, int from, int n, int team, unsigned* left_out, int* ids, float* ws) {
  const int lane = threadIdx.x & 63;
  unsigned first = 0, later = 0;                         // later: in a vector (or odd element) that another has marked
#pragma unroll
  for (int i = 0; i < Points<1>::N; ++i) {
    ids[i * WAVE + lane] = pt.id[i];
    ws[i * WAVE + lane] = pt.w[i];
    if (pt.id[i] >= from && pt.id[i] - from < n) {
      const Place<T> at = place_of(r, pt.id[i] - from, team);
      const bool known = atomicOr(left_out + at.lane, 1u << at.bit) >> at.bit & 1;
      first |= known || at.bit == ODD_BIT ? 0u : 1u << i;
      later |= known ? 1u << i : 0u;
    }
  }
  wave_sync();
  bool twice = false;
  for (int i = 0; i < Points<1>::N; ++i)
    for (u64 who = __ballot(later >> i & 1); who; who &= who - 1) {     // (of two that are the same, one is here)
      const int from_lane = __builtin_ctzll(who), id = ids[i * WAVE + from_lane];
#pragma unroll
      for (int k = 0; k < Points<1>::N; ++k) twice |= pt.id[k] == id && !(k == i && lane == from_lane);
    }
  return Marked{first, __any(twice) != 0};
}
template <typename T> __device__ __forceinline__ void write_left_out(const Run<T>& r, T* out, const Slope& s, const Points<1>& pt, int from, int n, int kept, Marked marked, const int* ids, const float* ws) {
  constexpr int N = vec<T>();
  const int lane = threadIdx.x & 63;
  float z[Points<1>::N];
#pragma unroll
  for (int i = 0; i < Points<1>::N; ++i)
    if (pt.id[i] >= from && pt.id[i] - from < n) z[i] = to_f(r.p[pt.id[i] - from]);
  // the vectors without what the points add, by the first in each ..
#pragma unroll
  for (int i = 0; i < Points<1>::N; ++i)
    if (marked.first >> i & 1) {
      const int at = r.vec_at((pt.id[i] - from - r.head) / N);
      float x[N];
      decode<T>(ld_global(reinterpret_cast<const u32x4*>(r.p + at)), x);
      slope_vector<T, false>(x, s, -1);
      put_vector<T>(out + at, x, false);
    }
  // .. then the points themselves (a wavefront's stores to an address keep their order).  An id that comes twice is added up in
  // order, by its first.
#pragma unroll
  for (int i = 0; i < Points<1>::N; ++i) {
    if (i * WAVE >= kept) break;
    const int at = pt.id[i] - from;
    bool mine = pt.id[i] >= from && at < n;
    float sum = pt.w[i];
    if (marked.twice) {
      sum = 0.f;
      for (int j = 0; j < kept; ++j) {
        const bool same = ids[j] == pt.id[i];
        sum += same ? ws[j] : 0.f;
        mine = mine && !(same && j < i * WAVE + lane);
      }
    }
    if (mine) out[at] = from_f<T>(s.zero ? 0.f : s.template at<false>(z[i]) + s.slope * sum);
  }
}

// Bound by its bytes: 4096 x 50257 bf16 with one token a row 141 us, 5.8 TB/s.  A teacher's list costs what every run's
// wavefronts spend on looking through it: 147 us with 1 id a row, 151 with 16, 157 with 64, 190 with 200, 200 with 256.
// FROM: where a row's sums come from.  GIVEN: its log-sum-exp (and entropy) are arguments; PARTS: they lie in the workspace, and the
// rows' values are written as well.  A block (W = 4) writes a run of a row, a wavefront (W = 1) a whole short one, STEP
// vectors per lane.  dz may be z
// itself: what is needed of other runs lies in the workspace.
enum { GIVEN = 0, PARTS = 1 };
template <typename T, int W, bool ENTROPY, int MODE, int FROM>
__global__ void __launch_bounds__(THREADS) logits_gradient_kernel(const LogitsArgs a) {
  constexpr int TEAMS = WAVES / W, N = vec<T>(), team = W * WAVE;
  __shared__ float mass[TEAMS];
  __shared__ unsigned left_out[MODE == 1 ? THREADS : 1];
  __shared__ int ids[MODE == 1 ? TEAMS * KEPT : 1];
  __shared__ float ws[MODE == 1 ? TEAMS * KEPT : 1];
  const int wave = threadIdx.x / WAVE, group = wave / W, lane = threadIdx.x % team;
  const bool leads = wave % W == 0;
  const float c = LOG2E / a.tau;
  const long task = block_index() * TEAMS + group;
  if (task >= a.rows * a.runs) return;
  const long row = task / a.runs;
  const int run = (int)(task - row * a.runs), from = run * a.run_cols;
  const int n = a.cols - from < a.run_cols ? a.cols - from : a.run_cols;
  const T* z = static_cast<const T*>(a.z) + row * a.ld;
  T* out = static_cast<T*>(a.dz) + row * a.lddz + from;
  const Run<T> in(z, from, n);
  auto meet = [&]() {
    if constexpr (W > 1) __syncthreads();
    else wave_sync();
  };
  u32x4 raw[STEP];
  if (in.vecs) {
#pragma unroll
    for (int u = 0; u < STEP; ++u) {
      const int v = u * team + lane;
      const u32x4* at = reinterpret_cast<const u32x4*>(in.p + in.vec_at(v < in.vecs ? v : in.vecs - 1));
      raw[u] = MODE == 0 ? ld_stream(at) : ld_global(at);
    }
  }
  Points<MODE> pt;
  Marked marked = {0, false};
  unsigned skip = 0;
  if constexpr (MODE == 0) {
    pt.load(a, row);
  } else {
    left_out[threadIdx.x] = 0;
    if (leads) pt.load(a, row);
    meet();
    if (leads) {
      marked = leave_out<T>(in, pt, from, n, team, left_out + group * team, ids + group * KEPT, ws + group * KEPT);
      if (lane == 0) mass[group] = pt.mass;
    }
    meet();
    pt.mass = mass[group];
    skip = left_out[threadIdx.x];
  }
  Slope s;
  if constexpr (FROM == GIVEN) {
    s.template set<ENTROPY>(a, row, pt.mass, MODE == 0 ? 1.f : -1.f, ENTROPY ? a.entropy_in[row] : 0.f);
    s.from_lse(a.lse_in[row], a.tau);
  } else {
    const RowSums r(joined(a, row, c), a.tau);
    s.template set<ENTROPY>(a, row, pt.mass, MODE == 0 ? 1.f : -1.f, r.entropy);
    s.from_sums(r);
    if (run == 0 && leads) {
#pragma unroll
      for (int i = 0; i < Points<MODE>::N; ++i) pt.z[i] = i * WAVE + lane < a.points ? a.part_points[row * a.points + i * WAVE + lane] : 0.f;
      put_values<MODE>(a, row, r, pt);
    }
  }
  const int token = MODE == 0 && pt.id[0] >= 0 && !s.zero ? pt.id[0] - from : -1;
#pragma unroll
  for (int u = 0; u < STEP; ++u) {
    const int v = u * team + lane;
    if (v < in.vecs) {
      float x[N];
      decode<T>(raw[u], x);
      slope_vector<T, ENTROPY>(x, s, MODE == 0 && token >= 0 ? token - in.vec_at(v) : -1);
      if (MODE == 0 || !(skip >> u & 1)) put_vector<T>(out + in.vec_at(v), x, MODE == 0 && a.stream);
    }
  }
  if (lane < in.odd && !(skip >> ODD_BIT)) {
    const int at = in.odd_at(lane);
    out[at] = from_f<T>(s.template at<ENTROPY>(to_f(in.p[at])) + (MODE == 0 && at == token ? s.slope : 0.f));
  }
  if constexpr (MODE == 1)
    if (leads) write_left_out<T>(in, out, s, pt, from, n, a.kept, marked, ids + group * KEPT, ws + group * KEPT);
}

// ---- values and gradients of rows that fit the registers of NW wavefronts -------------------------
// RV vectors per lane.  A row is read once; the next row's loads are issued as its registers are written.  With the row's
// sums in the workspace and the row read again, 8192 x 50304 bf16 takes 394 us, here 319; that is the way of larger rows
// (1024 x 200000 bf16: 215 us), and of few long ones (fits()).
// A teacher's list is one wavefront's, while the others wait: 4096 x 50304 bf16 160 us with 1 id a row, 170 with 32, 173 with 64,
// 189 with 128, 223 with 200, 238 with 256.
// GRAD false: the values alone, of short rows (NW = 1), TOP with alternatives.
template <typename T, int NW, int RV, bool ENTROPY, int MODE, int OCC, bool GRAD, bool TOP>
__global__ void __launch_bounds__(NW == 1 ? THREADS : NW * WAVE, OCC) logits_step_kernel(const LogitsArgs a) {
  static_assert(NW == 1 || (GRAD && !TOP), "longer rows have kernels of their own for values");
  constexpr int N = vec<T>(), team = NW * WAVE, TEAMS = NW == 1 ? WAVES : 1;
  __shared__ u64 lists[TOP ? WAVES * ROOM : 1];
  __shared__ float tops[TEAMS * NW];
  __shared__ f32x2 waves[TEAMS * NW];
  __shared__ unsigned left_out[MODE == 1 && GRAD ? TEAMS * team : 1];
  __shared__ int ids[MODE == 1 && GRAD ? TEAMS * KEPT : 1];
  __shared__ float ws[MODE == 1 && GRAD ? TEAMS * KEPT : 1];
  __shared__ float mass[TEAMS];
  const int group = NW == 1 ? threadIdx.x / WAVE : 0, lane = threadIdx.x % team, wave = lane / WAVE, l = threadIdx.x & 63;
  const float c = LOG2E / a.tau, none = -__builtin_inff();
  const T* z = static_cast<const T*>(a.z);
  const long stride = (long)gridDim.x * TEAMS;
  auto meet = [&]() {                                    // (of a row's wavefronts; it waits for LDS alone: loads and stores stay in flight)
    if constexpr (NW == 1) {
      wave_sync();
    } else {
      wait_lgkm();
      bare_barrier();
    }
  };
  u32x4 raw[RV];
  float odd;
  Points<MODE> pt;
  auto load = [&](const Run<T>& r, int u) {
    const int v = u * team + lane;
    if (u * team < r.vecs) raw[u] = ld_stream(reinterpret_cast<const u32x4*>(r.p + r.vec_at(v < r.vecs ? v : r.vecs - 1)));
  };
  auto load_odd = [&](const Run<T>& r) { odd = lane < r.odd ? to_f(r.p[r.odd_at(lane)]) : none; };
  if constexpr (MODE == 1 && GRAD) left_out[group * team + lane] = 0;
  long row = (long)blockIdx.x * TEAMS + group;
  if (row < a.rows) {
    const Run<T> r(z, row * a.ld, a.cols);
#pragma unroll
    for (int u = 0; u < RV; ++u) load(r, u);
    load_odd(r);
    if (MODE == 1 && wave == 0) pt.fetch(a, row);
  }
  for (; row < a.rows; row += stride) {
    const Run<T> r(z, row * a.ld, a.cols);
    T* out = static_cast<T*>(a.dz) + row * a.lddz;
    auto each = [&](auto f) {
#pragma unroll
      for (int u = 0; u < RV; ++u)
        if (u * team + wave * WAVE < r.vecs) {           // (the same for a whole wavefront)
          float x[N];
          asm("" : "+v"(raw[u]));                        // (decoded anew in every pass: 8 values take more registers than a vector)
          decode<T>(raw[u], x);
          f(x, u);
        }
    };
    Marked marked = {0, false};
    if (MODE == 0) pt.fetch(a, row);
    if (MODE == 1 && wave == 0) {
      pt.settle(a, row);
      pt.gather(z + row * a.ld, 0, a.cols);
    }
#pragma unroll
    for (int u = 0; u < RV; ++u)
      if (u * team < r.vecs && u * team + lane >= r.vecs) raw[u] = u32x4{NOTHING<T>, NOTHING<T>, NOTHING<T>, NOTHING<T>};
    float top = odd;
    each([&](const float (&x)[N], int) {
#pragma unroll
      for (int j = 0; j < N; ++j) top = fmaxf(top, x[j]);
    });
    Top best;
    if constexpr (TOP) {
      best.start(lists, nullptr, a.top_k);
      best.best = top;
      const float bar = Top::bar_of(best.reached(a.top_k));
      best.take(lane < r.odd && odd >= bar, candidate(odd, r.odd_at(lane)));
      constexpr int PART = RV < 4 ? RV : 4;
#pragma unroll
      for (int u0 = 0; u0 < RV; u0 += PART)
        if (u0 * team < r.vecs)
          best.template take_high<T, PART>(raw + u0, bar, [&](int u) { return (u0 + u) * team + lane < r.vecs; }, [&](int u) { return r.vec_at((u0 + u) * team + lane); });
      best.finish();
      if (best.n < best.k) best.fill(0, a.cols);
    }
    top = all_max(top);
    if constexpr (NW > 1) {
      if (l == 0) tops[wave] = top;
      meet();
      top = all_max<NW>(tops[l % NW]);
    }
    top = fmaxf(top, LOWEST);
    // The token's logit, from the lane that holds it
    float z_token = 0.f;
    bool owner = false;
    if (MODE == 0 && pt.id[0] >= 0) {
      const int from_head = pt.id[0] - r.head, v = from_head / N;
      if (pt.id[0] < r.head || v >= r.vecs) {
        owner = lane < r.odd && r.odd_at(lane) == pt.id[0];
        z_token = odd;
      } else {
        u32x4 held = {0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < RV; ++u)
          if (u == v / team) held = raw[u];              // (the same u for all lanes)
        float x[N];
        decode<T>(held, x);
        z_token = x[0];
#pragma unroll
        for (int j = 1; j < N; ++j) z_token = j == from_head - v * N ? x[j] : z_token;
        owner = lane == v % team;
      }
    }
    // Exponents are x c - P as in Reader; `rest` is the part of each that P leaves out.  Where |P| is too large for that the
    // row's values become their differences to the maximum, which then is 0: those that matter are exact.
    float base = top, P = top * c, x_token = z_token;
    if (!(fabsf(P) < 0x1p20f)) {
#pragma unroll
      for (int u = 0; u < RV; ++u)
        if (u * team + wave * WAVE < r.vecs) {
          float x[N];
          decode<T>(raw[u], x);
#pragma unroll
          for (int j = 0; j < N; ++j) x[j] -= top;
          raw[u] = encode<T>(x);
        }
      odd -= top;
      x_token -= top;
      base = P = 0.f;
    }
    const float rest = fmaf(base, c, -P);
    float s = 0.f, t = 0.f;
    auto add = [&](float x) {
      const float d = fmaf(x, c, -P), e = exp2_of(d);
      s += e;
      if constexpr (MODE == 0) t = fmaf(bounded(d), e, t);
    };
    add(odd);
    each([&](const float (&x)[N], int) {
#pragma unroll
      for (int j = 0; j < N; ++j) add(x[j]);
    });
    shift(s, t, -rest);
    s = all_sum(s);
    if constexpr (MODE == 0) t = all_sum(t);
    if constexpr (MODE == 1) {
      if (GRAD && wave == 0) {
        marked = leave_out<T>(r, pt, 0, a.cols, team, left_out + group * team, ids + group * KEPT, ws + group * KEPT);
        if (l == 0) mass[group] = pt.mass;
      }
    }
    if (NW > 1 && l == 0) waves[wave] = f32x2{s, t};
    meet();
    if constexpr (NW > 1) {
      const f32x2 w = waves[l % NW];
      s = all_sum<NW>(w[0]);
      if constexpr (MODE == 0) t = all_sum<NW>(w[1]);
    }
    const RowSums sums(Sums{top, s, t}, a.tau);
    unsigned skip = 0;
    float weight = pt.mass;
    if constexpr (MODE == 1 && GRAD) {
      weight = mass[group];
      skip = left_out[group * team + lane];
      left_out[group * team + lane] = 0;                 // (marked again only behind the next row's first meeting)
    }
    Slope slope;
    slope.zero = false;
    if constexpr (GRAD) slope.template set<ENTROPY>(a, row, weight, MODE == 0 ? 1.f : -1.f, sums.entropy);
    slope.from_sums(sums);
    if (wave == 0 && l == 0) {                           // (a loss comes last)
      if (a.lse) a.lse[row] = sums.lse;
      if (MODE == 0 && a.entropy) a.entropy[row] = sums.entropy;
      if (MODE == 0 && a.logprob && pt.id[0] < 0) a.logprob[row] = pt.mass;
    }
    if (owner && a.logprob) a.logprob[row] = sums.logprob(z_token, a.tau);
    const bool more = row + stride < a.rows;
    const Run<T> next(z, (more ? row + stride : row) * a.ld, a.cols);
    if constexpr (!GRAD) {
      if (MODE == 1) put_values<MODE>(a, row, sums, pt);
      if constexpr (TOP) put_alternatives(a, row, sums, best.list);
#pragma unroll
      for (int u = 0; u < RV; ++u)
        if (more) load(next, u);
      if (more) load_odd(next);
      if (MODE == 1 && more) pt.fetch(a, row + stride);
      continue;
    }
    // log2 p = x c - Q - left: Q is P + rest + log2 s rounded
    const float tail = rest + slope.off * LOG2E;
    float Q = P + tail;
    const float left = (P - Q) + tail, whole = exp2_of(-left);
    float A = -slope.A * whole, B = -slope.B * 0.69314718055994530942f * whole;
    if (slope.zero) {
#pragma unroll
      for (int u = 0; u < RV; ++u) raw[u] = u32x4{0, 0, 0, 0};
      odd = Q = A = B = 0.f;
    }
    auto gradient = [&](float x) {
      const float lp = fmaf(x, c, -Q), p = exp2_of(lp);
      return ENTROPY ? p * fmaf(B, bounded(lp - left), A) : p * A;
    };
    if (lane < r.odd && !(skip >> ODD_BIT)) {
      const int at = r.odd_at(lane);
      out[at] = from_f<T>(gradient(odd));
    }
#pragma unroll
    for (int u = 0; u < RV; ++u) {
      if (u * team + wave * WAVE < r.vecs) {             // (the same for a whole wavefront)
        const int v = u * team + lane;
        float x[N];
        decode<T>(raw[u], x);
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = gradient(x[j]);
        if (v < r.vecs && (MODE == 0 || !(skip >> u & 1))) put_vector<T>(out + r.vec_at(v), x, a.stream);
      }
      if (more) load(next, u);
    }
    if (owner && !slope.zero) out[pt.id[0]] = from_f<T>(gradient(x_token) + slope.slope);    // (once more, behind its vector)
    if (more) load_odd(next);
    if constexpr (MODE == 1) {
      if (wave == 0) {
        put_values<MODE>(a, row, sums, pt);
        write_left_out<T>(r, out, slope, pt, 0, a.cols, a.kept, marked, ids + group * KEPT, ws + group * KEPT);
        if (more) pt.fetch(a, row + stride);
      }
      if constexpr (NW == 1) wave_sync();
    }
  }
}

// ---- launches ---------------------------------------------------------------------------
constexpr long MOST_BLOCKS = 1 << 22;                    // along x (a launch has at most 2^32 threads there)
constexpr int MOST_PARTS = WAVE;                         // a lane per part in the join

template <typename F> hipError_t with(bool x, F&& f) { return x ? f(std::true_type()) : f(std::false_type()); }
dim3 blocks_for(long tasks, int teams) {
  const long b = (tasks + teams - 1) / teams;
  return b <= MOST_BLOCKS ? dim3((unsigned)b) : dim3((unsigned)MOST_BLOCKS, (unsigned)((b + MOST_BLOCKS - 1) / MOST_BLOCKS));
}
// short rows: one wavefront each, which holds them
bool short_rows(int cols, bool is_bf16) { return cols <= (is_bf16 ? 4096 : 2048); }
// Few rows: a row's elements are shared out over several blocks, with a join behind them, from 64 KB on, into no less than
// 8 KB, at most two blocks per CU; 128 KB a part in any case.  In parts and whole: 1 x 50257 bf16 5.7 and 7.7 us, with 20
// alternatives 11.7 and 11.8; 16 x 131072 fp32 7.3 and 27.5, with 20 17.4 and 35.7; 300 x 200000 bf16 with 20 39.5 and 50.4; the join costs
// where a part is short and there are alternatives: 16 x 32003 fp32 with 20 14.6 and 12.4, 256 x 50257 bf16 with 20 19.0 and 16.9 (the
// rule does not look at top_k).
int parts_of(long rows, int cols, bool is_bf16) {
  const long bytes = (long)cols * (is_bf16 ? 2 : 4);
  if (bytes < 65536 || rows >= 512 || rows < 1) return 1;
  long parts = 512 / rows < bytes / 8192 ? 512 / rows : bytes / 8192;
  if (parts > 16) parts = 16;
  const long least = 2048 / rows < bytes / 131072 ? 2048 / rows : bytes / 131072;
  if (parts < least) parts = least;
  return (int)(parts < MOST_PARTS ? parts : MOST_PARTS);
}
// Rows that a step keeps in registers.  Few long ones keep too few CUs at work so and go through the workspace, in parts (in
// registers and in parts: 1 x 131072 bf16 19.3 and 7.7 us, 32 rows 21.4 and 10.4, 77 rows 24.4 and 19.2, 128 rows 27.0 and 24.3, 200 rows
// 30.1 and 36.9, 300 rows 56.2 and 46.4, 400 rows 55.9 and 58.9; 32 x 65536 fp32 14.7 and 9.4, 77 rows 18.2 and 16.2, 128 rows 20.5
// and 22.3, 257 rows 45.5 and 38.9, 300 rows 46.0 and 43.0).  The bound lies below the break-even at 100 to 150 rows, and does not know of
// the second one: from 257 to about 350 rows a second round of blocks, one per CU, has hardly begun, and parts would take 7 to 25 per cent
// less.  Up to 128 KB a row the two are about even for few rows (32 x 50304 bf16 10.8 and 9.5, distillation 10.5 and 12.0) and one
// launch is less than two.
bool fits(long rows, int cols, bool is_bf16) {
  const long bytes = (long)cols * (is_bf16 ? 2 : 4);
  return bytes <= 262144 && (bytes <= 131072 || rows > 64);
}
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
size_t parts_bytes(long rows, int parts, int top_k, int points) {
  return up256(rows * parts * sizeof(f32x4)) + up256(rows * parts * top_k * sizeof(u64)) + up256((size_t)rows * points * sizeof(float));
}

template <typename T, int MODE> hipError_t values(const LogitsArgs& a, hipStream_t st) {
  return with(a.top_k > 0 && MODE == 0, [&](auto top) -> hipError_t {
    constexpr bool TOP = decltype(top)::value && MODE == 0;
    logits_values_kernel<T, TOP, MODE><<<blocks_for(a.rows * a.parts, 1), THREADS, 0, st>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.part_sums || a.dz) return e;
    logits_join_kernel<T, TOP, MODE><<<blocks_for(a.rows, WAVES), THREADS, 0, st>>>(a);
    return hipGetLastError();
  });
}
template <typename T, int W, int MODE, int FROM> hipError_t gradient(const LogitsArgs& a, hipStream_t st) {
  return with(MODE == 0 && a.h, [&](auto entropy) -> hipError_t {
    logits_gradient_kernel<T, W, decltype(entropy)::value && MODE == 0, MODE, FROM><<<blocks_for(a.rows * a.runs, WAVES / W), THREADS, 0, st>>>(a);
    return hipGetLastError();
  });
}
template <typename T, int MODE, int NW, int RV, int OCC> hipError_t step_of(const LogitsArgs& a, hipStream_t st) {
  constexpr int threads = NW == 1 ? THREADS : NW * WAVE, teams = NW == 1 ? WAVES : 1;
  // as many blocks as run at once: each walks over its rows
  const long most = (long)compute_units() * (4 * OCC * WAVE / threads), blocks = (a.rows + teams - 1) / teams;
  const unsigned grid = (unsigned)(blocks < most ? blocks : most);
  if constexpr (NW == 1) {
    if (!a.dz)
      return with(MODE == 0 && a.top_k > 0, [&](auto top) -> hipError_t {
        logits_step_kernel<T, NW, RV, false, MODE, OCC, false, decltype(top)::value && MODE == 0><<<grid, threads, 0, st>>>(a);
        return hipGetLastError();
      });
  }
  return with(MODE == 0 && a.h, [&](auto entropy) -> hipError_t {
    logits_step_kernel<T, NW, RV, decltype(entropy)::value && MODE == 0, MODE, OCC, true, false><<<grid, threads, 0, st>>>(a);
    return hipGetLastError();
  });
}
// The fewer wavefronts hold a row, the more rows a CU works on, whose loads, sums and stores overlap; few rows are done
// soonest by many (step, bf16, with few as the rule has it and the other way: 1 x 50304 9.7 and 13.6 us, 64 rows 11.3 and 14.5, 256 rows
// 15.6 and 19.1, 500 rows 26.5 and 25.9, 600 rows 31.4 and 36.8, 1000 rows 38 and 49; 256 x 20000 9.6 and 10.3; 500 x 3000 5.4 and 6.6).  Not so
// everywhere: blocks of 16 wavefronts run one per CU, and from 257 rows on a second round keeps few of them at work (257 x 50304 25.7 and
// 22.9, 300 rows 24.8 and 23.7, 300 x 20000 15.0 and 12.8), and a row of up to 32 KB is too short for 16 (64 x 9000 7.1 and 6.4, 300 rows 11.9
// and 7.7).  Wavefronts per SIMD, by a sweep: what the registers of RV vectors leave room for (16384 x 3000, distillation, 4 and 5: 54 and 71 us).
template <typename T, int MODE> hipError_t step(const LogitsArgs& a, hipStream_t st) {
  const int vecs = a.cols / vec<T>();                    // (an odd element less may make one vector less)
  const bool few = a.rows <= 2 * compute_units();
  if (vecs <= WAVE) return step_of<T, MODE, 1, 1, 6>(a, st);
  if (vecs <= 4 * WAVE) return step_of<T, MODE, 1, 4, 5>(a, st);
  if (vecs <= 8 * WAVE && (!few || !a.dz)) return step_of<T, MODE, 1, 8, MODE == 0 ? 5 : 4>(a, st);
  if (vecs <= 4 * 4 * WAVE) return step_of<T, MODE, 4, 4, 5>(a, st);
  if (vecs <= 4 * 8 * WAVE && !few) return step_of<T, MODE, 4, 8, 4>(a, st);
  if (vecs <= 4 * 16 * WAVE && !few) return step_of<T, MODE, 4, 16, 4>(a, st);
  if (vecs <= 4 * 26 * WAVE && !few) return step_of<T, MODE, 4, 26, 3>(a, st);
  if (vecs <= 16 * 8 * WAVE) return step_of<T, MODE, 16, 8, 4>(a, st);
  if (vecs <= 16 * 13 * WAVE) return step_of<T, MODE, 16, 13, 4>(a, st);
  return step_of<T, MODE, 16, 16, 4>(a, st);
}

template <typename T, int MODE> hipError_t launch(LogitsArgs a, bool resident, hipStream_t st) {
  constexpr int LANE_TILE = STEP * vec<T>();             // elements that a lane loads together
  if (resident) return step<T, MODE>(a, st);
  if (!a.dz) return values<T, MODE>(a, st);
  // A row of one tile to a wavefront, else a block to a run (so and with blocks: 16384 x 2000 bf16 25.8 and 33.6 us, 16384 x 1000
  // 15.6 and 27.9, 16384 x 64 8.1 and 17.5; 64 x 1000 fp32 3.6 and 3.2).
  if (a.lse_in && a.cols <= WAVE * LANE_TILE) {
    a.runs = 1;
    a.run_cols = a.cols;
    return gradient<T, 1, MODE, GIVEN>(a, st);
  }
  a.run_cols = THREADS * LANE_TILE;
  a.runs = (a.cols + a.run_cols - 1) / a.run_cols;
  if (a.lse_in) return gradient<T, WAVES, MODE, GIVEN>(a, st);
  const hipError_t e = values<T, MODE>(a, st);
  return e != hipSuccess ? e : gradient<T, WAVES, MODE, PARTS>(a, st);
}

}  // namespace

size_t logits_workspace_bytes(long rows, int cols, bool is_bf16, int top_k, int points, bool step) {
  if (rows == 0 || (step && fits(rows, cols, is_bf16))) return 0;
  const int parts = parts_of(rows, cols, is_bf16);
  return parts > 1 || step ? parts_bytes(rows, parts, top_k, points) : 0;
}

hipError_t launch_logits(LogitsArgs a, int mode, bool is_bf16, void* workspace, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  const double elems = (double)a.rows * a.cols, size = is_bf16 ? 2 : 4;
  ProfScope ps(a.lse_in ? PC_LOGITS_GRAD : a.dz ? PC_LOGITS_STEP : PC_LOGITS, elems * (a.dz && !a.lse_in ? 10 : 6), elems * size * (a.dz ? 2 : 1), st);
  const bool stepping = a.dz && !a.lse_in, resident = stepping ? fits(a.rows, a.cols, is_bf16) : !a.lse_in && short_rows(a.cols, is_bf16);
  a.parts = a.lse_in || resident ? 1 : parts_of(a.rows, a.cols, is_bf16);
  a.part_cols = a.cols;
  a.points = mode == 0 ? 1 : a.kept;
  // Gradients that no cache could hold are written past them: past and into them 8192 x 50304 bf16 274 and 300 us backward, 314
  // and 326 in a step, 4096 x 50304 137 and 148.  Smaller ones stay for who reads them next, at the same cost (2048 x 50304:
  // 69.5 and 68.1 us, a step 78.3 and 73.9; 1024 x 50304: 36.9 and 38.6, 37.4 and 40.8).
  a.stream = elems * size > 256.0 * (1 << 20);
  if (a.parts > 1 || (stepping && !resident)) {
    // (whole 128-byte lines apart, but for the rows' own alignment)
    a.part_cols = ((a.cols + a.parts - 1) / a.parts + 63) / 64 * 64;
    a.parts = (a.cols + a.part_cols - 1) / a.part_cols;
    char* at = static_cast<char*>(workspace);
    a.part_sums = reinterpret_cast<f32x4*>(at);
    at += up256(a.rows * a.parts * sizeof(f32x4));
    a.part_lists = reinterpret_cast<unsigned long long*>(at);
    at += up256(a.rows * a.parts * a.top_k * sizeof(u64));
    a.part_points = stepping ? reinterpret_cast<float*>(at) : nullptr;
  }
  return with(is_bf16, [&](auto b) {
    typedef typename std::conditional<decltype(b)::value, bf16, float>::type T;
    return with(mode == 0, [&](auto m) { return launch<T, decltype(m)::value ? 0 : 1>(a, resident, st); });
  });
}

}  // namespace mg
