// Scores of tokens from logits: log probability of given words, log-sum-exp, entropy and the likeliest words; and the gradient of the logits.
//
// Every logit is read once.  With x the logits, m their maximum, e = scale (x - m), l = sum exp e and w = sum (exp e) e:
//     lse = scale m + log l,   logp = e_y - log l,   entropy = log l - w / l   (in base 2 inside),
// kept against a running maximum by each lane of its own elements.  The difference is taken before the scale: it is 0 at the maximum whatever its size, so rows and forbidden words at
// large finite numbers (-1e10, the type's lowest) come out as they should.  (From a product of the maximum, e = x scale - fl(m scale) is its rounding, beyond 128 at numbers of 3e9.)
//   The likeliest words: while the row is read, each lane keeps the largest number of its elements, the step (32 or 16 elements) where it came first, and the
// largest of the other steps: nine instructions a step.  The n_top-th of the lanes' largest is a bound that n_top words reach, and only those n_top lanes
// can have others: they read that step again (and, the few whose second largest reaches the bound, the others), and what reaches the bound, about n_top words,
// is sorted.  An entry is the number, as a whole one of the same order, over the complement of its index: equal numbers go by the lowest index, rows of equal
// numbers (masked ones) give a bound that few words reach like any other, and any way of dealing the elements out gives the same words.
//   A row is a wave's where there are many, else several waves' or several work-groups', whose sums and lists are joined.
//   Measured: 4001 x 128256 bf16, 20 words 226 us (4.5 TB/s, vector unit 88 % busy; without words 182, 5.6 TB/s); 4096 x 32000 fp32 without words 98 us (5.4 TB/s); 60 x 32000, 8 words
// 12.5 us, of which the words are 4.5.  Lists that are kept in order while a row is read took 318 us in the first case.
#include <algorithm>
#include <type_traits>

#include "cache.hpp"
#include "kernels.hpp"

namespace burst {

namespace {

typedef __attribute__((ext_vector_type(8))) float f32x8;

constexpr int kMostSegments = 16;      // work-groups of a row
constexpr int64_t kScoresUnits = 256;   // compute units
constexpr float kNothing = -1000.f;    // exp2 of this is 0: in place of -inf where it is multiplied with such a zero

// A number and its index as one whole number: greater numbers first, among equals (0 and -0 are) the lower index.  0: no entry.
__device__ __forceinline__ uint64_t entry_of(float x, int32_t index) {
  uint32_t bits = __builtin_bit_cast(uint32_t, x);
  bits = bits == 0x80000000u ? 0u : bits;
  const uint32_t order = bits >> 31 ? ~bits : bits | 0x80000000u;
  return (uint64_t)order << 32 | (uint32_t)~index;
}
__device__ __forceinline__ float number_of(uint64_t entry) {
  const uint32_t order = (uint32_t)(entry >> 32);
  return entry == 0 ? -INFINITY : __builtin_bit_cast(float, order >> 31 ? order & 0x7fffffffu : ~order);
}
__device__ __forceinline__ bool is_nan(float x) { return (__builtin_bit_cast(uint32_t, x) & 0x7fffffffu) > 0x7f800000u; }

// One stage of a bitonic network over the lanes: of the two lanes that STEP parts, the one below keeps the larger if `larger_below`.
template <int STEP>
__device__ __forceinline__ uint64_t exchanged(uint64_t x, bool larger_below, int lane) {
  const uint64_t y = (uint64_t)of_lane_xor<STEP>((uint32_t)(x >> 32)) << 32 | of_lane_xor<STEP>((uint32_t)x);
  return (x > y) == (((lane & STEP) == 0) == larger_below) ? x : y;
}
template <int STEP>
__device__ __forceinline__ uint64_t exchanged_down(uint64_t x, bool larger_below, int lane) {   // stages STEP, STEP / 2, .. 1
  x = exchanged<STEP>(x, larger_below, lane);
  if constexpr (STEP > 1) x = exchanged_down<STEP / 2>(x, larger_below, lane);
  return x;
}
// A bitonic sequence sorted, the largest in lane 0
__device__ __forceinline__ uint64_t merged_down(uint64_t x, int lane) { return exchanged_down<32>(x, true, lane); }
template <bool DOWN>
__device__ __forceinline__ uint64_t sorted(uint64_t x, int lane) {
  x = exchanged_down<1>(x, ((lane & 2) == 0) == DOWN, lane);
  x = exchanged_down<2>(x, ((lane & 4) == 0) == DOWN, lane);
  x = exchanged_down<4>(x, ((lane & 8) == 0) == DOWN, lane);
  x = exchanged_down<8>(x, ((lane & 16) == 0) == DOWN, lane);
  x = exchanged_down<16>(x, ((lane & 32) == 0) == DOWN, lane);
  return exchanged_down<32>(x, DOWN, lane);
}
// The 64 largest of a list and of entries sorted the other way round
__device__ __forceinline__ uint64_t joined(uint64_t list, uint64_t up, int lane) { return merged_down(list > up ? list : up, lane); }

// From differences of logits to base-2 exponents (finite for the largest scales too: 0 has to stay 0)
__device__ __forceinline__ float exponents_of(float scale) { return fminf(scale * kLog2e, 3.4028235e38f); }

// What a part of a row comes to.
struct RowSums {
  float m, l, w;   // largest logit; with e = to_log2 (x - m): sum of exp2(e), sum of exp2(e) e
  __device__ __forceinline__ void join(const RowSums& o, float to_log2) {
    const float top = fmaxf(m, o.m);
    const float d0 = m == top ? 0.f : fmaxf((m - top) * to_log2, kNothing), d1 = o.m == top ? 0.f : fmaxf((o.m - top) * to_log2, kNothing);
    const float f0 = __builtin_amdgcn_exp2f(d0), f1 = __builtin_amdgcn_exp2f(d1);
    w = (w + l * d0) * f0 + (o.w + o.l * d1) * f1;
    l = l * f0 + o.l * f1;
    m = top;
  }
  template <int STEP>
  __device__ __forceinline__ void join_lane_xor(float to_log2) {
    auto other = [](float x) { return __builtin_bit_cast(float, of_lane_xor<STEP>(__builtin_bit_cast(uint32_t, x))); };
    join(RowSums{other(m), other(l), other(w)}, to_log2);
  }
  __device__ __forceinline__ void join_lanes(float to_log2) {
    join_lane_xor<1>(to_log2);
    join_lane_xor<2>(to_log2);
    join_lane_xor<4>(to_log2);
    join_lane_xor<8>(to_log2);
    join_lane_xor<16>(to_log2);
    join_lane_xor<32>(to_log2);
  }
};

// A row of logits as vectors of 16 bytes from the aligned address at or below its first element on.
template <bool F32>
struct RowVectors {
  static constexpr int VEC = F32 ? 4 : 8;
  const char* row;      // its first element
  int32_t before, vocab;   // elements of the first vector that lie before it
  __device__ __forceinline__ void init(const void* logits, int64_t at, int32_t words) {   // at: the row's first element
    before = (int32_t)(at & (VEC - 1));
    row = (const char*)logits + at * (F32 ? 4 : 2);
    vocab = words;
  }
  __device__ __forceinline__ void init(const ScoresParams& p, int64_t token) { init(p.logits, token * p.ld, p.vocab); }
  __device__ __forceinline__ int32_t vectors() const { return (int32_t)(((int64_t)before + vocab + VEC - 1) / VEC); }
  __device__ __forceinline__ float element(int32_t i) const {
    return F32 ? ((const float*)row)[i] : __builtin_bit_cast(float, (uint32_t)((const uint16_t*)row)[i] << 16);
  }
  // Vector j, elements VEC j - before ..; those outside the row are -inf.
  __device__ __forceinline__ u32x4 load(int64_t j) const {
    const int64_t e0 = j * VEC - before;
    if (e0 >= 0 && e0 + VEC <= vocab) return *reinterpret_cast<const u32x4*>(row + e0 * (F32 ? 4 : 2));
    u32x4 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (F32) {
        x[i] = e0 + i >= 0 && e0 + i < vocab ? ((const uint32_t*)row)[e0 + i] : 0xff800000u;
      } else {
        const uint32_t lo = e0 + 2 * i >= 0 && e0 + 2 * i < vocab ? ((const uint16_t*)row)[e0 + 2 * i] : 0xff80u;
        const uint32_t hi = e0 + 2 * i + 1 >= 0 && e0 + 2 * i + 1 < vocab ? ((const uint16_t*)row)[e0 + 2 * i + 1] : 0xff80u;
        x[i] = lo | hi << 16;
      }
    }
    return x;
  }
  static __device__ __forceinline__ float value(const u32x4& x, int i) {
    const uint32_t word = F32 ? x[i] : x[i / 2];
    return __builtin_bit_cast(float, F32 ? word : i & 1 ? word & 0xffff0000u : word << 16);
  }
};

// What a lane remembers of its part of a row: the largest numbers of the steps where they are largest and next to largest, those steps (their first vector;
// among equals the first step), and the largest number of all others.
struct LaneBest {
  float best, second, third;
  int32_t step, second_step;
  __device__ __forceinline__ void see(float x, int32_t j0) {
    const bool first = x > best, next = x > second;
    third = fmaxf(third, fminf(second, x));
    second_step = first ? step : next ? j0 : second_step;
    second = fmaxf(second, fminf(best, x));
    step = first ? j0 : step;
    best = fmaxf(best, x);
  }
};

// A wave's part of a row, vectors v0 .. v1 - 1, 64 U in each step.
constexpr int U = 4;
template <bool F32, bool TOP>
__device__ __forceinline__ void scan_row(const RowVectors<F32>& row, int32_t v0, int32_t v1, float to_log2, int lane, RowSums& sums, LaneBest& top) {
  constexpr int VEC = RowVectors<F32>::VEC;
  sums = RowSums{-INFINITY, 0.f, 0.f};
  top = LaneBest{-INFINITY, -INFINITY, -INFINITY, v0, v0};
  bool masked = false;   // some number so far was -inf (or NaN)
  for (int32_t j0 = v0; j0 < v1; j0 += 64 * U) {
    u32x4 x[U];
    const u32x4 none = F32 ? u32x4{0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u} : u32x4{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u};
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = j0 + 64 * u + lane < v1 ? row.load(j0 + 64 * u + lane) : none;
    float most[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      auto y = [&](int i) { return RowVectors<F32>::value(x[u], i); };
      most[u] = max3(y(0), y(1), max3(y(2), y(3), -INFINITY));
      if constexpr (!F32) most[u] = max3(max3(y(4), y(5), most[u]), y(6), y(7));
    }
    static_assert(U == 4, "four of them");
    const float step = max3(max3(most[0], most[1], most[2]), most[3], -INFINITY);
    if constexpr (TOP) top.see(step, j0);
    // (a scale is positive: the largest logit is the largest exponent)
    const float m = fmaxf(sums.m, step), d = sums.m == m ? 0.f : fmaxf((sums.m - m) * to_log2, kNothing), f = __builtin_amdgcn_exp2f(d);
    sums.w = (sums.w + sums.l * d) * f;
    sums.l *= f;
    sums.m = m;
    const float base = m == -INFINITY ? 0.f : m;
    auto add = [&](auto masked_) {   // (a number at -inf has the weight 0, and 0 * -inf would be NaN)
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const float e = (RowVectors<F32>::value(x[u], i) - base) * to_log2, p = __builtin_amdgcn_exp2f(e);
          sums.l += p;
          sums.w = fmaf(p, decltype(masked_)::value ? fmaxf(e, kNothing) : e, sums.w);
        }
    };
    if (!masked) {   // without that care as long as there is none
      const float l = sums.l, w = sums.w;
      add(std::false_type());
      masked = __any(is_nan(sums.w)) != 0;
      if (masked) {
        sums.l = l;
        sums.w = w;
      }
    }
    if (masked) add(std::true_type());
  }
  sums.join_lanes(to_log2);
}

// Sums and lists of the work-group's waves, in wave 0.
template <int W, bool TOP>
__device__ __forceinline__ void join_waves(RowSums& sums, uint64_t& list, float to_log2, RowSums* sums_lds, uint64_t* lists, int wave, int lane) {
  if (lane == 0) sums_lds[wave] = sums;
  if (TOP) lists[64 * wave + lane] = list;
  __syncthreads();
#pragma unroll
  for (int s = 1; s < W; s <<= 1) {
    if (wave % (2 * s) == 0) {
      sums.join(sums_lds[wave + s], to_log2);
      if (lane == 0) sums_lds[wave] = sums;
      if (TOP) {
        list = joined(list, lists[64 * (wave + s) + 63 - lane], lane);
        lists[64 * wave + lane] = list;
      }
    }
    __syncthreads();
  }
}
// A lane's entry, in all of them
__device__ __forceinline__ uint64_t of_lane(uint64_t x, int lane) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, lane);
}

// The likeliest words of a part of a row that W waves have, vectors v0 .. v1 - 1 this one: a lane each of wave 0, the first in lane 0.  found: LDS, kFound entries
// and behind them their number (zero), of the waves together; lists: as for join_waves.  sums are joined on the way.
template <int W>
constexpr int kFound = W == 1 ? 256 : 1024;
template <bool F32, int W>
__device__ __forceinline__ uint64_t likeliest(const RowVectors<F32>& row, int32_t v0, int32_t v1, const LaneBest& top, int n_top, RowSums& sums, float to_log2,
                                              RowSums* sums_lds, uint64_t* lists, uint64_t* found, int* count, int wave, int lane) {
  constexpr int VEC = RowVectors<F32>::VEC;
  auto index = [&](int32_t j, int i) { return (int32_t)((int64_t)j * VEC - row.before + i); };
  auto is_word = [&](int32_t id, float y) { return (uint32_t)id < (uint32_t)row.vocab && !is_nan(y); };
  // The step with the lane's largest number again, and the first word there that has it
  u32x4 x[U];
#pragma unroll
  for (int u = 0; u < U; ++u) x[u] = top.step + 64 * u + lane < v1 ? row.load(top.step + 64 * u + lane) : u32x4{};
  uint64_t mine = 0;
#pragma unroll
  for (int u = U - 1; u >= 0; --u) {
    const int32_t j = top.step + 64 * u + lane;
    int32_t id = -1;
#pragma unroll
    for (int i = VEC - 1; i >= 0; --i) id = RowVectors<F32>::value(x[u], i) == top.best && (uint32_t)index(j, i) < (uint32_t)row.vocab ? index(j, i) : id;
    mine = id >= 0 && j < v1 ? entry_of(top.best, id) : mine;
  }
  uint64_t list = sorted<true>(mine, lane);
  uint64_t bound;
  if constexpr (W == 1) {
    bound = of_lane(list, n_top - 1);
  } else {
    join_waves<W, true>(sums, list, to_log2, sums_lds, lists, wave, lane);
    bound = lists[n_top - 1];
  }
  // What reaches it
  const float bound_number = number_of(bound);
  int n = 0;   // W = 1: found so far
  auto look = [&](const u32x4& x, int32_t j, bool active) {
    auto value = [&](int i) { return RowVectors<F32>::value(x, i); };
    float most = max3(value(0), value(1), max3(value(2), value(3), -INFINITY));
    if constexpr (!F32) most = max3(max3(value(4), value(5), most), value(6), value(7));
    if (!__any(active && most >= bound_number)) return;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const float y = value(i);
      const bool near = active && y >= bound_number;
      if (!__any(near)) continue;
      const uint64_t entry = entry_of(y, index(j, i));
      const bool passes = near && is_word(index(j, i), y) && entry >= bound;
      const uint64_t who = __ballot(passes);
      if (who == 0) continue;
      int at = n;
      if constexpr (W == 1) n += __builtin_popcountll(who);
      else at = __builtin_amdgcn_readlane(lane == __builtin_ctzll(who) ? atomicAdd(count, __builtin_popcountll(who)) : 0, __builtin_ctzll(who));
      at += __builtin_popcountll(who & ((1ull << lane) - 1));
      if (passes && at < kFound<W>) found[at] = entry;
    }
  };
  const bool has = mine != 0 && mine >= bound;
  if (__any(has)) {
#pragma unroll
    for (int u = 0; u < U; ++u) look(x[u], top.step + 64 * u + lane, has && top.step + 64 * u + lane < v1);
  }
  // (the step that a lane's second largest is from; it is the step above where there is no other, or nothing larger than -inf in it)
  const bool second = has && top.second >= bound_number && top.second_step != top.step;
  if (__any(second)) {
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = second && top.second_step + 64 * u + lane < v1 ? row.load(top.second_step + 64 * u + lane) : u32x4{};
#pragma unroll
    for (int u = 0; u < U; ++u) look(x[u], top.second_step + 64 * u + lane, second && top.second_step + 64 * u + lane < v1);
  }
  const bool more = has && top.third >= bound_number;
  if (__any(more)) {
    for (int32_t j = v0; j < v1; j += 64 * U) {
      const bool other = more && j != top.step && j != top.second_step;
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = other && j + 64 * u + lane < v1 ? row.load(j + 64 * u + lane) : u32x4{};
#pragma unroll
      for (int u = 0; u < U; ++u) look(x[u], j + 64 * u + lane, other && j + 64 * u + lane < v1);
    }
  }
  if constexpr (W > 1) {
    __syncthreads();
    n = *count;
  }
  if (n <= kFound<W>) {
    if (W > 1 && wave != 0) return 0;
    __builtin_amdgcn_wave_barrier();
    list = sorted<true>(lane < n ? found[lane] : 0, lane);
    for (int c = 64; c < n; c += 64) list = joined(list, sorted<false>(c + lane < n ? found[c + lane] : 0, lane), lane);
    return list;
  }
  // Too many (large numbers of which few lanes have all): the next one after the other, over the whole part each time
  uint64_t last = ~0ull;
  list = 0;
  for (int t = 0; t < n_top; ++t) {
    uint64_t next = 0;
    for (int32_t j = v0 + lane; j < v1; j += 64) {
      const u32x4 x = row.load(j);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float y = RowVectors<F32>::value(x, i);
        const uint64_t entry = is_word(index(j, i), y) ? entry_of(y, index(j, i)) : 0;
        if (entry < last && entry > next) next = entry;
      }
    }
    next = of_lane(sorted<true>(next, lane), 0);
    if constexpr (W > 1) {
      __syncthreads();
      if (lane == 0) found[wave] = next;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < W; ++w) next = found[w] > next ? found[w] : next;
    }
    if (lane == t) list = next;
    last = next;
  }
  return list;
}

// A token's results from its row's sums and list, by one wave.
template <bool F32>
__device__ __forceinline__ void write_scores(const ScoresParams& p, int64_t token, const RowSums& sums, uint64_t list, int lane) {
  const bool none = sums.l == 0.f;   // (every word at -inf; NaN is not)
  const float log_l = __builtin_amdgcn_logf(sums.l), ln_l = log_l * kLn2;
  if (lane == 0) {
    if (p.lse) p.lse[token] = none ? -INFINITY : fmaf(sums.m, p.scale, ln_l);
    if (p.entropy) p.entropy[token] = none ? 0.f : (log_l - sums.w / sums.l) * kLn2;
    if (p.logp) {
      const int64_t y = p.y[token];
      RowVectors<F32> row;
      row.init(p, token);
      p.logp[token] = y < 0 || y >= p.vocab ? 0.f : none ? -INFINITY : (row.element((int32_t)y) - sums.m) * p.scale - ln_l;
    }
  }
  if (lane < p.n_top) {
    const int64_t to = token * p.n_top + lane;
    if (p.top_ids) p.top_ids[to] = list == 0 ? 0 : (int64_t)(int32_t)~(uint32_t)list;   // (fewer words than n_top: the others are NaN)
    if (p.top_logp) p.top_logp[to] = none ? -INFINITY : (number_of(list) - sums.m) * p.scale - ln_l;
  }
}

// What a work-group leaves of its segment of a row: sums, then its list.
struct Partial {
  RowSums sums;
  int32_t unused;
};

// W waves for a segment of a row; with W = 1 four rows for a work-group of four waves.
template <bool F32, bool TOP, int W>
__global__ __launch_bounds__(64 * (W == 1 ? 4 : W)) void scores_kernel(ScoresParams p, int32_t segments) {
  constexpr int WAVES = W == 1 ? 4 : W;
  __shared__ uint64_t lists[TOP && W > 1 ? W * 64 : 1];
  __shared__ uint64_t found[W == 1 ? WAVES : 1][TOP ? kFound<W> : 1];
  __shared__ RowSums sums_lds[WAVES];
  __shared__ int count;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int64_t token = W == 1 ? (int64_t)blockIdx.x * WAVES + wave : (int64_t)((uint32_t)blockIdx.x / (uint32_t)segments);
  const int32_t segment = W == 1 ? 0 : (int32_t)((uint32_t)blockIdx.x - (uint32_t)token * (uint32_t)segments);
  if (token >= p.n_tokens) return;   // (W = 1: no barrier follows)
  if (TOP && W > 1 && threadIdx.x == 0) count = 0;
  RowVectors<F32> row;
  row.init(p, token);
  const int64_t vectors = row.vectors(), parts = (int64_t)segments * W, part = W == 1 ? 0 : (int64_t)segment * W + wave;
  const int32_t v0 = (int32_t)(vectors * part / parts), v1 = (int32_t)(vectors * (part + 1) / parts);
  RowSums sums;
  LaneBest top;
  uint64_t list = 0;
  const float to_log2 = exponents_of(p.scale);
  scan_row<F32, TOP>(row, v0, v1, to_log2, lane, sums, top);
  if constexpr (TOP) list = likeliest<F32, W>(row, v0, v1, top, p.n_top, sums, to_log2, sums_lds, lists, found[W == 1 ? wave : 0], &count, wave, lane);
  else if constexpr (W > 1) join_waves<W, false>(sums, list, to_log2, sums_lds, lists, wave, lane);
  if (W > 1 && wave != 0) return;
  if (segments == 1) {
    write_scores<F32>(p, token, sums, list, lane);
    return;
  }
  const int64_t at = token * segments + segment;
  if (lane == 0) ((Partial*)p.workspace)[at] = Partial{sums, 0};
  if (TOP && lane < p.n_top) ((uint64_t*)((Partial*)p.workspace + p.n_tokens * segments))[at * p.n_top + lane] = list;
}

// The segments of a row: a wave for each.
template <bool F32, bool TOP>
__global__ __launch_bounds__(64 * kMostSegments) void scores_join_kernel(ScoresParams p, int32_t segments) {
  __shared__ uint64_t lists[TOP ? kMostSegments * 64 : 1];
  __shared__ RowSums sums_lds[kMostSegments];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int64_t token = blockIdx.x, at = token * segments + wave;
  RowSums sums{-INFINITY, 0.f, 0.f};
  uint64_t list = 0;
  if (wave < segments) {
    sums = ((const Partial*)p.workspace)[at].sums;
    if (TOP && lane < p.n_top) list = ((const uint64_t*)((const Partial*)p.workspace + p.n_tokens * segments))[at * p.n_top + lane];
  }
  join_waves<kMostSegments, TOP>(sums, list, exponents_of(p.scale), sums_lds, lists, wave, lane);
  if (wave == 0) write_scores<F32>(p, token, sums, list, lane);
}

// How a row is dealt out: waves of a work-group, and work-groups.  us with 8 (20 where there are 300 tokens or more) words, bf16:
//   tokens x vocabulary          1 wave     4     16     16 x 4 work-groups and a join
//   1 x 32000                     24.2   11.2   13.3   16.8
//   1 x 128256                    62.2   23.0   19.3   17.4
//   1 x 262144                     120   38.3   26.6   18.1 (x 8: 16.5)
//   60 x 5000                     11.1    8.7   13.0
//   60 x 32000                    29.5   12.4   14.2   17.3
//   60 x 65000                    57.7   17.2   16.4   17.9
//   60 x 262144                    224   44.4   28.4   20.8 (x 8, which is more work-groups than compute units: 29.0)
//   300 x 32000                   39.3   17.0   26.4
//   800 x 128256                   149   65.7   84.2
//   16000 x 5000                  70.4    146    704
//   4001 x 32000                  80.1   75.9    198
//   4001 x 128256                  265    225    329
// Calls without words go by the same rule, which was not measured for them.
// (A launch has fewer than 2^32 threads, so the most tokens get a wave each, four of them a work-group.)
struct ScoresShape {
  int waves, segments;
};
ScoresShape scores_shape(int64_t n_tokens, int32_t vocab) {
  if (vocab <= 2048 || (n_tokens >= 2048 && vocab < 16384) || n_tokens >= (1 << 23)) return {1, 1};
  if (n_tokens > kScoresUnits || vocab < 65536) return {4, 1};
  if (vocab < 98304) return {16, 1};
  return {16, (int)std::max<int64_t>(1, std::min<int64_t>({kMostSegments, vocab / 32768, kScoresUnits / std::max<int64_t>(1, n_tokens)}))};
}

template <bool F32, bool TOP>
hipError_t launch(const ScoresParams& p, hipStream_t stream) {
  const ScoresShape s = scores_shape(p.n_tokens, p.vocab);
  if (s.waves == 1) hipLaunchKernelGGL((scores_kernel<F32, TOP, 1>), dim3((uint32_t)((p.n_tokens + 3) / 4)), dim3(256), 0, stream, p, 1);
  else if (s.waves == 4) hipLaunchKernelGGL((scores_kernel<F32, TOP, 4>), dim3((uint32_t)p.n_tokens), dim3(256), 0, stream, p, 1);
  else hipLaunchKernelGGL((scores_kernel<F32, TOP, 16>), dim3((uint32_t)(p.n_tokens * s.segments)), dim3(1024), 0, stream, p, s.segments);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || s.segments == 1) return e;
  hipLaunchKernelGGL((scores_join_kernel<F32, TOP>), dim3((uint32_t)p.n_tokens), dim3(64 * kMostSegments), 0, stream, p, s.segments);
  return hipGetLastError();
}

// ---- the gradient ----------------------------------------------------------------------------------------
// d x_j = scale * [ p_j (g_lse - g_logp - sum g_top - g_entropy (log p_j + entropy)) + g_logp [j = y] + sum over k of g_top,k [j = id_k] ]
// Every logit is read once and every gradient written once but for the few words that are named: their logits are read before anything is written (the
// gradient may take the logits' place), and their gradients written once more, whole, behind the others of their part of the row.
// Bound by memory: 4096 x 32000 fp32 202 us, 1.05 GB at 5.2 TB/s.  (Four runs of a thread loaded before the first is stored: 50 us more in fp32, nothing in bf16.)
//   A log probability is x scale - lse, off by lse's rounding, 2^-25 of it.  Where |lse| is beyond kFarLse (rows at large finite numbers: a lse of -1e10 is the same for one word and for
// 128256) that says too little or nothing, and the maximum and the sum are formed again from the row, by the threads of its first part, which then do the others' work too: nobody else
// reads a row that may be written in its place.  (4096 x 128256 bf16: 346 us, 374 with 16 such rows; 4096 x 32000 fp32: 227 us, 254 with 256, 828 with nothing else.)
constexpr float kFarLse = 4096.f;

struct RowSlope {
  float m, lse, entropy, g_all, g_entropy, scale;   // log p = scale (x - m) - lse
  bool none;   // a row all at -inf, or to be left out (it may hold anything)
  __device__ __forceinline__ float of_sum(float x) const {   // of the part without named words
    const float logp = fmaf(x - m, scale, -lse), p = __builtin_amdgcn_exp2f(logp * kLog2e);
    return none ? 0.f : p * fmaf(-g_entropy, fmaxf(logp, kNothing) + entropy, g_all);
  }
};

constexpr int kSlopeChunk = 8192;   // elements of a part of a row

// A value of each of a part's threads joined over all of them, in all of them.  lds: a number for each wave.
template <int T, class Join>
__device__ __forceinline__ float over_part(float x, Join join, float* lds) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) x = join(x, __shfl_xor(x, s, 64));
  if constexpr (T > 64) {
    __syncthreads();
    lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
#pragma unroll
    for (int i = 1; i < T / 64; ++i) x = join(x, lds[i]);
  }
  return x;
}

// T: threads of a part, of which a work-group of 256 has one or four.
template <bool F32, bool TO_F32, bool NT, int T>
__global__ __launch_bounds__(256) void scores_bwd_kernel(ScoresBwdParams p, int32_t chunks) {
  const int tid = T == 256 ? (int)threadIdx.x : (int)threadIdx.x & 63;
  const uint32_t part = T == 256 ? blockIdx.x : blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int64_t number = (int64_t)(part / (uint32_t)chunks), token = number < p.n_tokens ? number : p.n_tokens - 1;   // (the last work-group may have too many parts)
  const int32_t chunk = (int32_t)(part - (uint32_t)number * (uint32_t)chunks), vocab = number < p.n_tokens ? p.vocab : 0;
  const int64_t from = token * p.ld, to = token * p.ld_out;
  // Runs of 8 start at multiples of 8 of the logits' memory; of the gradient's too if its rows lie alike.
  const int32_t before = (int32_t)(from & 7), e_first = chunk * kSlopeChunk - before;
  __shared__ float joined_lds[T / 64];
  const bool alike = ((from ^ to) & 7) == 0;
  const int64_t y = p.y ? p.y[token] : -1;
  const bool has_y = y >= 0 && y < p.vocab && p.g_logp;
  RowSlope s;
  s.m = 0.f;
  s.lse = p.lse[token];
  s.none = s.lse == -INFINITY;
  const bool far = fabsf(s.lse) > kFarLse && !s.none;   // (the same for all threads of a part)
  if (far && chunk != 0) return;                        // (T = 256: of the whole work-group)
  s.entropy = p.g_entropy ? p.entropy[token] : 0.f;
  s.g_entropy = p.g_entropy ? p.g_entropy[token] : 0.f;
  s.scale = p.scale;
  const float g_logp = has_y ? p.g_logp[token] : 0.f;
  auto top_id = [&](int k) { return p.top_ids[token * p.n_top + k]; };
  auto is_word = [&](int64_t id) { return id >= 0 && id < vocab; };
  const int n_top = p.g_top ? p.n_top : 0;
  float g_all = (p.g_lse ? p.g_lse[token] : 0.f) - g_logp;
  for (int k = 0; k < n_top; ++k) g_all -= is_word(top_id(k)) ? p.g_top[token * p.n_top + k] : 0.f;
  s.g_all = g_all;
  const char* const row = (const char*)p.logits + from * (F32 ? 4 : 2);
  char* const out = (char*)p.d_logits + to * (TO_F32 ? 4 : 2);
  auto element = [&](int64_t i) { return F32 ? ((const float*)row)[i] : __builtin_bit_cast(float, (uint32_t)((const uint16_t*)row)[i] << 16); };
  auto put = [&](int64_t i, float x) {
    if (TO_F32) ((float*)out)[i] = x;
    else ((__bf16*)out)[i] = (__bf16)x;
  };

  if (far) {
    RowVectors<F32> again;
    again.init(p.logits, from, vocab);
    const int32_t vectors = again.vectors();
    const float to_log2 = exponents_of(p.scale);
    float m = -INFINITY, l = 0.f;
    for (int32_t j = tid; j < vectors; j += T) {
      const u32x4 x = again.load(j);
#pragma unroll
      for (int i = 0; i < RowVectors<F32>::VEC; ++i) m = fmaxf(m, RowVectors<F32>::value(x, i));
    }
    s.m = over_part<T>(m, [](float a, float b) { return fmaxf(a, b); }, joined_lds);
    for (int32_t j = tid; j < vectors; j += T) {
      const u32x4 x = again.load(j);
#pragma unroll
      for (int i = 0; i < RowVectors<F32>::VEC; ++i) l += __builtin_amdgcn_exp2f((RowVectors<F32>::value(x, i) - s.m) * to_log2);
    }
    s.lse = __builtin_amdgcn_logf(over_part<T>(l, [](float a, float b) { return a + b; }, joined_lds)) * kLn2;
  }
  const int32_t e_behind = e_first + (far ? chunks : 1) * kSlopeChunk;

  // The words that this thread has to write by itself, if they lie in this part of the row: the given one (thread 0), one of the likeliest
  int64_t named[2] = {tid == 0 && has_y ? y : -1, tid < n_top ? top_id(tid) : -1};
  float named_slope[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (!is_word(named[i]) || named[i] < e_first || named[i] >= e_behind) named[i] = -1;
    if (named[i] < 0) continue;
    float g = has_y && named[i] == y ? g_logp : 0.f;
    for (int k = 0; k < n_top; ++k) g += top_id(k) == named[i] ? p.g_top[token * p.n_top + k] : 0.f;
    named_slope[i] = s.none ? 0.f : (s.of_sum(element(named[i])) + g) * p.scale;
  }
  __syncthreads();

#pragma clang loop unroll(disable)
  for (int32_t e_part = e_first; e_part < e_behind; e_part += kSlopeChunk) {
#pragma unroll 4
    for (int r = 0; r < kSlopeChunk / (8 * T); ++r) {
      const int32_t e0 = e_part + (tid + T * r) * 8;
      if (e0 >= vocab) break;
      if (alike && e0 >= 0 && e0 + 8 <= vocab) {
        float x[8];
        if constexpr (F32) {
          const f32x4 a = load_as<f32x4, NT>(row + 4 * (int64_t)e0), b = load_as<f32x4, NT>(row + 4 * (int64_t)e0 + 16);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = i < 4 ? a[i & 3] : b[i & 3];
        } else {
          const u32x4 a = load_as<u32x4, NT>(row + 2 * (int64_t)e0);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = RowVectors<false>::value(a, i);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = s.of_sum(x[i]) * p.scale;
        if constexpr (TO_F32) {
          store_as<NT>(f32x4{x[0], x[1], x[2], x[3]}, out + 4 * (int64_t)e0);
          store_as<NT>(f32x4{x[4], x[5], x[6], x[7]}, out + 4 * (int64_t)e0 + 16);
        } else {
          bf16x8 z;
#pragma unroll
          for (int i = 0; i < 8; ++i) z[i] = (__bf16)x[i];
          store_as<NT>(z, out + 2 * (int64_t)e0);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (e0 + i >= 0 && e0 + i < vocab) put(e0 + i, s.of_sum(element(e0 + i)) * p.scale);
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (named[i] >= 0) put(named[i], named_slope[i]);
}

// Logits and gradients of more bytes than this are read and written without keeping their lines.  Of 32000 words in fp32, scores and gradient, kept / not:
// 400 tokens (102 MB) 35.3 / 39.6 us, 600 (154 MB) 52.4 / 49.8, 1200 101 / 82.7, 2400 196 / 179, 4096 312 / 296; 8192 in bf16 294 / 258.
constexpr int64_t kLargeBytes = 128 << 20;

int32_t parts_of_row(int32_t vocab) { return (int32_t)(((int64_t)vocab + 7 + kSlopeChunk - 1) / kSlopeChunk); }
// A launch has fewer than 2^32 threads; more tokens go to several, in multiples of 8: each begins at a multiple of 16 bytes then, whatever the rows' pitch.
int64_t tokens_of_launch(int32_t vocab) { return ((int64_t)1 << 23) / parts_of_row(vocab) / 8 * 8; }   // (at most 2^17 + 1 parts)

template <bool F32, bool TO_F32>
hipError_t launch_bwd(const ScoresBwdParams& p, hipStream_t stream) {
  const int32_t chunks = parts_of_row(p.vocab);
  const int64_t each = tokens_of_launch(p.vocab);
  // A wave for a row of few words (scores and gradient in us, bf16, a wave / four: 6107 x 357 16.4 / 24.3, 10211 x 1800 28.7 / 33.2, 10211 x 4154 68.6 / 77.0; in fp32 10211 x
  // 8000 219 / 177, 300 x 8000 20.0 / 15.0)
  const bool few = p.vocab <= 4608;
  const bool large = p.n_tokens * p.vocab * ((F32 ? 4 : 2) + (TO_F32 ? 4 : 2)) > kLargeBytes;
  for (int64_t first = 0; first < p.n_tokens; first += each) {
    ScoresBwdParams part = p;
    part.n_tokens = std::min(each, p.n_tokens - first);
    part.logits = (const char*)p.logits + first * p.ld * (F32 ? 4 : 2);
    part.d_logits = (char*)p.d_logits + first * p.ld_out * (TO_F32 ? 4 : 2);
    for (const float** x : {&part.lse, &part.entropy, &part.g_logp, &part.g_lse, &part.g_entropy})
      if (*x) *x += first;
    if (part.y) part.y += first;
    if (part.top_ids) part.top_ids += first * p.n_top;
    if (part.g_top) part.g_top += first * p.n_top;
    const int64_t parts = part.n_tokens * chunks;
    if (few) hipLaunchKernelGGL((scores_bwd_kernel<F32, TO_F32, false, 64>), dim3((uint32_t)((parts + 3) / 4)), dim3(256), 0, stream, part, chunks);
    else if (large) hipLaunchKernelGGL((scores_bwd_kernel<F32, TO_F32, true, 256>), dim3((uint32_t)parts), dim3(256), 0, stream, part, chunks);
    else hipLaunchKernelGGL((scores_bwd_kernel<F32, TO_F32, false, 256>), dim3((uint32_t)parts), dim3(256), 0, stream, part, chunks);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

int64_t scores_workspace_bytes(int64_t n_tokens, int32_t vocab, int32_t n_top) {
  const ScoresShape s = scores_shape(n_tokens, vocab);
  return s.segments == 1 ? 0 : n_tokens * s.segments * (int64_t)(sizeof(Partial) + 8 * n_top);
}

void scores_plan(int64_t n_tokens, int32_t vocab, int32_t out[2]) {
  const ScoresShape s = scores_shape(n_tokens, vocab);
  out[0] = s.waves;
  out[1] = s.segments;
}

int64_t scores_bwd_tokens(int32_t vocab) { return tokens_of_launch(vocab); }

hipError_t launch_scores(const ScoresParams& p, hipStream_t stream) {
  if (p.n_tokens == 0) return hipSuccess;
  if (p.n_top > 0) return p.is_f32 ? launch<true, true>(p, stream) : launch<false, true>(p, stream);
  return p.is_f32 ? launch<true, false>(p, stream) : launch<false, false>(p, stream);
}

hipError_t launch_scores_bwd(const ScoresBwdParams& p, hipStream_t stream) {
  if (p.is_f32) return p.out_is_f32 ? launch_bwd<true, true>(p, stream) : launch_bwd<true, false>(p, stream);
  return p.out_is_f32 ? launch_bwd<false, true>(p, stream) : launch_bwd<false, false>(p, stream);
}

}  // namespace burst
