// Scores of tokens from logits: log probability of given words, log-sum-exp, entropy and the likeliest words; and the gradient of the logits.
//
// Every logit is read once.  With x the logits times scale, m their maximum, l = sum exp(x - m) and w = sum exp(x - m) (x - m):
//     lse = m + log l,   logp = x_y - lse,   entropy = log l - w / l   (in base 2 inside),
// kept against a running maximum by each lane of its own elements.
//   The likeliest words: a wave has a list of 64, one a lane, in order.  The list starts from each lane's best element of the wave's first step, so its n_top-th
// is a bound that about n_top elements of that step pass; of each later step only what passes the bound is looked at (one comparison of a lane's
// maximum, which the sum needs anyway, for 8 or 4 elements), gathered in LDS, and taken into the list 64 at a time by a bitonic sort and merge.  An entry is
// the number, as a whole one of the same order, over the complement of its index: equal numbers go by the lowest index, and any way of dealing the
// elements out gives the same list.
//   A row is a wave's where there are many, else several waves' or several work-groups', whose sums and lists are joined.
#include <algorithm>

#include "cache.hpp"
#include "kernels.hpp"

namespace burst {

namespace {

typedef __attribute__((ext_vector_type(8))) float f32x8;

constexpr int kMostSegments = 16;      // work-groups of a row
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

// One stage of a bitonic network over the lanes: of the two lanes that `step` parts, the one below keeps the larger if `larger_below`.
__device__ __forceinline__ uint64_t exchanged(uint64_t x, int step, bool larger_below, int lane) {
  const uint64_t y = __shfl_xor((unsigned long long)x, step, 64);
  return (x > y) == (((lane & step) == 0) == larger_below) ? x : y;
}
// A bitonic sequence sorted, the largest in lane 0
__device__ __forceinline__ uint64_t merged_down(uint64_t x, int lane) {
#pragma unroll
  for (int step = 32; step >= 1; step >>= 1) x = exchanged(x, step, true, lane);
  return x;
}
template <bool DOWN>
__device__ __forceinline__ uint64_t sorted(uint64_t x, int lane) {
#pragma unroll
  for (int size = 2; size <= 64; size <<= 1)
#pragma unroll
    for (int step = size >> 1; step >= 1; step >>= 1) x = exchanged(x, step, ((lane & size) == 0 || size == 64) == DOWN, lane);
  return x;
}
// The 64 largest of a list and of entries sorted the other way round
__device__ __forceinline__ uint64_t joined(uint64_t list, uint64_t up, int lane) { return merged_down(list > up ? list : up, lane); }

// What a part of a row comes to.
struct RowSums {
  float m, l, w;   // of base-2 exponents: maximum, sum of exp2(x - m), sum of exp2(x - m) (x - m)
  __device__ __forceinline__ void join(const RowSums& o) {
    const float top = fmaxf(m, o.m);
    const float d0 = m == top ? 0.f : fmaxf(m - top, kNothing), d1 = o.m == top ? 0.f : fmaxf(o.m - top, kNothing);
    const float f0 = __builtin_amdgcn_exp2f(d0), f1 = __builtin_amdgcn_exp2f(d1);
    w = (w + l * d0) * f0 + (o.w + o.l * d1) * f1;
    l = l * f0 + o.l * f1;
    m = top;
  }
  __device__ __forceinline__ void join_lanes() {
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) join(RowSums{__shfl_xor(m, s, 64), __shfl_xor(l, s, 64), __shfl_xor(w, s, 64)});
  }
};

// A row of logits as vectors of 16 bytes from the aligned address at or below its first element on.
template <bool F32>
struct RowVectors {
  static constexpr int VEC = F32 ? 4 : 8;
  const char* row;      // its first element
  int32_t before, vocab;   // elements of the first vector that lie before it
  __device__ __forceinline__ void init(const ScoresParams& p, int64_t token) {
    const int64_t at = token * p.ld;
    before = (int32_t)(at & (VEC - 1));
    row = (const char*)p.logits + at * (F32 ? 4 : 2);
    vocab = p.vocab;
  }
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

// The list of a wave's likeliest words.
struct TopList {
  uint64_t list;       // a lane's entry, the largest in lane 0
  uint64_t bound;      // the n_top-th
  float bound_number;
  uint64_t* pending;   // LDS of the wave: fewer than 64, and what one vector of each lane may add
  int count, n_top, lane;
  __device__ __forceinline__ void set_bound() {
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)list, n_top - 1), hi = __builtin_amdgcn_readlane((uint32_t)(list >> 32), n_top - 1);
    bound = (uint64_t)hi << 32 | lo;
    bound_number = number_of(bound);
  }
  __device__ __forceinline__ void start(uint64_t best, uint64_t* lds, int n, int lane_) {
    pending = lds;
    n_top = n;
    lane = lane_;
    count = 0;
    list = sorted<true>(best, lane);
    set_bound();
  }
  __device__ __forceinline__ void offer(uint64_t entry, bool is_new) {
    const uint64_t passes = __ballot(is_new && entry > bound);
    if (passes == 0) return;
    if ((passes >> lane) & 1) pending[count + __builtin_popcountll(passes & ((1ull << lane) - 1))] = entry;
    count += __builtin_popcountll(passes);
  }
  // What is pending goes into the list, 64 at a time, until fewer than `rest` are left
  __device__ __forceinline__ void take(int rest) {
    int head = 0;
    __builtin_amdgcn_wave_barrier();
    while (count - head >= rest) {
      const uint64_t x = head + lane < count ? pending[head + lane] : 0;
      list = joined(list, sorted<false>(x, lane), lane);
      head += 64;
    }
    if (head == 0) return;
    set_bound();
    count = count > head ? count - head : 0;
    const uint64_t x = lane < count ? pending[head + lane] : 0;
    __builtin_amdgcn_wave_barrier();
    if (lane < count) pending[lane] = x;
    __builtin_amdgcn_wave_barrier();
  }
};

constexpr int kPending = 64 + 64 * 8;   // entries in LDS of a wave

// A wave's part of a row, vectors v0 .. v1 - 1.
template <bool F32, bool TOP>
__device__ __forceinline__ void scan_row(const RowVectors<F32>& row, int32_t v0, int32_t v1, float to_log2, int n_top, uint64_t* pending, int lane,
                                         RowSums& sums, uint64_t& list) {
  constexpr int VEC = RowVectors<F32>::VEC, U = 4;
  sums = RowSums{-INFINITY, 0.f, 0.f};
  TopList top;
  top.list = 0;
  auto index = [&](int32_t j, int i) { return (int32_t)((int64_t)j * VEC - row.before + i); };
  auto is_word = [&](int32_t id, float y) { return id >= 0 && id < row.vocab && !is_nan(y); };
  uint64_t best = 0;   // what the list starts from is not offered again
  if (TOP && v0 < v1) {
#pragma clang loop unroll(disable)
    for (int32_t j = v0 + lane; j < min(v1, v0 + 64 * U); j += 64) {
      const u32x4 x = row.load(j);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float y = RowVectors<F32>::value(x, i);
        const uint64_t entry = is_word(index(j, i), y) ? entry_of(y, index(j, i)) : 0;
        best = entry > best ? entry : best;
      }
    }
    top.start(best, pending, n_top, lane);
  }
  for (int32_t j0 = v0; j0 < v1; j0 += 64 * U) {
    u32x4 x[U];
    const u32x4 none = F32 ? u32x4{0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u} : u32x4{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u};
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = j0 + 64 * u + lane < v1 ? row.load(j0 + 64 * u + lane) : none;
    float most[U], step = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      most[u] = -INFINITY;
#pragma unroll
      for (int i = 0; i < VEC; ++i) most[u] = fmaxf(most[u], RowVectors<F32>::value(x[u], i));
      step = fmaxf(step, most[u]);
    }
    // (a scale is positive: the largest logit is the largest exponent)
    const float m = fmaxf(sums.m, step * to_log2), d = sums.m == m ? 0.f : fmaxf(sums.m - m, kNothing), f = __builtin_amdgcn_exp2f(d);
    sums.w = (sums.w + sums.l * d) * f;
    sums.l *= f;
    sums.m = m;
    const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float e = fmaf(RowVectors<F32>::value(x[u], i), to_log2, -base), p = __builtin_amdgcn_exp2f(e);
        sums.l += p;
        sums.w = fmaf(p, fmaxf(e, kNothing), sums.w);
      }
    if constexpr (TOP) {
      uint32_t some = 0;
#pragma unroll
      for (int u = 0; u < U; ++u) some |= __any(most[u] >= top.bound_number) ? 1u << u : 0u;
      while (some != 0) {   // (the vector is read again: a copy of this for each of them would cost the registers of all)
        const int u = __builtin_ctz(some);
        some &= some - 1;
        const bool inside = j0 + 64 * u + lane < v1;
        const u32x4 again = inside ? row.load(j0 + 64 * u + lane) : none;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const float y = RowVectors<F32>::value(again, i);
          const int32_t id = index(j0 + 64 * u + lane, i);
          const uint64_t entry = entry_of(y, id);
          top.offer(entry, inside && is_word(id, y) && entry != best);
        }
        top.take(64);
      }
    }
  }
  if constexpr (TOP) {
    if (v0 < v1) top.take(1);
    list = top.list;
  }
  sums.join_lanes();
}

// Sums and lists of the work-group's waves, in wave 0.
// lists: PITCH entries of LDS for each wave, the first 64 of them used.
template <int W, bool TOP, int PITCH>
__device__ __forceinline__ void join_waves(RowSums& sums, uint64_t& list, RowSums* sums_lds, uint64_t* lists, int wave, int lane) {
  if (lane == 0) sums_lds[wave] = sums;
  if (TOP) lists[PITCH * wave + lane] = list;
  __syncthreads();
#pragma unroll
  for (int s = 1; s < W; s <<= 1) {
    if (wave % (2 * s) == 0) {
      sums.join(sums_lds[wave + s]);
      if (lane == 0) sums_lds[wave] = sums;
      if (TOP) {
        list = joined(list, lists[PITCH * (wave + s) + 63 - lane], lane);
        lists[PITCH * wave + lane] = list;
      }
    }
    __syncthreads();
  }
}

// A token's results from its row's sums and list, by one wave.
template <bool F32>
__device__ __forceinline__ void write_scores(const ScoresParams& p, int64_t token, const RowSums& sums, uint64_t list, int lane) {
  const bool none = sums.l == 0.f;   // (every word at -inf; NaN is not)
  const float log_l = __builtin_amdgcn_logf(sums.l), lse = none ? -INFINITY : (sums.m + log_l) * kLn2;
  if (lane == 0) {
    if (p.lse) p.lse[token] = lse;
    if (p.entropy) p.entropy[token] = none ? 0.f : (log_l - sums.w / sums.l) * kLn2;
    if (p.logp) {
      const int64_t y = p.y[token];
      RowVectors<F32> row;
      row.init(p, token);
      p.logp[token] = y < 0 || y >= p.vocab ? 0.f : none ? -INFINITY : row.element((int32_t)y) * p.scale - lse;
    }
  }
  if (lane < p.n_top) {
    const int64_t to = token * p.n_top + lane;
    if (p.top_ids) p.top_ids[to] = list == 0 ? 0 : (int64_t)(int32_t)~(uint32_t)list;   // (fewer words than n_top: the others are NaN)
    if (p.top_logp) p.top_logp[to] = none ? -INFINITY : number_of(list) * p.scale - lse;
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
  __shared__ uint64_t pending[TOP ? WAVES : 1][kPending];
  __shared__ RowSums sums_lds[WAVES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int64_t token = W == 1 ? (int64_t)blockIdx.x * WAVES + wave : (int64_t)((uint32_t)blockIdx.x / (uint32_t)segments);
  const int32_t segment = W == 1 ? 0 : (int32_t)((uint32_t)blockIdx.x - (uint32_t)token * (uint32_t)segments);
  if (token >= p.n_tokens) return;   // (W = 1: no barrier follows)
  RowVectors<F32> row;
  row.init(p, token);
  const int64_t vectors = row.vectors(), parts = (int64_t)segments * W, part = W == 1 ? 0 : (int64_t)segment * W + wave;
  RowSums sums;
  uint64_t list = 0;
  scan_row<F32, TOP>(row, (int32_t)(vectors * part / parts), (int32_t)(vectors * (part + 1) / parts), p.scale * kLog2e, p.n_top, pending[TOP ? wave : 0], lane, sums,
                     list);
  if constexpr (W > 1) join_waves<W, TOP, kPending>(sums, list, sums_lds, pending[0], wave, lane);
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
  join_waves<kMostSegments, TOP, 64>(sums, list, sums_lds, lists, wave, lane);
  if (wave == 0) write_scores<F32>(p, token, sums, list, lane);
}

// How a row is dealt out: waves of a work-group, and work-groups.
struct ScoresShape {
  int waves, segments;
};
ScoresShape scores_shape(int64_t n_tokens, int32_t vocab) {
  if (n_tokens >= 2048) return {1, 1};
  if (n_tokens >= 512) return {4, 1};
  const int64_t steps = (int64_t)vocab / (16 * 64 * 4 * 4);   // of a work-group of 16 waves, 32-bit logits
  return {16, (int)std::max<int64_t>(1, std::min<int64_t>({kMostSegments, steps / 2, 512 / std::max<int64_t>(1, n_tokens)}))};
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
struct RowSlope {
  float lse, entropy, g_all, g_entropy, scale;
  bool none;   // a row all at -inf
  __device__ __forceinline__ float of_sum(float x) const {   // of the part without named words
    const float logp = fmaf(x, scale, -lse), p = none ? 0.f : __builtin_amdgcn_exp2f(logp * kLog2e);
    return p * fmaf(-g_entropy, fmaxf(logp, kNothing) + entropy, g_all);
  }
};

constexpr int kSlopeEach = 4, kSlopeChunk = 256 * 8 * kSlopeEach;   // runs of 8 elements of a thread; elements of a work-group

template <bool F32, bool TO_F32>
__global__ __launch_bounds__(256) void scores_bwd_kernel(ScoresBwdParams p, int32_t chunks) {
  const int64_t token = (int64_t)((uint32_t)blockIdx.x / (uint32_t)chunks);
  const int32_t chunk = (int32_t)((uint32_t)blockIdx.x - (uint32_t)token * (uint32_t)chunks);
  const int64_t from = token * p.ld, to = token * p.ld_out;
  // Runs of 8 start at multiples of 8 of the logits' memory; of the gradient's too if its rows lie alike.
  const int32_t before = (int32_t)(from & 7), e_first = chunk * kSlopeChunk - before;
  const bool alike = ((from ^ to) & 7) == 0;
  const int64_t y = p.y ? p.y[token] : -1;
  const bool has_y = y >= 0 && y < p.vocab && p.g_logp;
  RowSlope s;
  s.lse = p.lse[token];
  s.none = s.lse == -INFINITY;
  s.entropy = p.g_entropy ? p.entropy[token] : 0.f;
  s.g_entropy = p.g_entropy ? p.g_entropy[token] : 0.f;
  s.scale = p.scale;
  const float g_logp = has_y ? p.g_logp[token] : 0.f;
  auto top_id = [&](int k) { return p.top_ids[token * p.n_top + k]; };
  auto is_word = [&](int64_t id) { return id >= 0 && id < p.vocab; };
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

  // The word that this thread has to write by itself, if it lies in this part of the row: 0 is the given one, the others the likeliest
  const int mine = (int)threadIdx.x;
  int64_t named = -1;
  if (mine == 0 && has_y) named = y;
  if (mine >= 1 && mine <= n_top) named = top_id(mine - 1);
  if (!is_word(named) || named < e_first || named >= e_first + kSlopeChunk) named = -1;
  float named_slope = 0.f;
  if (named >= 0) {
    float g = named == y ? g_logp : 0.f;
    for (int k = 0; k < n_top; ++k) g += top_id(k) == named ? p.g_top[token * p.n_top + k] : 0.f;
    named_slope = s.none ? 0.f : (s.of_sum(element(named)) + g) * p.scale;
  }
  __syncthreads();

#pragma unroll
  for (int r = 0; r < kSlopeEach; ++r) {
    const int32_t e0 = e_first + ((int)threadIdx.x + 256 * r) * 8;
    if (e0 >= p.vocab) continue;
    if (alike && e0 >= 0 && e0 + 8 <= p.vocab) {
      float x[8];
      if constexpr (F32) {
        const f32x4 a = *reinterpret_cast<const f32x4*>(row + 4 * (int64_t)e0), b = *reinterpret_cast<const f32x4*>(row + 4 * (int64_t)e0 + 16);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < 4 ? a[i & 3] : b[i & 3];
      } else {
        const u32x4 a = *reinterpret_cast<const u32x4*>(row + 2 * (int64_t)e0);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = RowVectors<false>::value(a, i);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = s.of_sum(x[i]) * p.scale;
      if constexpr (TO_F32) {
        *reinterpret_cast<f32x4*>(out + 4 * (int64_t)e0) = f32x4{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<f32x4*>(out + 4 * (int64_t)e0 + 16) = f32x4{x[4], x[5], x[6], x[7]};
      } else {
        bf16x8 z;
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = (__bf16)x[i];
        *reinterpret_cast<bf16x8*>(out + 2 * (int64_t)e0) = z;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (e0 + i >= 0 && e0 + i < p.vocab) put(e0 + i, s.of_sum(element(e0 + i)) * p.scale);
    }
  }
  __syncthreads();
  if (named >= 0) put(named, named_slope);
}

template <bool F32, bool TO_F32>
hipError_t launch_bwd(const ScoresBwdParams& p, hipStream_t stream) {
  const int32_t chunks = (int32_t)(((int64_t)p.vocab + 7 + kSlopeChunk - 1) / kSlopeChunk);
  // A launch has fewer than 2^32 threads; more tokens go to several.
  const int64_t each = std::max<int64_t>(1, ((int64_t)1 << 23) / chunks);
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
    hipLaunchKernelGGL((scores_bwd_kernel<F32, TO_F32>), dim3((uint32_t)(part.n_tokens * chunks)), dim3(256), 0, stream, part, chunks);
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
