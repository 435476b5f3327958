// Building blocks of the attention of a few new tokens over a paged cache (tree.hip, tree_few.hip): what a sequence brings, how its rows are dealt out,
// and 32 columns (new tokens times query heads of a key head) of a wave with their products and softmax.
#pragma once
#include <algorithm>
#include <type_traits>
#include <utility>

#include "cache.hpp"
#include "kernels.hpp"
#include "mfma16.hpp"

namespace burst {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;

constexpr float kTreeStale = 8.f;  // a maximum may fall behind by a factor of 2^8
// As for one new token: no part of a weight is 0, or an infinity among the values would give NaN; each is about 2^-32 of the weight at least.
constexpr uint16_t kTreeLeastPart = 32 << 7;

// The arguments of a launch (its first parameter), to be loaded here: taken from the parameter itself, what the start, the loop and the end of a kernel need
// of them is held in scalar registers all at once, which are too few (50 to 100 of them were spilled to lanes of vector registers, and read back in the loop).
__device__ __forceinline__ const TreeParams& args_here() {
  typedef const __attribute__((address_space(4))) TreeParams* args_ptr;
  args_ptr p = (args_ptr)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const TreeParams*)p;
}

// The leading 16 bits of two numbers.
__device__ __forceinline__ u16x2 upper_halves(float x0, float x1) {
  return __builtin_bit_cast(u16x2, __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, x1), __builtin_bit_cast(uint32_t, x0), 0x07060302u));
}
// The lowest n bits, n of any size.
__device__ __forceinline__ uint64_t low_bits(int32_t n) { return n >= 64 ? ~0ull : n > 0 ? (1ull << n) - 1 : 0ull; }
// Of the 64 rows from t0 on those that are rows lo .. hi - 1.
__device__ __forceinline__ uint64_t rows_between(int32_t lo, int32_t hi, int32_t t0) { return low_bits(hi - t0) & ~low_bits(lo - t0); }
// Bit 0 of a word moved to bit s.
__device__ __forceinline__ uint64_t moved(uint64_t word, int32_t s) { return s >= 64 || s <= -64 ? 0ull : s >= 0 ? word << s : word >> -s; }
__device__ __forceinline__ uint64_t uniform(uint64_t x) {
  return (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(x >> 32)) << 32 | __builtin_amdgcn_readfirstlane((uint32_t)x);
}

// What a sequence brings: its tokens; rows hi that are there and below the bound; rows that are older than the new tokens; and of these the first that some
// token sees beside the first `sinks`.  Its units, of UNIT rows, are 0 .. ts - 1 and from tf on; a sequence without visible rows has one unit, which writes
// its empty result, one without tokens none.
struct TreeSeq {
  int32_t tokens, hi, older, lo, sinks, ts, tf, units;
  __device__ __forceinline__ void make_uniform() {
    for (int32_t* x : {&tokens, &hi, &older, &lo, &sinks, &ts, &tf, &units}) *x = __builtin_amdgcn_readfirstlane(*x);
  }
};
// ALIKE: all lanes ask for the same sequence, and look at a token each.
template <int UNIT, bool ALIKE>
__device__ __forceinline__ TreeSeq tree_seq(const TreeParams& p, int32_t b, int lane) {
  TreeSeq s;
  const int32_t n = p.tokens ? p.tokens[b] : p.sq, rows = p.cache.rows_of(b);
  s.tokens = n < 0 ? 0 : n > p.sq ? p.sq : n;
  s.hi = rows < p.max_rows ? rows : p.max_rows;
  s.older = p.elsewhere ? rows : rows - s.tokens;   // (negative: more tokens than rows)
  const int32_t old = s.older > 0 ? s.older : 0;
  int32_t lo = 0;
  if (p.first) {
    const int32_t* const first = p.first + b * p.first_sb;
    if constexpr (ALIKE) {
      const int32_t f = lane < p.sq ? first[lane] : 0;   // (asked for with the numbers above: not by s.tokens)
      lo = lane < s.tokens ? f : old;
      auto least = [&](auto step) {
        const int32_t x = (int32_t)of_lane_xor<decltype(step)::value>((uint32_t)lo);
        lo = x < lo ? x : lo;
      };
      least(std::integral_constant<int, 1>());
      least(std::integral_constant<int, 2>());
      least(std::integral_constant<int, 4>());
      least(std::integral_constant<int, 8>());
      least(std::integral_constant<int, 16>());
      least(std::integral_constant<int, 32>());
      lo = lo < old ? lo : old;
    } else {
      constexpr int N = 8;   // loads under way
      lo = old;
      for (int32_t i = 0; i < s.tokens; i += N) {
        int32_t f[N];
#pragma unroll
        for (int k = 0; k < N; ++k) f[k] = first[i + k < s.tokens ? i + k : i];
#pragma unroll
        for (int k = 0; k < N; ++k) lo = f[k] < lo ? f[k] : lo;
      }
    }
    lo = lo > 0 ? lo : 0;
  }
  s.sinks = p.sinks < old ? p.sinks : old;
  s.lo = lo <= s.sinks ? 0 : lo;   // (all older rows are one interval)
  const int32_t first_units = s.lo == 0 ? 0 : (s.sinks + UNIT - 1) / UNIT, te = (s.hi + UNIT - 1) / UNIT;
  s.ts = first_units < te ? first_units : te;
  const int32_t tf = s.lo / UNIT > s.ts ? s.lo / UNIT : s.ts;
  s.tf = tf < te ? tf : te;
  const int32_t units = s.ts + te - s.tf;
  s.units = s.tokens == 0 ? 0 : units > 0 ? units : 1;
  return s;
}

// Units dealt to `shares` work-groups: the first `more` of them get one more.
struct TreeDeal {
  int32_t each, more;
  __device__ __forceinline__ void init(int32_t units, int32_t shares) {
    each = __builtin_amdgcn_readfirstlane((int32_t)((uint32_t)units / (uint32_t)shares));
    more = units - each * shares;
  }
  __device__ __forceinline__ int32_t first(int32_t w) const { return w * each + (w < more ? w : more); }
  __device__ __forceinline__ int32_t owner(int32_t unit) const {
    const int32_t longer = more * (each + 1);
    return unit < longer ? (int32_t)((uint32_t)unit / (uint32_t)(each + 1)) : more + (int32_t)((uint32_t)(unit - longer) / (uint32_t)each);
  }
};

// The workspace: for each sequence its first owner and, times two, its last one, plus one if the first owner's piece is its second; and two pieces for
// every work-group, each (maximum, sum) and O of its columns relative to that maximum.
struct TreeSpace {
  int2* owners;
  float2* ml;
  float* o;
};

// A work-group's walk over its share: the units of all sequences one after the other.
template <int UNIT>
struct TreeWalk {
  TreeDeal deal;
  TreeSeq seq;
  int32_t b, at, unit, left, take;   // the sequence, its unit that comes next, that one's number over all sequences; units left, and of this sequence
  bool first_piece, whole;

  // False: nothing to do.  direct: share is a sequence.
  __device__ __forceinline__ bool init(const TreeParams& p, int32_t share, int32_t shares, bool direct, int lane) {
    b = share;
    at = unit = 0;
    left = 1;
    first_piece = true;
    if (direct) {
      seq = tree_seq<UNIT, true>(p, b, lane);
      seq.make_uniform();
      return seq.units > 0;
    }
    auto upto = [&](int32_t x) {   // sum over this lane and the ones below
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) {
        const int32_t y = __shfl_up(x, s, 64);
        x += lane >= s ? y : 0;
      }
      return x;
    };
    int32_t total = 0;   // (below 2^31, checked on the host)
    TreeSeq mine = {};
    for (int32_t b0 = 0; b0 < p.batch; b0 += 64) {
      mine = b0 + lane < p.batch ? tree_seq<UNIT, false>(p, b0 + lane, lane) : TreeSeq{};
      total += __builtin_amdgcn_readlane(upto(mine.units), 63);
    }
    deal.init(total, shares);
    unit = deal.first(share);
    left = deal.first(share + 1) - unit;
    if (left == 0) return false;
    int32_t passed = 0;
    for (int32_t b0 = 0;; b0 += 64) {   // (unit < total: one sequence has it)
      if (p.batch > 64) mine = b0 + lane < p.batch ? tree_seq<UNIT, false>(p, b0 + lane, lane) : TreeSeq{};
      const int32_t end = passed + upto(mine.units), begin = end - mine.units;
      const uint64_t has = __ballot(begin <= unit && unit < end);
      if (has != 0) {
        const int l = __builtin_ctzll(has);
        b = __builtin_amdgcn_readfirstlane(b0 + l);
        at = unit - __builtin_amdgcn_readlane(begin, l);
        for (auto [to, from] : {std::pair<int32_t*, int32_t*>{&seq.tokens, &mine.tokens}, {&seq.hi, &mine.hi}, {&seq.older, &mine.older}, {&seq.lo, &mine.lo},
                                {&seq.sinks, &mine.sinks}, {&seq.ts, &mine.ts}, {&seq.tf, &mine.tf}, {&seq.units, &mine.units}})
          *to = __builtin_amdgcn_readlane(*from, l);
        break;
      }
      passed = __builtin_amdgcn_readlane(end, 63);
    }
    return true;
  }
  // What is to be done of this sequence; notes its owners (one thread of the work-groups of a share)
  __device__ __forceinline__ void begin(bool direct, bool notes, const TreeSpace& ws, int32_t share) {
    take = direct ? seq.units : left < seq.units - at ? left : seq.units - at;
    whole = direct || (at == 0 && take == seq.units);
    if (notes && !direct && at == 0 && seq.units > 0) {
      const int32_t last = whole ? share : deal.owner(unit + seq.units - 1);
      ws.owners[b] = int2{share, 2 * last + (first_piece ? 0 : 1)};
    }
  }
  __device__ __forceinline__ bool next(const TreeParams& p, bool direct, int lane) {
    if (direct) return false;
    first_piece = false;
    unit += take;
    left -= take;
    at = 0;
    if (left <= 0) return false;
    seq = tree_seq<UNIT, true>(p, ++b, lane);
    seq.make_uniform();
    return true;
  }
  __device__ __forceinline__ int32_t row_of(int32_t u) const { return (u < seq.ts ? u : u - seq.ts + seq.tf) * UNIT; }
};

// What some token of a sequence sees of the 64 rows from t0 on.
struct TreeUnion {
  uint64_t word;
  int32_t older, lo, sinks, hi, inside;
  __device__ __forceinline__ void init(const TreeParams& p, const TreeSeq& s, int32_t b, int lane) {
    uint64_t w = 0;
    if (lane < s.tokens && !p.elsewhere) w = (p.seen ? p.seen[b * p.seen_sb + lane] : low_bits(lane + 1)) & low_bits(s.tokens);
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) w |= __shfl_xor((unsigned long long)w, i, 64);
    word = uniform(w);
    older = s.older;
    lo = s.lo;
    sinks = s.sinks;
    hi = s.hi;
    inside = s.older < s.hi ? s.older : s.hi;   // rows from lo up to here are all seen
  }
  __device__ __forceinline__ uint64_t rows(int32_t t0) const {
    if (t0 >= lo && t0 + 64 <= inside) return ~0ull;   // (most tiles: scalar arithmetic is a good part of a tile's time)
    return (rows_between(lo, older, t0) | rows_between(0, sinks, t0) | moved(word, older - t0)) & low_bits(hi - t0);
  }
};

// Operands of the products from a tile of 32 rows in LDS.  bf16 as elsewhere (mfma16.hpp); e4m3 as the bytes they are, made bf16 on the way to the product: half
// the LDS, twice the tiles under way.  A row of D bytes is D / 16 chunks, permuted by an exclusive or with a function of the row: 16 lanes of a
// row-wise read (8 bytes each) and the 8 rows of a transposing one (ds_read_b64_tr_b8: of 16 lanes lane r names row r / 2 and 8 bytes r % 2 of its chunk, and gets of column
// r those 8 rows) fall into different places of a bank line, those of two neighbours g too.
template <int D>
__device__ __forceinline__ int swz8(int row) {   // row of 32
  return D == 128 ? ((row >> 1) & 7) ^ ((row >> 4) & 1) << 2 : ((row >> 2) & 3) ^ ((row >> 4) & 1) << 1;
}
template <int D, bool F8>
struct TreeOperands {
  typedef __attribute__((ext_vector_type(2))) int i32x2;
  using Raw = std::conditional_t<F8, i32x2, bf16x8>;
  static constexpr int ROW = D * (F8 ? 1 : 2), TILE = 32 * ROW;
  OperandAddr<D> ad;
  uint32_t rows8, cols8;
  __device__ __forceinline__ void init(int lane) {
    const int r = lane & 15, g = lane >> 4;
    if constexpr (F8) {
      rows8 = r * ROW + ((swz8<D>(r) << 4) ^ (8 * g));       // k-step 0: row r, bytes 8 g ..
      const int j = r >> 1, row = j < 4 ? 4 * g + j : 16 + 4 * g + j - 4;
      cols8 = row * ROW + (swz8<D>(row) << 4) + 8 * (r & 1);   // column block 0
    } else {
      ad.init(lane);
    }
  }
  // Rows 16 mb + r, elements 32 ks + 8 g ..  `tile`: a multiple of 256
  __device__ __forceinline__ Raw row(uint32_t tile, int mb, int ks) const {
    if constexpr (F8) {
      // (16 rows on, the permutation is another one: swz8 of row 16 is a constant more)
      const uint32_t at = (tile + rows8) ^ (uint32_t)(32 * ks) ^ (uint32_t)(mb ? swz8<D>(16) << 4 : 0);
      return *reinterpret_cast<const __attribute__((address_space(3))) i32x2*>((lds_bytes)(uintptr_t)at + 16 * ROW * mb);
    } else {
      return rows_operand<D>(tile, ad, 16 * mb, ks);
    }
  }
  // Column 16 db + r, the 32 rows in packed-accumulator order
  __device__ __forceinline__ Raw col(uint32_t tile, int db) const {
    if constexpr (F8) {
      typedef __attribute__((address_space(3))) i32x2* tr_ptr;
      return __builtin_amdgcn_ds_read_tr8_b64_v2i32((tr_ptr)(uintptr_t)((tile + cols8) ^ (uint32_t)(16 * db)));
    } else {
      return cols_operand<D>(tile, ad, 0, db);
    }
  }
  static __device__ __forceinline__ bf16x8 wide(const Raw& x) {
    if constexpr (F8) {
      const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[0], 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[0], 1.0f, true);
      const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[1], 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[1], 1.0f, true);
      return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    } else {
      return x;
    }
  }
};

// 16 NB columns of a wave: column 16 nb + r of them is lane r's (and r + 16's, ..).  A column is a token and a query head; what it sees, its query,
// its running maximum (base 2, a whole number, so that a rescale changes no bit of P and O) and sums.
// PARTS: bf16 numbers that a P is multiplied in, three (all of its 24 bits) or two; AHEAD: operands fetched before they are used; CH: 32 rows at a time, or twice as many.
template <int D, bool F8, int NB, int PARTS, int AHEAD, int CH>
struct TreeColumns {
  static constexpr int MB = 2 * CH, DK = D / 32, DB = D / 16, HALF = TreeOperands<D, F8>::TILE;
  bf16x8 q[DK][NB];
  int32_t first[NB], latest, older, sinks;
  uint64_t word[NB];
  float to_log2, m[NB], l[NB];
  f32x4 acc[DB][NB], s[MB][NB];
  bf16x8 part[CH][NB][PARTS];

  // Columns from c0 on (those behind the sequence's last one are zeros)
  __device__ __forceinline__ void init(const TreeParams& p, const TreeSeq& seq, int32_t b, int32_t hk, int32_t group, int32_t c0, int lane) {
    const int r = lane & 15, g = lane >> 4;
    older = seq.older;
    sinks = p.sinks < seq.older ? p.sinks : seq.older;
    int32_t last = 0;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int32_t c = c0 + 16 * nb + r, i = c / group, h = hk * group + (c - i * group);
      const bool there = c < seq.tokens * group;
      first[nb] = there && p.first ? max(p.first[b * p.first_sb + i], 0) : 0;
      word[nb] = there && !p.elsewhere ? (p.seen ? p.seen[b * p.seen_sb + i] : low_bits(i + 1)) & low_bits(seq.tokens) : 0;
      last = max(first[nb], last);
      const __bf16* row = (const __bf16*)p.q.ptr + b * p.q.sb + i * p.q.ss + h * p.q.sh + 8 * g;
#pragma unroll
      for (int ks = 0; ks < DK; ++ks) q[ks][nb] = there ? *reinterpret_cast<const bf16x8*>(row + 32 * ks) : zero_operand();
      m[nb] = -INFINITY;
      l[nb] = 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db) acc[db][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int x = 1; x < 16; x <<= 1) last = max(last, __shfl_xor(last, x, 64));
    latest = __builtin_amdgcn_readfirstlane(last);
    to_log2 = p.scale * kLog2e * (F8 && p.cache.k_scale ? p.cache.k_scale[hk] : 1.f);
  }
  // Scores of the rows whose keys lie in LDS at kt
  __device__ __forceinline__ void scores(uint32_t kt, const TreeOperands<D, F8>& ops) {
    constexpr int N = DK * MB;
    typename TreeOperands<D, F8>::Raw a[N];
    MatrixPhase prio;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) a[i] = ops.row(kt + i % MB / 2 * HALF, i % 2, i / MB);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i + AHEAD < N) a[i + AHEAD] = ops.row(kt + (i + AHEAD) % MB / 2 * HALF, (i + AHEAD) % 2, (i + AHEAD) / MB);
      const bf16x8 x = ops.wide(a[i]);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) s[i % MB][nb] = mfma16(x, q[i / MB][nb], i < MB ? f32x4{0.f, 0.f, 0.f, 0.f} : s[i % MB][nb]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // Whether every column sees all of the rows from t0 on, if they are there
  __device__ __forceinline__ bool sees_all(int32_t t0) const { return t0 + 32 * CH <= older && (t0 >= latest || t0 + 32 * CH <= sinks); }
  // P of these rows (from t0 on; `there`: which of them are) as bf16 numbers that add up to it
  __device__ __forceinline__ void weights(int32_t t0, uint64_t there, int g) {
    const bool full = there == low_bits(32 * CH) && sees_all(t0);   // (wave-uniform)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float x[8 * CH], top = -INFINITY;
#pragma unroll
      for (int e = 0; e < 8 * CH; ++e) x[e] = s[e >> 2][nb][e & 3];
      if (!full) {
        const uint64_t sees = (rows_between(first[nb], older, t0) | rows_between(0, sinks, t0) | moved(word[nb], older - t0)) & there;
        const uint32_t bits[2] = {(uint32_t)sees >> (4 * g), (uint32_t)(sees >> 32) >> (4 * g)};
#pragma unroll
        for (int e = 0; e < 8 * CH; ++e) x[e] = (bits[e >> 3] >> (16 * ((e >> 2) & 1) + (e & 3))) & 1 ? x[e] : -INFINITY;
      }
#pragma unroll
      for (int e = 0; e < 8 * CH; ++e) top = fmaxf(top, x[e]);
      top *= to_log2;   // (positive)
      if (__any(top > m[nb] + kTreeStale)) {   // (the first rows: m is -inf)
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float up = fmaxf(m[nb], ceilf(top)), f = up == m[nb] ? 1.f : __builtin_amdgcn_exp2f(m[nb] - up);
        m[nb] = up;
        l[nb] *= f;
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[db][nb] *= f;
      }
      const float base = m[nb] == -INFINITY ? 0.f : m[nb];
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float* const y = x + 8 * c;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = __builtin_amdgcn_exp2f(fmaf(y[e], to_log2, -base));
        l[nb] += ((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]));
        static_assert(PARTS == 2 || PARTS == 3, "parts");
        u16x2 least[4];
#pragma unroll
        for (int n = 0; n < PARTS; ++n) {
          u32x4 words;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float &x0 = y[2 * i], &x1 = y[2 * i + 1];
            // (the last of two parts is rounded, to 2^-16 of P at most and either way; none is negative)
            u16x2 bits;
            if constexpr (PARTS == 2) bits = n == 0 ? upper_halves(x0, x1) : __builtin_bit_cast(u16x2, bf16x2{(__bf16)x0, (__bf16)x1});
            else bits = upper_halves(x0, x1);
            if (!F8 && n == 0) least[i] = __builtin_elementwise_sub_sat(bits, u16x2{kTreeLeastPart, kTreeLeastPart});
            if (!F8 && n != 0) bits = __builtin_elementwise_max(bits, least[i]);
            words[i] = __builtin_bit_cast(uint32_t, bits);
            x0 -= __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x0) & 0xffff0000u);   // (exact)
            x1 -= __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x1) & 0xffff0000u);
          }
          part[c][nb][n] = __builtin_bit_cast(bf16x8, words);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_sched_barrier(0);   // (one block of columns after the other: both at once take the registers of twice as many numbers)
    }
  }
  // O += V^T P, with the values of the rows in LDS at vt
  __device__ __forceinline__ void add(uint32_t vt, const TreeOperands<D, F8>& ops) {
    constexpr int N = CH * DB;
    typename TreeOperands<D, F8>::Raw a[N];
    MatrixPhase prio;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) a[i] = ops.col(vt, i);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i + AHEAD < N) a[i + AHEAD] = ops.col(vt + (i + AHEAD) / DB * HALF, (i + AHEAD) % DB);
      const bf16x8 v = ops.wide(a[i]);
#pragma unroll
      for (int n = 0; n < PARTS; ++n)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) acc[i % DB][nb] = mfma16(v, part[i / DB][nb][n], acc[i % DB][nb]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // The four lanes of a column have the sum over all its rows
  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      l[nb] += __shfl_xor(l[nb], 16, 64);
      l[nb] += __shfl_xor(l[nb], 32, 64);
    }
  }
};

// Elements d .. d + 3 of O of a column (c of key head hk) whose sums are whole, and with d = 0 its Lse.
template <bool F8>
__device__ __forceinline__ void tree_write(const TreeParams& p, int32_t b, int32_t hk, int32_t group, int32_t c, int d, f32x4 x, float m, float l) {
  const int32_t i = c / group, h = hk * group + (c - i * group);
  const float over = l == 0.f ? 0.f : (F8 && p.cache.v_scale ? p.cache.v_scale[hk] : 1.f) / l;
  const int64_t to = b * p.o.sb + i * p.o.ss + h * p.o.sh + d;
  x *= over;
  if (p.o.is_f32) *reinterpret_cast<f32x4*>((float*)p.o.ptr + to) = x;
  else *reinterpret_cast<bf16x4*>((__bf16*)p.o.ptr + to) = bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
  if (d == 0 && p.lse.ptr) p.lse.ptr[b * p.lse.sb + h * p.lse.sh + i] = l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

// Meets the other waves with all of this wave's LDS instructions done; loads stay under way.
__device__ __forceinline__ void lds_barrier() { stores_barrier<0>(); }

// A direct load of every lane's 16 bytes, from an address of its own, to lds + 16 * lane.
__device__ __forceinline__ void load_rows_to_lds(const char* at, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(at) : "memory");
}
// From a base of the wave and an offset of the lane, lines not kept.
__device__ __forceinline__ void load_to_lds_once(const char* base, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(lds), "v"(offset), "s"(base) : "memory");
}

// Runs of 16 rows of a sequence, as a wave brings them to LDS by direct loads, RPI rows with each: lane l row l / PER_ROW of them, 16 bytes of it.  HALVES: a wave brings
// runs to the first and the second half of a tile of 32 rows (which lie differently there); else always to one of them.
// PAGES16: pages are multiples of 16 rows, so a run lies in one page, and its place is scalar arithmetic; else each lane looks its rows up.
// What is brought: rows of which `rows` bits are set and that have a page.  Others: some rows that are there, whose keys are not looked at and whose values
// clear() makes zeros (they may hold NaN, which a P of 0 would not silence).
template <int D, bool F8, bool PAGES16, int HALVES>
struct TreeRun {
  static constexpr int kBytes = F8 ? 1 : 2, PER_ROW = D * kBytes / 16, RPI = 64 / PER_ROW, NI = 16 / RPI, BYTES = 16 * D * kBytes;
  const char *k_base, *v_base;
  const int32_t* table;
  int64_t s_page, s_row;
  int32_t hi, page_rows, n_pages;
  Divider by_page;
  uint32_t off[PAGES16 ? HALVES : 1][NI];   // of this lane's 16 bytes from the run's first row
  uint32_t piece[HALVES][NI];               // those alone (each lane's own rows)
  __device__ __forceinline__ static int row_in(int i, int lane) { return RPI * i + lane / PER_ROW; }
  // half0: the half that its runs go to (HALVES = 1)
  __device__ __forceinline__ void init(const CacheDev& c, int32_t b, int32_t hk, int32_t hi_, int half0, int lane) {
    hi = hi_;
    k_base = (const char*)c.k + hk * c.s_head * kBytes;
    v_base = (const char*)c.v + hk * c.s_head * kBytes;
    table = c.table + b * c.table_stride;
    s_page = c.s_page * kBytes;
    s_row = c.s_row * kBytes;
    page_rows = c.page_rows;
    n_pages = c.n_pages;
    by_page = c.by_page;
#pragma unroll
    for (int h = 0; h < HALVES; ++h)
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int row = row_in(i, lane), in = lane % PER_ROW;
        piece[h][i] = 16 * (F8 ? in ^ swz8<D>(row + 16 * (HALVES == 1 ? half0 : h)) : in ^ swz<D>(row));
        if constexpr (PAGES16) off[h][i] = row * (uint32_t)s_row + piece[h][i];
      }
  }
  // The pages of a run's rows.  PAGES16: of 64 / HALVES tiles at once, a lane for each run, as a scalar load for each tile would make every wait for LDS operands
  // a wait for that load too (they count in one counter, and it comes back in any order).
  static constexpr int TILES = PAGES16 ? 64 / HALVES : 1;
  struct Pages {
    int32_t page[PAGES16 ? 1 : HALVES * NI], from;
    uint64_t all, each[4];   // PAGES16, HALVES 1: tiles whose four runs have a page, and those of each run
  };
  // Of the 64 rows of tile u those whose run has a page (PAGES16, HALVES 1)
  __device__ __forceinline__ uint64_t with_page(const Pages& x, int32_t u) const {
    const int32_t i = u - x.from;
    if ((x.all >> i) & 1) return ~0ull;
    uint64_t rows = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) rows |= ((x.each[k] >> i) & 1) * (0xffffull << (16 * k));
    return rows;
  }
  // Of tile u (first_row(u): this wave's first row of it), if they have not been looked up; tiles come one after the other, the first one is `begin`.  run: this wave's
  // of the four of a tile (HALVES 1).
  template <class FirstRow>
  __device__ __forceinline__ void look_up(FirstRow first_row, int32_t u, int32_t begin, int32_t end, int run, int lane, Pages& x) const {
    if constexpr (PAGES16 && HALVES == 1) {
      if (u != begin && u != x.from + TILES) return;
      const int32_t row0 = first_row(u + lane) - 16 * run;
      int32_t page[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) page[k] = u + lane < end && row0 + 16 * k < hi ? table[by_page.quotient(row0 + 16 * k)] : -1;
#pragma unroll
      for (int k = 0; k < 4; ++k) asm volatile("" : "+v"(page[k]));   // (waited for here: at its uses the compiler would wait in every tile, for all loads under way)
      x.all = ~0ull;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x.each[k] = __ballot(page[k] >= 0 && page[k] < n_pages);
        x.all &= x.each[k];
      }
      x.page[0] = run == 0 ? page[0] : run == 1 ? page[1] : run == 2 ? page[2] : page[3];
      x.from = u;
    } else if constexpr (PAGES16) {
      if (u != begin && u != x.from + TILES) return;
      const int32_t tile = u + lane % TILES, row0 = first_row(tile) + 16 * (lane / TILES);
      x.page[0] = tile < end && row0 < hi ? table[by_page.quotient(row0)] : -1;
      asm volatile("" : "+v"(x.page[0]));   // (as above)
      x.from = u;
    } else {
#pragma unroll
      for (int h = 0; h < HALVES; ++h)
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const int32_t row = first_row(u) + 16 * h + row_in(i, lane);
          x.page[h * NI + i] = row < hi ? table[by_page.quotient(row)] : -1;
        }
    }
  }
  // Where the run lies, and which of its rows are brought (bits, the same in all lanes)
  struct Place {
    uint32_t there;
    int64_t at[PAGES16 ? 1 : NI];   // bytes, of the run's first row or of this lane's rows
  };
  // row0: first row of run h of tile u
  __device__ __forceinline__ void place(int32_t row0, uint32_t rows, int lane, const Pages& x, int32_t u, int h, Place& to) const {
    if constexpr (PAGES16) {
      const int32_t page = __builtin_amdgcn_readlane(x.page[0], u - x.from + TILES * h), in_page = row0 - by_page.quotient(row0) * page_rows;
      to.there = page >= 0 && page < n_pages ? rows : 0u;
      to.at[0] = to.there ? page * s_page + in_page * s_row : 0;
    } else {
      bool all = true;
      uint32_t mine = 0;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int32_t row = row0 + row_in(i, lane), in_page = row - by_page.quotient(row) * page_rows;
        const bool there = ((rows >> row_in(i, lane)) & 1) && x.page[h * NI + i] >= 0 && x.page[h * NI + i] < n_pages;
        to.at[i] = there ? x.page[h * NI + i] * s_page + in_page * s_row : 0;
        mine |= there ? 1u << i : 0u;
        all = all && there;
      }
      to.there = 0xffffu;
      if (!__all(all)) {
        to.there = 0;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const uint64_t v = __ballot((mine >> i) & 1u);
#pragma unroll
          for (int k = 0; k < RPI; ++k) to.there |= (uint32_t)((v >> (k * PER_ROW)) & 1u) << (RPI * i + k);
        }
      }
    }
  }
  template <bool VALUES>
  __device__ __forceinline__ void bring(const Place& x, int half, uint32_t lds, bool once) const {
    const char* const base = VALUES ? v_base : k_base;
    const int h = HALVES == 1 ? 0 : half;   // (known when compiled)
    if constexpr (!PAGES16) {
#pragma unroll
      for (int i = 0; i < NI; ++i) load_rows_to_lds(base + x.at[i] + piece[h][i], lds + 1024 * i);
    } else {
      const char* run = base + x.at[0];
      pin(run);
      if (once) {
#pragma unroll
        for (int i = 0; i < NI; ++i) load_to_lds_once(run, off[h][i], lds + 1024 * i);
      } else {
#pragma unroll
        for (int i = 0; i < NI; ++i) load_to_lds(run, off[h][i], lds + 1024 * i);
      }
    }
  }
  // Zeros for the rows of a run in LDS that were not brought
  static __device__ __forceinline__ void clear(char* lds, uint32_t there, int lane) {
    if (there == 0xffffu) return;
#pragma unroll
    for (int i = 0; i < NI; ++i)
      if (!((there >> row_in(i, lane)) & 1u)) *reinterpret_cast<u32x4*>(lds + 1024 * i + 16 * lane) = u32x4{0, 0, 0, 0};
  }
};

hipError_t launch_tree_few(const TreeParams& p, const TreeSpace& ws, int32_t columns, int32_t shares, bool direct, hipStream_t stream);
constexpr int kTreeFit = 512;      // work-groups of four waves that the chip holds at once, two a CU

}  // namespace burst
