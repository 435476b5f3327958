// Attention of a few new tokens of every sequence, a chain or a tree of drafts, over its rows in a paged cache.
//
// The new tokens times the query heads that share a key head are the columns of two products: S^T = K Q^T and O^T = V^T P^T, so a row of the
// cache that is read once serves them all.  A work-group of four waves takes 64 or 128 columns; tiles of 64 rows of K and V come into LDS, where
// their addresses go by the page table row by row, and each wave multiplies them for 32 columns (all 64 rows for 128 columns of the work-group, half
// of them for 64, whose halves are added up at the end).
//   Which rows a column sees is a 64-bit word for each tile: older rows from its first one on and the first rows of all, both intervals, and the
// new tokens' rows by the bits of its word, moved to where they stand in the tile.  A tile of which every column of a wave sees all rows does not
// look at them.
//   The running maximum is a whole number (base 2), so that a rescale changes no bit of P and O.  P goes in as bf16 numbers that add up to it: three for O
// in fp32, whose 24 bits they are, two for O in bf16 (16 bits, far below what the cast rounds).
//
// Work is cut into units of a tile and numbered over (sequence, tiles that some of its tokens see): a window leaves the tiles out that lie between the
// first rows and its own.  The units are dealt evenly to shares, a work-group each for every key head and block of columns; a piece that is
// a whole sequence is written out, others go to the workspace and tree_join_kernel adds them up in a fixed order.
#include <algorithm>

#include "cache.hpp"
#include "kernels.hpp"
#include "mfma16.hpp"

namespace burst {

namespace {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;

constexpr int kTreeRows = 64;      // rows of a tile
constexpr int kTreeWaves = 4;
constexpr float kTreeStale = 8.f;  // a maximum may fall behind by a factor of 2^8
// As for one new token: no part of a weight is 0, or an infinity among the values would give NaN; each is about 2^-32 of the weight at least.
constexpr uint16_t kTreeLeastPart = 32 << 7;
constexpr int kTreeFit = 512;      // work-groups that the chip holds at once, two a CU

// The lowest n bits, n of any size.
__device__ __forceinline__ uint64_t low_bits(int32_t n) { return n >= 64 ? ~0ull : n > 0 ? (1ull << n) - 1 : 0ull; }
// Bits of the tile at row t0 that are rows lo .. hi - 1.
__device__ __forceinline__ uint64_t tile_interval(int32_t lo, int32_t hi, int32_t t0) { return low_bits(hi - t0) & ~low_bits(lo - t0); }
// Bit 0 of a word moved to bit s of a tile.
__device__ __forceinline__ uint64_t moved(uint64_t word, int32_t s) { return s >= 64 || s <= -64 ? 0ull : s >= 0 ? word << s : word >> -s; }

// What a sequence brings: its tokens; rows hi that are there and below the bound; rows that are older than the new tokens; and of these the first that some
// token sees beside the first `sinks`.  Its units are tiles 0 .. ts - 1 and from tf on; a sequence without visible rows has one unit, which writes
// its empty result, one without tokens none.
struct TreeSeq {
  int32_t tokens, hi, older, lo, sinks, ts, tf, units;
};
__device__ __forceinline__ TreeSeq tree_seq(const TreeParams& p, int32_t b) {
  TreeSeq s;
  const int32_t n = p.tokens ? p.tokens[b] : p.sq, rows = p.cache.rows_of(b);
  s.tokens = n < 0 ? 0 : n > p.sq ? p.sq : n;
  s.hi = rows < p.max_rows ? rows : p.max_rows;
  s.older = p.elsewhere ? rows : rows - s.tokens;   // (negative: more tokens than rows)
  const int32_t old = s.older > 0 ? s.older : 0;
  int32_t lo = 0;
  if (p.first) {
    lo = old;
    for (int32_t i = 0; i < s.tokens; ++i) {
      const int32_t f = p.first[b * p.first_sb + i];
      lo = f < lo ? f : lo;
    }
    lo = lo > 0 ? lo : 0;
  }
  s.sinks = p.sinks < old ? p.sinks : old;
  s.lo = lo <= s.sinks ? 0 : lo;
  if (s.lo == 0) s.sinks = 0;   // all rows are one interval
  const int32_t te = (s.hi + kTreeRows - 1) / kTreeRows, ts = (s.sinks + kTreeRows - 1) / kTreeRows;
  s.ts = ts < te ? ts : te;
  const int32_t tf = s.lo / kTreeRows > s.ts ? s.lo / kTreeRows : s.ts;
  s.tf = tf < te ? tf : te;
  const int32_t units = s.ts + te - s.tf;
  s.units = s.tokens == 0 ? 0 : units > 0 ? units : 1;
  return s;
}
// (sinks and lo above say which tiles there are; whether a row is seen goes by the numbers as they were given)

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
struct TreeShape {
  int32_t columns, blocks, shares;   // columns of a work-group; blocks of them of a key head; shares of the units
  bool direct;                       // a share for every sequence, no workspace
  int64_t off_ml, off_o, bytes;
};
int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }
TreeShape tree_shape(int32_t batch, int32_t sq, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int64_t max_rows) {
  TreeShape s;
  const int32_t all = q_heads / kv_heads * sq;
  s.columns = all <= 64 ? 64 : 128;
  s.blocks = (all + s.columns - 1) / s.columns;
  const int64_t per_seq = (int64_t)kv_heads * s.blocks, max_units = std::max<int64_t>(1, (max_rows + kTreeRows - 1) / kTreeRows);
  s.direct = batch * per_seq >= kTreeFit || max_units <= 2;
  s.shares = (int32_t)(s.direct ? batch : std::min<int64_t>(batch * max_units, std::max<int64_t>(1, kTreeFit / per_seq)));
  const int64_t pieces = s.shares * per_seq * 2 * s.columns;
  s.off_ml = up256((int64_t)batch * 8);
  s.off_o = s.off_ml + up256(pieces * 8);
  s.bytes = s.direct ? 0 : s.off_o + pieces * head_dim * 4;
  return s;
}

// 16 numbers of e4m3 as two bf16 operands.
__device__ __forceinline__ void widened16(u32x4 x, bf16x8& lo, bf16x8& hi) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[w], 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[w], 1.0f, true);
    bf16x8& to = w < 2 ? lo : hi;
    to[4 * (w & 1)] = a[0];
    to[4 * (w & 1) + 1] = a[1];
    to[4 * (w & 1) + 2] = b[0];
    to[4 * (w & 1) + 3] = b[1];
  }
}

// A direct load of every lane's 16 bytes, from an address of its own, to lds + 16 * lane.
__device__ __forceinline__ void load_rows_to_lds(const char* at, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(at) : "memory");
}

template <int D, bool F8, int CW, int PARTS>
__global__ __launch_bounds__(64 * kTreeWaves, 2) void tree_kernel(TreeParams p, TreeSpace ws, int32_t blocks, int32_t shares, int32_t direct) {
  constexpr int RW = kTreeWaves / CW, HALVES = 2 / RW, MB = 2, NB = 2, DK = D / 32, DB = D / 16;
  constexpr int kBytes = F8 ? 1 : 2, TILE = kTreeRows * 2 * D, COLS = 32 * CW, AHEAD = 4;
  constexpr int PER_ROW = D * kBytes / 16, RPI = 64 / PER_ROW, NI = 16 / RPI;   // lanes of a row; rows of a load; loads of a wave's 16 rows
  extern __shared__ __attribute__((aligned(1024))) char smem[];   // [2][K tile, V tile], the rows that are there [2][wave], maxima and sums
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_bytes)smem;
  volatile uint16_t* const there_lds = (volatile uint16_t*)(smem + 4 * TILE);
  float2* const ml_lds = (float2*)(smem + 4 * TILE + 16);
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 15, g = lane >> 4;
  const int cw = wave % CW, rw = wave / CW;
  const int32_t group = p.q_heads / p.kv_heads, per_seq = p.kv_heads * blocks;

  // Blocks of columns of one (share, key head) read the same rows: they are work-groups of one XCD, as near each other as can be.
  const int32_t of8 = (int32_t)blockIdx.x / (8 * blocks), in8 = (int32_t)blockIdx.x - of8 * 8 * blocks, cb = in8 >> 3, sh = 8 * of8 + (in8 & 7);
  const int32_t share = sh / p.kv_heads, hk = sh - share * p.kv_heads, c0 = cb * COLS;
  if (share >= shares) return;

  // The first unit of this share: the units of all sequences one after the other
  TreeDeal deal;
  TreeSeq seq;
  int32_t b = share, at = 0, unit = 0, left = 1;
  if (direct) {
    seq = tree_seq(p, b);
  } else {
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
      mine = b0 + lane < p.batch ? tree_seq(p, b0 + lane) : TreeSeq{};
      total += __builtin_amdgcn_readlane(upto(mine.units), 63);
    }
    deal.init(total, shares);
    unit = deal.first(share);
    left = deal.first(share + 1) - unit;
    if (left == 0) return;
    int32_t passed = 0;
    for (int32_t b0 = 0;; b0 += 64) {   // (unit < total: one sequence has it)
      if (p.batch > 64) mine = b0 + lane < p.batch ? tree_seq(p, b0 + lane) : TreeSeq{};
      const int32_t end = passed + upto(mine.units), begin = end - mine.units;
      const uint64_t has = __ballot(begin <= unit && unit < end);
      if (has != 0) {
        const int l = __builtin_ctzll(has);
        b = b0 + l;
        at = unit - __builtin_amdgcn_readlane(begin, l);
        break;
      }
      passed = __builtin_amdgcn_readlane(end, 63);
    }
    seq = tree_seq(p, b);
  }

  OperandAddr<D> ad;
  ad.init(lane);
  // This lane's part of a tile: rows 16 wave + RPI i + lane / PER_ROW
  const int row_in = 16 * wave + lane / PER_ROW, piece_in = lane % PER_ROW;
  bool first_piece = true;

  while (left > 0) {
    b = __builtin_amdgcn_readfirstlane(b);
    seq.tokens = __builtin_amdgcn_readfirstlane(seq.tokens);
    seq.hi = __builtin_amdgcn_readfirstlane(seq.hi);
    seq.older = __builtin_amdgcn_readfirstlane(seq.older);
    seq.lo = __builtin_amdgcn_readfirstlane(seq.lo);
    seq.ts = __builtin_amdgcn_readfirstlane(seq.ts);
    seq.tf = __builtin_amdgcn_readfirstlane(seq.tf);
    seq.units = __builtin_amdgcn_readfirstlane(seq.units);
    const int32_t take = direct ? seq.units : left < seq.units - at ? left : seq.units - at;
    const bool whole = direct || (at == 0 && take == seq.units);
    if (!direct && hk == 0 && cb == 0 && at == 0 && tid == 0 && seq.units > 0) {
      const int32_t last = whole ? share : deal.owner(unit + seq.units - 1);
      ws.owners[b] = int2{share, 2 * last + (first_piece ? 0 : 1)};
    }

    if (take > 0 && c0 < seq.tokens * group) {
      const int32_t columns = seq.tokens * group, sinks = p.sinks < seq.older ? p.sinks : seq.older;
      const bool live = c0 + 32 * cw < columns;   // this wave has columns
      // What the columns see; what some token of the sequence sees, by lane = token
      int32_t first[NB];
      uint64_t word[NB], any_word = 0;
      bf16x8 q[DK][NB];
      int32_t latest = 0;
      auto word_of = [&](int32_t i) { return (p.seen ? p.seen[b * p.seen_sb + i] : low_bits(i + 1)) & low_bits(seq.tokens); };
      if (lane < seq.tokens) any_word = word_of(lane);
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) any_word |= __shfl_xor(any_word, s, 64);
      if (p.elsewhere) any_word = 0;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int32_t c = c0 + 32 * cw + 16 * nb + r, i = c / group, h = hk * group + (c - i * group);
        const bool there = c < columns;
        first[nb] = there && p.first ? max(p.first[b * p.first_sb + i], 0) : 0;
        word[nb] = there && !p.elsewhere ? word_of(i) : 0;
        latest = first[nb] > latest ? first[nb] : latest;
        const __bf16* row = (const __bf16*)p.q.ptr + b * p.q.sb + i * p.q.ss + h * p.q.sh + 8 * g;
#pragma unroll
        for (int ks = 0; ks < DK; ++ks) q[ks][nb] = there ? *reinterpret_cast<const bf16x8*>(row + 32 * ks) : zero_operand();
      }
#pragma unroll
      for (int s = 1; s < 16; s <<= 1) {
        const int32_t other = __shfl_xor(latest, s, 64);
        latest = other > latest ? other : latest;
      }
      latest = __builtin_amdgcn_readfirstlane(latest);
      const float to_log2 = p.scale * kLog2e * (F8 && p.cache.k_scale ? p.cache.k_scale[hk] : 1.f);
      const char* const k_base = (const char*)p.cache.k + hk * p.cache.s_head * kBytes;
      const char* const v_base = (const char*)p.cache.v + hk * p.cache.s_head * kBytes;
      const int32_t* const table = p.cache.table + b * p.cache.table_stride;

      float m[NB], l[NB];
      f32x4 acc[DB][NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        m[nb] = -INFINITY;
        l[nb] = 0.f;
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[db][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
      }

      auto tile_row = [&](int32_t u) { return (u < seq.ts ? u : u - seq.ts + seq.tf) * kTreeRows; };
      int32_t page[NI];
      auto look_up = [&](int32_t u) {   // the pages of this lane's rows
        const int32_t row0 = tile_row(u);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const int32_t row = row0 + row_in + RPI * i;
          page[i] = row < seq.hi ? table[p.cache.by_page.quotient(row)] : -1;
        }
      };
      u32x4 raw_k[F8 ? NI : 1], raw_v[F8 ? NI : 1];
      uint32_t mine = 0;           // of the tile under way: which of this lane's rows are there
      bool all_there = true;
      // Asks for a tile whose pages are known.  Rows that are not there or that no token sees: some row that is there, whose keys are not looked at and
      // whose values are made zeros (they may hold NaN, which a P of 0 would not silence).
      auto ask = [&](int32_t u, int slot) {
        const int32_t row0 = tile_row(u);
        mine = 0;
        const char *from_k[NI], *from_v[NI];
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const int32_t row = row0 + row_in + RPI * i, j = row - seq.older;
          const bool seen = j < 0 ? row >= seq.lo || row < sinks : ((any_word >> (j & 63)) & 1) != 0 && j < 64;
          const bool there = seen && page[i] >= 0 && page[i] < p.cache.n_pages;
          const int32_t in_page = row - p.cache.by_page.quotient(row) * p.cache.page_rows;
          const int64_t off = there ? (page[i] * p.cache.s_page + in_page * p.cache.s_row) * kBytes : 0;
          mine |= there ? 1u << i : 0u;
          const int piece = F8 ? piece_in : piece_in ^ swz<D>(row_in + RPI * i);   // (row0 is a multiple of 16)
          from_k[i] = k_base + off + 16 * piece;
          from_v[i] = v_base + off + 16 * piece;
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          if constexpr (F8) {
            raw_k[i] = *reinterpret_cast<const u32x4*>(from_k[i]);
            raw_v[i] = *reinterpret_cast<const u32x4*>(from_v[i]);
          } else {
            load_rows_to_lds(from_k[i], lds0 + slot * 2 * TILE + (wave * NI + i) * 1024);
            load_rows_to_lds(from_v[i], lds0 + slot * 2 * TILE + TILE + (wave * NI + i) * 1024);
          }
        }
        all_there = __all(mine == (1u << NI) - 1u);
        uint32_t bits = 0xffffu;
        if (!all_there) {
          bits = 0;
#pragma unroll
          for (int i = 0; i < NI; ++i) {
            const uint64_t v = __ballot((mine >> i) & 1u);
#pragma unroll
            for (int k = 0; k < RPI; ++k) bits |= (uint32_t)((v >> (k * PER_ROW)) & 1u) << (RPI * i + k);
          }
        }
        if (lane == 0) there_lds[slot * kTreeWaves + wave] = (uint16_t)bits;
      };
      // The tile that was asked for is in LDS, as far as this wave brings it
      auto arrive = [&](int slot) {
        if constexpr (F8) {
          char* const kt = smem + slot * 2 * TILE;
#pragma unroll
          for (int i = 0; i < NI; ++i) {
            const int row = row_in + RPI * i;
            if (!((mine >> i) & 1u)) raw_v[i] = u32x4{0, 0, 0, 0};
            bf16x8 x[2];
            const int at0 = row * 2 * D + ((2 * piece_in) ^ swz<D>(row)) * 16, at1 = row * 2 * D + ((2 * piece_in + 1) ^ swz<D>(row)) * 16;
            widened16(raw_k[i], x[0], x[1]);
            *reinterpret_cast<bf16x8*>(kt + at0) = x[0];
            *reinterpret_cast<bf16x8*>(kt + at1) = x[1];
            widened16(raw_v[i], x[0], x[1]);
            *reinterpret_cast<bf16x8*>(kt + TILE + at0) = x[0];
            *reinterpret_cast<bf16x8*>(kt + TILE + at1) = x[1];
          }
        } else {
          wait_loads<0>();
          if (!all_there) {
#pragma unroll
            for (int i = 0; i < NI; ++i)
              if (!((mine >> i) & 1u)) *reinterpret_cast<u32x4*>(smem + slot * 2 * TILE + TILE + (wave * NI + i) * 1024 + 16 * lane) = u32x4{0, 0, 0, 0};
          }
        }
      };

      look_up(at);
      ask(at, 0);
      if (take > 1) look_up(at + 1);
      int slot = 0;
      for (int32_t u = at; u < at + take; ++u, slot ^= 1) {
        arrive(slot);
        stores_loads_barrier<0>();
        const uint64_t there = *reinterpret_cast<const volatile uint64_t*>(there_lds + slot * kTreeWaves);
        if (u + 1 < at + take) {
          ask(u + 1, slot ^ 1);
          if (u + 2 < at + take) look_up(u + 2);
        }
        if (!live) continue;
        const uint32_t kt = lds0 + slot * 2 * TILE, vt = kt + TILE;
        const int32_t t0 = tile_row(u);
        const bool full = there == ~0ull && t0 + kTreeRows <= seq.older && (t0 >= latest || t0 + kTreeRows <= sinks);
        // 32 rows at a time: the scores and P of 64 do not fit in the registers beside the sums
#pragma clang loop unroll(disable)
        for (int half = 0; half < HALVES; ++half) {
          const int row0 = 32 * (RW == 2 ? rw : half);
          const uint32_t kh = kt + row0 * 2 * D, vh = vt + row0 * 2 * D;
          f32x4 s[MB][NB];
          {
            const f32x4 zero[MB] = {};
            bf16x8 ahead[AHEAD];
            rows_fetch<D, MB, AHEAD>(kh, ad, 0, ahead);
            rows_product<D, MB, NB, AHEAD>(kh, ad, 0, q, s, zero, ahead);
          }
          bf16x8 part[NB][PARTS];
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            float x[8], top = -INFINITY;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = s[e >> 2][nb][e & 3] * to_log2;
            if (!full) {
              uint64_t seen = tile_interval(first[nb], seq.older, t0) | tile_interval(0, sinks, t0) | moved(word[nb], seq.older - t0);
              const uint32_t bits = (uint32_t)((seen & there) >> row0) >> (4 * g);
#pragma unroll
              for (int e = 0; e < 8; ++e) x[e] = (bits >> (16 * (e >> 2) + (e & 3))) & 1 ? x[e] : -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, x[e]);
            if (__any(top > m[nb] + kTreeStale)) {   // (the first tile: m is -inf)
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
            for (int e = 0; e < 8; ++e) {
              x[e] = __builtin_amdgcn_exp2f(x[e] - base);
              l[nb] += x[e];
            }
            u16x2 least[4];
#pragma unroll
            for (int n = 0; n < PARTS; ++n) {
              u32x4 words;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                float &x0 = x[2 * i], &x1 = x[2 * i + 1];
                uint32_t two = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, x1), __builtin_bit_cast(uint32_t, x0), 0x07060302u);
                if (PARTS == 2 && n == 1) two = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x0, (__bf16)x1});   // (rounded: 2^-17 of P at most)
                u16x2 bits = __builtin_bit_cast(u16x2, two);
                if (!F8 && n == 0) least[i] = __builtin_elementwise_sub_sat(bits, u16x2{kTreeLeastPart, kTreeLeastPart});
                if (!F8 && n != 0) bits = __builtin_elementwise_max(bits, least[i]);
                words[i] = __builtin_bit_cast(uint32_t, bits);
                x0 -= __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x0) & 0xffff0000u);   // (exact)
                x1 -= __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x1) & 0xffff0000u);
              }
              part[nb][n] = __builtin_bit_cast(bf16x8, words);
            }
          }
          bf16x8 a[DB];
          MatrixPhase prio;
#pragma unroll
          for (int i = 0; i < AHEAD; ++i) a[i] = cols_operand<D>(vh, ad, 0, i);
#pragma unroll
          for (int i = 0; i < DB; ++i) {
            if (i + AHEAD < DB) a[i + AHEAD] = cols_operand<D>(vh, ad, 0, i + AHEAD);
#pragma unroll
            for (int n = 0; n < PARTS; ++n)
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) acc[i][nb] = mfma16(a[i], part[nb][n], acc[i][nb]);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }

      // Lane (r, g) has of column r elements 16 db + 4g ..  The halves of 64 columns' rows against the larger maximum of both.
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        l[nb] += __shfl_xor(l[nb], 16, 64);
        l[nb] += __shfl_xor(l[nb], 32, 64);
      }
      __syncthreads();
      if constexpr (RW == 2) {
        f32x4* const sums = reinterpret_cast<f32x4*>(smem) + cw * (DB * NB * 64) + lane;
        if (rw == 1) {
#pragma unroll
          for (int i = 0; i < DB * NB; ++i) sums[64 * i] = acc[i / NB][i % NB];
          if (g == 0) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) ml_lds[32 * cw + 16 * nb + r] = float2{m[nb], l[nb]};
          }
        }
        __syncthreads();
        if (rw == 0) {
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            const float2 other = ml_lds[32 * cw + 16 * nb + r];
            const float top = fmaxf(m[nb], other.x);
            const float f0 = m[nb] == top ? 1.f : __builtin_amdgcn_exp2f(m[nb] - top), f1 = other.x == top ? 1.f : __builtin_amdgcn_exp2f(other.x - top);
            m[nb] = top;
            l[nb] = l[nb] * f0 + other.y * f1;
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db][nb] = acc[db][nb] * f0 + sums[64 * (db * NB + nb)] * f1;
          }
        }
        __syncthreads();
      }
      if (rw == 0) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const int32_t in = 32 * cw + 16 * nb + r, c = c0 + in, i = c / group, h = hk * group + (c - i * group);
          if (c >= columns) continue;
          if (whole) {
            const float over = l[nb] == 0.f ? 0.f : (F8 && p.cache.v_scale ? p.cache.v_scale[hk] : 1.f) / l[nb];
            const int64_t to = b * p.o.sb + i * p.o.ss + h * p.o.sh + 4 * g;
#pragma unroll
            for (int db = 0; db < DB; ++db) {
              const f32x4 x = acc[db][nb] * over;
              if (p.o.is_f32) *reinterpret_cast<f32x4*>((float*)p.o.ptr + to + 16 * db) = x;
              else *reinterpret_cast<bf16x4*>((__bf16*)p.o.ptr + to + 16 * db) = bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
            }
            if (g == 0 && p.lse.ptr) p.lse.ptr[b * p.lse.sb + h * p.lse.sh + i] = l[nb] == 0.f ? -INFINITY : (m[nb] + __log2f(l[nb])) * kLn2;
          } else {
            const int64_t piece = (2 * ((int64_t)share * per_seq + hk * blocks + cb) + (first_piece ? 0 : 1)) * COLS + in;
#pragma unroll
            for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(ws.o + piece * D + 16 * db + 4 * g) = acc[db][nb];
            if (g == 0) ws.ml[piece] = float2{m[nb], l[nb]};
          }
        }
      }
    }
    if (direct) break;
    first_piece = false;
    unit += take;
    left -= take;
    at = 0;
    if (left > 0) seq = tree_seq(p, ++b);
  }
}

// A (sequence, new token, query head) whose rows several work-groups had: their pieces added up.  D / 4 threads for each.
template <int D, int COLS>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeParams p, TreeSpace ws, int32_t blocks) {
  constexpr int LANES = D / 4;
  const int64_t row = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LANES;
  const int lane = threadIdx.x % LANES;
  const int32_t h = (int32_t)(row % p.q_heads), group = p.q_heads / p.kv_heads, hk = h / group;
  const int64_t bi = row / p.q_heads;
  const int32_t b = (int32_t)(bi / p.sq), i = (int32_t)(bi - (int64_t)b * p.sq);
  if (b >= p.batch) return;
  int32_t tokens = p.tokens ? p.tokens[b] : p.sq;
  if (i >= tokens) return;
  const int2 owners = ws.owners[b];
  const int32_t w0 = owners.x, w1 = owners.y >> 1, skip = owners.y & 1;
  if (w0 == w1) return;   // written out by its only owner
  const int32_t c = i * group + (h - hk * group), hb = hk * blocks + c / COLS, per_seq = p.kv_heads * blocks;
  auto piece = [&](int32_t w) { return (2 * ((int64_t)w * per_seq + hb) + (w == w0 ? skip : 0)) * COLS + c % COLS; };
  float top = -INFINITY, sum = 0.f;
  for (int32_t w = w0; w <= w1; ++w) top = fmaxf(top, ws.ml[piece(w)].x);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int32_t w = w0; w <= w1; ++w) {
    const int64_t at = piece(w);
    const float2 ml = ws.ml[at];
    const float f = ml.x == top ? 1.f : __builtin_amdgcn_exp2f(ml.x - top);
    sum += ml.y * f;
    o += *reinterpret_cast<const f32x4*>(ws.o + at * D + 4 * lane) * f;
  }
  o *= sum == 0.f ? 0.f : (p.cache.v_scale ? p.cache.v_scale[hk] : 1.f) / sum;
  const int64_t to = b * p.o.sb + i * p.o.ss + h * p.o.sh + 4 * lane;
  if (p.o.is_f32) *reinterpret_cast<f32x4*>((float*)p.o.ptr + to) = o;
  else *reinterpret_cast<bf16x4*>((__bf16*)p.o.ptr + to) = bf16x4{(__bf16)o[0], (__bf16)o[1], (__bf16)o[2], (__bf16)o[3]};
  if (lane == 0 && p.lse.ptr) p.lse.ptr[b * p.lse.sb + h * p.lse.sh + i] = sum == 0.f ? -INFINITY : (top + __log2f(sum)) * kLn2;
}

TreeShape shape_of(const TreeParams& p) { return tree_shape(p.batch, p.sq, p.q_heads, p.kv_heads, p.head_dim, p.max_rows); }

template <int D, bool F8, int CW, int PARTS>
hipError_t launch(const TreeParams& p, hipStream_t stream) {
  constexpr int LDS = 4 * kTreeRows * 2 * D + 16 + 64 * 8;
  const TreeShape s = shape_of(p);
  char* const space = (char*)p.workspace;
  const TreeSpace ws{(int2*)space, (float2*)(space + s.off_ml), (float*)(space + s.off_o)};
  const int64_t pairs = ((int64_t)s.shares * p.kv_heads + 7) / 8 * 8;
  hipLaunchKernelGGL((tree_kernel<D, F8, CW, PARTS>), dim3((uint32_t)(pairs * s.blocks)), dim3(64 * kTreeWaves), LDS, stream, p, ws, s.blocks, s.shares,
                     s.direct ? 1 : 0);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || s.direct) return e;
  const int64_t rows = (int64_t)p.batch * p.sq * p.q_heads;
  hipLaunchKernelGGL((tree_join_kernel<D, 32 * CW>), dim3((uint32_t)((rows * (D / 4) + 255) / 256)), dim3(256), 0, stream, p, ws, s.blocks);
  return hipGetLastError();
}
template <int D, bool F8>
hipError_t launch(const TreeParams& p, hipStream_t stream) {
  if (shape_of(p).columns == 64) return launch<D, F8, 2, 3>(p, stream);
  return p.o.is_f32 ? launch<D, F8, 4, 3>(p, stream) : launch<D, F8, 4, 2>(p, stream);
}
template <int D>
hipError_t launch(const TreeParams& p, hipStream_t stream) {
  return p.cache.is_f8 ? launch<D, true>(p, stream) : launch<D, false>(p, stream);
}

}  // namespace

int64_t tree_workspace_bytes(int32_t batch, int32_t sq, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int64_t max_rows) {
  return tree_shape(batch, sq, q_heads, kv_heads, head_dim, max_rows).bytes;
}

void tree_plan(const TreeParams& p, int32_t out[3]) {
  const TreeShape s = shape_of(p);
  out[0] = s.shares;
  out[1] = s.columns;
  out[2] = s.direct;
}

hipError_t launch_tree(const TreeParams& p, hipStream_t stream) {
  return p.head_dim == 128 ? launch<128>(p, stream) : launch<64>(p, stream);
}

}  // namespace burst
