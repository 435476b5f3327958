// Attention of one new token of every sequence over its rows in a paged cache.
//
// The bytes of the cache bound it: each key/value element is read once and takes part in 2 (group) products, so the kernel is built
// to keep loads under way, and the arithmetic only has to stay out of their way.
//
//   A wave takes tiles of 32 rows of one key head for the 16 (or 32) query heads that share it.  S^T = K Q^T and O^T = V^T P^T run on
//   v_mfma_f32_16x16x32_bf16 with rows of the cache loaded straight into the operands' registers, no LDS in between: 16 lanes of a K load
//   take 64 bytes each of 16 rows (an A operand as it is), 16 lanes of a V load a whole row.  Lane (r, g) then has for 8 keys the same
//   D / 16 elements of V, and one v_perm for every two of them makes them the A operand whose k index is the key: the keys that S^T leaves
//   in this lane's accumulators (16 (e / 4) + 4g + e % 4), so P needs no exchange between lanes either.
//   The running maximum of a column is a whole number (base 2), so that a rescale by 2^n changes no bit of P and O, and which rows
//   another wave or work-group took has no influence but roundings in fp32 (of S minus the maximum, and the order of sums).  P goes in whole, as the three bf16 numbers that its
//   24 bits are (in two parts O was 4.9e-6 off 64 bits, in three 1.1e-6, as elementary operations in 32 bits; the time is the same: the matrix
//   pipe is busy a sixth of it).
//
//   Work is cut into units of a tile for each wave and numbered over (sequence, rows).  The units are dealt evenly to shares, a work-group each for
//   every key head, as many as the chip holds at once, whatever the sequences' lengths are: each finds its first unit by a scan
//   over the sequences.  A piece that is a whole (sequence, key head) is written out; what a work-group has of others goes to the
//   workspace, two pieces at most, and decode_join_kernel adds the pieces up in a fixed order.  Half as many work-groups as fit: e4m3 212 -> 239
//   us, one and a half times as many 212 -> 232, twice as many 228.  Two tiles under way in a wave instead of one: no gain (the
//   CU's own rate of loads, about 50 GB/s, is what a short sequence waits for, and the memory a long one).
//
// Measured (rows x key heads, a cache of its own for each of three calls in turn): 131072 x 32 bf16 320 us, 6.72 TB/s (a copy reaches 5.2, a
// fill 6.9); 32 sequences of 32768 and fewer x 8 in e4m3 135 us, 5.3 TB/s (128-byte rows of heads side by side; head by head 5.7); 64
// of 4096 and fewer x 8 65 us, 5.1 TB/s; 32768 x 8 32 us, 4.2 TB/s, of which 5 us are the second kernel and 6 the first loads.
// Pages of a multiple of 16 rows, whose size else does not matter, against others (65536 x 8, heads side by side; a row's address by each lane and a
// shuffle): bf16 54 us and 58-62, e4m3 40 and 42-45; direct, 16 sequences of 1000 x 8, 20.8 and 24.9.  Query heads over a key head (4 x 131072 x 1 of 128,
// floor 52 us): 1 to 16 51-53 us, 17 to 32 (queries in LDS) 56-59, 33 to 64 98-101, as every 32 read the keys and values for themselves.
#include "cache.hpp"
#include "kernels.hpp"
#include "mfma16.hpp"

namespace burst {

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
// Read by scalar loads: a vector load of a page's number would have to be waited for together with all tiles asked for before it.
typedef const __attribute__((address_space(4))) int32_t* scalar_table;

constexpr int kTileRows = 32, kDealtWaves = 4;
constexpr int kDirectWaves = 8;
constexpr float kStale = 8.f;   // a maximum may fall behind by a factor of 2^8: P, O and their sums stay far inside fp32
// No part of a weight is 0 (as the second would be of a power of two), or an infinity among the values would give NaN: each is about 2^-32 of the
// weight at least, which stays below what fp32 rounds.  (e4m3 has no infinity.)  In bits of bf16, which grow with the number:
constexpr uint16_t kLeastPart = 32 << 7;
constexpr int kCus = 256;
// Waves that share a SIMD, by the registers that one takes (also: work-groups of four waves that share a CU).
constexpr int waves_per_simd(int head_dim, bool f8, int nc) { return nc == 2 ? 2 : 2 + (head_dim == 64) + f8; }

// What a sequence's share of the work is.  It starts at a multiple of the tile, so that the halves of a tile lie in one page each where
// pages are multiples of 16 rows; a sequence without rows has one unit, which writes its empty result.
struct SeqRows {
  int32_t lo, hi, start, units;
};
__device__ __forceinline__ SeqRows seq_rows(const DecodeParams& p, int32_t n, int32_t first, int unit_rows) {
  SeqRows s;
  const int32_t most = p.max_rows;   // (at most table_cols * page_rows, checked on the host)
  s.hi = n < 0 ? 0 : n > most ? most : n;
  s.lo = first < 0 ? 0 : first < s.hi ? first : s.hi;
  s.start = s.lo & ~(kTileRows - 1);
  s.units = s.lo < s.hi ? (s.hi - s.start + unit_rows - 1) / unit_rows : 1;
  return s;
}
__device__ __forceinline__ SeqRows seq_rows_of(const DecodeParams& p, int32_t b, int unit_rows) {
  return seq_rows(p, p.cache.rows[b], p.first_row ? p.first_row[b] : 0, unit_rows);
}

// Units dealt to `shares` work-groups: the first `more` of them get one more.
struct Deal {
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

// Heads of a cache row that the waves of a work-group take beside each other, 512 bytes where they lie side by side.
constexpr int heads_side_by_side(int head_dim, bool f8) { return head_dim == 128 && !f8 ? 2 : 4; }

// The workspace: for each sequence its first owner and, times two, its last one, plus one if the first owner's piece is its second (an owner is
// a share of the units; every block of columns of every key head has the same shares); and two pieces for every work-group, each (maximum,
// sum) and O of its columns relative to that maximum.
struct DecodeSpace {
  int2* owners;
  float2* ml;
  float* o;
  int32_t columns;   // of a piece: min(group, 16 NC)
};

struct DecodeShape {
  int32_t blocks, shares;   // blocks of columns of a key head; shares of a block's units, a work-group each
  int32_t columns;
  bool direct;              // a work-group for every (sequence, key head, block of columns), no workspace
  int64_t off_ml, off_o, bytes;
};
static int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }
static int columns_of(int32_t group) { return group <= 16 ? 16 : 32; }
static DecodeShape decode_shape(int32_t batch, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int64_t max_rows, bool f8, int heads) {
  DecodeShape s;
  const int32_t group = q_heads / kv_heads, wide = columns_of(group);
  s.blocks = (group + wide - 1) / wide;
  s.columns = group < wide ? group : wide;
  const int64_t per_seq = (int64_t)kv_heads * s.blocks, unit = kTileRows * kDealtWaves / heads, max_units = (max_rows + unit - 1) / unit;
  // The line between the two: a work-group for each (sequence, key head) saves the scan and the second kernel, and reads its rows by itself.  bf16,
  // heads of 128, direct and dealt: one sequence x 8 heads, 512 rows 9.7 and 11.4 us, 1024 rows 14.3 and 11.5; heads of 64, 1024 rows 10.2
  // and 10.4; e4m3, 32 sequences x 8, 1024 rows 16.2 and 24, 2048 rows 34.5 and 41; bf16, 64 sequences x 8, 1024 rows 56 and 55, of
  // that and less 39 and 38.
  const int64_t head_bytes = max_rows * head_dim * (f8 ? 2 : 4);
  s.direct = head_bytes <= (batch * per_seq < kCus ? 256 << 10 : 512 << 10);
  const int64_t fit = std::max<int64_t>(1, kCus * waves_per_simd(head_dim, f8, wide / 16) * heads / per_seq);
  s.shares = (int32_t)(s.direct ? batch : std::min<int64_t>(batch * max_units, fit));
  const int64_t pieces = s.shares * per_seq * 2 * s.columns;
  s.off_ml = up256((int64_t)batch * 8);
  s.off_o = s.off_ml + up256(pieces * 8);
  s.bytes = s.direct ? 0 : s.off_o + pieces * head_dim * 4;
  return s;
}
int64_t decode_workspace_bytes(int32_t batch, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int64_t max_rows) {
  int64_t most = 0;
  for (bool f8 : {false, true})
    for (int heads : {1, heads_side_by_side(head_dim, f8)})
      most = std::max(most, decode_shape(batch, q_heads, kv_heads, head_dim, max_rows, f8, heads).bytes);
  return most;
}
static DecodeSpace space_of(const DecodeShape& s, void* workspace) {
  char* ws = (char*)workspace;
  return DecodeSpace{(int2*)ws, (float2*)(ws + s.off_ml), (float*)(ws + s.off_o), s.columns};
}

// 8 numbers of e4m3 (two words) as a bf16 operand.
__device__ __forceinline__ bf16x8 widened(uint32_t w0, uint32_t w1) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.0f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.0f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A tile's keys and values in a wave's registers.  NT (where work is dealt): the lines are not kept, as there are more than the chip keeps until the
// next call; 131072 rows x 32 heads 374 -> 334 us, 16 x 16384 x 8 202 -> 179, 32768 x 8 38.9 -> 35.9 (head by head).  Where a sequence
// is short they are, for the next call: 1024 rows x 8 heads 14.6 us kept, 19.8 not.
template <int D, bool F8, bool NT>
struct Tile {
  static constexpr int kBytes = F8 ? 1 : 2;
  static constexpr int KW = D * kBytes / 64;         // 16-byte pieces of a K row in a lane
  static constexpr int VW = D * kBytes / 64;         // words of a V row in a lane (D / 16 elements)
  u32x4 k[2][KW];
  uint32_t v[8][VW];

  // The A operand of half t and k-step kk: row 16 t + r, elements 32 kk + 8g .. (bf16), 64 (kk / 2) + 16 g + 8 (kk % 2) .. (e4m3).
  __device__ __forceinline__ bf16x8 k_operand(int t, int kk) const {
    if constexpr (F8) return widened(k[t][kk / 2][2 * (kk & 1)], k[t][kk / 2][2 * (kk & 1) + 1]);
    else return __builtin_bit_cast(bf16x8, k[t][kk]);
  }
  __device__ __forceinline__ static int q_element(int g, int kk) { return F8 ? 64 * (kk / 2) + 16 * g + 8 * (kk & 1) : 32 * kk + 8 * g; }
  __device__ __forceinline__ void load_k(int t, const char* row) {   // of this lane: row 16 t + r, its piece g
#pragma unroll
    for (int i = 0; i < KW; ++i) k[t][i] = load_as<u32x4, NT>(row + 64 * i);
  }
  __device__ __forceinline__ void load_v(int e, const char* row) {   // of this lane: key e, elements D / 16 r ..
    if constexpr (VW == 4) {
      const u32x4 x = load_as<u32x4, NT>(row);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[e][i] = x[i];
    } else if constexpr (VW == 2) {
      const u32x2 x = load_as<u32x2, NT>(row);
      v[e][0] = x[0];
      v[e][1] = x[1];
    } else {
      v[e][0] = load_as<uint32_t, NT>(row);
    }
  }
};

// A 32-bit offset that the compiler takes as new here: added to a scalar base it becomes an operand of the load, where one extended to 64
// bits outside the loop would be added by the vector unit and take two registers.
__device__ __forceinline__ uint32_t offset_here(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Where a tile's rows lie, and which of them are seen (a bit for each).
struct TilePlace {
  uint32_t seen;
  const char* half_k[2];   // pages of a multiple of 16 rows: first row of each half
  const char* half_v[2];
  int64_t row;             // any pages: bytes to this lane's row (lane % 32)
};

// The sequence that holds the first unit of a work-group, found by a scan over all.
struct FirstUnit {
  SeqRows seq;
  int32_t b, at;   // the sequence, and which of its units
};

template <int D, bool F8, int NC, bool PAGES16, bool DIRECT, int HEADS>
__global__ __launch_bounds__(DIRECT ? 64 * kDirectWaves : 64 * kDealtWaves, waves_per_simd(D, F8, NC)) void decode_kernel(DecodeParams p, DecodeSpace ws,
                                                                                                         int32_t blocks, int32_t shares) {
  constexpr int KK = D / 32, DT = D / 16, kBytes = F8 ? 1 : 2, kWaves = DIRECT ? kDirectWaves : kDealtWaves, kRowWaves = kWaves / HEADS, kUnit = kRowWaves * kTileRows;
  __shared__ float part_o[kWaves][16][D + 4];
  __shared__ float2 part_ml[kWaves][NC * 16];
  constexpr bool kQInLds = NC == 2;   // two blocks of 16 queries do not fit in the registers beside their sums
  __shared__ bf16x8 q_lds[kQInLds ? HEADS : 1][kQInLds ? NC * KK : 1][64];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 15, g = lane >> 4;
  const int32_t group = p.q_heads / p.kv_heads, per_seq = p.kv_heads * blocks;
  const int head_wave = wave % HEADS, row_wave = wave / HEADS;

  // Heads next to each other are work-groups next to each other: their rows lie side by side in most caches, and are read at the same time.
  const int32_t share = (int32_t)blockIdx.x / (per_seq / HEADS), hb = (int32_t)blockIdx.x - share * (per_seq / HEADS);
  const int32_t hk0 = hb / blocks * HEADS, cb = hb % blocks, c0 = cb * 16 * NC;   // the first head; first of the block's columns in a group
  const int32_t hk = hk0 + head_wave;                                           // this wave's head

  SeqRows seq;
  int32_t b, at = 0;
  int32_t unit = 0, left = 1;
  Deal deal;
  if constexpr (DIRECT) {
    b = share;
    seq = seq_rows_of(p, b, kUnit);
  } else {
    __shared__ int32_t scan[kWaves];
    __shared__ FirstUnit found;
    auto upto = [&](int32_t x) {   // sum over this lane and the ones below
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) {
        const int32_t y = __shfl_up(x, s, 64);
        x += lane >= s ? y : 0;
      }
      return x;
    };
    if (p.batch <= 64) {   // each wave by itself
      const SeqRows mine = lane < p.batch ? seq_rows_of(p, lane, kUnit) : SeqRows{};
      const int32_t end = upto(mine.units), begin = end - mine.units;
      deal.init(__builtin_amdgcn_readlane(end, 63), shares);
      unit = deal.first(share);
      left = deal.first(share + 1) - unit;
      if (left == 0) return;
      b = __builtin_ctzll(__ballot(begin <= unit && unit < end));   // (one lane)
      at = unit - __builtin_amdgcn_readlane(begin, b);
      seq = SeqRows{__builtin_amdgcn_readlane(mine.lo, b), __builtin_amdgcn_readlane(mine.hi, b), __builtin_amdgcn_readlane(mine.start, b),
                    __builtin_amdgcn_readlane(mine.units, b)};
    } else {
      int32_t total = 0;   // (below 2^31, checked on the host)
      SeqRows mine = {};
      for (int32_t b0 = 0; b0 < p.batch; b0 += 256) {
        mine = b0 + tid < p.batch ? seq_rows_of(p, b0 + tid, kUnit) : SeqRows{};
        const int32_t sum = upto(mine.units);
        if (lane == 63) scan[wave] = sum;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) total += scan[w];
        __syncthreads();
      }
      deal.init(__builtin_amdgcn_readfirstlane(total), shares);
      unit = deal.first(share);
      left = deal.first(share + 1) - unit;
      if (left == 0) return;
      int32_t passed = 0;
      for (int32_t b0 = 0; b0 < p.batch; b0 += 256) {
        if (p.batch > 256) mine = b0 + tid < p.batch ? seq_rows_of(p, b0 + tid, kUnit) : SeqRows{};
        const int32_t sum = upto(mine.units);
        if (lane == 63) scan[wave] = sum;
        __syncthreads();
        int32_t begin = passed + sum - mine.units;
        for (int w = 0; w < kWaves; ++w) {
          begin += w < wave ? scan[w] : 0;
          passed += scan[w];
        }
        if (begin <= unit && unit < begin + mine.units) found = FirstUnit{mine, b0 + tid, unit - begin};   // (one thread)
        __syncthreads();
        if (passed > unit) break;
      }
      b = __builtin_amdgcn_readfirstlane(found.b);
      seq.lo = __builtin_amdgcn_readfirstlane(found.seq.lo);
      seq.hi = __builtin_amdgcn_readfirstlane(found.seq.hi);
      seq.start = __builtin_amdgcn_readfirstlane(found.seq.start);
      seq.units = __builtin_amdgcn_readfirstlane(found.seq.units);
      at = __builtin_amdgcn_readfirstlane(found.at);
    }
  }

  const uint32_t row_bytes = (uint32_t)p.cache.s_row * kBytes;
  const uint32_t k_lane = r * row_bytes + 16 * g, v_lane = 4 * g * row_bytes + DT * kBytes * r;
  bool first_piece = true;

  while (left > 0) {
    const int32_t take = DIRECT ? seq.units : left < seq.units - at ? left : seq.units - at;
    const bool whole = DIRECT || (at == 0 && take == seq.units);
    if constexpr (!DIRECT) {
      if (hb == 0 && at == 0 && tid == 0) {
        const int32_t last = whole ? share : deal.owner(unit + seq.units - 1);
        ws.owners[b] = int2{share, 2 * last + (first_piece ? 0 : 1)};
      }
    }

    bf16x8 q[kQInLds ? 1 : NC][KK];
    if (!kQInLds || row_wave == 0) {
#pragma unroll
      for (int nc = 0; nc < NC; ++nc) {
        const int32_t c = c0 + 16 * nc + r;
        const __bf16* row = (const __bf16*)p.q.ptr + b * p.q.sb + (int64_t)(hk * group + c) * p.q.sh;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          const bf16x8 x = c < group ? *reinterpret_cast<const bf16x8*>(row + Tile<D, F8, !DIRECT>::q_element(g, kk)) : bf16x8{};
          if constexpr (kQInLds) q_lds[head_wave][nc * KK + kk][lane] = x;
          else q[nc][kk] = x;
        }
      }
    }
    if constexpr (kQInLds) __syncthreads();
    const float to_log2 = p.scale * kLog2e * (F8 && p.cache.k_scale ? p.cache.k_scale[hk] : 1.f);
    const char* k_base = (const char*)p.cache.k + hk * p.cache.s_head * kBytes;
    const char* v_base = (const char*)p.cache.v + hk * p.cache.s_head * kBytes;
    const int32_t* table = p.cache.table + b * p.cache.table_stride;
    const scalar_table pages = (scalar_table)table;

    float m[NC], l[NC];
    f32x4 acc[NC][DT];
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
      m[nc] = -INFINITY;
      l[nc] = 0.f;
#pragma unroll
      for (int j = 0; j < DT; ++j) acc[nc][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // this wave's tiles: from t on every kRowWaves-th one, below t1
    const int32_t t1 = seq.units == at + take ? seq.hi : seq.start + (at + take) * kUnit;
    int32_t t = seq.start + at * kUnit + row_wave * kTileRows;

    // The pages of a tile as the table says them: of its two halves, or of this lane's row (lane % 32).  Asked for up to the bound, not the
    // sequence's end, so that the first look-up does not wait for that.
    auto look_up = [&](int32_t row0, int32_t (&page)[2]) {
      if constexpr (PAGES16) {
        page[0] = row0 < p.max_rows ? pages[p.cache.by_page.quotient(row0)] : -1;
        page[1] = row0 + 16 < p.max_rows ? pages[p.cache.by_page.quotient(row0 + 16)] : -1;
      } else {
        const int32_t row = row0 + (lane & 31);
        page[0] = row < p.max_rows ? table[p.cache.by_page.quotient(row)] : -1;
      }
    };
    auto place = [&](int32_t row0, const int32_t (&page)[2], TilePlace& x) {
      // rows of the tile that the sequence has
      const int32_t below = seq.hi - row0, above = seq.lo - row0;
      uint32_t seen = below >= 32 ? ~0u : below > 0 ? (1u << below) - 1u : 0u;
      if (above > 0) seen &= ~0u << above;   // (start is at most 31 before lo)
      if constexpr (PAGES16) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          int64_t off = 0;   // a half without a page: any rows that are there, unseen
          const int32_t row = row0 + 16 * h;
          if (row < seq.hi && page[h] >= 0 && page[h] < p.cache.n_pages) {
            const int32_t in_page = row - p.cache.by_page.quotient(row) * p.cache.page_rows;
            off = (page[h] * p.cache.s_page + in_page * p.cache.s_row) * kBytes;
          } else {
            seen &= h ? 0x0000ffffu : 0xffff0000u;
          }
          x.half_k[h] = k_base + off;
          x.half_v[h] = v_base + off;
        }
        x.seen = seen;
      } else {
        const int32_t row = row0 + (lane & 31), in_page = row - p.cache.by_page.quotient(row) * p.cache.page_rows;
        const bool there = row < seq.hi && page[0] >= 0 && page[0] < p.cache.n_pages;
        x.seen = seen & (uint32_t)__ballot(there);
        x.row = there ? (page[0] * p.cache.s_page + in_page * p.cache.s_row) * kBytes : 0;
      }
    };
    Tile<D, F8, !DIRECT> tile;
    auto load_k = [&](const TilePlace& x) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if constexpr (PAGES16) tile.load_k(h, x.half_k[h] + offset_here(k_lane));
        else tile.load_k(h, k_base + __shfl(x.row, 16 * h + r, 64) + 16 * g);
      }
    };
    auto load_v = [&](const TilePlace& x) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (PAGES16) tile.load_v(e, x.half_v[e >> 2] + offset_here(v_lane + (e & 3) * row_bytes));
        else tile.load_v(e, v_base + __shfl(x.row, 16 * (e >> 2) + 4 * g + (e & 3), 64) + DT * kBytes * r);
      }
    };

    int32_t page[2] = {-1, -1};
    TilePlace now;
    look_up(t, page);
    if (t < t1) {
      place(t, page, now);
      load_k(now);
      load_v(now);
      look_up(t + kUnit, page);
    }
    for (; t < t1; t += kUnit) {
      // (pages of any size: behind the last tile row 0 of page 0 is asked for, by all lanes; with a condition there the compiler forgets registers
      // that are still to be read, which the build refuses)
      const bool more = !PAGES16 || t + kUnit < t1;
      f32x4 s[NC][2];
      if constexpr (kQInLds) asm volatile("" ::: "memory");   // (or the compiler reads the queries once, into registers)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          const bf16x8 a = tile.k_operand(h, kk);
#pragma unroll
          for (int nc = 0; nc < NC; ++nc) {
            bf16x8 qv;
            if constexpr (kQInLds) qv = q_lds[head_wave][nc * KK + kk][lane];
            else qv = q[nc][kk];
            s[nc][h] = mfma16(a, qv, kk == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[nc][h]);
          }
        }
      const uint32_t seen = now.seen;
      if (more) {
        place(t + kUnit, page, now);
        load_k(now);
        look_up(t + 2 * kUnit, page);
      }
      // this lane's keys: bit 16 (e / 4) + 4g + e % 4
      const uint32_t bits = ((seen >> (4 * g)) & 15u) | ((seen >> (4 * g + 12)) & 0xf0u);
      bf16x8 p_part[NC][3];
#pragma unroll
      for (int nc = 0; nc < NC; ++nc) {
        float x[8], top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = s[nc][e >> 2][e & 3] * to_log2;
        if (seen != ~0u) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = (bits >> e) & 1u ? x[e] : -INFINITY;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, x[e]);
        if (__any(top > m[nc] + kStale)) {   // (the first tile: m is -inf)
          top = fmaxf(top, __shfl_xor(top, 16, 64));
          top = fmaxf(top, __shfl_xor(top, 32, 64));
          const float up = fmaxf(m[nc], ceilf(top)), f = up == m[nc] ? 1.f : __builtin_amdgcn_exp2f(m[nc] - up);
          m[nc] = up;
          l[nc] *= f;
#pragma unroll
          for (int j = 0; j < DT; ++j) acc[nc][j] *= f;
        }
        const float base = m[nc] == -INFINITY ? 0.f : m[nc];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[e] = __builtin_amdgcn_exp2f(x[e] - base);
          l[nc] += x[e];
        }
        u16x2 least[4];
#pragma unroll
        for (int part = 0; part < 3; ++part) {
          u32x4 words;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t two = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, x[2 * i + 1]), __builtin_bit_cast(uint32_t, x[2 * i]), 0x07060302u);
            u16x2 bits2 = __builtin_bit_cast(u16x2, two);   // (of words[i] itself the bit cast would take the vector's first word)
            if (!F8 && part == 0) least[i] = __builtin_elementwise_sub_sat(bits2, u16x2{kLeastPart, kLeastPart});
            if (!F8 && part != 0) bits2 = __builtin_elementwise_max(bits2, least[i]);
            words[i] = __builtin_bit_cast(uint32_t, bits2);
          }
          p_part[nc][part] = __builtin_bit_cast(bf16x8, words);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] -= __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x[e]) & 0xffff0000u);   // (exact)
        }
      }
      // rows that are not seen may hold NaN, which a P of 0 would not silence
      if (seen != ~0u) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int i = 0; i < Tile<D, F8, !DIRECT>::VW; ++i) tile.v[e][i] = (bits >> e) & 1u ? tile.v[e][i] : 0u;
      }
      uint32_t v2[8][DT / 2];   // as bf16: words of two elements
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (F8) {
#pragma unroll
          for (int i = 0; i < DT / 4; ++i) {
            v2[e][2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(tile.v[e][i], 1.0f, false));
            v2[e][2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(tile.v[e][i], 1.0f, true));
          }
        } else {
#pragma unroll
          for (int i = 0; i < DT / 2; ++i) v2[e][i] = tile.v[e][i];
        }
      }
#pragma unroll
      for (int j = 0; j < DT; ++j) {
        u32x4 a;
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = __builtin_amdgcn_perm(v2[2 * i + 1][j / 2], v2[2 * i][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
        const bf16x8 av = __builtin_bit_cast(bf16x8, a);
#pragma unroll
        for (int nc = 0; nc < NC; ++nc) {
#pragma unroll
          for (int part = 0; part < 3; ++part) acc[nc][j] = mfma16(av, p_part[nc][part], acc[nc][j]);
        }
      }
      if (more) load_v(now);
    }

    // The waves' sums against their largest maximum.  Lane (r, g) has of column r the elements DT (4g + v) + j.
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
      l[nc] += __shfl_xor(l[nc], 16, 64);
      l[nc] += __shfl_xor(l[nc], 32, 64);
      if (g == 0) part_ml[wave][16 * nc + r] = float2{m[nc], l[nc]};
    }
    __syncthreads();
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kRowWaves; ++w) top = fmaxf(top, part_ml[w * HEADS + head_wave][16 * nc + r].x);
      const float f = m[nc] == top ? 1.f : __builtin_amdgcn_exp2f(m[nc] - top);
#pragma unroll
      for (int v = 0; v < 4; ++v)
#pragma unroll
        for (int j = 0; j < DT; j += 4)
          *reinterpret_cast<f32x4*>(&part_o[wave][r][DT * (4 * g + v) + j]) =
              f32x4{acc[nc][j][v] * f, acc[nc][j + 1][v] * f, acc[nc][j + 2][v] * f, acc[nc][j + 3][v] * f};
      __syncthreads();
      for (int i = tid; i < HEADS * 16 * (D / 4); i += 64 * kWaves) {
        const int hw = i / (16 * (D / 4)), c = i / (D / 4) % 16, d = i % (D / 4) * 4, column = c0 + 16 * nc + c, head = hk0 + hw;
        if (column >= group) continue;
        float most = -INFINITY, sum = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kRowWaves; ++w) most = fmaxf(most, part_ml[w * HEADS + hw][16 * nc + c].x);
#pragma unroll
        for (int w = 0; w < kRowWaves; ++w) {
          const float2 ml = part_ml[w * HEADS + hw][16 * nc + c];
          sum += ml.y * (ml.x == most ? 1.f : __builtin_amdgcn_exp2f(ml.x - most));
          o += *reinterpret_cast<const f32x4*>(&part_o[w * HEADS + hw][c][d]);
        }
        if (whole) {
          const int32_t h = head * group + column;
          const float over = sum == 0.f ? 0.f : (F8 && p.cache.v_scale ? p.cache.v_scale[head] : 1.f) / sum;
          const int64_t to = b * p.o.sb + h * p.o.sh + d;
          o *= over;
          if (p.o.is_f32) *reinterpret_cast<f32x4*>((float*)p.o.ptr + to) = o;
          else *reinterpret_cast<bf16x4*>((__bf16*)p.o.ptr + to) = bf16x4{(__bf16)o[0], (__bf16)o[1], (__bf16)o[2], (__bf16)o[3]};
          if (d == 0 && p.lse.ptr) p.lse.ptr[b * p.lse.sb + h * p.lse.sh] = sum == 0.f ? -INFINITY : (most + __log2f(sum)) * kLn2;
        } else {
          const int64_t piece = (2 * ((int64_t)share * per_seq + head * blocks + cb) + (first_piece ? 0 : 1)) * ws.columns + 16 * nc + c;
          *reinterpret_cast<f32x4*>(ws.o + piece * D + d) = o;
          if (d == 0) ws.ml[piece] = float2{most, sum};
        }
      }
      __syncthreads();
    }
    if constexpr (DIRECT) break;
    first_piece = false;
    unit += take;
    left -= take;
    at = 0;
    if (left > 0) seq = seq_rows_of(p, ++b, kUnit);
  }
}

// A (sequence, query head) whose rows several work-groups had: their pieces added up.
template <int D, int NC, int THREADS>
__global__ __launch_bounds__(THREADS) void decode_join_kernel(DecodeParams p, DecodeSpace ws, int32_t blocks) {
  constexpr int LANES = D / 4, ROWS = THREADS / LANES;
  __shared__ float top_w[THREADS / 64];
  __shared__ f32x4 part[ROWS][LANES];
  __shared__ float sums[ROWS];
  const int32_t b = (int32_t)blockIdx.x / p.q_heads, h = (int32_t)blockIdx.x - b * p.q_heads, group = p.q_heads / p.kv_heads;
  const int32_t hk = h / group, column = h - hk * group, cb = column / (16 * NC), c = column - cb * 16 * NC;
  const int2 owners = ws.owners[b];
  const int32_t w0 = owners.x, w1 = owners.y >> 1, skip = owners.y & 1;
  if (w0 == w1) return;   // written out by its only owner
  const int32_t per_seq = p.kv_heads * blocks, hb = hk * blocks + cb;
  auto piece = [&](int32_t w) { return (2 * ((int64_t)w * per_seq + hb) + (w == w0 ? skip : 0)) * ws.columns + c; };
  const int lane = threadIdx.x % LANES, row = threadIdx.x / LANES;
  constexpr int U = THREADS > 256 ? 4 : 8;   // pieces under way for a thread; the first ones while the largest maximum is looked for
  f32x4 x[U];
  float2 ml[U];
  auto load = [&](int32_t w) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (w + u * ROWS <= w1) {
        const int64_t at = piece(w + u * ROWS);
        x[u] = *reinterpret_cast<const f32x4*>(ws.o + at * D + 4 * lane);
        ml[u] = ws.ml[at];
      }
    }
  };
  load(w0 + row);
  float top = -INFINITY;
  for (int32_t w = w0 + threadIdx.x; w <= w1; w += THREADS) top = fmaxf(top, ws.ml[piece(w)].x);
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) top = fmaxf(top, __shfl_xor(top, s, 64));
  if ((threadIdx.x & 63) == 0) top_w[threadIdx.x >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < THREADS / 64; ++i) top = fmaxf(top, top_w[i]);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float sum = 0.f;
  for (int32_t w = w0 + row; w <= w1; w += U * ROWS) {
    if (w > w0 + row) load(w);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (w + u * ROWS > w1) continue;
      const float f = ml[u].x == top ? 1.f : __builtin_amdgcn_exp2f(ml[u].x - top);
      sum += ml[u].y * f;
      o += x[u] * f;
    }
  }
  part[row][lane] = o;
  if (lane == 0) sums[row] = sum;
  __syncthreads();
  if (row != 0) return;
#pragma unroll 4
  for (int i = 1; i < ROWS; ++i) {
    o += part[i][lane];
    sum += sums[i];
  }
  o *= sum == 0.f ? 0.f : (p.cache.v_scale ? p.cache.v_scale[hk] : 1.f) / sum;
  const int64_t to = b * p.o.sb + h * p.o.sh + 4 * lane;
  if (p.o.is_f32) *reinterpret_cast<f32x4*>((float*)p.o.ptr + to) = o;
  else *reinterpret_cast<bf16x4*>((__bf16*)p.o.ptr + to) = bf16x4{(__bf16)o[0], (__bf16)o[1], (__bf16)o[2], (__bf16)o[3]};
  if (lane == 0 && p.lse.ptr) p.lse.ptr[b * p.lse.sb + h * p.lse.sh] = sum == 0.f ? -INFINITY : (top + __log2f(sum)) * kLn2;
}

// Heads whose rows a work-group takes together: several where they lie side by side and there are four units of 128 rows and more for each
// work-group, by the bound.  32 sequences of 16384 rows, 8 heads in e4m3: 223 us one by one, 204 in fours; 16 in bf16: 206 and 188 in
// twos; 16 heads of 64: 209 and 186 in fours.  A work-group has a piece for each of them, so short ones lose: one sequence, 8 heads of 128 in
// bf16, 8192 rows 19.7 and 22.2, 32768 rows 38.5 and 38.6, 65536 rows 62 and 60.
static int heads_together(const DecodeParams& p) {
  const int side = heads_side_by_side(p.head_dim, p.cache.is_f8 != 0);
  const int64_t most = (int64_t)p.batch * p.kv_heads * ((p.max_rows + 127) / 128);
  const int waves = waves_per_simd(p.head_dim, p.cache.is_f8 != 0, columns_of(p.q_heads / p.kv_heads) / 16);
  return p.kv_heads % side == 0 && p.cache.s_head == p.head_dim && most >= 4ll * kCus * waves ? side : 1;
}

void decode_plan(const DecodeParams& p, int32_t out[3]) {
  const int heads = heads_together(p);
  const DecodeShape s = decode_shape(p.batch, p.q_heads, p.kv_heads, p.head_dim, p.max_rows, p.cache.is_f8 != 0, heads);
  out[0] = s.shares;
  out[1] = s.direct ? 1 : heads;
  out[2] = s.direct;
}

template <int D, bool F8, int NC, bool PAGES16>
static hipError_t launch(const DecodeParams& p, hipStream_t stream) {
  constexpr int kSide = heads_side_by_side(D, F8);
  const int heads = heads_together(p);
  const DecodeShape s = decode_shape(p.batch, p.q_heads, p.kv_heads, D, p.max_rows, F8, heads);
  const dim3 grid((uint32_t)((int64_t)s.shares * p.kv_heads * s.blocks / (s.direct ? 1 : heads)));
  if (s.direct) {
    hipLaunchKernelGGL((decode_kernel<D, F8, NC, PAGES16, true, 1>), grid, dim3(64 * kDirectWaves), 0, stream, p, DecodeSpace{}, s.blocks, s.shares);
    return hipGetLastError();
  }
  const DecodeSpace ws = space_of(s, p.workspace);
  if (heads > 1) hipLaunchKernelGGL((decode_kernel<D, F8, NC, PAGES16, false, kSide>), grid, dim3(64 * kDealtWaves), 0, stream, p, ws, s.blocks, s.shares);
  else hipLaunchKernelGGL((decode_kernel<D, F8, NC, PAGES16, false, 1>), grid, dim3(64 * kDealtWaves), 0, stream, p, ws, s.blocks, s.shares);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // Threads for the pieces of a sequence: a share or two where there are as many sequences as shares, all of them where there is one.  A wave takes
  // 16 pieces (heads of 128) at once.  64 sequences, 64 shares: 69 us with 256 threads, 65.5 with 64; one sequence of one head, 512 shares:
  // the join alone 12 us with 256, 8 with 1024.
  const dim3 joins((uint32_t)(p.batch * p.q_heads));
  if (s.shares > 64 * p.batch) hipLaunchKernelGGL((decode_join_kernel<D, NC, 1024>), joins, dim3(1024), 0, stream, p, ws, s.blocks);
  else if (s.shares > 16 * p.batch) hipLaunchKernelGGL((decode_join_kernel<D, NC, 256>), joins, dim3(256), 0, stream, p, ws, s.blocks);
  else hipLaunchKernelGGL((decode_join_kernel<D, NC, 64>), joins, dim3(64), 0, stream, p, ws, s.blocks);
  return hipGetLastError();
}

template <int D, bool F8>
static hipError_t launch(const DecodeParams& p, hipStream_t stream) {
  const bool wide = columns_of(p.q_heads / p.kv_heads) == 32;
  if (p.cache.page_rows % 16 == 0) return wide ? launch<D, F8, 2, true>(p, stream) : launch<D, F8, 1, true>(p, stream);
  return wide ? launch<D, F8, 2, false>(p, stream) : launch<D, F8, 1, false>(p, stream);
}

template <int D>
static hipError_t launch(const DecodeParams& p, hipStream_t stream) {
  return p.cache.is_f8 ? launch<D, true>(p, stream) : launch<D, false>(p, stream);
}

hipError_t launch_decode(const DecodeParams& p, hipStream_t stream) {
  return p.head_dim == 128 ? launch<128>(p, stream) : launch<64>(p, stream);
}

}  // namespace burst
