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
//   The running maximum of a column is a whole number (base 2), so that a rescale by 2^n changes no bit of P and O, and which
//   rows another wave or work-group took has no influence but the order of fp32 sums.  P goes in whole, as the three bf16 numbers that its
//   24 bits are; the matrix pipe has the time for it.
//
//   Work is cut into units of 128 rows (a tile for each wave), numbered over (sequence, key head, rows), and dealt evenly to as many
//   work-groups as the chip holds at once, whatever the sequences' lengths are: each finds its first unit by a scan over
//   the sequences.  A piece that is a whole (sequence, key head) is written out; what a work-group has of others goes to the workspace,
//   two pieces at most, and decode_join_kernel adds the pieces up in a fixed order.
#include "cache.hpp"
#include "kernels.hpp"
#include "mfma16.hpp"

namespace burst {

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

constexpr int kWaves = 4, kTileRows = 32, kUnitRows = kWaves * kTileRows;
constexpr float kStale = 8.f;   // a maximum may fall behind by a factor of 2^8: P, O and their sums stay far inside fp32
constexpr int kCus = 256;
// Work-groups that share a CU, by the registers that a wave takes.
constexpr int groups_per_cu(int head_dim, bool f8, int nc) { return nc == 2 ? 2 : head_dim == 64 ? 4 : f8 ? 3 : 2; }

// What a sequence's share of the work is.  It starts at a multiple of the tile, so that the halves of a tile lie in one page each where
// pages are multiples of 16 rows; a sequence without rows has one unit, which writes its empty result.
struct SeqRows {
  int32_t lo, hi, start, units;
};
__device__ __forceinline__ SeqRows seq_rows(const DecodeParams& p, int32_t n, int32_t first) {
  SeqRows s;
  const int32_t most = p.max_rows;   // (at most table_cols * page_rows, checked on the host)
  s.hi = n < 0 ? 0 : n > most ? most : n;
  s.lo = first < 0 ? 0 : first < s.hi ? first : s.hi;
  s.start = s.lo & ~(kTileRows - 1);
  s.units = s.lo < s.hi ? (s.hi - s.start + kUnitRows - 1) / kUnitRows : 1;
  return s;
}
__device__ __forceinline__ SeqRows seq_rows_of(const DecodeParams& p, int32_t b) {
  return seq_rows(p, p.cache.rows[b], p.first_row ? p.first_row[b] : 0);
}

// Units dealt to `groups` work-groups: the first `more` of them get one more.
struct Deal {
  int64_t each, more;
  __device__ __forceinline__ void init(int64_t units, int32_t groups) {
    each = units >> 32 ? units / groups : (int64_t)((uint32_t)units / (uint32_t)groups);
    more = units - each * groups;
  }
  __device__ __forceinline__ int64_t first(int32_t w) const { return w * each + (w < more ? w : more); }
  __device__ __forceinline__ int32_t owner(int64_t unit) const {
    const int64_t longer = more * (each + 1);
    const int64_t x = unit < longer ? unit : unit - longer, y = unit < longer ? each + 1 : each;
    const int64_t n = (x | y) >> 32 ? x / y : (int64_t)((uint32_t)x / (uint32_t)y);
    return (int32_t)(unit < longer ? n : more + n);
  }
};

// The workspace: units of all, units before each sequence, and two pieces for every work-group, each (maximum, sum) and O of its
// columns relative to that maximum.
struct DecodeSpace {
  int64_t* units;
  int64_t* before;
  float2* ml;
  float* o;
  int32_t columns;   // of a piece: min(group, 16 NC)
};

struct DecodeShape {
  int32_t blocks, groups;   // blocks of columns of a key head, work-groups
  int32_t columns, max_units;
  int64_t off_before, off_ml, off_o, bytes;
};
static int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }
static int columns_of(int32_t group) { return group <= 16 ? 16 : 32; }
static DecodeShape decode_shape(int32_t batch, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int64_t max_rows, bool f8) {
  DecodeShape s;
  const int32_t group = q_heads / kv_heads, wide = columns_of(group);
  s.blocks = (group + wide - 1) / wide;
  s.columns = group < wide ? group : wide;
  s.max_units = (int32_t)std::max<int64_t>(1, (max_rows + kUnitRows - 1) / kUnitRows);
  const int64_t most = (int64_t)batch * kv_heads * s.blocks * s.max_units;
  s.groups = (int32_t)std::min<int64_t>(most, kCus * groups_per_cu(head_dim, f8, wide / 16));
  s.off_before = 256;
  s.off_ml = s.off_before + up256((int64_t)batch * 8);
  s.off_o = s.off_ml + up256((int64_t)s.groups * 2 * s.columns * 8);
  s.bytes = s.max_units == 1 ? 0 : s.off_o + (int64_t)s.groups * 2 * s.columns * head_dim * 4;   // (a single unit is never shared)
  return s;
}
int64_t decode_workspace_bytes(int32_t batch, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int64_t max_rows) {
  return std::max(decode_shape(batch, q_heads, kv_heads, head_dim, max_rows, false).bytes,
                  decode_shape(batch, q_heads, kv_heads, head_dim, max_rows, true).bytes);
}
static DecodeSpace space_of(const DecodeShape& s, void* workspace) {
  char* ws = (char*)workspace;
  return DecodeSpace{(int64_t*)ws, (int64_t*)(ws + s.off_before), (float2*)(ws + s.off_ml), (float*)(ws + s.off_o), s.columns};
}

// 8 numbers of e4m3 (two words) as a bf16 operand.
__device__ __forceinline__ bf16x8 widened(uint32_t w0, uint32_t w1) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.0f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.0f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A tile's keys and values in a wave's registers.
template <int D, bool F8>
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
    for (int i = 0; i < KW; ++i) k[t][i] = *reinterpret_cast<const u32x4*>(row + 64 * i);
  }
  __device__ __forceinline__ void load_v(int e, const char* row) {   // of this lane: key e, elements D / 16 r ..
    if constexpr (VW == 4) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(row);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[e][i] = x[i];
    } else if constexpr (VW == 2) {
      const u32x2 x = *reinterpret_cast<const u32x2*>(row);
      v[e][0] = x[0];
      v[e][1] = x[1];
    } else {
      v[e][0] = *reinterpret_cast<const uint32_t*>(row);
    }
  }
};

// Where a tile's rows lie, and which of them are seen (a bit for each).
struct TilePlace {
  uint32_t seen;
  const char* half_k[2];   // pages of a multiple of 16 rows: first row of each half
  const char* half_v[2];
  int64_t row;             // any pages: bytes to this lane's row (lane % 32)
};

template <int D, bool F8, int NC, bool PAGES16>
__global__ __launch_bounds__(256, groups_per_cu(D, F8, NC)) void decode_kernel(DecodeParams p, DecodeSpace ws, int32_t blocks, int32_t groups) {
  constexpr int KK = D / 32, DT = D / 16, kBytes = F8 ? 1 : 2;
  __shared__ float part_o[kWaves][16][D + 4];
  __shared__ float2 part_ml[kWaves][NC * 16];
  __shared__ int64_t scan[kWaves + 2];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 15, g = lane >> 4;
  const int32_t group = p.q_heads / p.kv_heads, per_seq = p.kv_heads * blocks;

  // All units, and the sequence that holds this work-group's first one.
  int64_t total = 0;
  int32_t mine = 0;
  for (int32_t b0 = 0; b0 < p.batch; b0 += 256) {
    mine = b0 + tid < p.batch ? seq_rows_of(p, b0 + tid).units : 0;
    int32_t sum = mine;   // (at most 2^23 units a sequence, 64 of them)
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x, 64);
    if (lane == 0) scan[wave] = sum;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) total += scan[w];
    __syncthreads();
  }
  Deal deal;
  deal.init(total * per_seq, groups);
  int64_t unit = deal.first(blockIdx.x), left = deal.first(blockIdx.x + 1) - unit;
  if (left == 0) return;
  int64_t passed = 0;
  for (int32_t b0 = 0; b0 < p.batch; b0 += 256) {
    if (p.batch > 256) mine = b0 + tid < p.batch ? seq_rows_of(p, b0 + tid).units : 0;
    int32_t upto = mine;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
      const int32_t y = __shfl_up(upto, x, 64);
      upto += lane >= x ? y : 0;
    }
    if (lane == 63) scan[wave] = upto;
    __syncthreads();
    int64_t before = passed;
    for (int w = 0; w < kWaves; ++w) {
      before += w < wave ? scan[w] : 0;
      passed += scan[w];
    }
    const int64_t end = before + upto, begin = end - mine;
    if (begin * per_seq <= unit && unit < end * per_seq) {   // (one thread: a sequence without units is none of the batch)
      scan[kWaves] = begin;
      scan[kWaves + 1] = b0 + tid;
    }
    __syncthreads();
    if (passed * per_seq > unit) break;
  }
  int64_t before = scan[kWaves];
  int32_t b = __builtin_amdgcn_readfirstlane((int32_t)scan[kWaves + 1]);
  if (ws.units && blockIdx.x == 0 && tid == 0) *ws.units = total;

  SeqRows seq = seq_rows_of(p, b);
  int64_t in_seq = unit - before * per_seq;
  int32_t hb = __builtin_amdgcn_readfirstlane((int32_t)(in_seq / seq.units));
  int32_t at = __builtin_amdgcn_readfirstlane((int32_t)(in_seq - (int64_t)hb * seq.units));

  const uint32_t row_bytes = (uint32_t)p.cache.s_row * kBytes;
  const uint32_t k_lane = r * row_bytes + 16 * g, v_lane = 4 * g * row_bytes + DT * kBytes * r;
  bool first_piece = true;

  while (left > 0) {
    const int32_t take = (int32_t)(left < seq.units - at ? left : seq.units - at);
    const int32_t hk = hb / blocks, c0 = (hb - hk * blocks) * 16 * NC;   // first of the block's columns in its group
    const bool whole = at == 0 && take == seq.units;
    if (ws.units && hb == 0 && at == 0 && tid == 0) ws.before[b] = before;

    bf16x8 q[NC][KK];
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
      const int32_t c = c0 + 16 * nc + r;
      const __bf16* row = (const __bf16*)p.q.ptr + b * p.q.sb + (int64_t)(hk * group + c) * p.q.sh;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
        q[nc][kk] = c < group ? *reinterpret_cast<const bf16x8*>(row + Tile<D, F8>::q_element(g, kk)) : bf16x8{};
    }
    const float to_log2 = p.scale * kLog2e * (F8 && p.cache.k_scale ? p.cache.k_scale[hk] : 1.f);
    const char* k_base = (const char*)p.cache.k + hk * p.cache.s_head * kBytes;
    const char* v_base = (const char*)p.cache.v + hk * p.cache.s_head * kBytes;
    const int32_t* table = p.cache.table + b * p.cache.table_stride;

    float m[NC], l[NC];
    f32x4 acc[NC][DT];
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
      m[nc] = -INFINITY;
      l[nc] = 0.f;
#pragma unroll
      for (int j = 0; j < DT; ++j) acc[nc][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // this wave's tiles: every fourth from t0 on, below t1
    const int32_t t1 = seq.units == at + take ? seq.hi : seq.start + (at + take) * kUnitRows;
    int32_t t = seq.start + at * kUnitRows + wave * kTileRows;

    auto page_of = [&](int32_t row) -> int32_t {   // (the whole wave's row)
      if (row >= seq.hi) return -1;
      const int32_t page = table[p.cache.by_page.quotient(row)];
      return __builtin_amdgcn_readfirstlane(page >= 0 && page < p.cache.n_pages ? page : -1);
    };
    auto place = [&](int32_t row0, const int32_t (&page)[2], TilePlace& x) {
      // rows of the tile that the sequence has
      const int32_t below = seq.hi - row0, above = seq.lo - row0;
      uint32_t seen = below >= 32 ? ~0u : (1u << below) - 1u;
      if (above > 0) seen &= ~0u << above;   // (start is at most 31 before lo)
      if constexpr (PAGES16) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          int64_t off = 0;   // a half without a page: any rows that are there, unseen
          if (page[h] >= 0) {
            const int32_t row = row0 + 16 * h, in_page = row - p.cache.by_page.quotient(row) * p.cache.page_rows;
            off = (page[h] * p.cache.s_page + in_page * p.cache.s_row) * kBytes;
          } else {
            seen &= h ? 0x0000ffffu : 0xffff0000u;
          }
          x.half_k[h] = k_base + off;
          x.half_v[h] = v_base + off;
        }
        x.seen = seen;
      } else {
        const int32_t row = row0 + (lane & 31);
        int64_t off = -1;
        if (row < seq.hi) off = p.cache.row_offset(b, row);
        x.seen = seen & (uint32_t)__ballot(off >= 0);
        x.row = off >= 0 ? off * kBytes : 0;
      }
    };
    Tile<D, F8> tile;
    auto load_k = [&](const TilePlace& x) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if constexpr (PAGES16) tile.load_k(h, x.half_k[h] + k_lane);
        else tile.load_k(h, k_base + __shfl(x.row, 16 * h + r, 64) + 16 * g);
      }
    };
    auto load_v = [&](const TilePlace& x) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (PAGES16) tile.load_v(e, x.half_v[e >> 2] + (v_lane + (e & 3) * row_bytes));
        else tile.load_v(e, v_base + __shfl(x.row, 16 * (e >> 2) + 4 * g + (e & 3), 64) + DT * kBytes * r);
      }
    };

    int32_t page[2] = {-1, -1};
    TilePlace now;
    if (t < t1) {
      if constexpr (PAGES16) {
        page[0] = page_of(t);
        page[1] = page_of(t + 16);
      }
      place(t, page, now);
      load_k(now);
      load_v(now);
      if constexpr (PAGES16) {
        page[0] = page_of(t + kUnitRows);
        page[1] = page_of(t + kUnitRows + 16);
      }
    }
    for (; t < t1; t += kUnitRows) {
      const bool more = t + kUnitRows < t1;
      f32x4 s[NC][2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          const bf16x8 a = tile.k_operand(h, kk);
#pragma unroll
          for (int nc = 0; nc < NC; ++nc) s[nc][h] = mfma16(a, q[nc][kk], kk == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[nc][h]);
        }
      const uint32_t seen = now.seen;
      if (more) {
        place(t + kUnitRows, page, now);
        load_k(now);
        if constexpr (PAGES16) {
          page[0] = page_of(t + 2 * kUnitRows);
          page[1] = page_of(t + 2 * kUnitRows + 16);
        }
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
#pragma unroll
        for (int part = 0; part < 3; ++part) {
          u32x4 words;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            words[i] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, x[2 * i + 1]), __builtin_bit_cast(uint32_t, x[2 * i]), 0x07060302u);
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
          for (int i = 0; i < Tile<D, F8>::VW; ++i) tile.v[e][i] = (bits >> e) & 1u ? tile.v[e][i] : 0u;
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

    // The four waves' sums against their largest maximum.  Lane (r, g) has of column r the elements DT (4g + v) + j.
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
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, part_ml[w][16 * nc + r].x);
      const float f = m[nc] == top ? 1.f : __builtin_amdgcn_exp2f(m[nc] - top);
#pragma unroll
      for (int v = 0; v < 4; ++v)
#pragma unroll
        for (int j = 0; j < DT; j += 4)
          *reinterpret_cast<f32x4*>(&part_o[wave][r][DT * (4 * g + v) + j]) =
              f32x4{acc[nc][j][v] * f, acc[nc][j + 1][v] * f, acc[nc][j + 2][v] * f, acc[nc][j + 3][v] * f};
      __syncthreads();
      for (int i = tid; i < 16 * (D / 4); i += 256) {
        const int c = i / (D / 4), d = i % (D / 4) * 4, column = c0 + 16 * nc + c;
        if (column >= group) continue;
        float most = -INFINITY, sum = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) most = fmaxf(most, part_ml[w][16 * nc + c].x);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float2 ml = part_ml[w][16 * nc + c];
          sum += ml.y * (ml.x == most ? 1.f : __builtin_amdgcn_exp2f(ml.x - most));
          o += *reinterpret_cast<const f32x4*>(&part_o[w][c][d]);
        }
        if (whole) {
          const int32_t h = hk * group + column;
          const float over = sum == 0.f ? 0.f : (F8 && p.cache.v_scale ? p.cache.v_scale[hk] : 1.f) / sum;
          const int64_t to = b * p.o.sb + h * p.o.sh + d;
          o *= over;
          if (p.o.is_f32) *reinterpret_cast<f32x4*>((float*)p.o.ptr + to) = o;
          else *reinterpret_cast<bf16x4*>((__bf16*)p.o.ptr + to) = bf16x4{(__bf16)o[0], (__bf16)o[1], (__bf16)o[2], (__bf16)o[3]};
          if (d == 0 && p.lse.ptr) p.lse.ptr[b * p.lse.sb + h * p.lse.sh] = sum == 0.f ? -INFINITY : (most + __log2f(sum)) * kLn2;
        } else {
          const int64_t piece = (int64_t)(2 * blockIdx.x + (first_piece ? 0 : 1)) * ws.columns + 16 * nc + c;
          *reinterpret_cast<f32x4*>(ws.o + piece * D + d) = o;
          if (d == 0) ws.ml[piece] = float2{most, sum};
        }
      }
      __syncthreads();
    }
    first_piece = false;
    left -= take;
    at = 0;
    if (left > 0 && ++hb == per_seq) {
      hb = 0;
      before += seq.units;
      seq = seq_rows_of(p, ++b);
    }
  }
}

// A (sequence, query head) whose rows several work-groups had: their pieces added up.
template <int D, int NC>
__global__ __launch_bounds__(256) void decode_join_kernel(DecodeParams p, DecodeSpace ws, int32_t blocks, int32_t groups, int32_t f8) {
  constexpr int LANES = D / 4, ROWS = 256 / LANES;
  __shared__ float top_w[4];
  __shared__ f32x4 part[ROWS][LANES];
  __shared__ float sums[ROWS];
  const int32_t b = blockIdx.x / p.q_heads, h = blockIdx.x - b * p.q_heads, group = p.q_heads / p.kv_heads;
  const int32_t hk = h / group, column = h - hk * group, cb = column / (16 * NC), c = column - cb * 16 * NC;
  const int32_t per_seq = p.kv_heads * blocks, units = seq_rows_of(p, b).units;
  Deal deal;
  deal.init(*ws.units * per_seq, groups);
  const int64_t unit = ws.before[b] * per_seq + (int64_t)(hk * blocks + cb) * units;
  const int32_t w0 = deal.owner(unit), w1 = deal.owner(unit + units - 1);
  if (w0 == w1) return;   // written out by its only owner
  const int32_t skip = deal.first(w0) < unit ? 1 : 0;   // the first owner has something else before it
  auto piece = [&](int32_t w) { return (int64_t)(2 * w + (w == w0 ? skip : 0)) * ws.columns + c; };
  float top = -INFINITY;
  for (int32_t w = w0 + threadIdx.x; w <= w1; w += 256) top = fmaxf(top, ws.ml[piece(w)].x);
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
  if ((threadIdx.x & 63) == 0) top_w[threadIdx.x >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(top_w[0], top_w[1]), fmaxf(top_w[2], top_w[3]));
  const int lane = threadIdx.x % LANES, row = threadIdx.x / LANES;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float sum = 0.f;
  for (int32_t w = w0 + row; w <= w1; w += ROWS) {
    const float2 ml = ws.ml[piece(w)];
    const float f = ml.x == top ? 1.f : __builtin_amdgcn_exp2f(ml.x - top);
    sum += ml.y * f;
    o += *reinterpret_cast<const f32x4*>(ws.o + piece(w) * D + 4 * lane) * f;
  }
  part[row][lane] = o;
  if (lane == 0) sums[row] = sum;
  __syncthreads();
  if (row != 0) return;
  for (int i = 1; i < ROWS; ++i) {
    o += part[i][lane];
    sum += sums[i];
  }
  o *= sum == 0.f ? 0.f : (f8 && p.cache.v_scale ? p.cache.v_scale[hk] : 1.f) / sum;
  const int64_t to = b * p.o.sb + h * p.o.sh + 4 * lane;
  if (p.o.is_f32) *reinterpret_cast<f32x4*>((float*)p.o.ptr + to) = o;
  else *reinterpret_cast<bf16x4*>((__bf16*)p.o.ptr + to) = bf16x4{(__bf16)o[0], (__bf16)o[1], (__bf16)o[2], (__bf16)o[3]};
  if (lane == 0 && p.lse.ptr) p.lse.ptr[b * p.lse.sb + h * p.lse.sh] = sum == 0.f ? -INFINITY : (top + __log2f(sum)) * kLn2;
}

template <int D, int NC>
static hipError_t launch(const DecodeParams& p, hipStream_t stream) {
  const DecodeShape s = decode_shape(p.batch, p.q_heads, p.kv_heads, D, p.max_rows, p.cache.is_f8 != 0);
  DecodeSpace ws = {};
  if (s.bytes > 0) ws = space_of(s, p.workspace);
  const dim3 grid(s.groups), block(256);
  const bool pages16 = p.cache.page_rows % 16 == 0;
  if (p.cache.is_f8) {
    if (pages16) hipLaunchKernelGGL((decode_kernel<D, true, NC, true>), grid, block, 0, stream, p, ws, s.blocks, s.groups);
    else hipLaunchKernelGGL((decode_kernel<D, true, NC, false>), grid, block, 0, stream, p, ws, s.blocks, s.groups);
  } else {
    if (pages16) hipLaunchKernelGGL((decode_kernel<D, false, NC, true>), grid, block, 0, stream, p, ws, s.blocks, s.groups);
    else hipLaunchKernelGGL((decode_kernel<D, false, NC, false>), grid, block, 0, stream, p, ws, s.blocks, s.groups);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || s.max_units == 1) return e;
  hipLaunchKernelGGL((decode_join_kernel<D, NC>), dim3((uint32_t)(p.batch * p.q_heads)), block, 0, stream, p, ws, s.blocks, s.groups,
                     p.cache.is_f8);
  return hipGetLastError();
}

hipError_t launch_decode(const DecodeParams& p, hipStream_t stream) {
  const bool wide = columns_of(p.q_heads / p.kv_heads) == 32;
  if (p.head_dim == 128) return wide ? launch<128, 2>(p, stream) : launch<128, 1>(p, stream);
  return wide ? launch<64, 2>(p, stream) : launch<64, 1>(p, stream);
}

}  // namespace burst
