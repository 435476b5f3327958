// Attention of a few new tokens of every sequence, a chain or a tree of drafts, over its rows in a paged cache.
//
// The new tokens times the query heads that share a key head are the columns of two products: S^T = K Q^T and O^T = V^T P^T, so a row of the
// cache that is read once serves them all.  Up to 32 columns (tree_few.hip) the cache's bytes bound it, more of them (here) the products and the exponentials.
// A work-group of four waves takes 64 or 128 columns; tiles of 64 rows of K and V come into LDS by direct loads, where their addresses go by the page table, and
// each wave multiplies them for 32 columns (all 64 rows for 128 columns of the work-group, half of them for 64, whose halves are added up at the end).
//   Which rows a column sees is a 64-bit word for each tile: older rows from its first one on and the first rows of all, both intervals, and the
// new tokens' rows by the bits of its word, moved to where they stand in the tile.  A tile of which every column of a wave sees all rows does not
// look at them.
//   The running maximum is a whole number (base 2), so that a rescale changes no bit of P and O.  P goes in as the three bf16 numbers that its 24 bits are; with more
// than 32 columns and O in bf16 as two, which hold it to 2^-16: far below the 2^-8 that the cast of O rounds, so that one token more, which may bring a sequence here from
// tree_few.hip, changes no result by more than that.  (4 x 32768 rows, 512 columns, head_dim 128: three parts 486 us in bf16 and 460 in e4m3, two 398 and 381; one, which is off by
// 2^-9 of each number, 298 and 289.)
//
// Work is cut into units of a tile and numbered over (sequence, tiles that some of its tokens see): a window leaves the tiles out that lie between the
// first rows and its own.  The units are dealt evenly to shares, a work-group each for every key head and block of columns; a piece that is
// a whole sequence is written out, others go to the workspace and tree_join_kernel adds them up in a fixed order.
//
// Measured, with the join: 4 sequences of 32768 rows, 64 tokens, 64 query heads over 8 (512 columns, bf16) 391-404 us, three products executed for two at 1020-1050 TFLOP/s, matrix pipe 50 % busy,
// vector unit 53 %.  Scalar work on
// masks and pages is kept out of the tiles (looked up tile by tile it took 8 % more).  Two teams of waves that take products and exponentials in turn gave nothing where each team brought tiles of its
// own, nor did 256 columns a work-group (both with P in one part); teams over one set of tiles, as in a step of the ring, were not tried.  16 sequences of up to 4096 rows, 12 tokens, 32 over 8 heads: 25 us and a join of 6.5; 32 of up to 49152, a
// window of 16384, 8 tokens, 64 over 8 heads, e4m3 165 us, 4.7 TB/s.
#include "tree.hpp"

namespace burst {

namespace {

constexpr int kTreeRows = 64;      // rows of a tile
constexpr int kTreeWaves = 4;      // of a work-group, two of which share a CU
constexpr int tree_slots(int head_dim, bool f8) { return (1 << 16) / (2 * kTreeRows * head_dim * (f8 ? 1 : 2)); }   // 64 KiB

// CW: waves side by side, of 32 columns each; the other way they share a tile's rows.
template <int D, bool F8, bool PAGES16, int CW, int PARTS>
__global__ __launch_bounds__(64 * kTreeWaves, 2) void tree_kernel(TreeParams, TreeSpace ws, int32_t blocks, int32_t shares, int32_t direct) {
  constexpr int RW = kTreeWaves / CW, CH = RW == 1 && PARTS <= 2 ? 2 : 1, PASSES = 2 / RW / CH;
  using Columns = TreeColumns<D, F8, 2, PARTS, D == 128 && !F8 && !PAGES16 ? 2 : 4, CH>;   // (registers)
  using Run = TreeRun<D, F8, PAGES16, 1>;
  using Operands = TreeOperands<D, F8>;
  constexpr int NB = 2, DB = Columns::DB, HALF = Operands::TILE, TILE = 2 * HALF, COLS = 32 * CW;
  constexpr int SLOTS = tree_slots(D, F8), LOADS = 2 * Run::NI * (SLOTS - 2);   // tiles in LDS; loads that may be under way when one is there
  extern __shared__ __attribute__((aligned(1024))) char smem[];   // [SLOTS][K tile, V tile], the rows that are there [SLOTS][4 runs], maxima and sums
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_bytes)smem;
  // (through the address space: a volatile access by a generic pointer is a flat one, which waits for all loads under way)
  typedef volatile __attribute__((address_space(3))) uint16_t* lds_u16;
  typedef volatile __attribute__((address_space(3))) uint64_t* lds_u64;
  const lds_bytes there_lds = (lds_bytes)smem + SLOTS * 2 * TILE;
  float2* const ml_lds = (float2*)(smem + SLOTS * 2 * TILE + SLOTS * 8);
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 15, g = lane >> 4;
  const int cw = wave % CW, rw = wave / CW;
  const TreeParams& sizes = args_here();
  const int32_t kv_heads = sizes.kv_heads, group = sizes.q_heads / kv_heads;

  // Blocks of columns of one (share, key head) read the same rows: they are work-groups of one XCD, as near each other as can be.
  const int32_t of8 = (int32_t)((uint32_t)blockIdx.x / (uint32_t)(8 * blocks)), in8 = (int32_t)blockIdx.x - of8 * 8 * blocks, cb = in8 >> 3, sh = 8 * of8 + (in8 & 7);
  const int32_t share = (int32_t)((uint32_t)sh / (uint32_t)kv_heads), hk = sh - share * kv_heads, c0 = cb * COLS;
  if (share >= shares) return;

  TreeWalk<kTreeRows> walk;
  if (!walk.init(args_here(), share, shares, direct != 0, lane)) return;
  Operands ops;
  ops.init(lane);
  do {
    walk.begin(direct != 0, hk == 0 && cb == 0 && tid == 0, ws, share);
    const int32_t b = walk.b, columns = walk.seq.tokens * group;
    if (walk.take <= 0 || c0 >= columns) continue;
    const bool live = c0 + 32 * cw < columns;   // this wave has columns
    Columns x;
    x.init(args_here(), walk.seq, b, hk, group, c0 + 32 * cw, lane);
    TreeUnion some;
    some.init(args_here(), walk.seq, b, lane);
    Run run;
    run.init(args_here().cache, b, hk, walk.seq.hi, wave & 1, lane);

    // A wave brings 16 rows of a tile, SLOTS - 1 tiles before it is multiplied
    const bool once = blocks == 1 && direct == 0;   // lines are not kept where rows are many and no other work-group reads them
    typename Run::Pages pages;
    const int32_t end = walk.at + walk.take;
    uint32_t there[SLOTS];   // of the tiles under way: this wave's rows; all rows (PAGES16: each wave looks at all pages; else the waves tell each other)
    uint64_t rows_of[SLOTS];
    auto look_up = [&](int32_t u) { run.look_up([&](int32_t v) { return walk.row_of(v) + 16 * wave; }, u, walk.at, end, wave, lane, pages); };
    auto ask = [&](int32_t u, int slot, uint64_t& rows) {
      const int32_t row0 = walk.row_of(u);
      rows = some.rows(row0);
      if constexpr (PAGES16) rows &= run.with_page(pages, u);
      typename Run::Place place;
      run.place(row0 + 16 * wave, (uint32_t)(rows >> (16 * wave)) & 0xffffu, lane, pages, u, 0, place);
      const uint32_t kt = lds0 + slot * 2 * TILE + wave * Run::BYTES;
      run.template bring<false>(place, 0, kt, once);
      run.template bring<true>(place, 0, kt + TILE, once);
      if (!PAGES16 && lane == 0) ((lds_u16)there_lds)[slot * 4 + wave] = (uint16_t)place.there;
      return place.there;
    };
    look_up(walk.at);
#pragma unroll
    for (int i = 0; i + 1 < SLOTS; ++i) {
      there[i] = 0xffffu;
      if (walk.at + i < end) {
        there[i] = ask(walk.at + i, i, rows_of[i]);
        if (walk.at + i + 1 < end) look_up(walk.at + i + 1);
      }
    }
    int slot = 0;
    for (int32_t u = walk.at; u < end; ++u) {
      const int next_slot = (slot + SLOTS - 1) & (SLOTS - 1);
      if (u + SLOTS - 2 < end) wait_loads<LOADS>();
      else wait_loads<0>();
      char* const tile = smem + slot * 2 * TILE;
      Run::clear(tile + TILE + wave * Run::BYTES, there[0], lane);
      lds_barrier();            // the tile is there, and all waves have left the one before
      uint64_t rows_there = rows_of[0];
      if constexpr (!PAGES16) rows_there = uniform(((lds_u64)there_lds)[slot]);
#pragma unroll
      for (int i = 0; i + 2 < SLOTS; ++i) {
        there[i] = there[i + 1];
        rows_of[i] = rows_of[i + 1];
      }
      if (u + SLOTS - 1 < end) {
        there[SLOTS - 2] = ask(u + SLOTS - 1, next_slot, rows_of[SLOTS - 2]);
        if (u + SLOTS < end) look_up(u + SLOTS);
      }
      if (live) {
        const uint32_t kt = lds0 + slot * 2 * TILE;
        const int32_t t0 = walk.row_of(u);
#pragma clang loop unroll(disable)
        for (int i = 0; i < PASSES; ++i) {   // (with P in three parts the scores and P of 64 rows do not fit in the registers beside the sums)
          const int half = RW == 2 ? rw : i;
          x.scores(kt + half * HALF, ops);
          x.weights(t0 + 32 * half, rows_there >> (32 * half) & low_bits(32 * CH), g);
          x.add(kt + TILE + half * HALF, ops);
        }
      }
      slot = (slot + 1) & (SLOTS - 1);
    }
    x.finish();

    // Lane (r, g) has of column r elements 16 db + 4g ..  The halves of 64 columns' rows against the larger maximum of both.
    __syncthreads();
    if constexpr (RW == 2) {
      f32x4* const sums = reinterpret_cast<f32x4*>(smem) + cw * (DB * NB * 64) + lane;
      if (rw == 1) {
#pragma unroll
        for (int i = 0; i < DB * NB; ++i) sums[64 * i] = x.acc[i / NB][i % NB];
        if (g == 0) {
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) ml_lds[32 * cw + 16 * nb + r] = float2{x.m[nb], x.l[nb]};
        }
      }
      __syncthreads();
      if (rw == 0) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const float2 other = ml_lds[32 * cw + 16 * nb + r];
          const float top = fmaxf(x.m[nb], other.x);
          const float f0 = x.m[nb] == top ? 1.f : __builtin_amdgcn_exp2f(x.m[nb] - top), f1 = other.x == top ? 1.f : __builtin_amdgcn_exp2f(other.x - top);
          x.m[nb] = top;
          x.l[nb] = x.l[nb] * f0 + other.y * f1;
#pragma unroll
          for (int db = 0; db < DB; ++db) x.acc[db][nb] = x.acc[db][nb] * f0 + sums[64 * (db * NB + nb)] * f1;
        }
      }
      __syncthreads();
    }
    if (rw == 0) {
      const TreeParams& p = args_here();
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int32_t in = 32 * cw + 16 * nb + r, c = c0 + in;
        if (c >= columns) continue;
        if (walk.whole) {
#pragma unroll
          for (int db = 0; db < DB; ++db) tree_write<F8>(p, b, hk, group, c, 16 * db + 4 * g, x.acc[db][nb], x.m[nb], x.l[nb]);
        } else {
          const int64_t piece = (2 * (((int64_t)share * kv_heads + hk) * blocks + cb) + (walk.first_piece ? 0 : 1)) * COLS + in;
#pragma unroll
          for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(ws.o + piece * D + 16 * db + 4 * g) = x.acc[db][nb];
          if (g == 0) ws.ml[piece] = float2{x.m[nb], x.l[nb]};
        }
      }
    }
  } while (walk.next(args_here(), direct != 0, lane));
}

// A (sequence, new token, query head) whose rows several work-groups had: their pieces added up, in a fixed order.  GROUPS times D / 4 threads take every
// GROUPS-th piece each, four at a time against a running maximum; with GROUPS > 1 their sums meet in LDS.
template <int D, int COLS, int GROUPS>
__global__ __launch_bounds__(GROUPS == 1 ? 256 : GROUPS * D / 4) void tree_join_kernel(TreeParams p, TreeSpace ws, int32_t blocks) {
  constexpr int LANES = D / 4, U = 4, OUTPUTS = GROUPS == 1 ? 256 / LANES : 1;
  __shared__ f32x4 part[GROUPS == 1 ? 1 : GROUPS][LANES];
  __shared__ float2 part_ml[GROUPS];
  const int lane = threadIdx.x % LANES, group_of = GROUPS == 1 ? 0 : threadIdx.x / LANES;
  const uint32_t row = blockIdx.x * OUTPUTS + (GROUPS == 1 ? threadIdx.x / LANES : 0);   // (below 2^25, checked on the host)
  const int32_t bi = (int32_t)(row / (uint32_t)p.q_heads), h = (int32_t)row - bi * p.q_heads, group = p.q_heads / p.kv_heads, hk = h / group;
  const int32_t b = bi / p.sq, i = bi - b * p.sq;
  if (b >= p.batch) return;
  const int32_t tokens = p.tokens ? p.tokens[b] : p.sq;
  const int2 owners = ws.owners[b];   // (not written for a sequence without tokens)
  if (i >= tokens) return;
  const int32_t w0 = owners.x, w1 = owners.y >> 1, skip = owners.y & 1;
  if (w0 == w1) return;   // written out by its only owner
  const int32_t c = i * group + (h - hk * group), hb = hk * blocks + c / COLS, per_seq = p.kv_heads * blocks;
  auto piece = [&](int32_t w) { return (2 * ((int64_t)w * per_seq + hb) + (w == w0 ? skip : 0)) * COLS + c % COLS; };
  float top = -INFINITY, sum = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int32_t w = w0 + group_of; w <= w1; w += U * GROUPS) {
    float2 ml[U];
    f32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = piece(min(w + u * GROUPS, w1));
      ml[u] = ws.ml[at];
      x[u] = *reinterpret_cast<const f32x4*>(ws.o + at * D + 4 * lane);
    }
    float up = top;
#pragma unroll
    for (int u = 0; u < U; ++u) up = fmaxf(up, w + u * GROUPS <= w1 ? ml[u].x : -INFINITY);
    const float f0 = top == up ? 1.f : __builtin_amdgcn_exp2f(top - up);
    top = up;
    sum *= f0;
    o *= f0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (w + u * GROUPS > w1) continue;
      const float f = ml[u].x == top ? 1.f : __builtin_amdgcn_exp2f(ml[u].x - top);
      sum += ml[u].y * f;
      o += x[u] * f;
    }
  }
  if constexpr (GROUPS > 1) {
    part[group_of][lane] = o;
    if (lane == 0) part_ml[group_of] = float2{top, sum};
    __syncthreads();
    if (group_of != 0) return;
    top = -INFINITY;
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) top = fmaxf(top, part_ml[k].x);
    sum = 0.f;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int k = 0; k < GROUPS; ++k) {
      const float f = part_ml[k].x == top ? 1.f : __builtin_amdgcn_exp2f(part_ml[k].x - top);
      sum += part_ml[k].y * f;
      o += part[k][lane] * f;
    }
  }
  if (p.cache.is_f8) tree_write<true>(p, b, hk, group, c, 4 * lane, o, top, sum);
  else tree_write<false>(p, b, hk, group, c, 4 * lane, o, top, sum);
}

// How a call is dealt.
struct TreeShape {
  int32_t columns, blocks, shares;   // columns of a work-group; blocks of them of a key head; shares of the units
  bool direct;                       // a share for every sequence, no workspace
  int64_t off_ml, off_o, bytes;
};
int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }
TreeShape tree_shape(int32_t batch, int32_t sq, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int64_t max_rows) {
  TreeShape s;
  const int32_t all = q_heads / kv_heads * sq;
  s.columns = all <= 16 ? 16 : all <= 32 ? 32 : all <= 64 ? 64 : 128;
  s.blocks = (all + s.columns - 1) / s.columns;
  const int64_t per_seq = (int64_t)kv_heads * s.blocks, unit = s.columns <= 32 ? 128 : 64, max_units = std::max<int64_t>(1, (max_rows + unit - 1) / unit);
  // A work-group for a whole sequence where they fill the chip, or where its tiles take less time than dealing them out, a second launch and the join of pieces: the
  // more sequences there are, the longer those take.  us, whole / dealt, bf16, head_dim 128:
  //   80 columns   32 work-groups: 256 rows 14.6 / 15.1, 512 21.8 / 17.7;   64: 512 22.6 / 22.4, 1024 37.1 / 25.8;   128: 512 23.1 / 25.5, 1024 37.5 / 31.2;
  //                240: 1024 40.5 / 46.0, 2048 69.5 / 69.9, 4096 128 / 113, of up to 1024 rows 37.3 / 30.3, of up to 4096 125 / 47.1
  //   16 columns   64 work-groups: 512 rows 10.6 / 14.2, 1024 13.4 / 18.5, 4096 47.8 / 32.0;   240: 1024 29.3 / 31.7, of up to 1024 15.5 / 22.9, of up to 4096 50.5 / 35.8
  //   16 columns   2 work-groups: 1024 rows 12.5 / 12.5;   32 columns, e4m3: 16.2 / 14.3;   16 columns, head_dim 64: 2040 rows 15.0 / 12.0, 12 work-groups of 777 10.4 / 11.0
  // From kTreeFit work-groups on every sequence is whole.  That costs nothing where they are alike, and time where they are not: 512 work-groups, 80 columns, 1024 rows 61.6 / 61.4, 4096 206 / 205,
  // of up to 4096 rows 130 / 83.5;   40 columns, of up to 7487 rows 187 / 125;   16 columns, 1024 rows 51.8 / 47.7, of up to 1024 27.7 / 30.7, of up to 4096 91 / 64.5.
  const int64_t groups = batch * per_seq, whole = s.columns <= 32 ? s.columns == 16 || groups >= 64 ? 1024 : 768 : std::max({(int64_t)256, std::min((int64_t)512, 8 * groups), 4 * groups});
  s.direct = groups >= kTreeFit || max_rows <= whole;
  s.shares = (int32_t)(s.direct ? batch : std::min<int64_t>(batch * max_units, std::max<int64_t>(1, kTreeFit / per_seq)));
  const int64_t pieces = s.shares * per_seq * 2 * s.columns;
  s.off_ml = up256((int64_t)batch * 8);
  s.off_o = s.off_ml + up256(pieces * 8);
  s.bytes = s.direct ? 0 : s.off_o + pieces * head_dim * 4;
  return s;
}
TreeShape shape_of(const TreeParams& p) { return tree_shape(p.batch, p.sq, p.q_heads, p.kv_heads, p.head_dim, p.max_rows); }

template <int D, bool F8, bool PAGES16, int CW, int PARTS>
hipError_t launch_columns(const TreeParams& p, const TreeShape& s, const TreeSpace& ws, hipStream_t stream) {
  constexpr int SLOTS = tree_slots(D, F8), LDS = SLOTS * (2 * kTreeRows * D * (F8 ? 1 : 2) + 8) + 64 * 8;
  static_assert(LDS >= 2 * 32 * D * 4 + 64 * 8, "sums of two waves fit where the tiles were");
  const int64_t pairs = ((int64_t)s.shares * p.kv_heads + 7) / 8 * 8;
  hipLaunchKernelGGL((tree_kernel<D, F8, PAGES16, CW, PARTS>), dim3((uint32_t)(pairs * s.blocks)), dim3(64 * kTreeWaves), LDS, stream, p, ws, s.blocks, s.shares,
                     s.direct ? 1 : 0);
  return hipGetLastError();
}
template <int D, bool F8, bool PAGES16>
hipError_t launch_kernel(const TreeParams& p, const TreeShape& s, const TreeSpace& ws, hipStream_t stream) {
  // P in two parts where O is bf16, else in three
  if (s.columns == 64) return p.o.is_f32 ? launch_columns<D, F8, PAGES16, 2, 3>(p, s, ws, stream) : launch_columns<D, F8, PAGES16, 2, 2>(p, s, ws, stream);
  return p.o.is_f32 ? launch_columns<D, F8, PAGES16, 4, 3>(p, s, ws, stream) : launch_columns<D, F8, PAGES16, 4, 2>(p, s, ws, stream);
}
// Threads for the pieces of a sequence, of which it has as many as shares if it is the only long one.
template <int D, int COLS>
hipError_t launch_join(const TreeParams& p, const TreeShape& s, const TreeSpace& ws, hipStream_t stream) {
  const int64_t rows = (int64_t)p.batch * p.sq * p.q_heads;
  if (s.shares > 64 * p.batch) hipLaunchKernelGGL((tree_join_kernel<D, COLS, 16>), dim3((uint32_t)rows), dim3(16 * D / 4), 0, stream, p, ws, s.blocks);
  else if (s.shares > 8 * p.batch) hipLaunchKernelGGL((tree_join_kernel<D, COLS, 4>), dim3((uint32_t)rows), dim3(4 * D / 4), 0, stream, p, ws, s.blocks);
  else hipLaunchKernelGGL((tree_join_kernel<D, COLS, 1>), dim3((uint32_t)((rows * (D / 4) + 255) / 256)), dim3(256), 0, stream, p, ws, s.blocks);
  return hipGetLastError();
}
template <int D, bool F8>
hipError_t launch(const TreeParams& p, hipStream_t stream) {
  const TreeShape s = shape_of(p);
  char* const space = (char*)p.workspace;
  const TreeSpace ws{(int2*)space, (float2*)(space + s.off_ml), (float*)(space + s.off_o)};
  hipError_t e;
  if (s.columns <= 32) e = launch_tree_few(p, ws, s.columns, s.shares, s.direct, stream);
  else e = p.cache.page_rows % 16 == 0 ? launch_kernel<D, F8, true>(p, s, ws, stream) : launch_kernel<D, F8, false>(p, s, ws, stream);
  if (e != hipSuccess || s.direct) return e;
  if (s.columns == 16) return launch_join<D, 16>(p, s, ws, stream);
  if (s.columns == 32) return launch_join<D, 32>(p, s, ws, stream);
  return s.columns == 64 ? launch_join<D, 64>(p, s, ws, stream) : launch_join<D, 128>(p, s, ws, stream);
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
