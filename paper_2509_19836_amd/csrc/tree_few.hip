// Attention of a few new tokens over a paged cache where they are up to 32 columns (new tokens times query heads of a key head): the cache's bytes bound it.
//
// Each wave has tiles of 32 rows of its own and all columns: it brings its keys and values to its own part of LDS and meets the others only at the end,
// so loads stay under way everywhere.
//   Measured: a sequence's 131072 rows, 32 heads, 4 tokens, bf16 319 us, 6.7 TB/s.  12 heads over 777 rows of 64, 5 tokens: 10.4 us, most of it one work-group's own chain
// of page table, loads, products and join.
#include "tree.hpp"

namespace burst {

namespace {

constexpr int few_slots(int head_dim, bool f8) { return (1 << 14) / (2 * 32 * head_dim * (f8 ? 1 : 2)); }   // 16 KiB a wave

// NB: blocks of 16 columns.  NW: waves of a work-group, four where rows are dealt to many.
template <int D, bool F8, bool PAGES16, int NB, int NW>
__global__ __launch_bounds__(64 * NW, 2) void tree_few_kernel(TreeParams, TreeSpace ws, int32_t shares, int32_t direct) {
  using Columns = TreeColumns<D, F8, NB, 3, D == 128 && !F8 && !PAGES16 && NB == 2 ? 1 : 4, 1>;   // (registers)
  using Run = TreeRun<D, F8, PAGES16, 2>;
  using Operands = TreeOperands<D, F8>;
  constexpr int DB = Columns::DB, UNIT = 32 * NW, TILE = Operands::TILE, NI = Run::NI;
  constexpr int SLOTS = few_slots(D, F8), LOADS = 2 * NI * (2 * SLOTS - 1);   // tiles under way; loads behind those that a product waits for
  extern __shared__ __attribute__((aligned(1024))) char smem[];   // [wave][slot][K tile, V tile], maxima and sums [wave][16 NB]
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 15, g = lane >> 4;
  char* const tiles = smem + wave * SLOTS * 2 * TILE;
  const uint32_t tiles0 = (uint32_t)(uintptr_t)(lds_bytes)tiles;
  float2* const ml_lds = (float2*)(smem + NW * SLOTS * 2 * TILE);
  const TreeParams& sizes = args_here();
  const int32_t kv_heads = sizes.kv_heads, group = sizes.q_heads / kv_heads;
  const int32_t share = (int32_t)((uint32_t)blockIdx.x / (uint32_t)kv_heads), hk = (int32_t)blockIdx.x - share * kv_heads;

  TreeWalk<UNIT> walk;
  if (!walk.init(args_here(), share, shares, direct != 0, lane)) return;
  Operands ops;
  ops.init(lane);
  do {
    walk.begin(direct != 0, hk == 0 && tid == 0, ws, share);
    if (walk.take <= 0) continue;
    const int32_t b = walk.b, columns = walk.seq.tokens * group;
    Columns x;
    x.init(args_here(), walk.seq, b, hk, group, 0, lane);
    TreeUnion some;
    some.init(args_here(), walk.seq, b, lane);
    Run run;
    run.init(args_here().cache, b, hk, walk.seq.hi, 0, lane);

    // This wave's tiles: rows of unit u from 32 wave on, two runs of 16.  Tile u + SLOTS takes the place of tile u: its keys are asked for when the scores of u
    // have been formed, its values when the products with P are done.
    const bool once = direct == 0;   // lines are not kept where rows are many
    typename Run::Pages pages;
    typename Run::Place place[2];
    const int32_t end = walk.at + walk.take;
    uint32_t there[SLOTS];
    auto first_row = [&](int32_t u) { return walk.row_of(u) + 32 * wave; };
    constexpr bool EARLY = PAGES16 || F8 || D == 64 || NB == 1;   // (else the pages' numbers find no registers beside the products)
    auto look_up = [&](int32_t u) {
      if (EARLY) run.look_up(first_row, u, walk.at, end, 0, lane, pages);
    };
    auto put = [&](int32_t u) {
      if (!EARLY) run.look_up(first_row, u, walk.at, end, 0, lane, pages);
      const uint32_t rows = (uint32_t)some.rows(first_row(u));
#pragma unroll
      for (int h = 0; h < 2; ++h) run.place(first_row(u) + 16 * h, (rows >> (16 * h)) & 0xffffu, lane, pages, u, h, place[h]);
      return place[0].there | place[1].there << 16;
    };
    auto ask_k = [&](uint32_t kt) {
#pragma unroll
      for (int h = 0; h < 2; ++h) run.template bring<false>(place[h], h, kt + Run::BYTES * h, once);
    };
    auto ask_v = [&](uint32_t vt) {
#pragma unroll
      for (int h = 0; h < 2; ++h) run.template bring<true>(place[h], h, vt + Run::BYTES * h, once);
    };
    look_up(walk.at);
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
      there[i] = 0;
      if (walk.at + i < end) {
        there[i] = put(walk.at + i);
        ask_k(tiles0 + i * 2 * TILE);
        ask_v(tiles0 + i * 2 * TILE + TILE);
        if (walk.at + i + 1 < end) look_up(walk.at + i + 1);
      }
    }
    int slot = 0;
    for (int32_t u = walk.at; u < end; ++u) {
      const bool more = u + SLOTS < end;
      const uint32_t kt = tiles0 + slot * 2 * TILE, vt = kt + TILE, now = there[0];
      if (more) wait_loads<LOADS>();
      else wait_loads<0>();
      x.scores(kt, ops);
#pragma unroll
      for (int i = 0; i + 1 < SLOTS; ++i) there[i] = there[i + 1];
      if (more) {
        there[SLOTS - 1] = put(u + SLOTS);
        ask_k(kt);
        if (u + SLOTS + 1 < end) look_up(u + SLOTS + 1);
      }
      x.weights(first_row(u), now, g);
      if (more) wait_loads<LOADS>();
#pragma unroll
      for (int h = 0; h < 2; ++h) Run::clear(tiles + (slot * 2 + 1) * TILE + Run::BYTES * h, (now >> (16 * h)) & 0xffffu, lane);
      x.add(vt, ops);
      if (more) ask_v(vt);
      slot = (slot + 1) & (SLOTS - 1);
    }
    x.finish();
    const TreeParams& p = args_here();

    // The waves' sums against their largest maximum; where their tiles were
    if (g == 0) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) ml_lds[16 * NB * wave + 16 * nb + r] = float2{x.m[nb], x.l[nb]};
    }
    f32x4* const sums = reinterpret_cast<f32x4*>(smem);   // [wave][block of 16 elements][column block][lane]
    constexpr int PITCH = SLOTS * 2 * TILE / 16;
    static_assert(DB * NB * 64 <= PITCH, "a wave's sums fit where its tiles were");
#pragma unroll
    for (int i = 0; i < DB * NB; ++i) sums[wave * PITCH + i * 64 + lane] = x.acc[i / NB][i % NB];
    __syncthreads();
    for (int i = tid; i < DB * NB * 64; i += 64 * NW) {
      const int at = i / 64, l = i % 64, nb = at % NB, c = 16 * nb + l % 16, d = 16 * (at / NB) + 4 * (l / 16);
      if (c >= columns) continue;
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) top = fmaxf(top, ml_lds[16 * NB * w + c].x);
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float2 ml = ml_lds[16 * NB * w + c];
        const float f = ml.x == top ? 1.f : __builtin_amdgcn_exp2f(ml.x - top);
        sum += ml.y * f;
        o += sums[w * PITCH + at * 64 + l] * f;
      }
      if (walk.whole) {
        tree_write<F8>(p, b, hk, group, c, d, o, top, sum);
      } else {
        const int64_t piece = (2 * ((int64_t)share * kv_heads + hk) + (walk.first_piece ? 0 : 1)) * (16 * NB) + c;
        *reinterpret_cast<f32x4*>(ws.o + piece * D + d) = o;
        if (d == 0) ws.ml[piece] = float2{top, sum};
      }
    }
    __syncthreads();
  } while (walk.next(args_here(), direct != 0, lane));
}

template <int D, bool F8, bool PAGES16, int NB, int NW>
hipError_t launch_kernel(const TreeParams& p, const TreeSpace& ws, int32_t shares, bool direct, hipStream_t stream) {
  constexpr int LDS = NW * ((1 << 14) + 16 * NB * 8);
  const int64_t groups = (int64_t)shares * p.kv_heads;
  hipLaunchKernelGGL((tree_few_kernel<D, F8, PAGES16, NB, NW>), dim3((uint32_t)groups), dim3(64 * NW), LDS, stream, p, ws, shares, direct ? 1 : 0);
  return hipGetLastError();
}
template <int D, bool F8, bool PAGES16, int NB>
hipError_t launch_waves(const TreeParams& p, const TreeSpace& ws, int32_t shares, bool direct, hipStream_t stream) {
  // Where a work-group has a whole sequence, eight waves if it has tiles for them and a CU to itself, else few enough that its others find room.  us with 1, 2, 4
  // and 8 waves (bf16, head_dim 128 if not said):
  //   4 heads x 3 sequences of 30 rows   7.9, 7.5, 7.2, 8.1;   of 120 rows   10.9, 8.4, 7.1, 8.4;   of 500 rows   24.1, 15.0, 10.5, 9.5
  //   16 x 128 of 31 (e4m3, 31 tokens)   18.7, 30.8, 41.4, 73.6;   8 x 128 of up to 75 (head_dim 64)   12.3, 10.9, 15.1, 26.5
  //   8 x 64 of up to 200   16.4, 12.8, 11.4, 15.3;   8 x 128 of up to 1000   78.0, 59.7, 56.2, 66.5;   of up to 8000   518, 352, 281, 292
  // (A launch has fewer than 2^32 threads: the most sequences get a wave each.)
  const int32_t tiles = (p.max_rows + 31) / 32;
  const int64_t groups = (int64_t)shares * p.kv_heads;
  const bool many = groups >= kTreeFit;
  if (direct && !many && tiles > 4) return launch_kernel<D, F8, PAGES16, NB, 8>(p, ws, shares, direct, stream);
  if (direct && many && (tiles <= 1 || groups >= 1 << 24)) return launch_kernel<D, F8, PAGES16, NB, 1>(p, ws, shares, direct, stream);
  if (direct && many && tiles <= 4) return launch_kernel<D, F8, PAGES16, NB, 2>(p, ws, shares, direct, stream);
  return launch_kernel<D, F8, PAGES16, NB, 4>(p, ws, shares, direct, stream);
}
template <int D, bool F8, bool PAGES16>
hipError_t launch(const TreeParams& p, const TreeSpace& ws, int32_t columns, int32_t shares, bool direct, hipStream_t stream) {
  return columns == 16 ? launch_waves<D, F8, PAGES16, 1>(p, ws, shares, direct, stream) : launch_waves<D, F8, PAGES16, 2>(p, ws, shares, direct, stream);
}
template <int D, bool F8>
hipError_t launch(const TreeParams& p, const TreeSpace& ws, int32_t columns, int32_t shares, bool direct, hipStream_t stream) {
  return p.cache.page_rows % 16 == 0 ? launch<D, F8, true>(p, ws, columns, shares, direct, stream)
                                     : launch<D, F8, false>(p, ws, columns, shares, direct, stream);
}

}  // namespace

hipError_t launch_tree_few(const TreeParams& p, const TreeSpace& ws, int32_t columns, int32_t shares, bool direct, hipStream_t stream) {
  if (p.head_dim == 128) return p.cache.is_f8 ? launch<128, true>(p, ws, columns, shares, direct, stream) : launch<128, false>(p, ws, columns, shares, direct, stream);
  return p.cache.is_f8 ? launch<64, true>(p, ws, columns, shares, direct, stream) : launch<64, false>(p, ws, columns, shares, direct, stream);
}

}  // namespace burst
