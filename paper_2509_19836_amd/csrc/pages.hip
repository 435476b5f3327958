// Pages of a cache copied, and rows of its sequences moved to the front, in all layers of a model at once.
//
// Both move bytes and nothing else: 16 of them a thread and access, as many accesses under way as a thread has registers for, and neighbouring
// threads side by side in the order in which a page lies in memory.
//   Measured: 64 pages of 64 rows, 32 layers, 8 heads (537 MB read, as many written) 212 us, 5.07 TB/s, what a large copy reaches; with 32 sequences' up to 16 rows in 32 layers
// a keep takes 6.6 to 6.9 us, which the host's issue of a call from Python just hides; the copy of three pages in two layers 4.5 to 4.8, and 5.8 a call.
#include <algorithm>

#include "cache.hpp"
#include "kernels.hpp"

namespace burst {

namespace {

// The arguments of a launch are read with a variable index through their own pointer (the compiler would copy them to scratch memory otherwise).
template <class Params>
__device__ __forceinline__ const Params& kernel_args() {
  typedef const __attribute__((address_space(4))) Params* args_ptr;
  return *(const Params*)(args_ptr)__builtin_amdgcn_kernarg_segment_ptr();
}

// A page's part as pieces of 16 bytes: `inner` of a row (or head) one after the other, then `middle` heads (or rows), then the other of the two.
struct PagePieces {
  Divider by_piece, by_head;   // pieces of a head's row; heads
  int32_t per_head, heads;
  // Bytes from the page's first element to piece i of rows `rows`
  __device__ __forceinline__ int64_t at(int32_t i, int32_t rows, const LayersDev& c) const {
    const int32_t piece = i - by_piece.quotient(i) * per_head, rest = by_piece.quotient(i);
    int32_t row, head;
    if (c.head_outer) {
      head = rest / rows;
      row = rest - head * rows;
    } else {
      row = by_head.quotient(rest);
      head = rest - row * heads;
    }
    return row * c.s_row + head * c.s_head + 16 * (int64_t)piece;
  }
};

constexpr int kCopyEach = 8;   // pieces of a thread

__global__ __launch_bounds__(256) void cache_copy_pages_kernel(CopyPagesParams p, PagePieces pieces, int32_t parts) {
  const CopyPagesParams& args = kernel_args<CopyPagesParams>();
  const int32_t n = (int32_t)((uint32_t)blockIdx.x / (uint32_t)parts), part = (int32_t)blockIdx.x - n * parts;
  const int32_t from = p.moves[3 * (int64_t)n], to = p.moves[3 * (int64_t)n + 1];
  int32_t rows = p.moves[3 * (int64_t)n + 2];
  rows = rows < p.layers.page_rows ? rows : p.layers.page_rows;
  if (from < 0 || from >= p.layers.n_pages || to < 0 || to >= p.layers.n_pages || from == to || rows <= 0) return;
  char* const base = (char*)(blockIdx.y & 1 ? args.layers.v[blockIdx.y >> 1] : args.layers.k[blockIdx.y >> 1]);
  const char* const src = base + from * p.layers.s_page;
  char* const dst = base + to * p.layers.s_page;
  const int32_t total = rows * pieces.heads * pieces.per_head, first = part * (256 * kCopyEach) + (int32_t)threadIdx.x;
  int64_t at[kCopyEach];
  u32x4 x[kCopyEach];
#pragma unroll
  for (int e = 0; e < kCopyEach; ++e) {
    const int32_t i = first + 256 * e;
    if (i < total) {
      at[e] = pieces.at(i, rows, p.layers);
      x[e] = *reinterpret_cast<const u32x4*>(src + at[e]);
    }
  }
#pragma unroll
  for (int e = 0; e < kCopyEach; ++e)
    if (first + 256 * e < total) *reinterpret_cast<u32x4*>(dst + at[e]) = x[e];
}

// A work-group has some pieces of all rows that a sequence keeps: all of them are read before the first is written, so a row may be another's
// source and destination.
constexpr int kKeepEach = 4;

__global__ __launch_bounds__(256) void cache_keep_rows_kernel(KeepRowsParams p, PagePieces pieces, int32_t per_row, int32_t pieces_each) {
  const KeepRowsParams& args = kernel_args<KeepRowsParams>();
  const int32_t b = (int32_t)blockIdx.z, first_piece = (int32_t)blockIdx.x * pieces_each;
  char* const base = (char*)(blockIdx.y & 1 ? args.cache.layers.v[blockIdx.y >> 1] : args.cache.layers.k[blockIdx.y >> 1]);
  int32_t n = p.new_rows ? p.new_rows[b] : p.sq, kept = p.kept[b];
  n = n < 0 ? 0 : n > p.sq ? p.sq : n;
  kept = kept < n ? kept : n;
  const int32_t rows = p.cache.dev.rows_of(b), older = rows - n;
  const int32_t here = min(pieces_each, per_row - first_piece);
  char* to[kKeepEach];
  u32x4 x[kKeepEach];
#pragma unroll
  for (int e = 0; e < kKeepEach; ++e) {
    const int32_t item = (int32_t)threadIdx.x + 256 * e, i = item / pieces_each, in = item - i * pieces_each;
    to[e] = nullptr;
    if (i >= kept || in >= here) continue;
    const int32_t j = p.from[b * p.from_sb + i];
    if (j < 0 || j >= n || j == i || older + i < 0 || older + j < 0) continue;
    const int64_t source = p.cache.dev.row_offset(b, older + j), target = p.cache.dev.row_offset(b, older + i);
    if (source < 0 || target < 0) continue;
    const int32_t piece = first_piece + in, head = pieces.by_piece.quotient(piece);
    const int64_t off = head * p.cache.layers.s_head + 16 * (int64_t)(piece - head * pieces.per_head);
    x[e] = *reinterpret_cast<const u32x4*>(base + source * p.cache.layers.bytes + off);
    to[e] = base + target * p.cache.layers.bytes + off;
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < kKeepEach; ++e)
    if (to[e]) *reinterpret_cast<u32x4*>(to[e]) = x[e];
}

PagePieces pieces_of(const LayersDev& c) {
  PagePieces x;
  x.per_head = c.head_dim * c.bytes / 16;
  x.heads = c.kv_heads;
  x.by_piece.init((uint32_t)x.per_head);
  x.by_head.init((uint32_t)x.heads);
  return x;
}

}  // namespace

hipError_t launch_cache_copy_pages(const CopyPagesParams& p, hipStream_t stream) {
  const PagePieces pieces = pieces_of(p.layers);
  const int64_t total = (int64_t)p.layers.page_rows * pieces.heads * pieces.per_head;   // (below 2^31, checked on the host)
  const int32_t parts = (int32_t)((total + 256 * kCopyEach - 1) / (256 * kCopyEach));
  // A launch has fewer than 2^32 threads; more pages go to several.
  const int64_t each = std::max<int64_t>(1, ((int64_t)1 << 31) / (256 * (int64_t)parts * 2 * p.layers.n));
  for (int64_t first = 0; first < p.n_moves; first += each) {
    CopyPagesParams part = p;
    part.moves += 3 * first;
    const int64_t n = std::min<int64_t>(each, p.n_moves - first);
    hipLaunchKernelGGL(cache_copy_pages_kernel, dim3((uint32_t)(n * parts), 2 * p.layers.n), dim3(256), 0, stream, part, pieces, parts);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_cache_keep_rows(const KeepRowsParams& p, hipStream_t stream) {
  if (p.sq == 0) return hipSuccess;
  const PagePieces pieces = pieces_of(p.cache.layers);
  const int32_t per_row = pieces.heads * pieces.per_head, pieces_each = std::min(per_row, 256 * kKeepEach / p.sq);
  constexpr int64_t kMaxZ = 65535;
  for (int64_t b0 = 0; b0 < p.batch; b0 += kMaxZ) {
    KeepRowsParams part = p;
    part.from += b0 * p.from_sb;
    part.kept += b0;
    if (part.new_rows) part.new_rows += b0;
    part.cache.dev.table += b0 * p.cache.dev.table_stride;
    part.cache.dev.rows += b0;
    hipLaunchKernelGGL(cache_keep_rows_kernel, dim3((uint32_t)((per_row + pieces_each - 1) / pieces_each), 2 * p.cache.layers.n, (uint32_t)std::min(kMaxZ, p.batch - b0)),
                       dim3(256), 0, stream, part, pieces, per_row, pieces_each);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace burst
