// Parameter blocks, launchers and shared device code of the rotation by positions and of the paged key-value cache.
#pragma once
#include "common.hpp"

namespace burst {

// n / d for 0 <= n < 2^31 without a division (Granlund, Montgomery: Division by Invariant Integers using Multiplication): with
// 2^(s-1) < d <= 2^s and m = ceil(2^(31+s) / d) the quotient is floor(m * n / 2^(31+s)), and m fits in 32 bits.
struct Divider {
  uint32_t d, mul, shift;
  void init(uint32_t d_) {
    d = d_;
    shift = 0;
    while (((uint64_t)1 << shift) < d) ++shift;
    mul = shift == 0 ? 0u : (uint32_t)((((uint64_t)1 << (31 + shift)) + d - 1) / d);
  }
  __host__ __device__ __forceinline__ int32_t quotient(int32_t n) const {
    return shift == 0 ? n : (int32_t)((uint32_t)(((uint64_t)(uint32_t)n * mul) >> 32) >> (shift - 1));
  }
};

// NT: of a tensor that is larger than what stays on the chip until it is next asked for, no line is kept.
template <class T, bool NT>
__device__ __forceinline__ T load_as(const void* at) {
  if constexpr (NT) return __builtin_nontemporal_load(reinterpret_cast<const T*>(at));
  else return *reinterpret_cast<const T*>(at);
}
template <bool NT, class T>
__device__ __forceinline__ void store_as(T x, void* at) {
  if constexpr (NT) __builtin_nontemporal_store(x, reinterpret_cast<T*>(at));
  else *reinterpret_cast<T*>(at) = x;
}

// The value of the lane that differs by STEP.  By the vector unit's own moves, not through LDS: a stage of a network over the lanes in a quarter of the time.
template <int STEP>
__device__ __forceinline__ uint32_t of_lane_xor(uint32_t x) {
  if constexpr (STEP == 1) return __builtin_amdgcn_mov_dpp(x, 0xb1, 0xf, 0xf, false);         // quad_perm [1, 0, 3, 2]
  else if constexpr (STEP == 2) return __builtin_amdgcn_mov_dpp(x, 0x4e, 0xf, 0xf, false);    // quad_perm [2, 3, 0, 1]
  else if constexpr (STEP == 4) return __builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp(x, 0x141, 0xf, 0xf, false), 0x1b, 0xf, 0xf, false);   // 8 lanes, then 4, the other way round
  else if constexpr (STEP == 8) return __builtin_amdgcn_mov_dpp(x, 0x128, 0xf, 0xf, false);   // row_ror 8
  else if constexpr (STEP == 16) {
    const auto y = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return (threadIdx.x & 16) ? y[0] : y[1];
  } else {
    const auto y = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return (threadIdx.x & 32) ? y[0] : y[1];
  }
}

struct RopeDev {
  const float* inv_freq;
  const int32_t* positions;
  int64_t s_axis, s_b;
  int32_t n_axes, rotary_dim;   // rotary_dim 0: no rotation
  int32_t adjacent, inverse;
  uint8_t axes[16];             // two bits for each of four pairs
};

struct RopeParams {
  int32_t batch, sq, q_heads, kv_heads, head_dim;
  RopeDev rope;
  TensorDev q, q_out, k, k_out;   // k.ptr == nullptr: q alone
};

struct CacheDev {
  void* k;
  void* v;
  int64_t s_page, s_row, s_head;   // elements
  int32_t is_f8;
  int32_t n_pages, page_rows, table_cols;
  const int32_t* table;
  int64_t table_stride;
  const int32_t* rows;
  const float* k_scale;
  const float* v_scale;
  Divider by_page;

  // Rows of a sequence, as the interface limits them.
  __device__ __forceinline__ int32_t rows_of(int32_t b) const {
    const int32_t n = rows[b], most = table_cols * page_rows;   // (at most 2^30, checked on the host)
    return n < 0 ? 0 : n > most ? most : n;
  }
  // First element of the head rows of row t < table_cols * page_rows; -1: the table has no page there.
  __device__ __forceinline__ int64_t row_offset(int32_t b, int32_t t) const {
    const int32_t col = by_page.quotient(t);
    const int32_t page = table[b * table_stride + col];
    if (page < 0 || page >= n_pages) return -1;
    return page * s_page + (int64_t)(t - col * page_rows) * s_row;
  }
};

struct AppendParams {
  int32_t batch, sq, q_heads, kv_heads, head_dim;
  RopeDev rope;
  TensorDev k, v, q, q_out;   // q.ptr == nullptr: keys and values alone
  const int32_t* new_rows;
  CacheDev cache;
};

struct DecodeParams {
  int32_t batch, q_heads, kv_heads, head_dim;
  int32_t max_rows;
  float scale;
  TensorDev q, o;
  RowvecDev lse;              // ptr == nullptr: not wanted
  const int32_t* first_row;   // nullptr: 0
  CacheDev cache;
  void* workspace;
};

struct TreeParams {
  int32_t batch, sq, q_heads, kv_heads, head_dim;
  int32_t max_rows;
  float scale;
  TensorDev q, o;
  RowvecDev lse;              // ptr == nullptr: not wanted
  const uint64_t* seen;       // nullptr: a chain
  int64_t seen_sb;
  const int32_t* first;       // nullptr: 0
  int64_t first_sb;
  const int32_t* tokens;      // nullptr: sq
  int32_t sinks, elsewhere;
  CacheDev cache;
  void* workspace;
};

// The keys and values of some layers, alike but for where they are.
constexpr int kLayersOfLaunch = 64;
struct LayersDev {
  void* k[kLayersOfLaunch];
  void* v[kLayersOfLaunch];
  int32_t n, kv_heads, head_dim, page_rows, n_pages;
  int32_t bytes;                     // of an element
  int32_t head_outer;                // heads are further apart than rows
  int64_t s_page, s_row, s_head;     // bytes
};
struct CopyPagesParams {
  LayersDev layers;
  const int32_t* moves;   // [n_moves][3]: from, to, rows
  int32_t n_moves;
};
struct KeepRowsParams {
  struct {
    LayersDev layers;
    CacheDev dev;         // (k and v are not read)
  } cache;
  int32_t batch, sq;
  const int32_t* from;
  int64_t from_sb;
  const int32_t* new_rows;   // nullptr: sq
  const int32_t* kept;
};

hipError_t launch_rope(const RopeParams& p, hipStream_t stream);
hipError_t launch_cache_append(const AppendParams& p, hipStream_t stream);
hipError_t launch_decode(const DecodeParams& p, hipStream_t stream);
void decode_plan(const DecodeParams& p, int32_t out[3]);   // burst_attn_decode_plan
int64_t decode_workspace_bytes(int32_t batch, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int64_t max_rows);
hipError_t launch_tree(const TreeParams& p, hipStream_t stream);
void tree_plan(const TreeParams& p, int32_t out[3]);   // burst_attn_tree_plan
int64_t tree_workspace_bytes(int32_t batch, int32_t sq, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int64_t max_rows);
hipError_t launch_cache_copy_pages(const CopyPagesParams& p, hipStream_t stream);
hipError_t launch_cache_keep_rows(const KeepRowsParams& p, hipStream_t stream);

}  // namespace burst
