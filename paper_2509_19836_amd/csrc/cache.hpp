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

hipError_t launch_rope(const RopeParams& p, hipStream_t stream);
hipError_t launch_cache_append(const AppendParams& p, hipStream_t stream);
hipError_t launch_decode(const DecodeParams& p, hipStream_t stream);
void decode_plan(const DecodeParams& p, int32_t out[3]);   // burst_attn_decode_plan
int64_t decode_workspace_bytes(int32_t batch, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int64_t max_rows);

}  // namespace burst
