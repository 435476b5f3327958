// Attention of one new token of every sequence over its rows in a paged cache.
#include "cache.hpp"
#include "kernels.hpp"
#include "mfma16.hpp"

namespace burst {

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// 8 numbers of a cache row as fp32.
template <bool F8>
__device__ __forceinline__ void cache8(const void* base, int64_t off, float (&x)[8]) {
  if constexpr (F8) {
    const u32x2 w = *reinterpret_cast<const u32x2*>((const uint8_t*)base + off);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.0f, false);
      const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.0f, true);
      x[4 * i] = (float)a[0];
      x[4 * i + 1] = (float)a[1];
      x[4 * i + 2] = (float)b[0];
      x[4 * i + 3] = (float)b[1];
    }
  } else {
    const bf16x8 w = *reinterpret_cast<const bf16x8*>((const __bf16*)base + off);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)w[i];
  }
}

// One work-group a (sequence, query head): groups of D / 8 lanes take a row each, 8 elements a lane, with a running maximum and sum
// of their own; they meet in LDS.
template <int D, bool F8>
__global__ __launch_bounds__(256) void decode_rows_kernel(DecodeParams p) {
  constexpr int LANES = D / 8, GROUPS = 256 / LANES;
  __shared__ float part_o[GROUPS][D + 2];
  const int b = blockIdx.x / p.q_heads, hq = blockIdx.x - b * p.q_heads, hk = hq / (p.q_heads / p.kv_heads);
  const int c = threadIdx.x % LANES, grp = threadIdx.x / LANES;
  const int32_t n = p.cache.rows_of(b), hi = n < p.max_rows ? n : p.max_rows;
  int32_t lo = p.first_row ? p.first_row[b] : 0;
  lo = lo < 0 ? 0 : lo < hi ? lo : hi;
  const bf16x8 qv = *reinterpret_cast<const bf16x8*>((const __bf16*)p.q.ptr + b * p.q.sb + hq * p.q.sh + 8 * c);
  const float to_log2 = p.scale * kLog2e * (F8 && p.cache.k_scale ? p.cache.k_scale[hk] : 1.f);
  float m = -INFINITY, l = 0.f, acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  for (int32_t t = lo + grp; t < hi; t += GROUPS) {
    const int64_t row = p.cache.row_offset(b, t);
    if (row < 0) continue;
    float kx[8], vx[8], s = 0.f;
    cache8<F8>(p.cache.k, row + hk * p.cache.s_head + 8 * c, kx);
    cache8<F8>(p.cache.v, row + hk * p.cache.s_head + 8 * c, vx);
#pragma unroll
    for (int e = 0; e < 8; ++e) s += (float)qv[e] * kx[e];
#pragma unroll
    for (int x = 1; x < LANES; x <<= 1) s += __shfl_xor(s, x, 64);
    s *= to_log2;
    const float mm = fmaxf(m, s), safe = mm == -INFINITY ? 0.f : mm;
    const float old = exp2f(m - safe), w = exp2f(s - safe);
    m = mm;
    l = l * old + w;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = acc[e] * old + w * vx[e];
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) part_o[grp][8 * c + e] = acc[e];
  if (c == 0) {
    part_o[grp][D] = m;
    part_o[grp][D + 1] = l;
  }
  __syncthreads();
  if (threadIdx.x >= D) return;
  float top = -INFINITY, total = 0.f, o = 0.f;
  for (int g = 0; g < GROUPS; ++g) top = fmaxf(top, part_o[g][D]);
  const float safe = top == -INFINITY ? 0.f : top;
  for (int g = 0; g < GROUPS; ++g) {
    const float w = exp2f(part_o[g][D] - safe);
    total += w * part_o[g][D + 1];
    o += w * part_o[g][threadIdx.x];
  }
  o = total == 0.f ? 0.f : o / total * (F8 && p.cache.v_scale ? p.cache.v_scale[hk] : 1.f);
  const int64_t at = b * p.o.sb + hq * p.o.sh + threadIdx.x;
  if (p.o.is_f32) ((float*)p.o.ptr)[at] = o;
  else ((__bf16*)p.o.ptr)[at] = (__bf16)o;
  if (p.lse.ptr && threadIdx.x == 0) p.lse.ptr[b * p.lse.sb + hq * p.lse.sh] = total == 0.f ? -INFINITY : (top + log2f(total)) * kLn2;
}

int64_t decode_workspace_bytes(int32_t, int32_t, int32_t, int32_t, int64_t) { return 0; }

hipError_t launch_decode(const DecodeParams& p, hipStream_t stream) {
  const dim3 grid((uint32_t)(p.batch * p.q_heads));
  const bool f8 = p.cache.is_f8 != 0;
  if (p.head_dim == 128) {
    if (f8) hipLaunchKernelGGL((decode_rows_kernel<128, true>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((decode_rows_kernel<128, false>), grid, dim3(256), 0, stream, p);
  } else {
    if (f8) hipLaunchKernelGGL((decode_rows_kernel<64, true>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((decode_rows_kernel<64, false>), grid, dim3(256), 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace burst
