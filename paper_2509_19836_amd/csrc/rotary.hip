// The rotation by positions, on its own (queries and keys, or their gradients) and on the way into a paged cache.
//
// A thread takes 16 elements of a head, two runs of 8 that lie half the rotated part apart: as (i, i + rotary_dim / 2) eight pairs, as (2i, 2i + 1)
// four pairs of either run.  The elements behind the rotated part are copied by threads that take two runs half of that part apart.  So 8
// threads that sit next to each other read and write 128 bytes in a row, whatever is a pair.  Angle, sine and cosine depend on the token
// alone: a thread forms those of its pairs once and takes them through its share of the token's heads, so the kernels stay bound by the
// bytes they move.
#include "cache.hpp"
#include "kernels.hpp"

namespace burst {

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4u;   // 4-byte aligned in memory

struct Turn {
  float c[8], s[8];
};

// Sine and cosine of a thread's 8 pairs at one token, rounded to fp32 once.  The angle in whole turns, position * inv_freq / 2 pi, is
// formed in 64 bits by three roundings, off by 3 * 2^-53 of itself: 7e-7 radians at position 2^31 with frequency 1, where 32 bits would lose the
// place on the circle from about 10^5 on.
// What is left of it after the whole turns, and then after the quarter turns, is within +-pi / 4, where the Taylor series of sine to
// x^11 and cosine to x^10 are off by less than 1e-11 and 2e-10.
__device__ __forceinline__ void turn_of(const RopeDev& r, int slot, int32_t b, int32_t row, Turn& t) {
  int32_t pos[3];
#pragma unroll
  for (int a = 0; a < 3; ++a) pos[a] = a < r.n_axes ? r.positions[a * r.s_axis + b * r.s_b + row] : 0;
  const int first = r.adjacent ? 4 * slot : 8 * slot, second = r.adjacent ? r.rotary_dim / 4 + 4 * slot : 8 * slot + 4;
  const f32x4u f0 = *reinterpret_cast<const f32x4u*>(r.inv_freq + first);
  const f32x4u f1 = *reinterpret_cast<const f32x4u*>(r.inv_freq + second);
  const uint32_t axes = r.axes[first / 4] | (uint32_t)r.axes[second / 4] << 8;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t a = (axes >> (2 * j)) & 3u;
    const int32_t p = a == 0 ? pos[0] : a == 1 ? pos[1] : pos[2];
    double turns = (double)p * (double)(j < 4 ? f0[j & 3] : f1[j & 3]) * 0.15915494309189533577;   // 1 / 2 pi
    turns -= rint(turns);
    const double quarter = rint(4. * turns), y = fma(-0.25, quarter, turns) * 6.28318530717958647693, z = y * y;
    const float sy = (float)fma(y * z, fma(z, fma(z, fma(z, fma(z, -1. / 39916800., 1. / 362880.), -1. / 5040.), 1. / 120.), -1. / 6.), y);
    const float cy = (float)fma(z, fma(z, fma(z, fma(z, fma(z, -1. / 3628800., 1. / 40320.), -1. / 720.), 1. / 24.), -0.5), 1.);
    const int n = (int)quarter;
    const float s = n & 1 ? cy : sy, c = n & 1 ? sy : cy;
    t.s[j] = ((n & 2) != 0) != (r.inverse != 0) ? -s : s;
    t.c[j] = (n + 1) & 2 ? -c : c;
  }
}

// The two runs of 8 elements of a thread, from the head's first element.
struct SlotPlace {
  int lo, hi;
  bool turned;
  __device__ __forceinline__ void init(int rotary_dim, int head_dim, int slot) {
    turned = 16 * slot < rotary_dim;
    const int start = turned ? 0 : rotary_dim, part = turned ? rotary_dim : head_dim - rotary_dim, in = slot - start / 16;
    lo = start + 8 * in;
    hi = lo + part / 2;
  }
};

// 16 elements as they lie in memory.
template <bool F32, bool NT>
struct Raw {
  u32x4 w[F32 ? 4 : 2];
  __device__ __forceinline__ void load(const void* ptr, int64_t off, const SlotPlace& at) {
    if constexpr (F32) {
      const float* x = (const float*)ptr + off;
      w[0] = load_as<u32x4, NT>(x + at.lo);
      w[1] = load_as<u32x4, NT>(x + at.lo + 4);
      w[2] = load_as<u32x4, NT>(x + at.hi);
      w[3] = load_as<u32x4, NT>(x + at.hi + 4);
    } else {
      const __bf16* x = (const __bf16*)ptr + off;
      w[0] = load_as<u32x4, NT>(x + at.lo);
      w[1] = load_as<u32x4, NT>(x + at.hi);
    }
  }
  __device__ __forceinline__ float value(int i) const {   // (i is known when compiled)
    const uint32_t word = F32 ? w[i / 4][i % 4] : w[i / 8][i % 8 / 2];   // (a bit cast of w[..][..] itself would take the vector's first word)
    return __builtin_bit_cast(float, F32 ? word : i & 1 ? word & 0xffff0000u : word << 16);
  }
};

// Where 16 results go: fp32, bf16, or e4m3 over a scale.
enum class To { kF32, kBf16, kF8 };
template <To TO, bool NT>
__device__ __forceinline__ void store16(void* ptr, int64_t off, const SlotPlace& at, const float (&y)[16], float scale) {
  if constexpr (TO == To::kF32) {
    float* x = (float*)ptr + off;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      store_as<NT>(f32x4{y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]}, x + (i < 2 ? at.lo : at.hi) + 4 * (i & 1));
  } else if constexpr (TO == To::kBf16) {
    __bf16* x = (__bf16*)ptr + off;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      bf16x8 z;
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = (__bf16)y[8 * h + e];
      store_as<NT>(z, x + (h ? at.hi : at.lo));
    }
  } else {
    uint8_t* to = (uint8_t*)ptr + off;
    float z[16];
    // A scale at either end of fp32, whose reciprocal is no normal number: it and what it divides go by 2^64 towards 1.  (By their exponents: factors
    // would be multiplied with the reciprocal first.)
    const int nearer = scale < 0x1p-100f ? 64 : scale > 0x1p100f ? -64 : 0;
    const float by = __builtin_ldexpf(scale, nearer), over = 1.f / by;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      // y / scale: the product with the reciprocal and what is left of y, as long as that is finite
      const float x = __builtin_ldexpf(y[i], nearer), near = x * over, s = fabsf(near) < 1e4f ? fmaf(fmaf(-near, by, x), over, near) : near;
      z[i] = s != s ? s : fminf(fmaxf(s, -448.f), 448.f);   // (the conversion itself makes NaN of what is too large)
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x2 out;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        int two = __builtin_amdgcn_cvt_pk_fp8_f32(z[8 * h + 4 * w], z[8 * h + 4 * w + 1], 0, false);
        out[w] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(z[8 * h + 4 * w + 2], z[8 * h + 4 * w + 3], two, true);
      }
      *reinterpret_cast<u32x2*>(to + (h ? at.hi : at.lo)) = out;
    }
  }
}

// Each product is rounded by itself, not one of the two fused into the difference: turning by a and by -a are then the same sums of the
// same numbers, and elementary operations in 32 bits give the same result.
// (What is not turned keeps its bits: no multiplication by 1 and 0, which a neighbour's infinity would make a NaN of.)
template <bool F32, bool NT>
__device__ __forceinline__ void turned(const Raw<F32, NT>& raw, const Turn& t, bool adjacent, bool turn, float (&y)[16]) {
#pragma clang fp contract(off)
#pragma unroll
  for (int i = 0; i < 16; ++i) y[i] = raw.value(i);
  if (!turn) return;
  if (adjacent) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float a = y[2 * j], b = y[2 * j + 1];
      y[2 * j] = a * t.c[j] - b * t.s[j];
      y[2 * j + 1] = b * t.c[j] + a * t.s[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float a = y[j], b = y[8 + j];
      y[j] = a * t.c[j] - b * t.s[j];
      y[8 + j] = b * t.c[j] + a * t.s[j];
    }
  }
}

// How a work-group of 256 threads is shared: 2^slots_log2 slots of a head, 2^heads_log2 heads side by side, the rest tokens.
struct TokenShare {
  int slots_log2, heads_log2;
  __host__ __device__ __forceinline__ int tokens() const { return 256 >> (slots_log2 + heads_log2); }
};

// A thread's share of a token's heads.
template <bool F32, To TO, bool NT>
__device__ __forceinline__ void turn_heads(const RopeDev& r, const Turn& t, const SlotPlace& at, const void* from, int64_t from_off,
                                           int64_t from_sh, void* to, int64_t to_off, int64_t to_sh, int first, int step, int heads,
                                           const float* scale) {
  constexpr int U = F32 ? 2 : 4;   // heads whose loads are under way together
  for (int h0 = first; h0 < heads; h0 += U * step) {
    Raw<F32, NT> raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (h0 + u * step < heads) raw[u].load(from, from_off + (h0 + u * step) * from_sh, at);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u * step;
      if (h < heads) {
        float y[16];
        turned(raw[u], t, r.adjacent != 0, at.turned, y);
        store16<TO, NT>(to, to_off + h * to_sh, at, y, TO == To::kF8 && scale ? scale[h] : 1.f);
      }
    }
  }
}

template <bool NT>
__device__ __forceinline__ void turn_tensor(const RopeDev& r, const Turn& t, const SlotPlace& at, const TensorDev& x, const TensorDev& y,
                                            int32_t b, int32_t row, int first, int step, int heads) {
  const int64_t from = b * x.sb + row * x.ss, to = b * y.sb + row * y.ss;
  if (x.is_f32) {
    if (y.is_f32) turn_heads<true, To::kF32, NT>(r, t, at, x.ptr, from, x.sh, y.ptr, to, y.sh, first, step, heads, nullptr);
    else turn_heads<true, To::kBf16, NT>(r, t, at, x.ptr, from, x.sh, y.ptr, to, y.sh, first, step, heads, nullptr);
  } else {
    if (y.is_f32) turn_heads<false, To::kF32, NT>(r, t, at, x.ptr, from, x.sh, y.ptr, to, y.sh, first, step, heads, nullptr);
    else turn_heads<false, To::kBf16, NT>(r, t, at, x.ptr, from, x.sh, y.ptr, to, y.sh, first, step, heads, nullptr);
  }
}

template <bool NT>
__global__ __launch_bounds__(256) void rope_kernel(RopeParams p, TokenShare share, int32_t first) {
  const int slot = threadIdx.x & ((1 << share.slots_log2) - 1), step = 1 << share.heads_log2;
  const int head = (threadIdx.x >> share.slots_log2) & (step - 1);
  const int64_t token = first + (int64_t)blockIdx.x * share.tokens() + (threadIdx.x >> (share.slots_log2 + share.heads_log2));
  if (token >= (int64_t)p.batch * p.sq) return;
  const int32_t b = (int32_t)token / p.sq, row = (int32_t)token - b * p.sq;   // (batch * sq < 2^31, checked on the host)
  SlotPlace at;
  at.init(p.rope.rotary_dim, p.head_dim, slot);
  Turn t;
  if (at.turned) turn_of(p.rope, slot, b, row, t);
  turn_tensor<NT>(p.rope, t, at, p.q, p.q_out, b, row, head, step, p.q_heads);
  if (p.k.ptr) turn_tensor<NT>(p.rope, t, at, p.k, p.k_out, b, row, head, step, p.kv_heads);
}

// Whether lines are kept: not where a call moves more than the 256 MiB that the chip keeps and every access takes whole lines, 8 threads of 16
// bytes.  16384 rows x 64 heads of 128, bf16: 102 us kept, 94 not; 4096 x 40: 17.1 kept, 18.6 not; with half lines, of 64 elements
// turned out of 128, 103 kept and 113 not.  (The 32 bytes that a thread takes of fp32 are two accesses: 172 and 157 us from fp32 to bf16, 16384
// x 72, but 221 and 232 from fp32 to fp32.)
static bool streams(int64_t bytes, int32_t head_dim, const RopeDev& r) {
  return bytes > ((int64_t)256 << 20) && head_dim == 128 && (r.rotary_dim == 128 || r.rotary_dim == 0);
}

// Heads that a thread takes one after the other: the more, the fewer times sine and cosine are formed; the fewer, the more threads there are.  One
// where these do not fill the chip twice over (256 tokens of 40 heads: 6.0 us, by fours 6.8; 16 tokens 5.6, 6.5), two of bf16 where
// lines are not kept and there are about as many key heads, or threads would wait while others take those (16384 x 32 + 32 heads: 90.6 us, by
// fours 95.4, by ones 121; appended, 16000 x 32 + 32: 137, by fours 144, but 16384 x 64 + 8: 132 and 115), four otherwise (4096 x 40: 16.7 us, by twos 18.2, by
// eights 17.9; 4 x 8192 x 24 heads of 64: 43.1, 43.3, 46.8; fp32 to bf16, 16384 x 72: 159, 161, 162).
static TokenShare token_share(int32_t head_dim, int32_t heads, int64_t tokens, bool by_twos) {
  TokenShare s{head_dim == 128 ? 3 : 2, 0};
  const int64_t all = tokens * heads * (head_dim / 16);
  const int each = all <= 2 * 256 * 256 ? 1 : by_twos ? 2 : 4;
  while (s.slots_log2 + s.heads_log2 < 8 && (each << s.heads_log2) < heads) ++s.heads_log2;
  return s;
}

// A launch has fewer than 2^32 threads; more tokens than these are for go to several.
template <class Params>
static hipError_t launch_tokens(void (*kernel)(Params, TokenShare, int32_t), const Params& p, TokenShare share, int64_t total, hipStream_t stream) {
  const int64_t each = (int64_t)share.tokens() << 23;   // 2^31 threads
  for (int64_t first = 0; first < total; first += each) {
    const int64_t grid = (std::min(each, total - first) + share.tokens() - 1) / share.tokens();
    hipLaunchKernelGGL(kernel, dim3((uint32_t)grid), dim3(256), 0, stream, p, share, (int32_t)first);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_rope(const RopeParams& p, hipStream_t stream) {
  const int64_t total = (int64_t)p.batch * p.sq;
  if (total == 0) return hipSuccess;
  auto bytes = [&](const TensorDev& x, const TensorDev& y, int32_t heads) {
    return x.ptr ? total * heads * p.head_dim * ((x.is_f32 ? 4 : 2) + (y.is_f32 ? 4 : 2)) : (int64_t)0;
  };
  const bool f32_to_f32 = (p.q.is_f32 && p.q_out.is_f32) || (p.k.ptr && p.k.is_f32 && p.k_out.is_f32);
  const bool nt = !f32_to_f32 && streams(bytes(p.q, p.q_out, p.q_heads) + bytes(p.k, p.k_out, p.kv_heads), p.head_dim, p.rope);
  const TokenShare share = token_share(p.head_dim, p.q_heads, total, nt && !p.q.is_f32 && 2 * p.kv_heads >= p.q_heads);
  return launch_tokens(nt ? rope_kernel<true> : rope_kernel<false>, p, share, total, stream);
}

// A token's keys (turned) and values into its row of the cache, and its queries (turned) to q_out.
template <bool NT>
__global__ __launch_bounds__(256) void cache_append_kernel(AppendParams p, TokenShare share, int32_t first) {
  const int slot = threadIdx.x & ((1 << share.slots_log2) - 1), step = 1 << share.heads_log2;
  const int head = (threadIdx.x >> share.slots_log2) & (step - 1);
  const int64_t token = first + (int64_t)blockIdx.x * share.tokens() + (threadIdx.x >> (share.slots_log2 + share.heads_log2));
  if (token >= (int64_t)p.batch * p.sq) return;
  const int32_t b = (int32_t)token / p.sq, i = (int32_t)token - b * p.sq;
  int32_t fresh = p.new_rows ? p.new_rows[b] : p.sq;
  fresh = fresh < 0 ? 0 : fresh > p.sq ? p.sq : fresh;
  if (i >= fresh) return;
  SlotPlace at, as_is;
  at.init(p.rope.rotary_dim, p.head_dim, slot);
  as_is.init(0, p.head_dim, slot);
  Turn t;
  if (at.turned) turn_of(p.rope, slot, b, i, t);
  if (p.q.ptr)
    turn_heads<false, To::kBf16, NT>(p.rope, t, at, p.q.ptr, b * p.q.sb + i * p.q.ss, p.q.sh, p.q_out.ptr, b * p.q_out.sb + i * p.q_out.ss,
                                 p.q_out.sh, head, step, p.q_heads, nullptr);
  const int32_t row = p.cache.rows_of(b) - fresh + i;
  const int64_t to = row < 0 ? -1 : p.cache.row_offset(b, row);
  if (to < 0) return;
  const int64_t k = b * p.k.sb + i * p.k.ss, v = b * p.v.sb + i * p.v.ss;
  if (p.cache.is_f8) {
    turn_heads<false, To::kF8, NT>(p.rope, t, at, p.k.ptr, k, p.k.sh, p.cache.k, to, p.cache.s_head, head, step, p.kv_heads, p.cache.k_scale);
    turn_heads<false, To::kF8, NT>(p.rope, t, as_is, p.v.ptr, v, p.v.sh, p.cache.v, to, p.cache.s_head, head, step, p.kv_heads, p.cache.v_scale);
  } else {
    turn_heads<false, To::kBf16, NT>(p.rope, t, at, p.k.ptr, k, p.k.sh, p.cache.k, to, p.cache.s_head, head, step, p.kv_heads, nullptr);
    turn_heads<false, To::kBf16, NT>(p.rope, t, as_is, p.v.ptr, v, p.v.sh, p.cache.v, to, p.cache.s_head, head, step, p.kv_heads, nullptr);
  }
}

hipError_t launch_cache_append(const AppendParams& p, hipStream_t stream) {
  const int64_t total = (int64_t)p.batch * p.sq;
  if (total == 0) return hipSuccess;
  const int64_t bytes = total * p.head_dim * ((p.q.ptr ? 4 * p.q_heads : 0) + 2 * p.kv_heads * (p.cache.is_f8 ? 3 : 4));
  const bool nt = streams(bytes, p.head_dim, p.rope);
  const TokenShare share = token_share(p.head_dim, p.q.ptr ? p.q_heads : p.kv_heads, total, nt && (!p.q.ptr || 2 * p.kv_heads >= p.q_heads));
  return launch_tokens(nt ? cache_append_kernel<true> : cache_append_kernel<false>, p, share, total, stream);
}

}  // namespace burst
