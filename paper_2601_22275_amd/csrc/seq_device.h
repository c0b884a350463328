// Device pieces of the bf16 token-sequence kernels (seq_mfma.hip, seq_token.hip, seq_bwd.hip); everything has internal linkage.
#pragma once
#include <type_traits>

#include "seq.h"

namespace vm {

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr float NEG_BIG = -3.402823466e38f;  // the reference of a row that has seen nothing: below any finite logit, and finite, so that -inf - reference is -inf

template <int I, int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    static_for<I + 1, N>(f);
  }
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
  bf16x2 r;
  r[0] = (__bf16)a;
  r[1] = (__bf16)b;
  uint32_t u;
  __builtin_memcpy(&u, &r, 4);
  return u;
}

// Row maximum of a 32-key sub-tile: 16 logits in the lane, 16 in lane ^ 32
__device__ __forceinline__ float subtile_max(const f32x16& s) {
  float m0 = fmaxf(fmaxf(s[0], s[1]), s[2]), m1 = fmaxf(fmaxf(s[3], s[4]), s[5]);
  float m2 = fmaxf(fmaxf(s[6], s[7]), s[8]), m3 = fmaxf(fmaxf(s[9], s[10]), s[11]);
  m0 = fmaxf(fmaxf(m0, s[12]), s[13]);
  m1 = fmaxf(fmaxf(m1, s[14]), s[15]);
  const unsigned u = __float_as_uint(fmaxf(fmaxf(m0, m1), fmaxf(m2, m3)));
  const auto sw = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}

// Whether the 32 rows at LDS address `at` hold a bf16 that is not finite (all lanes of a wave together)
template <int ROW_BYTES>
__device__ __forceinline__ bool odd_values(unsigned at) {
  typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
  typedef __attribute__((address_space(3))) const u32x4* lds_u32x4_ptr;
  typedef __attribute__((__vector_size__(2 * sizeof(uint16_t)))) uint16_t u16x2;
  u16x2 largest = {0, 0};
#pragma unroll
  for (int i = 0; i < 32 * ROW_BYTES; i += 1024) {
    const u32x4 w = *(lds_u32x4_ptr)(unsigned long long)(at + i + 16 * (threadIdx.x & 63));
#pragma unroll
    for (int e = 0; e < 4; ++e) largest = __builtin_elementwise_max(largest, __builtin_bit_cast(u16x2, w[e] & 0x7fff7fffu));
  }
  return __any(max(largest[0], largest[1]) >= 0x7f80);
}

// Where a key's row and its value's lie
struct alignas(16) RowAt {
  const bf16_t *k, *v;
};

}  // namespace

}  // namespace vm
