// The 4-bit cache: what its entry points share.  Sixteen neighbouring values x of a head are held as sixteen 4-bit floats c (sign, two
// bits of exponent, one of mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6) and one 8-bit scale s (four bits of exponent, three of mantissa):
//   s = e4m3(max |x| / (6 g)), from 2^-9 to 448,   c = e2m1(x / (s g)),   held: c s g,   g the pool's scale, a power of two.
// c s has at most six significant bits and lies in [2^-10, 2688], or is 0: exact in fp16, and c s g in bf16.
#pragma once
#include "common.cuh"
#include <cuda_fp16.h>
#include <cstring>

namespace efim {

// A power of two between 2^-60 and 2^60: then x / g and c s g are exact wherever they matter.
inline bool good_pool_scale(float g) {
  uint32_t bits;
  memcpy(&bits, &g, 4);
  const int exponent = (int)(bits >> 23) - 127;             // (a sign or NaN falls out of the range)
  return (bits & 0x7fffff) == 0 && exponent >= -60 && exponent <= 60;
}

inline efim_status check_cache4(const efim_cache4_desc* c) {
  if (!c || !c->d_k_codes || !c->d_v_codes || !c->d_k_scales || !c->d_v_scales) return EFIM_ERR_INVALID_ARG;
  if (c->num_pages <= 0 || c->num_q_heads <= 0 || c->num_kv_heads <= 0) return EFIM_ERR_INVALID_ARG;
  if (c->num_q_heads % c->num_kv_heads != 0) return EFIM_ERR_INVALID_ARG;
  if (c->num_kv_heads > 32767) return EFIM_ERR_UNSUPPORTED;
  if ((long long)c->num_pages * c->num_kv_heads > 0x7fffffffLL) return EFIM_ERR_UNSUPPORTED;
  if (c->page_size != 16) return EFIM_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return EFIM_ERR_UNSUPPORTED;
  if ((reinterpret_cast<uintptr_t>(c->d_k_codes) | reinterpret_cast<uintptr_t>(c->d_v_codes) |
       reinterpret_cast<uintptr_t>(c->d_k_scales) | reinterpret_cast<uintptr_t>(c->d_v_scales)) & 127)
    return EFIM_ERR_INVALID_ARG;
  return good_pool_scale(c->k_scale) && good_pool_scale(c->v_scale) ? EFIM_OK : EFIM_ERR_INVALID_ARG;
}

// bytes of one (page, kv head): 16 tokens' codes, and their scales
__host__ __device__ constexpr int kv4_code_bytes(int D) { return 16 * D / 2; }
__host__ __device__ constexpr int kv4_scale_bytes(int D) { return 16 * D / 16; }

// two 8-bit scales (the low 16 bits) as fp16
__device__ __forceinline__ uint32_t scales_to_half2(uint32_t two) {
  uint32_t r;
  asm("{\n.reg .b16 h;\ncvt.u16.u32 h, %1;\ncvt.rn.f16x2.e4m3x2 %0, h;\n}" : "=r"(r) : "r"(two));
  return r;
}
// the eight codes of a word as fp16: pair i is codes 2i (low half) and 2i + 1
__device__ __forceinline__ void codes_to_half2(uint32_t word, uint32_t* r) {
  asm("{\n.reg .b8 a, b, c, d;\nmov.b32 {a, b, c, d}, %4;\ncvt.rn.f16x2.e2m1x2 %0, a;\ncvt.rn.f16x2.e2m1x2 %1, b;\n"
      "cvt.rn.f16x2.e2m1x2 %2, c;\ncvt.rn.f16x2.e2m1x2 %3, d;\n}"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(word));
}
__device__ __forceinline__ __half2 as_half2(uint32_t x) { return *reinterpret_cast<const __half2*>(&x); }
__device__ __forceinline__ uint32_t mul_half2(uint32_t a, __half2 b) {
  const __half2 r = __hmul2(as_half2(a), b);
  return *reinterpret_cast<const uint32_t*>(&r);
}

// a word of codes (8 values of one block) as bf16
__device__ __forceinline__ uint4 kv4_to_bf16(uint32_t codes, uint32_t scale_byte, float g) {
  const float s = __half2float(__ushort_as_half((unsigned short)scales_to_half2(scale_byte))) * g;
  uint32_t h[4], r[4];
  codes_to_half2(codes, h);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 f = __half22float2(as_half2(h[e]));
    r[e] = pack_bf16x2(f.x * s, f.y * s);
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}

// Page `page` of all heads, keys and values, to page `to` of two bf16 pools (either may be null), by the threads of a CTA: a word of codes, 16 bytes of the
// result, a thread, so that neighbours read and write side by side; four of them on their way.
template <int D, int THREADS>
__device__ __forceinline__ void kv4_page_to_bf16(const uint8_t* k_codes, const uint8_t* v_codes, const uint8_t* k_scales, const uint8_t* v_scales,
                                                 float k_scale, float v_scale, size_t page, size_t to, int Hkv, uint16_t* k_out, uint16_t* v_out) {
  constexpr int AT_ONCE = 4;
  const int words = Hkv * (16 * D / 8);               // of a pool's page
#pragma unroll
  for (int pool = 0; pool < 2; ++pool) {
    uint4* out = reinterpret_cast<uint4*>(pool ? v_out : k_out);
    if (!out) continue;
    const uint32_t* codes = reinterpret_cast<const uint32_t*>(pool ? v_codes : k_codes) + page * words;
    const uint8_t* scales = (pool ? v_scales : k_scales) + page * (words / 2);
    const float g = pool ? v_scale : k_scale;
    out += to * words;
    for (int u0 = threadIdx.x; u0 < words; u0 += AT_ONCE * THREADS) {
      uint32_t w[AT_ONCE], s[AT_ONCE];
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i)
        if (u0 + i * THREADS < words) {
          w[i] = *(codes + u0 + i * THREADS);
          s[i] = *(scales + (u0 + i * THREADS) / 2);
        }
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i)
        if (u0 + i * THREADS < words) out[u0 + i * THREADS] = kv4_to_bf16(w[i], s[i], g);
    }
  }
}

}  // namespace efim
