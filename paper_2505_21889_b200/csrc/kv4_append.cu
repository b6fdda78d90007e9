// efim_kv4_append: the new tokens' q and k normalised (where the model does that) and rotated, k and v put into the pages of a 4-bit
// cache; efim_kv4_unpack: pages of such a cache as bf16.
#include "kv4.cuh"
#include "token_place.cuh"
#include <float.h>
#include <algorithm>
#include <type_traits>

namespace efim {

struct Kv4AppendParams {
  const uint16_t* q;        // rows of [Hq][D], q_stride elements apart; may be null
  const uint16_t* k;        // rows of [Hkv][D]
  const uint16_t* v;
  long long q_stride, k_stride, v_stride;
  uint16_t* q_out;          // [T][Hq][D]
  uint8_t *k_codes, *v_codes;       // [pages][Hkv][16][D/2]
  uint8_t *k_scales, *v_scales;     // [pages][Hkv][16][D/16]
  const void* q_weight;     // [D] bf16 or fp32, or null
  const void* k_weight;
  const int32_t* cached_len;
  const int32_t* q_indptr;
  const int32_t* block_table;
  const float* cos_sin;     // [max_position][D] or null
  int32_t* status;
  float eps, weight_offset, k_inv, v_inv;   // the pools' scales, inverted
  float key_error;          // how far fp32 may be off in a key, of the terms it is the sum of
  int batch, max_pages_per_seq, total_new_tokens;
  int num_pages, Hq, Hkv, max_position, interleaved, weight_f32, normed;
  int warps;                // of a token
  int ahead;                // a token's rows are sent for into L2 by its first and last warp
  int early_next;           // let the next kernel start its set-up while this one runs
};

constexpr int KV4_APPEND_THREADS = 256, KV4_APPEND_CTAS = 3;     // threads; CTAs that an SM holds, by 80 registers

// A value that is the same in a warp's lanes, in a form that tells the compiler so: what depends on it is computed once a warp.
__device__ __forceinline__ int kv4_uniform(int x) { return __reduce_max_sync(0xffffffffu, x); }

// 8 weights from position d on, as the products take them
__device__ __forceinline__ void kv4_load_weights(const void* weight, int f32, float offset, int d, float2* w) {
  if (!weight) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = make_float2(1.f, 1.f);
    return;
  }
  if (f32) {
    const float4* src = reinterpret_cast<const float4*>(static_cast<const float*>(weight) + d);
    const float4 u = src[0], v = src[1];
    w[0] = make_float2(u.x, u.y);
    w[1] = make_float2(u.z, u.w);
    w[2] = make_float2(v.x, v.y);
    w[3] = make_float2(v.z, v.w);
  } else {
    const uint4 u = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(weight) + d);
    const uint32_t p[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = make_float2(bf16lo(p[i]), bf16hi(p[i]));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = add2(w[i], make_float2(offset, offset));
}

// Eight of a block's sixteen values (bf16 numbers; the other eight are the neighbour lane's) to a word of codes and the block's scale.
// Rounding without divisions.  The largest value a is compared with 6 g times the borders between scales, and each x with the borders t s g
// between codes: all of these are numbers of at most 8 significant bits, so two of them are equal or at least 2^-8 of them apart.  The
// quotients a / (6 g) and x / (s g), as products with approximate inverses, are within 2^-21; rounded, to 14 significant bits and to a
// multiple of 2^-12 (by the sum with 3/2 2^11), they are a border where it is one, else on the right side of it.
__device__ __forceinline__ uint32_t kv4_quantize(const uint32_t* w, float inv_g, uint32_t* scale) {
  float2 x[4];
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = make_float2(bf16lo(w[i]), bf16hi(w[i]));
    top = max_nan(max_nan(top, fabsf(x[i].x)), fabsf(x[i].y));
  }
  top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 1));
  const float quotient = top * (inv_g * 0.16666667f);
  float s = __uint_as_float((__float_as_uint(quotient) + 0x200u) & ~0x3ffu);
  if (!(s >= 0.001953125f)) s = top == top ? 0.001953125f : top;              // (a NaN stays: the block is NaN)
  uint32_t s8, sf;
  asm("{\n.reg .b16 h;\ncvt.rn.satfinite.e4m3x2.f32 h, %2, %3;\ncvt.u32.u16 %0, h;\ncvt.rn.f16x2.e4m3x2 %1, h;\n}"
      : "=r"(s8), "=r"(sf) : "f"(0.f), "f"(s));
  *scale = s8 & 0xff;
  float inv_s;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv_s) : "f"(__half2float(__ushort_as_half((unsigned short)sf))));
  inv_s *= inv_g;                                                              // (a power of two)
  constexpr float TO_GRID = 1.5f * 2048.f;
  float y[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 z = add2(add2(mul2(x[i], make_float2(inv_s, inv_s)), make_float2(TO_GRID, TO_GRID)), make_float2(-TO_GRID, -TO_GRID));
    y[2 * i] = copysignf(z.x, x[i].x);
    y[2 * i + 1] = copysignf(z.y, x[i].y);
  }
  uint32_t codes;
  asm("{\n.reg .b8 a, b, c, d;\ncvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\ncvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\ncvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\nmov.b32 %0, {a, b, c, d};\n}"
      : "=r"(codes) : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
  return codes;
}

// A lane's 16 values of a head as codes and scales.
struct Kv4Codes { uint32_t c0, c1, s0, s1; };
__device__ __forceinline__ Kv4Codes kv4_quantize_both(const uint32_t* w, float inv_g) {
  Kv4Codes z;
  z.c0 = kv4_quantize(w, inv_g, &z.s0);
  z.c1 = kv4_quantize(w + 4, inv_g, &z.s1);
  return z;
}

// A key by its definition: normed and rotated in 64 bits, rounded to fp32 and that to bf16.  `row` and `cs` (or null) are the lane's first vector of
// the head and its first rotary value.  Called by whole warps.
template <int D>
__device__ __forceinline__ Kv4Codes kv4_key_in_64_bits(const uint4* row, const void* weight, const float* cs, int j, int normed, int weight_f32,
                                                    int interleaved, float eps, float offset, float inv_g) {
  constexpr int HALF = D / 16;
  const uint4 a = row[0], b = row[HALF];
  const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  double r = 1.;
  if (normed) {
    double ss = 0.;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double lo = bf16lo(w[e]), hi = bf16hi(w[e]);
      ss = fma(lo, lo, fma(hi, hi, ss));
    }
#pragma unroll
    for (int d = HALF / 2; d > 0; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
    r = rsqrt(ss / D + eps);
  }
  auto value = [&](int e, int odd) {                     // of w[e]: dim 2e + odd of the lane's first eight, then of its second
    double x = odd ? bf16hi(w[e]) : bf16lo(w[e]);
    if (normed) {
      x *= r;
      if (weight) {
        const int d = (j + e / 4 * HALF) * 8 + e % 4 * 2 + odd;
        x *= (weight_f32 ? (double)static_cast<const float*>(weight)[d] : (double)bf16lo(static_cast<const uint16_t*>(weight)[d])) + offset;
      }
    }
    return x;
  };
  uint32_t y[8];
  if (!cs) {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = pack_bf16x2((float)value(e, 0), (float)value(e, 1));
  } else if (interleaved) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double x0 = value(e, 0), x1 = value(e, 1), c = cs[e / 4 * (D / 4) + e % 4], s = cs[D / 2 + e / 4 * (D / 4) + e % 4];
      y[e] = pack_bf16x2((float)(x0 * c - x1 * s), (float)(x1 * c + x0 * s));
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float lo[2], hi[2];
#pragma unroll
      for (int odd = 0; odd < 2; ++odd) {
        const double x0 = value(e, odd), x1 = value(4 + e, odd), c = cs[2 * e + odd], s = cs[D / 2 + 2 * e + odd];
        lo[odd] = (float)(x0 * c - x1 * s);
        hi[odd] = (float)(x1 * c + x0 * s);
      }
      y[e] = pack_bf16x2(lo[0], lo[1]);
      y[4 + e] = pack_bf16x2(hi[0], hi[1]);
    }
  }
  return kv4_quantize_both(y, inv_g);
}

// A token's q, k and v heads go to its warps in groups of 512 / D heads.  A lane holds vector j of a head row and its partner
// j + D/16, as in efim_qk_norm_append, so either pairing of the rotation stays inside the lane; two neighbours hold a block of sixteen.
//
// Keys are what norm and rotation give in 64 bits, in codes: whole numbers, so an error of fp32 next to a border is a code off, or a block.  fp32 knows how far
// it may be off (key_error); where both ends of that have the same codes and scales they are the key's, else the group of heads is done again in
// 64 bits behind the loop.  At 32/8 heads x 128 with norms three groups of keys in four have a value whose ends round to different bf16 numbers (without, one in three), one in 160
// has ends of different codes (one in 700).
//
// Bound: with many tokens the instructions (75 % of the issue slots): 25,600 tokens at 32/8 heads x 128 with norms 113 us (5.0 TB/s), 102 by keys in fp32.
// What brought it there, as replayed from a graph, keys in fp32: warp-wide values marked as such 118 -> 113, rows sent for ahead 111, a warp a
// token instead of three 102.  Of the 64 bits: every group whose ends round differently again 143, those of different codes 124 (a call inside the loop)
// -> 117 (behind the loop) -> 113 (in line).  Timed by events around single calls: divisions and value by value 134, neither 125; all keys in
// 64 bits 179.  Not kept: 64 registers (four CTAs an SM, 48 bytes spilled) 115 where 78 registers took 113; a promise of three CTAs to the compiler, which then
// takes 76 registers instead of 80 and more instructions, 125.
// With few tokens a chain of dependent loads: 64 tokens at 28/4 3.0 us.
template <int D>
__global__ void __launch_bounds__(KV4_APPEND_THREADS) kv4_append_kernel(const Kv4AppendParams p) {
  constexpr int HALF = D / 16;                  // lanes that have a head
  constexpr int HW = 32 / HALF;
  const int lane = threadIdx.x & 31;
  const int flat = blockIdx.x * (KV4_APPEND_THREADS / 32) + kv4_uniform(threadIdx.x >> 5);
  const int t = flat / p.warps, part = flat % p.warps;
  pdl_wait();
  if (p.early_next) pdl_launch();
  if (t >= p.total_new_tokens || t >= *(p.q_indptr + p.batch)) return;
  const int nq = p.q ? p.Hq : 0, nk = nq + p.Hkv, nh = nk + p.Hkv;
  const int j = lane % HALF, sub = lane / HALF, step = p.warps * HW;
  const uint4* qin = reinterpret_cast<const uint4*>(p.q + (p.q ? t * p.q_stride : 0)) + j;
  const uint4* kin = reinterpret_cast<const uint4*>(p.k + t * p.k_stride) + j;
  const uint4* vin = reinterpret_cast<const uint4*>(p.v + t * p.v_stride) + j;
  uint4 a, b;
  auto fetch = [&](int h) {
    a = b = make_uint4(0, 0, 0, 0);
    if (h < nh) {
      const uint4* row = h < nq ? qin + h * (D / 8) : h < nk ? kin + (h - nq) * (D / 8) : vin + (h - nk) * (D / 8);
      a = ldg_stream(row);
      b = ldg_stream(row + HALF);
    }
  };
  const int base0 = part * HW;
  if (p.ahead && lane == 0) {
    if (part == 0 && p.q) prefetch_l2(p.q + t * p.q_stride, nq * D * 2LL);
    if (part == p.warps - 1) {
      prefetch_l2(p.k + t * p.k_stride, p.Hkv * D * 2LL);
      prefetch_l2(p.v + t * p.v_stride, p.Hkv * D * 2LL);
    }
  }
  fetch(base0 + sub);
  const TokenPlace at = find_token(p.q_indptr, p.cached_len, p.batch, t, lane);
  const int pos = kv4_uniform(at.pos), page_idx = pos >> 4;
  const bool in_table = !p.cos_sin || (pos >= 0 && pos < p.max_position);
  bool placed = pos >= 0 && page_idx < p.max_pages_per_seq && in_table;   // k and v have a place in the cache
  int page = 0;
  if (!placed) {
    if (lane == 0 && p.status) atomicOr(p.status, EFIM_DEV_BAD_POSITION);
  } else {
    page = *(p.block_table + (size_t)at.seq * p.max_pages_per_seq + page_idx);
  }
  float2 c[4], s[4];
  float key_error = p.key_error;                // times |x| + |y| of a pair: how far its rotated values may be off
  if (p.cos_sin && in_table) {
    // 8 pairs: (f, f + D/2) from f = 8 j on, or the 4 + 4 neighbours of the two vectors
    const float* cs = p.cos_sin + (size_t)pos * D + j * (p.interleaved ? 4 : 8);
    const int second = p.interleaved ? D / 4 : 4;
    auto four = [](const float* src, float2* to) {
      const float4 u = *reinterpret_cast<const float4*>(src);
      to[0] = make_float2(u.x, u.y);
      to[1] = make_float2(u.z, u.w);
    };
    four(cs, c);
    four(cs + second, c + 2);
    four(cs + D / 2, s);
    four(cs + D / 2 + second, s + 2);
    float most = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) most = fmaxf(most, fmaxf(fmaxf(fabsf(c[e].x), fabsf(c[e].y)), fmaxf(fabsf(s[e].x), fabsf(s[e].y))));
    key_error *= most;
  }
  if (placed && (page < 0 || page >= p.num_pages)) {
    if (lane == 0 && p.status) atomicOr(p.status, EFIM_DEV_BAD_PAGE);
    placed = false;
  }
  const size_t row0 = (size_t)page * p.Hkv * 16 + (pos & 15);              // + h * 16: rows of the pools
  auto store = [&](int h, const Kv4Codes& z) {
    if (h >= nq && h < nh && placed) {
      const bool key = h < nk;
      const size_t row = row0 + (size_t)(h - (key ? nq : nk)) * 16;
      uint8_t* codes = (key ? p.k_codes : p.v_codes) + row * (D / 2) + j * 4;
      *reinterpret_cast<uint32_t*>(codes) = z.c0;
      *reinterpret_cast<uint32_t*>(codes + D / 4) = z.c1;
      if ((j & 1) == 0) {
        uint8_t* scales = (key ? p.k_scales : p.v_scales) + row * (D / 16) + j / 2;
        scales[0] = (uint8_t)z.s0;
        scales[D / 32] = (uint8_t)z.s1;
      }
    }
  };
  int key_group = 0;                                   // of the groups that have keys
  uint32_t again = 0;                                  // those that fp32 does not decide, a bit each (a warp has fewer than 16 groups)
#pragma unroll 1
  for (int base = base0; base < nh; base += step) {    // (the same for a warp's lanes: the sums below are the whole warp's)
    const int h = base + sub;
    uint32_t y[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    uint32_t inner[8] = {};
    const bool key = h >= nq && h < nk && placed;
    bool unsure = false, lost = false;             // fp32 does not say which bf16 number one of a key's values is; its bounds do not hold
    if (base + step < nh) fetch(h + step);
    if (base < nk) {
      float2 x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = make_float2(bf16lo(y[e]), bf16hi(y[e]));
      if (p.normed) {
        auto squares = [&]() {
          float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
          for (int e = 0; e < 8; ++e) s2 = fma2(x[e], x[e], s2);
          float ss = s2.x + s2.y;
#pragma unroll
          for (int d = HALF / 2; d > 0; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
          return ss;
        };
        float ss = squares(), eps = p.eps;
        if (__any_sync(0xffffffffu, !(ss <= FLT_MAX))) {
          // Squares of values beyond 1e18 leave fp32: such heads are taken 2^-70 as large (exact, and eps no longer counts beside
          // them).  A row with an infinity or a NaN stays what the formula makes of it.
          lost = !(ss <= FLT_MAX);
          const float down = lost ? 8.470329472543003e-22f : 1.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = mul2(x[e], make_float2(down, down));
          if (lost) eps = 0.f;
          ss = squares();
        }
        const float r = rsqrtf(fmaf(ss, 1.f / D, eps));
        const float2 rr = make_float2(r, r);
        const void* weight = h < nq ? p.q_weight : p.k_weight;
        float2 w[4];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          kv4_load_weights(weight, p.weight_f32, p.weight_offset, (j + half * HALF) * 8, w);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[4 * half + e] = mul2(mul2(x[4 * half + e], rr), w[e]);
        }
      }
      // Rotation and rounding.  Of a key y is what a value becomes that is as much larger as fp32 may be off, `inner` one that is as much smaller.
      auto turn = [&](auto is_key) {
        constexpr bool KEY = decltype(is_key)::value;
        float2 terms = make_float2(0.f, 0.f);
        auto round = [&](int e, float2 v, float2 t) {
          if (!KEY) {
            y[e] = pack_bf16x2(v.x, v.y);
          } else {
            const float2 off = mul2(t, make_float2(copysignf(key_error, v.x), copysignf(key_error, v.y)));
            const float2 far = add2(v, off), near = sub2(v, off);
            y[e] = pack_bf16x2(far.x, far.y);
            inner[e] = pack_bf16x2(near.x, near.y);
            unsure |= y[e] != inner[e];
          }
        };
        if (!p.cos_sin) {
          if (p.normed) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float2 t = make_float2(fabsf(x[e].x), fabsf(x[e].y));
              terms = add2(terms, t);
              round(e, x[e], t);
            }
          }
        } else if (!in_table) {
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = 0;     // no rotation for this row: a query of zeros
        } else if (!p.interleaved) {
          const float2 minus = make_float2(-1.f, -1.f);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 lo = fma2(x[e], c[e], mul2(mul2(x[4 + e], s[e]), minus)), hi = fma2(x[4 + e], c[e], mul2(x[e], s[e]));
            const float2 t = make_float2(fabsf(x[e].x) + fabsf(x[4 + e].x), fabsf(x[e].y) + fabsf(x[4 + e].y));
            terms = add2(terms, t);
            round(e, lo, t);
            round(4 + e, hi, t);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float ce = e % 2 ? c[e / 2].y : c[e / 2].x, se = e % 2 ? s[e / 2].y : s[e / 2].x, t = fabsf(x[e].x) + fabsf(x[e].y);
            round(e, make_float2(fmaf(x[e].x, ce, -(x[e].y * se)), fmaf(x[e].y, ce, x[e].x * se)), make_float2(t, t));
            terms = add2(terms, make_float2(t, t));
          }
        }
        if (KEY) {
          const float sum = terms.x + terms.y;
          lost |= !(sum <= 1.2676506e30f);          // 2^100: beyond it products with a scaled table's values may leave fp32
          if (sum == 0.f) unsure = false;           // (zeros, whatever their signs)
        }
      };
      if (h < nq) turn(std::false_type());
      else if (h < nk) turn(std::true_type());     // (a value stays as it is)
      if (h < nq) {
        uint4* dst = reinterpret_cast<uint4*>(p.q_out + ((size_t)t * p.Hq + h) * D + j * 8);
        dst[0] = make_uint4(y[0], y[1], y[2], y[3]);
        dst[HALF] = make_uint4(y[4], y[5], y[6], y[7]);
      }
    }
    if (base + HW <= nq) continue;                 // query heads alone
    const float inv = h < nk ? p.k_inv : p.v_inv;
    const Kv4Codes z = kv4_quantize_both(y, inv);
    store(h, z);
    if (base >= nk) continue;
    if (__any_sync(0xffffffffu, key && (unsure || lost))) {
      // Codes and scales rise with their values' sizes: where those of both ends are the same, so are those between them.
      const Kv4Codes u = kv4_quantize_both(inner, inv);
      if (__any_sync(0xffffffffu, key && (lost || z.c0 != u.c0 || z.c1 != u.c1 || z.s0 != u.s0 || z.s1 != u.s1))) again |= 1u << key_group;
    }
    ++key_group;
  }
  if (again) {
    key_group = 0;
#pragma unroll 1
    for (int base = base0; base < nk; base += step) {
      if (base + HW <= nq) continue;
      if (again >> key_group++ & 1) {
        const int h = base + sub;
        const bool key = h >= nq && h < nk && placed;
        const Kv4Codes z = kv4_key_in_64_bits<D>(kin + (key ? h - nq : 0) * (D / 8), p.k_weight,
                                                 p.cos_sin && in_table ? p.cos_sin + (size_t)pos * D + j * (p.interleaved ? 4 : 8) : nullptr, j, p.normed,
                                                 p.weight_f32, p.interleaved, p.eps, p.weight_offset, p.k_inv);
        if (key) store(h, z);
      }
    }
  }
}

// ---- pages read back
struct Kv4UnpackParams {
  const uint8_t *k_codes, *v_codes, *k_scales, *v_scales;
  uint16_t *k_out, *v_out;          // [n][Hkv][16][D] bf16; either may be null
  const int32_t* pages;
  int32_t* status;
  float k_scale, v_scale;
  int num_pages, Hkv;
};

constexpr int KV4_UNPACK_THREADS = 256;

// One page a CTA.  Bound: HBM's writes (1,600 pages of 8 heads x 128, 134 MB: 23 us; 16 bytes of codes a thread, 64 of the result, 34).
template <int D>
__global__ void __launch_bounds__(KV4_UNPACK_THREADS) kv4_unpack_kernel(const Kv4UnpackParams p) {
  pdl_wait();
  pdl_launch();
  const int i = blockIdx.x;
  const int page = p.pages[i];
  if (page < 0 || page >= p.num_pages) {
    if (threadIdx.x == 0 && p.status) atomicOr(p.status, EFIM_DEV_BAD_PAGE);
    return;
  }
  kv4_page_to_bf16<D, KV4_UNPACK_THREADS>(p.k_codes, p.v_codes, p.k_scales, p.v_scales, p.k_scale, p.v_scale, page, i, p.Hkv, p.k_out, p.v_out);
}

}  // namespace efim

extern "C" efim_status efim_kv4_append(const efim_cache4_desc* cache, const efim_batch_desc* batch, const efim_qk_norm_desc* norm,
                                       const efim_rope_desc* rope, const void* d_q, int64_t q_stride, const void* d_k, int64_t k_stride,
                                       const void* d_v, int64_t v_stride, void* d_q_out, int32_t* d_status, void* stream) {
  using namespace efim;
  efim_status st = check_cache4(cache);
  if (st != EFIM_OK) return st;
  if (!batch) return EFIM_ERR_INVALID_ARG;
  st = check_batch(nullptr, batch, false);
  if (st != EFIM_OK) return st;
  if (norm && (!(norm->eps > 0.f) || !(norm->eps <= FLT_MAX) || (norm->weight_f32 != 0 && norm->weight_f32 != 1))) return EFIM_ERR_INVALID_ARG;
  if (batch->batch == 0 || batch->total_new_tokens == 0) return EFIM_OK;
  const long long D = cache->head_dim, q_row = cache->num_q_heads * D, kv_row = cache->num_kv_heads * D, T = batch->total_new_tokens;
  auto address = [](const void* x) { return reinterpret_cast<uintptr_t>(x); };
  if (!d_k || !d_v || !d_q != !d_q_out) return EFIM_ERR_INVALID_ARG;
  if ((address(d_q) | address(d_k) | address(d_v) | address(d_q_out)) & 15) return EFIM_ERR_INVALID_ARG;
  if (norm && ((address(norm->d_q_weight) | address(norm->d_k_weight)) & 15)) return EFIM_ERR_INVALID_ARG;
  if ((d_q && (q_stride < q_row || q_stride % 8)) || k_stride < kv_row || k_stride % 8 || v_stride < kv_row || v_stride % 8)
    return EFIM_ERR_INVALID_ARG;
  if (rope && rope->d_cos_sin && (rope->max_position <= 0 || (address(rope->d_cos_sin) & 15))) return EFIM_ERR_INVALID_ARG;
  if (d_q) {
    // Rows of the result must not lie where another token's are still to be read: in place (packed rows), or apart.
    const uintptr_t lo = address(d_q_out), hi = lo + T * q_row * 2;
    auto meets = [&](const void* x, long long stride, long long row) {
      return address(x) < hi && lo < address(x) + ((T - 1) * stride + row) * 2;
    };
    const bool in_place = d_q_out == d_q && q_stride == q_row;
    if ((!in_place && meets(d_q, q_stride, q_row)) || meets(d_k, k_stride, kv_row) || meets(d_v, v_stride, kv_row))
      return EFIM_ERR_INVALID_ARG;
  }
  Kv4AppendParams p{};
  p.q = static_cast<const uint16_t*>(d_q);
  p.k = static_cast<const uint16_t*>(d_k);
  p.v = static_cast<const uint16_t*>(d_v);
  p.q_stride = q_stride;
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.q_out = static_cast<uint16_t*>(d_q_out);
  p.k_codes = static_cast<uint8_t*>(cache->d_k_codes);
  p.v_codes = static_cast<uint8_t*>(cache->d_v_codes);
  p.k_scales = static_cast<uint8_t*>(cache->d_k_scales);
  p.v_scales = static_cast<uint8_t*>(cache->d_v_scales);
  p.k_inv = 1.f / cache->k_scale;
  p.v_inv = 1.f / cache->v_scale;
  if (norm) {
    p.normed = 1;
    p.q_weight = norm->d_q_weight;
    p.k_weight = norm->d_k_weight;
    p.weight_f32 = norm->weight_f32;
    p.weight_offset = norm->weight_offset;
    p.eps = norm->eps;
  }
  // Bounds of the error of fp32, u = 2^-24: the rotation's product and sum 2 u of |a c| + |b s|; a norm before them 13.5 u (twelve sums of squares and the mean 13 u, of
  // which the inverse root has half and 4 u of its own, a weight's sum, two products).
  p.key_error = norm ? 9.5367431640625e-07f : 2.384185791015625e-07f;          // 16 u, 4 u
  p.cached_len = batch->d_cached_len;
  p.q_indptr = batch->d_q_indptr;
  p.block_table = batch->d_block_table;
  if (rope && rope->d_cos_sin) {
    p.cos_sin = rope->d_cos_sin;
    p.max_position = rope->max_position;
    p.interleaved = rope->interleaved;
  }
  p.status = d_status;
  p.batch = batch->batch;
  p.max_pages_per_seq = batch->max_pages_per_seq;
  p.total_new_tokens = batch->total_new_tokens;
  p.num_pages = cache->num_pages;
  p.Hq = cache->num_q_heads;
  p.Hkv = cache->num_kv_heads;
  const int hw = 512 / D, heads = (d_q ? cache->num_q_heads : 0) + 2 * cache->num_kv_heads, groups = (heads + hw - 1) / hw;
  const long long resident = (long long)KV4_APPEND_CTAS * (KV4_APPEND_THREADS / 32) * sm_count();
  // Warps of a token: as many as are resident at once, up to one for every group of heads; with more tokens one, or from 16 groups on one for every ten.
  // Microseconds with 1 / 2 / 3 / 4: 25,600 tokens at 32/8 heads x 128 (12 groups) 113 / 117 / 125 / 137, 12,800 at 64/8 (20) 98 / 92 / 93 / 99, at 32/32 (24) 126 / 126 /
  // 128 / 129; 592 tokens at 32/8 with 6 warps 6.4, with 8, a few of which are a second wave, 8.3, 1,184 with 3 8.5, with 4 10.8.
  // Rows sent for ahead where there are several waves: 25,600 at 28/4 84 -> 72, with norms 88 -> 84.
  // (No warp has more than 15 groups: the kernel marks them in a word.)
  p.warps = (int)std::min<long long>(groups, std::max<long long>(groups >= 16 ? (groups + 9) / 10 : 1, resident / T));
  const long long ctas = (T * p.warps + KV4_APPEND_THREADS / 32 - 1) / (KV4_APPEND_THREADS / 32);
  if (ctas > 0x7fffffffLL / (KV4_APPEND_THREADS / 32)) return EFIM_ERR_UNSUPPORTED;    // (warps are counted in 32 bits)
  p.ahead = T * p.warps > 4 * resident;
  p.early_next = ctas <= sm_count();
  auto launch = [&](auto kernel) {
    return launch_pdl(kernel, dim3((unsigned)ctas), dim3(KV4_APPEND_THREADS), 0, static_cast<cudaStream_t>(stream), p);
  };
  EFIM_CUDA_TRY(D == 128 ? launch(kv4_append_kernel<128>) : launch(kv4_append_kernel<64>));
  return EFIM_OK;
}

extern "C" efim_status efim_kv4_unpack(const efim_cache4_desc* cache, const int32_t* d_pages, int32_t num, void* d_k_out, void* d_v_out,
                                       int32_t* d_status, void* stream) {
  using namespace efim;
  const efim_status st = check_cache4(cache);
  if (st != EFIM_OK) return st;
  if (num < 0) return EFIM_ERR_INVALID_ARG;
  if (num == 0) return EFIM_OK;
  if (!d_pages || (!d_k_out && !d_v_out) || ((reinterpret_cast<uintptr_t>(d_k_out) | reinterpret_cast<uintptr_t>(d_v_out)) & 15))
    return EFIM_ERR_INVALID_ARG;
  Kv4UnpackParams p{};
  p.k_codes = static_cast<const uint8_t*>(cache->d_k_codes);
  p.v_codes = static_cast<const uint8_t*>(cache->d_v_codes);
  p.k_scales = static_cast<const uint8_t*>(cache->d_k_scales);
  p.v_scales = static_cast<const uint8_t*>(cache->d_v_scales);
  p.k_out = static_cast<uint16_t*>(d_k_out);
  p.v_out = static_cast<uint16_t*>(d_v_out);
  p.pages = d_pages;
  p.status = d_status;
  p.k_scale = cache->k_scale;
  p.v_scale = cache->v_scale;
  p.num_pages = cache->num_pages;
  p.Hkv = cache->num_kv_heads;
  EFIM_CUDA_TRY(cache->head_dim == 128 ? launch_pdl(kv4_unpack_kernel<128>, dim3(num), dim3(KV4_UNPACK_THREADS), 0, static_cast<cudaStream_t>(stream), p)
                                       : launch_pdl(kv4_unpack_kernel<64>, dim3(num), dim3(KV4_UNPACK_THREADS), 0, static_cast<cudaStream_t>(stream), p));
  return EFIM_OK;
}
