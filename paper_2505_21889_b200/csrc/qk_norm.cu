// efim_qk_norm_append: what efim_kv_append does, for models that normalise every query and key head before the rotation: root
// mean square norm of a head's values, weight, rotation by the position and the scatter of k/v into the paged cache, in one pass
// over the projection's output.  q, k and v may be views of one buffer (rows further apart than they are long).
//
//   y_d = x_d (mean_e x_e^2 + eps)^(-1/2) (w_d + offset),  then the pairs of y are rotated; one rounding to bf16 at the end.
#include "token_place.cuh"
#include <float.h>
#include <algorithm>

namespace efim {

struct QkNormParams {
  const uint16_t* q;        // rows of [Hq][D], q_stride elements apart; may be null
  const uint16_t* k;        // rows of [Hkv][D]
  const uint16_t* v;
  long long q_stride, k_stride, v_stride;
  uint16_t* q_out;          // [T][Hq][D]
  uint16_t* k_pool;         // [pages][Hkv][16][D]
  uint16_t* v_pool;
  const void* q_weight;     // [D] bf16 or fp32, or null
  const void* k_weight;
  const int32_t* cached_len;
  const int32_t* q_indptr;
  const int32_t* block_table;
  const float* cos_sin;     // [max_position][D] or null
  int32_t* status;
  float eps, weight_offset;
  int batch, max_pages_per_seq, total_new_tokens;
  int num_pages, Hq, Hkv, max_position, interleaved, weight_f32;
  int warps;                // of a token
  int ahead;                // a token's rows are sent for into L2 by its first and last warp
  int early_next;           // let the next kernel start its set-up while this one runs
};

constexpr int QK_NORM_THREADS = 256;

// A value that is the same in a warp's lanes, in a form that tells the compiler so (it cannot know of the warp's index): what depends
// on it is computed once a warp, and its branches are not compiled for lanes that part.
__device__ __forceinline__ int uniform(int x) { return __reduce_max_sync(0xffffffffu, x); }

// 8 weights from position d on, as the products take them
__device__ __forceinline__ void load_weights(const void* weight, int f32, float offset, int d, float2* w) {
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

// A token's q and k heads go to its warps (WARPS, or p.warps where that is 0) in groups of HW = 512 / D, v's vectors, which are
// copied, to their lanes.  A lane holds vector j of a head row and its partner j + D/16 (16 values), so D/16 lanes have a head: the sum of
// squares is 16 products in a lane and log2(D/16) shuffles, and either pairing of the rotation stays inside the lane, whose rotary
// values are loaded once.  A warp's first rows are on their way before its token's sequence is looked up, then the next group's while
// one is computed.
//
// Bound: HBM with many tokens (25,600 at 32/8 heads x 128: 99 us, 6.4 TB/s), and close to it the instructions (2.8 a clock, with the products
// two at a time; one by one 15 % more of them and 1 us): 64 registers and four CTAs an SM even with a few bytes spilled (three CTAs 2-5 %
// longer with many tokens, two 16 %), weights taken from L1 when they are needed (held in registers the kernel spilled and took 25 %
// longer, in shared memory as fp32 5 %), warp-wide values marked as such.
// Not kept: a warp that walks several tokens in a row (code of one loop more: 40 % longer), two groups on their way (2-3 %),
// v's heads in the groups' loop (8 %), warps of v's alone (6 %).
template <int D, int WARPS>
__global__ void __launch_bounds__(QK_NORM_THREADS, 4) qk_norm_append_kernel(const QkNormParams p) {
  constexpr int VEC = D / 8, HALF = VEC / 2;    // 16-byte vectors of a head row, lanes that have it
  constexpr int HW = 32 / HALF;
  constexpr int COPIES = WARPS == 1 ? 4 : 2;    // vectors of v in flight per lane
  const int lane = threadIdx.x & 31;
  const int flat = blockIdx.x * (QK_NORM_THREADS / 32) + uniform(threadIdx.x >> 5);
  const int warps = WARPS ? WARPS : p.warps;
  const int t = flat / warps, part = flat % warps;
  pdl_wait();
  if (p.early_next) pdl_launch();
  if (t >= p.total_new_tokens) return;
  const int nq = p.q ? p.Hq : 0, nh = nq + p.Hkv;
  const int j = lane % HALF, sub = lane / HALF, step = warps * HW;
  const uint4* qin = reinterpret_cast<const uint4*>(p.q + (p.q ? t * p.q_stride : 0)) + j;
  const uint4* kin = reinterpret_cast<const uint4*>(p.k + t * p.k_stride) + j;
  const uint4* vin = reinterpret_cast<const uint4*>(p.v + t * p.v_stride);
  const int n_vec = p.Hkv * VEC, v0 = part * 32 + lane, v_step = warps * 32;
  const int base0 = part * HW;
  uint4 a, b, v[COPIES];                        // the next head's vectors, v's
  auto fetch = [&](int h) {
    a = b = make_uint4(0, 0, 0, 0);
    if (h < nh) {
      const uint4* row = h < nq ? qin + h * VEC : kin + (h - nq) * VEC;
      a = ldg_stream(row);
      b = ldg_stream(row + HALF);
    }
  };
  auto fetch_v = [&](int u0) {
#pragma unroll
    for (int i = 0; i < COPIES; ++i)
      if (u0 + v_step * i < n_vec) v[i] = ldg_stream(vin + u0 + v_step * i);
  };
  if (p.ahead && lane == 0) {
    if (part == 0 && p.q) prefetch_l2(p.q + t * p.q_stride, nq * D * 2LL);
    if (part == warps - 1) {
      prefetch_l2(p.k + t * p.k_stride, p.Hkv * D * 2LL);
      prefetch_l2(p.v + t * p.v_stride, p.Hkv * D * 2LL);
    }
  }
  fetch(base0 + sub);
  fetch_v(v0);

  const TokenPlace at = find_token(p.q_indptr, p.cached_len, p.batch, t, lane);
  const int pos = uniform(at.pos), page_idx = pos >> 4;
  const bool in_table = !p.cos_sin || (pos >= 0 && pos < p.max_position);
  bool placed = pos >= 0 && page_idx < p.max_pages_per_seq && in_table;   // k and v have a place in the cache
  int page = 0;
  if (!placed) {
    if (lane == 0 && p.status) atomicOr(p.status, EFIM_DEV_BAD_POSITION);
  } else {
    page = *(p.block_table + (size_t)at.seq * p.max_pages_per_seq + page_idx);
  }
  float2 c[4], s[4];
  if (p.cos_sin && in_table && base0 < nh) {
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
  }
  if (placed && (page < 0 || page >= p.num_pages)) {
    if (lane == 0 && p.status) atomicOr(p.status, EFIM_DEV_BAD_PAGE);
    placed = false;
  }
  const size_t pool_tok = ((size_t)page * p.Hkv) * 16 * D + (size_t)(pos & 15) * D;   // + h * 16 * D
  if (placed) {
    for (int u0 = v0; u0 < n_vec; u0 += COPIES * v_step) {
      if (u0 != v0) fetch_v(u0);
#pragma unroll
      for (int i = 0; i < COPIES; ++i) {
        const int u = u0 + v_step * i;
        if (u < n_vec) *reinterpret_cast<uint4*>(p.v_pool + pool_tok + (size_t)(u / VEC) * 16 * D + (u % VEC) * 8) = v[i];
      }
    }
  }
  uint16_t* q_out = p.q_out + (size_t)t * p.Hq * D + j * 8;
#pragma unroll 1
  for (int base = base0; base < nh; base += step) {    // (the same for a warp's lanes: the sums below are the whole warp's)
    const int h = base + sub;
    float2 x[8];
    {
      const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = make_float2(bf16lo(w[e]), bf16hi(w[e]));
    }
    if (base + step < nh) fetch(h + step);
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
      const float down = ss <= FLT_MAX ? 1.f : 8.470329472543003e-22f;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = mul2(x[e], make_float2(down, down));
      if (down != 1.f) eps = 0.f;
      ss = squares();
    }
    if (h >= nh || (h >= nq && !placed)) continue;
    const float r = rsqrtf(fmaf(ss, 1.f / D, eps));
    const float2 rr = make_float2(r, r);
    // (from L1 after a warp's first heads: in registers beside the rotary values they made the kernel spill)
    const void* weight = h < nq ? p.q_weight : p.k_weight;
    float2 w[4];
    load_weights(weight, p.weight_f32, p.weight_offset, j * 8, w);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = mul2(mul2(x[e], rr), w[e]);
    load_weights(weight, p.weight_f32, p.weight_offset, (j + HALF) * 8, w);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[4 + e] = mul2(mul2(x[4 + e], rr), w[e]);
    uint32_t y[8];
    if (!p.cos_sin) {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = pack_bf16x2(x[e].x, x[e].y);
    } else if (!in_table) {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = 0;     // no rotation for this row: a query of zeros
    } else if (!p.interleaved) {
      const float2 minus = make_float2(-1.f, -1.f);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 lo = fma2(x[e], c[e], mul2(mul2(x[4 + e], s[e]), minus)), hi = fma2(x[4 + e], c[e], mul2(x[e], s[e]));
        y[e] = pack_bf16x2(lo.x, lo.y);
        y[4 + e] = pack_bf16x2(hi.x, hi.y);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float ce = e % 2 ? c[e / 2].y : c[e / 2].x, se = e % 2 ? s[e / 2].y : s[e / 2].x;
        y[e] = pack_bf16x2(fmaf(x[e].x, ce, -(x[e].y * se)), fmaf(x[e].y, ce, x[e].x * se));
      }
    }
    uint4* dst = reinterpret_cast<uint4*>(h < nq ? q_out + h * D : p.k_pool + pool_tok + (size_t)(h - nq) * 16 * D + j * 8);
    dst[0] = make_uint4(y[0], y[1], y[2], y[3]);
    dst[HALF] = make_uint4(y[4], y[5], y[6], y[7]);
  }
}

}  // namespace efim

extern "C" efim_status efim_qk_norm_append(const efim_cache_desc* cache, const efim_batch_desc* batch, const efim_qk_norm_desc* norm,
                                           const efim_rope_desc* rope, const void* d_q, int64_t q_stride, const void* d_k,
                                           int64_t k_stride, const void* d_v, int64_t v_stride, void* d_q_out, int32_t* d_status,
                                           void* stream) {
  using namespace efim;
  efim_status st = check_cache(cache);
  if (st != EFIM_OK) return st;
  st = check_batch(cache, batch, false);
  if (st != EFIM_OK) return st;
  if (!norm || !(norm->eps > 0.f) || !(norm->eps <= FLT_MAX) || (norm->weight_f32 != 0 && norm->weight_f32 != 1))
    return EFIM_ERR_INVALID_ARG;
  if (batch->batch == 0 || batch->total_new_tokens == 0) return EFIM_OK;
  const long long D = cache->head_dim, q_row = cache->num_q_heads * D, kv_row = cache->num_kv_heads * D, T = batch->total_new_tokens;
  auto address = [](const void* x) { return reinterpret_cast<uintptr_t>(x); };
  if (!d_k || !d_v || !d_q != !d_q_out) return EFIM_ERR_INVALID_ARG;
  if ((address(d_q) | address(d_k) | address(d_v) | address(d_q_out) | address(norm->d_q_weight) | address(norm->d_k_weight)) & 15)
    return EFIM_ERR_INVALID_ARG;
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
  QkNormParams p{};
  p.q = static_cast<const uint16_t*>(d_q);
  p.k = static_cast<const uint16_t*>(d_k);
  p.v = static_cast<const uint16_t*>(d_v);
  p.q_stride = q_stride;
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.q_out = static_cast<uint16_t*>(d_q_out);
  p.k_pool = static_cast<uint16_t*>(cache->d_k_pool);
  p.v_pool = static_cast<uint16_t*>(cache->d_v_pool);
  p.q_weight = norm->d_q_weight;
  p.k_weight = norm->d_k_weight;
  p.weight_f32 = norm->weight_f32;
  p.weight_offset = norm->weight_offset;
  p.eps = norm->eps;
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
  // Warps of a token: as many as are resident at once, up to one for every group of q's and k's heads; with more tokens one, or from
  // ten groups on one for every five.  Microseconds with 1 / 2 / 4 / 10 (or a warp per group): 64 tokens at 32/8 heads x 128 8.3 / 5.5 / 4.3 / 2.7,
  // 2,304 at 28/4 10.2 / 9.4 / 9.7 / 11.7, at 32/8 13.8 / 12.1 / 12.8 / 15.4, at 32/32 25.3 / 22.1 / 21.3 / 23.0, 12,800 at 28/4 41.9 / 43.4 / 46.2 / 57,
  // at 32/8 54.3 / 54.8 / 58.6 / 72, at 32/32 107 / 109 / 104 / 113.
  const int hw = 512 / D, heads = (d_q ? cache->num_q_heads : 0) + cache->num_kv_heads, groups = (heads + hw - 1) / hw;
  const long long resident = 4LL * (QK_NORM_THREADS / 32) * sm_count();
  p.warps = (int)std::min<long long>(groups, std::max<long long>(groups >= 10 ? (groups + 4) / 5 : 1, resident / T));
  const long long ctas = (T * p.warps + QK_NORM_THREADS / 32 - 1) / (QK_NORM_THREADS / 32);
  if (ctas > 0x7fffffffLL) return EFIM_ERR_UNSUPPORTED;
  // From several waves on, where a token has several warps: 9,600 tokens at 32/8 42.8 -> 42.0, 25,600 104 -> 99, at 32/32 206 -> 199, at 64/8 177 -> 164;
  // but 3,200 at 32/32 28.9 -> 29.9, one wave of 2,304 21.8 -> 23.1, a warp a token 12,800 at 28/4 41.9 -> 44.1.
  p.ahead = p.warps > 1 && T * p.warps > 4 * resident;
  p.early_next = ctas <= sm_count();
  auto launch = [&](auto kernel) {
    return launch_pdl(kernel, dim3((unsigned)ctas), dim3(QK_NORM_THREADS), 0, static_cast<cudaStream_t>(stream), p);
  };
  EFIM_CUDA_TRY(D == 128 ? (p.warps == 1   ? launch(qk_norm_append_kernel<128, 1>)
                            : p.warps == 2 ? launch(qk_norm_append_kernel<128, 2>)
                                           : launch(qk_norm_append_kernel<128, 0>))
                         : (p.warps == 1   ? launch(qk_norm_append_kernel<64, 1>)
                            : p.warps == 2 ? launch(qk_norm_append_kernel<64, 2>)
                                           : launch(qk_norm_append_kernel<64, 0>)));
  return EFIM_OK;
}
