// efim_qk_norm_append: what efim_kv_append does, for models that normalise every query and key head before the rotation: root
// mean square norm of a head's values, weight, rotation by the position and the scatter of k/v into the paged cache, in one pass
// over the projection's output.  q, k and v may be views of one buffer (rows further apart than they are long).
//
//   y_d = x_d (mean_e x_e^2 + eps)^(-1/2) (w_d + offset),  then the pairs of y are rotated; one rounding to bf16 at the end.
#include "token_place.cuh"
#include <float.h>

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
  int early_next;           // let the next kernel start its set-up while this one runs
};

constexpr int QK_NORM_THREADS = 256;

// 8 weights from position d on, as the products take them
__device__ __forceinline__ void load_weights(const void* weight, int f32, float offset, int d, float* w) {
  if (!weight) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 1.f;
    return;
  }
  if (f32) {
    const float4* src = reinterpret_cast<const float4*>(static_cast<const float*>(weight) + d);
    *reinterpret_cast<float4*>(w) = src[0];
    *reinterpret_cast<float4*>(w + 4) = src[1];
  } else {
    const uint4 u = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(weight) + d);
    const uint32_t p[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[2 * i] = bf16lo(p[i]);
      w[2 * i + 1] = bf16hi(p[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] += offset;
}

// WPT warps per new token.  A lane holds vector j of a head row and its partner j + D/16 (both halves of the row, 16 values), so
// D/16 lanes have a head: the sum of squares is 16 products in a lane and log2(D/16) shuffles, and either pairing of the rotation
// stays inside the lane.  Its rotary values are loaded once, its weights once for q and once for k.
template <int D, int WPT>
__global__ void __launch_bounds__(QK_NORM_THREADS, 3) qk_norm_append_kernel(const QkNormParams p) {
  constexpr int VEC = D / 8, HALF = VEC / 2;    // 16-byte vectors of a head row, lanes that have it
  constexpr int LANES = 32 * WPT;
  constexpr int HW = 32 / HALF, HP = WPT * HW;  // heads that a warp, and a token's warps, have at once
  constexpr int COPIES = WPT == 1 ? 4 : 2;      // vectors of v in flight per lane
  const int lane = threadIdx.x % LANES, wl = threadIdx.x & 31;
  const int t = blockIdx.x * (QK_NORM_THREADS / LANES) + threadIdx.x / LANES;
  pdl_wait();
  if (p.early_next) pdl_launch();
  if (t >= p.total_new_tokens) return;
  const int nq = p.q ? p.Hq : 0, nh = nq + p.Hkv, n_vec = p.Hkv * VEC;
  const uint4* qin = reinterpret_cast<const uint4*>(p.q + (p.q ? t * p.q_stride : 0));
  const uint4* kin = reinterpret_cast<const uint4*>(p.k + t * p.k_stride);
  const uint4* vin = reinterpret_cast<const uint4*>(p.v + t * p.v_stride);
  const int j = lane % HALF;
  // the warp's first head, the same for its lanes, and this lane's among the warp's
  const int base0 = (lane >> 5) * HW, sub = wl / HALF;
  uint4 a[2], b[2], v[COPIES];
  auto fetch_heads = [&](int base) {            // vectors of heads base + sub and base + sub + HP
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int h = base + sub + i * HP;
      a[i] = b[i] = make_uint4(0, 0, 0, 0);
      if (h < nh) {
        const uint4* row = (h < nq ? qin + h * VEC : kin + (h - nq) * VEC) + j;
        a[i] = ldg_stream(row);
        b[i] = ldg_stream(row + HALF);
      }
    }
  };
  auto fetch_copy = [&](int u0) {
#pragma unroll
    for (int i = 0; i < COPIES; ++i)
      if (u0 + LANES * i < n_vec) v[i] = ldg_stream(vin + u0 + LANES * i);
  };
  fetch_heads(base0);
  fetch_copy(lane);
  // what the products take from the weights, for the heads of one kind
  float w[16];
  int kind = -1;
  auto weights_for = [&](int want) {
    if (kind == want) return;
    kind = want;
    const void* weight = want ? p.k_weight : p.q_weight;
    load_weights(weight, p.weight_f32, p.weight_offset, j * 8, w);
    load_weights(weight, p.weight_f32, p.weight_offset, (j + HALF) * 8, w + 8);
  };
  weights_for(base0 + sub >= nq);

  const TokenPlace at = find_token(p.q_indptr, p.cached_len, p.batch, t, wl);
  const int pos = at.pos, page_idx = pos >> 4;
  const bool in_table = !p.cos_sin || (pos >= 0 && pos < p.max_position);
  bool placed = pos >= 0 && page_idx < p.max_pages_per_seq && in_table;   // k and v have a place in the cache
  int page = 0;
  if (!placed) {
    if (lane == 0 && p.status) atomicOr(p.status, EFIM_DEV_BAD_POSITION);
  } else {
    page = *(p.block_table + (size_t)at.seq * p.max_pages_per_seq + page_idx);
  }
  float c[8], s[8];
  if (p.cos_sin && in_table) {
    // 8 pairs: (f, f + D/2) from f = 8 j on, or the 4 + 4 neighbours of the two vectors
    const float* cs = p.cos_sin + (size_t)pos * D + j * (p.interleaved ? 4 : 8);
    const int second = p.interleaved ? D / 4 : 4;
    *reinterpret_cast<float4*>(c) = *reinterpret_cast<const float4*>(cs);
    *reinterpret_cast<float4*>(c + 4) = *reinterpret_cast<const float4*>(cs + second);
    *reinterpret_cast<float4*>(s) = *reinterpret_cast<const float4*>(cs + D / 2);
    *reinterpret_cast<float4*>(s + 4) = *reinterpret_cast<const float4*>(cs + D / 2 + second);
  }
  if (placed && (page < 0 || page >= p.num_pages)) {
    if (lane == 0 && p.status) atomicOr(p.status, EFIM_DEV_BAD_PAGE);
    placed = false;
  }
  const size_t pool_tok = ((size_t)page * p.Hkv) * 16 * D + (size_t)(pos & 15) * D;   // + h * 16 * D
  if (placed) {
    for (int u0 = lane; u0 < n_vec; u0 += COPIES * LANES) {
      if (u0 != lane) fetch_copy(u0);
#pragma unroll
      for (int i = 0; i < COPIES; ++i) {
        const int u = u0 + LANES * i;
        if (u < n_vec) *reinterpret_cast<uint4*>(p.v_pool + pool_tok + (size_t)(u / VEC) * 16 * D + (u % VEC) * 8) = v[i];
      }
    }
  }
  uint4* q_out = reinterpret_cast<uint4*>(p.q_out + (size_t)t * p.Hq * D);
  for (int base = base0; base < nh; base += 2 * HP) {
    if (base != base0) fetch_heads(base);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int h = base + sub + i * HP;
      if (base + i * HP >= nh) break;           // the whole warp
      float x[16];
      {
        const uint32_t* wa = reinterpret_cast<const uint32_t*>(&a[i]);
        const uint32_t* wb = reinterpret_cast<const uint32_t*>(&b[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[2 * e] = bf16lo(wa[e]);
          x[2 * e + 1] = bf16hi(wa[e]);
          x[8 + 2 * e] = bf16lo(wb[e]);
          x[8 + 2 * e + 1] = bf16hi(wb[e]);
        }
      }
      auto squares = [&]() {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) ss = fmaf(x[e], x[e], ss);
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
        for (int e = 0; e < 16; ++e) x[e] *= down;
        if (down != 1.f) eps = 0.f;
        ss = squares();
      }
      if (h >= nh || (h >= nq && !placed)) continue;
      const float r = rsqrtf(fmaf(ss, 1.f / D, eps));
      weights_for(h >= nq);
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = x[e] * r * w[e];
      uint32_t y[8];
      if (!p.cos_sin) {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
      } else if (!in_table) {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = 0;   // no rotation for this row: a query of zeros
      } else if (!p.interleaved) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          y[e / 2] = pack_bf16x2(fmaf(x[e], c[e], -(x[8 + e] * s[e])), fmaf(x[e + 1], c[e + 1], -(x[9 + e] * s[e + 1])));
          y[4 + e / 2] = pack_bf16x2(fmaf(x[8 + e], c[e], x[e] * s[e]), fmaf(x[9 + e], c[e + 1], x[e + 1] * s[e + 1]));
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          y[e] = pack_bf16x2(fmaf(x[2 * e], c[e], -(x[2 * e + 1] * s[e])), fmaf(x[2 * e + 1], c[e], x[2 * e] * s[e]));
      }
      uint4* dst = h < nq ? q_out + h * VEC : reinterpret_cast<uint4*>(p.k_pool + pool_tok + (size_t)(h - nq) * 16 * D);
      dst[j] = make_uint4(y[0], y[1], y[2], y[3]);
      dst[j + HALF] = make_uint4(y[4], y[5], y[6], y[7]);
    }
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
  const long long resident = 3 * sm_count();
  const long long vectors = ((d_q ? cache->num_q_heads : 0) + 2LL * cache->num_kv_heads) * (D / 8);   // of the rows that a token moves
  const int wpt = T <= resident ? 8 : T <= 2 * resident || vectors >= 1024 ? 4 : vectors >= 384 || T <= 4 * resident ? 2 : 1;
  const unsigned grid = (unsigned)((T * wpt * 32 + QK_NORM_THREADS - 1) / QK_NORM_THREADS);
  p.early_next = grid <= (unsigned)sm_count();
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  auto launch = [&](auto kernel) { return launch_pdl(kernel, dim3(grid), dim3(QK_NORM_THREADS), 0, s, p); };
  auto launch_d = [&](auto dim) {
    constexpr int DIM = decltype(dim)::value;
    return wpt == 1   ? launch(qk_norm_append_kernel<DIM, 1>)
           : wpt == 2 ? launch(qk_norm_append_kernel<DIM, 2>)
           : wpt == 4 ? launch(qk_norm_append_kernel<DIM, 4>)
                      : launch(qk_norm_append_kernel<DIM, 8>);
  };
  EFIM_CUDA_TRY(D == 128 ? launch_d(std::integral_constant<int, 128>{}) : launch_d(std::integral_constant<int, 64>{}));
  return EFIM_OK;
}
