// efim_verify_drafts: which of a step's drafted tokens the target model's distributions accept, and the token that follows them.
//
// Row i of a sequence holds the target's distribution p_i after the step's token i; the draft it judges is token i + 1, drawn from
// q_i (or with certainty).  With u_i uniform in [0, 1) and e exponential, all given:
//   draft x is accepted  iff  u_i q_i(x) < p_i(x)                     (then its distribution is min(p, q) in that branch)
//   at the first row that accepts nothing, or the last one: next = argmax_j r_j / e_j,  r = (p - q)^+ or, behind the last draft, p
// (argmax_j r_j / e_j is a draw from r / sum r: the smallest of exponential times with rates r_j.)  Together the emitted tokens are
// distributed as if the target had been sampled token by token.  At temperature 0: accepted while the draft is the row's argmax.
//
// One thread-block cluster per sequence, each CTA with a slice of the vocabulary.  It walks the rows until one refuses, so what
// lies behind a refusal is not read; per group of rows the CTAs swap their (maximum, sum, argmax) through distributed shared
// memory and all of them decide alike.  The race for the next token then runs over the slices of that one row, which its CTAs
// have just read (L2).  No workspace, nothing kept between calls.
#include "cluster.cuh"
#include <float.h>

namespace efim {

constexpr int VERIFY_THREADS = 512;
constexpr int VERIFY_WARPS = VERIFY_THREADS / 32;
constexpr int VERIFY_MAX_CTAS = 8;       // of a cluster
constexpr int VERIFY_MAX_GROUP = 8;      // rows that are looked at together

struct VerifyParams {
  const void* target;       // rows of [vocab], target_stride elements apart
  const int32_t* row_indptr;
  const int32_t* tokens;    // [total_rows]
  const float* draft_probs; // rows of [vocab], or null: drafts that are certain
  const float* uniform;     // [total_rows]
  const float* noise;       // rows of [vocab], one per sequence, or null: every sequence greedy
  const float* temperature; // [batch], or null: 1
  int32_t* accepted;
  int32_t* next_token;
  int32_t* out_tokens;      // [batch][out_stride] or null
  float* out_logprobs;      // the same
  int32_t* status;
  long long target_stride, draft_stride, noise_stride;
  int batch, total_rows, vocab, out_stride, group;
};

enum { TARGET_BF16 = EFIM_TARGET_LOGITS_BF16, TARGET_F32 = EFIM_TARGET_LOGITS_F32, TARGET_PROBS = EFIM_TARGET_PROBS_F32 };
template <int KIND> struct TargetOf { using type = float; };
template <> struct TargetOf<TARGET_BF16> { using type = uint16_t; };

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Mass of a row's values seen so far: the largest, the sum of 2^((x - m) c), and the first place of the largest (where asked for).
// A NaN among the values makes the sum NaN; values of -inf have no mass; at +inf those values share all of it.
struct Mass {
  float m, l;
  int at;
};
__device__ __forceinline__ float weight_of(float x, float m, float c) {
  if (m == INFINITY) return x == INFINITY ? 1.f : x == x ? 0.f : x;
  return exp2_fast((x - (m == -INFINITY ? 0.f : m)) * c);
}
__device__ __forceinline__ void join(Mass& a, const Mass& b, float c) {
  const float m = fmaxf(a.m, b.m);
  if (m == -INFINITY) {
    a.l += b.l;                                       // 0, or NaN
  } else {
    const float fa = weight_of(a.m, m, c), fb = weight_of(b.m, m, c);
    a.l = fmaf(a.l, fa, b.l * fb);
  }
  if (b.m > a.m || (b.m == a.m && b.at < a.at)) a.at = b.at;
  a.m = m;
}

// Adds `N` values, value e standing at place at0 + e.
template <int N>
__device__ __forceinline__ void add_values(Mass& s, const float* x, int at0, int place_step, int per_vec, float c, bool want_at) {
  float top = x[0];
#pragma unroll
  for (int e = 1; e < N; ++e) top = fmaxf(top, x[e]);
  if (top > s.m) {
    if (s.m != -INFINITY) s.l *= weight_of(s.m, top, c);
    s.m = top;
    if (want_at) {
      int at = 0x7fffffff;
#pragma unroll
      for (int e = N - 1; e >= 0; --e)
        if (x[e] == top) at = at0 + (e / per_vec) * place_step + e % per_vec;
      s.at = at;
    }
  }
  if (s.m == INFINITY) {
#pragma unroll
    for (int e = 0; e < N; ++e) s.l += weight_of(x[e], s.m, c);
  } else {
    const float m = s.m == -INFINITY ? 0.f : s.m;
#pragma unroll
    for (int e = 0; e < N; ++e) s.l += exp2_fast((x[e] - m) * c);
  }
}

// The mass of places [begin, end) of a row, by `lanes` lanes; this is lane `id` of them.
template <typename T>
__device__ __forceinline__ Mass row_mass(const T* row, int begin, int end, int id, int lanes, float c, bool want_at) {
  constexpr int EPV = 16 / sizeof(T), U = 4;          // values of a 16-byte vector, vectors in flight
  Mass s{-INFINITY, 0.f, 0x7fffffff};
  if (begin >= end) return s;
  const int n = end - begin;
  const T* p = row + begin;
  const int lead = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(T));
  const int n_vec = (n - lead) / EPV, tail = lead + n_vec * EPV;
  if (id < lead) {
    const float x = as_float(p[id]);
    add_values<1>(s, &x, begin + id, 0, 1, c, want_at);
  }
  const uint4* vec = reinterpret_cast<const uint4*>(p + lead);
  for (int v0 = id; v0 < n_vec; v0 += U * lanes) {
    uint4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (v0 + u * lanes < n_vec) {
        w[u] = ldg_stream(vec + v0 + u * lanes);
      } else {
        const uint32_t low = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;   // -inf
        w[u] = make_uint4(low, low, low, low);
      }
    }
    float x[U * EPV];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t q[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 2) {
          x[u * EPV + 2 * e] = bf16lo(q[e]);
          x[u * EPV + 2 * e + 1] = bf16hi(q[e]);
        } else {
          x[u * EPV + e] = __uint_as_float(q[e]);
        }
      }
    }
    add_values<U * EPV>(s, x, begin + lead + v0 * EPV, lanes * EPV, EPV, c, want_at);
  }
  if (tail + id < n) {                                // fewer than a vector's
    const float x = as_float(p[tail + id]);
    add_values<1>(s, &x, begin + tail + id, 0, 1, c, want_at);
  }
  return s;
}

// Times of the race: the largest r / e wins, the lowest place among equals.  0 for places that cannot win.
__device__ __forceinline__ unsigned long long race_key(float r, float e, int at) {
  const float t = r / e;
  return r > 0.f && t > 0.f ? (unsigned long long)__float_as_uint(t) << 32 | (0xffffffffu - (uint32_t)at) : 0ull;
}

struct RowResult {
  float m, l, draft_logprob;
  int at, ok;
};

template <int KIND>
__global__ void __launch_bounds__(VERIFY_THREADS, 2) verify_kernel(const VerifyParams p) {
  using T = typename TargetOf<KIND>::type;
  __shared__ __align__(16) uint4 s_part[2][VERIFY_MAX_GROUP][VERIFY_MAX_CTAS];    // of every CTA of the cluster, by turns
  __shared__ Mass s_warp[VERIFY_WARPS];
  __shared__ RowResult s_row[VERIFY_MAX_GROUP];
  __shared__ ulonglong2 s_key[VERIFY_WARPS];
  __shared__ __align__(16) ulonglong2 s_keys[VERIFY_MAX_CTAS];
  __shared__ int s_stop;

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = cluster_rank(), ctas = cluster_size();
  const int s = blockIdx.x / ctas;
  cluster_arrive();
  pdl_wait();
  pdl_launch();
  const int r0 = *(p.row_indptr + s), r1 = *(p.row_indptr + s + 1);
  const T* target = static_cast<const T*>(p.target);
  const bool rows_ok = r0 >= 0 && r1 <= p.total_rows && r0 <= r1;
  const int n = rows_ok ? r1 - r0 : 0;
  // slices are whole multiples of 16 bytes of every operand, so that they are as aligned as the rows
  const int slice = ((p.vocab + (int)ctas - 1) / (int)ctas + 63) & ~63;
  const int begin = min(p.vocab, (int)rank * slice), end = min(p.vocab, begin + slice);
  float inv = 1.f;
  bool greedy = KIND != TARGET_PROBS && !p.noise;
  if (KIND != TARGET_PROBS && p.noise && p.temperature) {
    const float t = *(p.temperature + s);
    greedy = !(t > 0.f);
    inv = greedy ? 1.f : fminf(1.f / t, FLT_MAX);
  }
  const float c = fminf(inv * 1.4426950408889634f, FLT_MAX);

  cluster_wait();

  // ---- rows until one accepts nothing
  int stop = n - 1, turn = 0, status = rows_ok ? 0 : EFIM_DEV_BAD_POSITION;
  RowResult last{};
  if (KIND == TARGET_PROBS) {
    // the rows' probabilities are there: only the drafts' are looked up
    for (int i0 = 0; i0 < n - 1; i0 += VERIFY_THREADS) {
      if (tid == 0) s_stop = n - 1;
      __syncthreads();
      const int i = i0 + tid;
      bool bad = false;
      float px = 0.f;
      if (i < n - 1) {
        const int x = *(p.tokens + r0 + i + 1);
        bad = x < 0 || x >= p.vocab;
        float q = 1.f;
        if (!bad) {
          px = as_float(target[(r0 + i) * p.target_stride + x]);
          if (p.draft_probs) q = p.draft_probs[(r0 + i) * p.draft_stride + x];
        }
        if (!(*(p.uniform + r0 + i) * q < px)) atomicMin(&s_stop, i);
      }
      __syncthreads();
      stop = s_stop;
      if (i < stop && rank == 0) {
        if (p.out_logprobs && i < p.out_stride) p.out_logprobs[(size_t)s * p.out_stride + i] = logf(px);
      }
      if (i == stop && bad && rank == 0) status |= EFIM_DEV_BAD_TOKEN;
      __syncthreads();
      if (stop < n - 1) break;
    }
  } else if (n > 0) {
    int group = p.group;
    while (group > 1 && group / 2 >= n) group /= 2;
    const int per_row = VERIFY_WARPS / group;         // warps of a row
    for (int i0 = 0; i0 < n; i0 += group, turn ^= 1) {
      const int mine = i0 + warp / per_row;
      Mass mass{-INFINITY, 0.f, 0x7fffffff};
      if (mine < n)
        mass = row_mass<T>(target + (r0 + mine) * p.target_stride, begin, end, (warp % per_row) * 32 + lane, per_row * 32, c, greedy);
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) {
        const Mass o{__shfl_xor_sync(0xffffffffu, mass.m, d), __shfl_xor_sync(0xffffffffu, mass.l, d),
                     __shfl_xor_sync(0xffffffffu, mass.at, d)};
        join(mass, o, c);
      }
      if (lane == 0) s_warp[warp] = mass;
      __syncthreads();
      // warp w sends row w's mass of this slice to every CTA
      if (warp < group) {
        Mass sum = s_warp[warp * per_row];
        for (int w = 1; w < per_row; ++w) join(sum, s_warp[warp * per_row + w], c);
        if (lane < (int)ctas)
          store_remote(remote_smem(&s_part[turn][warp][rank], lane),
                       make_uint4(__float_as_uint(sum.m), __float_as_uint(sum.l), sum.at, 0));
      }
      // the draft's value and its distribution's, on their way meanwhile
      const int i = i0 + warp;
      int x = -1;
      float u = 0.f, q = 1.f, logit = -INFINITY;
      if (warp < group && i < n - 1) {
        x = *(p.tokens + r0 + i + 1);
        if (x >= 0 && x < p.vocab) {
          logit = as_float(target[(r0 + i) * p.target_stride + x]);
          if (!greedy) {
            u = *(p.uniform + r0 + i);
            if (p.draft_probs) q = p.draft_probs[(r0 + i) * p.draft_stride + x];
          }
        }
      }
      cluster_sync();
      if (warp < group) {
        Mass sum{-INFINITY, 0.f, 0x7fffffff};
        for (int k = 0; k < (int)ctas; ++k) {
          const uint4 w = s_part[turn][warp][k];
          join(sum, Mass{__uint_as_float(w.x), __uint_as_float(w.y), (int)w.z}, c);
        }
        if (lane == 0) {
          const bool any = sum.l > 0.f;                // (not NaN either)
          float px = 0.f;
          if (any && logit != -INFINITY) px = (sum.m == INFINITY ? (logit == INFINITY ? 1.f : 0.f) : expf((logit - sum.m) * inv)) / sum.l;
          RowResult r;
          r.m = sum.m;
          r.l = sum.l;
          r.at = sum.at;
          r.ok = i < n - 1 && any && (greedy ? sum.at == x : u * q < px);
          r.draft_logprob = sum.m == INFINITY ? logf(px) : (logit - sum.m) * inv - logf(sum.l);
          s_row[warp] = r;
          if (i < n - 1 && (x < 0 || x >= p.vocab)) s_row[warp].ok = -1;    // refused for what it is
        }
      }
      __syncthreads();
      int stopped = -1;
      for (int k = 0; k < group && i0 + k < n; ++k) {
        if (s_row[k].ok <= 0) {
          stopped = k;
          break;
        }
      }
      const int good = stopped < 0 ? group : stopped;
      if (rank == 0 && tid < good && p.out_logprobs && i0 + tid < p.out_stride)
        p.out_logprobs[(size_t)s * p.out_stride + i0 + tid] = s_row[tid].draft_logprob;
      if (stopped >= 0) {
        stop = i0 + stopped;
        last = s_row[stopped];
        if (last.ok < 0) status |= EFIM_DEV_BAD_TOKEN;
        break;
      }
    }
  }

  // ---- the next token
  unsigned long long key = 0, all = 0;                 // of what the draft leaves, of the target's distribution
  const bool judged = stop >= 0 && stop < n - 1;       // the row refused a draft
  const bool sound = n > 0 && (KIND == TARGET_PROBS || last.l > 0.f);
  if (sound && !greedy) {
    const T* row = target + (r0 + stop) * p.target_stride;
    const float* noise = p.noise + s * p.noise_stride;
    const float* q = judged && p.draft_probs ? p.draft_probs + (r0 + stop) * p.draft_stride : nullptr;
    const int gone = judged && !p.draft_probs ? *(p.tokens + r0 + stop + 1) : -1;
    const float total = last.l;
    auto probability = [&](float x) {
      if (KIND == TARGET_PROBS) return x;
      return (last.m == INFINITY ? (x == INFINITY ? 1.f : 0.f) : expf((x - last.m) * inv)) / total;
    };
    auto take = [&](float x, float e, float qx, int at) {
      const float pr = probability(x);
      const unsigned long long k = race_key(pr, e, at);
      all = max(all, k);
      if (q) key = max(key, race_key(pr - qx, e, at));
      else if (at != gone) key = max(key, k);
    };
    constexpr int U = 4;
    for (int a0 = begin + tid; a0 < end; a0 += U * VERIFY_THREADS) {
      float x[U], e[U], qx[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = a0 + u * VERIFY_THREADS;
        if (at < end) {
          x[u] = as_float(row[at]);
          e[u] = noise[at];
          qx[u] = q ? q[at] : 0.f;
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (a0 + u * VERIFY_THREADS < end) take(x[u], e[u], qx[u], a0 + u * VERIFY_THREADS);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      key = max(key, __shfl_xor_sync(0xffffffffu, key, d));
      all = max(all, __shfl_xor_sync(0xffffffffu, all, d));
    }
    if (lane == 0) s_key[warp] = make_ulonglong2(key, all);
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < VERIFY_WARPS; ++w) {
        key = max(key, s_key[w].x);
        all = max(all, s_key[w].y);
      }
      store_remote(remote_smem(&s_keys[rank].x, 0), key);
      store_remote(remote_smem(&s_keys[rank].y, 0), all);
    }
    cluster_sync();
  }
  if (rank != 0) return;
  if (tid == 0) {
    int next = -1;
    if (sound && greedy) {
      next = last.at;
    } else if (sound) {
      for (int k = 0; k < (int)ctas; ++k) {
        key = max(key, s_keys[k].x);
        all = max(all, s_keys[k].y);
      }
      if (!key) key = all;                             // the draft's distribution leaves nothing: rounding alone refused it
      if (key) next = (int)(0xffffffffu - (uint32_t)key);
    }
    float logprob = 0.f;
    if (next >= 0) {
      const float x = as_float(target[(r0 + stop) * p.target_stride + next]);
      logprob = KIND == TARGET_PROBS ? logf(x) : last.m == INFINITY ? -logf(last.l) : (x - last.m) * inv - logf(last.l);
    } else if (n > 0) {
      status |= EFIM_DEV_NO_TOKEN;
    }
    const int acc = max(stop, 0);
    p.accepted[s] = acc;
    p.next_token[s] = next;
    if (acc < p.out_stride) {
      if (p.out_tokens) p.out_tokens[(size_t)s * p.out_stride + acc] = next;
      if (p.out_logprobs) p.out_logprobs[(size_t)s * p.out_stride + acc] = logprob;
    }
    if (status && p.status) atomicOr(p.status, status);
  }
  for (int i = tid; i < p.out_stride; i += VERIFY_THREADS) {
    if (i < stop) {
      if (p.out_tokens) p.out_tokens[(size_t)s * p.out_stride + i] = *(p.tokens + r0 + i + 1);
    } else if (i > max(stop, 0)) {
      if (p.out_tokens) p.out_tokens[(size_t)s * p.out_stride + i] = -1;
      if (p.out_logprobs) p.out_logprobs[(size_t)s * p.out_stride + i] = 0.f;
    }
  }
}

}  // namespace efim

extern "C" efim_status efim_verify_drafts(const efim_verify_desc* d, int32_t* d_accepted, int32_t* d_next_token,
                                          int32_t* d_out_tokens, float* d_out_logprobs, int32_t out_stride, int32_t* d_status,
                                          void* stream) {
  using namespace efim;
  if (!d || d->batch < 0 || d->total_rows < 0 || d->vocab <= 0) return EFIM_ERR_INVALID_ARG;
  if (d->target_kind < EFIM_TARGET_LOGITS_BF16 || d->target_kind > EFIM_TARGET_PROBS_F32) return EFIM_ERR_INVALID_ARG;
  if (d->batch == 0) return EFIM_OK;
  if (!d->d_row_indptr || !d_accepted || !d_next_token) return EFIM_ERR_INVALID_ARG;
  if ((d_out_tokens || d_out_logprobs) ? out_stride <= 0 : out_stride < 0) return EFIM_ERR_INVALID_ARG;
  if (d->total_rows > 0) {
    const int size = d->target_kind == EFIM_TARGET_LOGITS_BF16 ? 2 : 4;
    if (!d->d_target || !d->d_tokens || d->target_stride < d->vocab) return EFIM_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(d->d_target) % size) return EFIM_ERR_INVALID_ARG;
    if (d->target_kind == EFIM_TARGET_PROBS_F32 && (!d->d_noise || d->d_temperature)) return EFIM_ERR_INVALID_ARG;
    if (d->d_noise && (!d->d_uniform || d->noise_stride < d->vocab)) return EFIM_ERR_INVALID_ARG;
    if (d->d_draft_probs && d->draft_stride < d->vocab) return EFIM_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(d->d_noise) | reinterpret_cast<uintptr_t>(d->d_draft_probs)) & 3) return EFIM_ERR_INVALID_ARG;
  }
  VerifyParams p{};
  p.target = d->d_target;
  p.row_indptr = d->d_row_indptr;
  p.tokens = d->d_tokens;
  p.draft_probs = d->d_draft_probs;
  p.uniform = d->d_uniform;
  p.noise = d->d_noise;
  p.temperature = d->d_temperature;
  p.accepted = d_accepted;
  p.next_token = d_next_token;
  p.out_tokens = d_out_tokens;
  p.out_logprobs = d_out_logprobs;
  p.status = d_status;
  p.target_stride = d->target_stride;
  p.draft_stride = d->draft_stride;
  p.noise_stride = d->noise_stride;
  p.batch = d->batch;
  p.total_rows = d->total_rows;
  p.vocab = d->vocab;
  p.out_stride = d_out_tokens || d_out_logprobs ? out_stride : 0;
  // as many CTAs a sequence as fill the GPU, of at least 2048 places each
  const int slots = 2 * sm_count();
  int ctas = VERIFY_MAX_CTAS;
  while (ctas > 1 && ((long long)d->batch * ctas > 4LL * slots || d->vocab / ctas < 2048)) ctas /= 2;
  p.group = (long long)d->batch * ctas <= slots ? VERIFY_MAX_GROUP : 1;
  if ((long long)d->batch * ctas > 0x7fffffffLL) return EFIM_ERR_UNSUPPORTED;
  auto launch = [&](auto kernel) {
    return launch_clusters(kernel, ctas, dim3((unsigned)(d->batch * ctas)), dim3(VERIFY_THREADS), static_cast<cudaStream_t>(stream), p);
  };
  EFIM_CUDA_TRY(d->target_kind == EFIM_TARGET_LOGITS_BF16  ? launch(verify_kernel<TARGET_BF16>)
                : d->target_kind == EFIM_TARGET_LOGITS_F32 ? launch(verify_kernel<TARGET_F32>)
                                                           : launch(verify_kernel<TARGET_PROBS>));
  return EFIM_OK;
}
