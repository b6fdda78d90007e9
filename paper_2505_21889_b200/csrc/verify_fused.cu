// efim_verify_drafts in one kernel, for few sequences and vocabularies of up to eight CTAs' threads with 16 bytes of a row each: a
// cluster per sequence.  Rows are looked at up to eight at a time, by some of a CTA's warps each; the CTAs swap the rows' masses through
// distributed shared memory and all of them judge alike; the race then runs over the row's values that each CTA has in L1.
//
// Bound: a chain of latencies - the row ranges, the rows, two exchanges over the cluster - and with many sequences the rows' bytes.
#include "cluster.cuh"
#include "verify.cuh"
#include <algorithm>

namespace efim {

constexpr int FUSED_THREADS = 512;
constexpr int FUSED_WARPS = FUSED_THREADS / 32;
constexpr int FUSED_ROWS = 8;            // that are looked at together
constexpr int FUSED_MOST_CTAS = 8;       // of a cluster
static_assert(FUSED_MOST_CTAS * FUSED_THREADS * 16 == FUSED_MOST_BYTES, "16 bytes of a row per thread");

// The mass of places [begin, end) of a row, by `lanes` lanes of which this is one, each seeing its places in rising order.  fetch() sends
// for the first vectors, so that other loads can follow before mass() waits.  The values stay in L1.
template <typename T, int U>
struct Slice {
  static constexpr int EPV = 16 / sizeof(T);
  static constexpr uint32_t LOW = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;        // -inf
  uint4 w[U];
  const T* p;
  int begin, n, first, n_vec, id, lanes;
  __device__ __forceinline__ void vectors(int v) {
    const uint4* vec = reinterpret_cast<const uint4*>(p + first);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      w[u] = make_uint4(LOW, LOW, LOW, LOW);
      if (v + u * lanes < n_vec) w[u] = vec[v + u * lanes];
    }
  }
  __device__ __forceinline__ void fetch(const T* row, int begin_, int end, int id_, int lanes_) {
    begin = begin_;
    n = max(0, end - begin);
    id = id_;
    lanes = lanes_;
    p = row + begin;
    first = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(T));
    n_vec = (n - first) / EPV;
    vectors(id);
  }
  __device__ __forceinline__ Mass mass(const Scale& sc) {
    Mass s = no_mass();
#pragma unroll 1
    for (int v = id;;) {
      float top = -INFINITY;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < EPV / 2; ++e) top = fmaxf(top, fmaxf(pair_of<T>(w[u], e).x, pair_of<T>(w[u], e).y));
      if (top > s.m) {
        s.l *= shift(s.m, top, sc.c);
        s.m = top;
        if (sc.greedy) {
#pragma unroll
          for (int u = U - 1; u >= 0; --u)
#pragma unroll
            for (int e = EPV / 2 - 1; e >= 0; --e) {
              const float2 x = pair_of<T>(w[u], e);
              const int at = begin + first + (v + u * lanes) * EPV + 2 * e;
              if (x.y == top) s.at = at + 1;
              if (x.x == top) s.at = at;
            }
        }
      }
      const bool plain = has_ref(s.m, sc.c);
      const float ref = plain ? -rintf(s.m * sc.c) : 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (v - (id & 31) + u * lanes >= n_vec) break;                     // the whole warp
#pragma unroll
        for (int e = 0; e < EPV / 2; ++e) {
          const float2 x = pair_of<T>(w[u], e);
          s.l += exp2_fast(plain ? fmaf(x.x, sc.c, ref) : below_ref(x.x, s.m, sc.c));
          s.l += exp2_fast(plain ? fmaf(x.y, sc.c, ref) : below_ref(x.y, s.m, sc.c));
        }
      }
      v += U * lanes;
      if (v >= n_vec) break;
      vectors(v);
    }
    // of a slice that is not aligned: a value a lane of those before and behind its vectors
    const int rest = first + n_vec * EPV, at = id < first ? id : rest + id - first;
    if (at < n) {
      const float x = as_float(p[at]);
      if (x >= s.m) {
        s.l *= shift(s.m, x, sc.c);
        s.at = x > s.m ? begin + at : min(s.at, begin + at);
        s.m = x;
      }
      s.l += exp2_fast(below_ref(x, s.m, sc.c));
    }
    return s;
  }
};

template <int KIND, int PER_SM>
__global__ void __launch_bounds__(FUSED_THREADS, PER_SM) verify_fused_kernel(const VerifyParams p) {
  using T = typename TargetOf<KIND>::type;
  constexpr int N = 16 / sizeof(T);      // places of a thread
  __shared__ Mass s_warp[FUSED_WARPS];
  __shared__ __align__(16) uint4 s_part[2][FUSED_ROWS][FUSED_MOST_CTAS];     // of every CTA of the cluster, by turns
  __shared__ RowResult s_row[FUSED_ROWS];
  __shared__ unsigned long long s_key[FUSED_WARPS], s_keys[2][FUSED_MOST_CTAS];

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)cluster_rank(), ctas = (int)cluster_size();
  const int s = blockIdx.x / ctas;
  cluster_arrive();
  pdl_wait();
  pdl_launch();
  const int r0 = *(p.row_indptr + s), r1 = *(p.row_indptr + s + 1);
  const bool rows_ok = r0 >= 0 && r1 <= p.total_rows && r0 <= r1;
  const int n = rows_ok ? r1 - r0 : 0;
  const Scale sc = KIND == TARGET_PROBS ? Scale{1.f, false} : scale_of(p, s);
  const T* target = static_cast<const T*>(p.target);
  const int begin = (rank * FUSED_THREADS + tid) * N, count = max(0, min(N, p.vocab - begin));

  // N values of this thread's places; past the vocabulary `none`
  auto fetch = [&](const auto* row, float none, float* x) {
    using V = std::remove_cv_t<std::remove_pointer_t<decltype(row)>>;
    if (count == N && !(reinterpret_cast<uintptr_t>(row) & 15)) {
      if constexpr (sizeof(V) == 2) {
        const uint4 w = *reinterpret_cast<const uint4*>(row + begin);
        const uint32_t q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[2 * e] = bf16lo(q[e]);
          x[2 * e + 1] = bf16hi(q[e]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < N / 4; ++e) *reinterpret_cast<float4*>(x + 4 * e) = *reinterpret_cast<const float4*>(row + begin + 4 * e);
      }
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = e < count ? as_float(row[begin + e]) : none;
    }
  };
  __align__(16) float noise[N];
  if (p.noise) fetch(p.noise + s * p.noise_stride, 0.f, noise);

  // ---- rows until one accepts nothing
  int stop = -1;
  RowResult last{};
  bool joined = false;
#pragma unroll 1
  for (int i0 = 0, turn = 0; i0 < n && stop < 0; i0 += FUSED_ROWS, turn ^= 1) {
    const int rows = min(FUSED_ROWS, n - i0);
    // warp u judges row u: its draft, on its way meanwhile
    const int i = i0 + warp;
    const bool any = warp < rows && i < n - 1;
    const int token = any ? *(p.tokens + r0 + i + 1) : -1;
    const int per_row = FUSED_WARPS / rows, mine = warp / per_row;       // warps of a row
    Slice<T, PER_SM == 1 ? 6 : 3> slice;             // (six vectors a lane: one of five rows by three warps)
    if (KIND != TARGET_PROBS && mine < rows)
      slice.fetch(target + (r0 + i0 + mine) * p.target_stride, rank * FUSED_THREADS * N, min(p.vocab, (rank + 1) * FUSED_THREADS * N),
                  (warp % per_row) * 32 + lane, per_row * 32);
    const Draft d = draft_of<KIND>(p, r0 + i, token, any, sc);
    Mass sum = no_mass();
    if (KIND != TARGET_PROBS) {
      if (mine < rows) {
        sum = warp_join(slice.mass(sc), sc.c, sc.greedy);
        if (lane == 0) s_warp[warp] = sum;
      }
      __syncthreads();
      if (warp < rows) sum = warp_join(lane < per_row ? s_warp[warp * per_row + lane] : no_mass(), sc.c, sc.greedy);
      if (ctas > 1) {
        if (!joined) cluster_wait();
        joined = true;
        if (warp < rows && lane < ctas)
          store_remote(remote_smem(&s_part[turn][warp][rank], lane), make_uint4(__float_as_uint(sum.m), __float_as_uint(sum.l), sum.at, 0));
        cluster_sync();
        if (warp < rows) {
          sum = no_mass();
          if (lane < ctas) {
            const uint4 v = s_part[turn][warp][lane];
            sum = Mass{__uint_as_float(v.x), __uint_as_float(v.y), (int)v.z};
          }
          sum = warp_join(sum, sc.c, sc.greedy);
        }
      }
    }
    if (warp < rows) {
      const RowResult row = judge<KIND>(sum, d, sc);
      if (lane == 0) s_row[warp] = row;
    }
    __syncthreads();
    int good = 0;
    while (good < rows && s_row[good].ok > 0) ++good;
    if (rank == 0 && p.out_logprobs && tid < good && i0 + tid < p.out_stride)
      p.out_logprobs[(size_t)s * p.out_stride + i0 + tid] = s_row[tid].logprob;
    if (good < rows) {
      stop = i0 + good;
      last = s_row[good];
    }
    __syncthreads();
  }
  if (!joined && ctas > 1) cluster_wait();

  // ---- the next token
  const bool sound = n > 0 && (KIND == TARGET_PROBS || last.l > 0.f), judged = stop < n - 1;
  int next = -1;
  __align__(16) float x[N];              // of the row it stops at: from L1
  if (sound) fetch(target + (r0 + stop) * p.target_stride, -INFINITY, x);
  if (sound && sc.greedy) {
    next = last.at;
  } else if (sound) {
    const bool dense = judged && p.draft_probs;
    __align__(16) float q[N];
#pragma unroll
    for (int e = 0; e < N; ++e) q[e] = 0.f;
    if (dense) fetch(p.draft_probs + (r0 + stop) * p.draft_stride, 0.f, q);
    int gone = judged && !dense ? last.draft : -1;
    // once, or, where the draft's distribution leaves nothing (rounding alone refused it), again over the target's own
    for (int round = 0; round < 2 && next < 0; ++round) {
      Race<KIND> race({last.m, last.l, sc.c}, gone, 0.f);
      if (race.estimates()) {
        float estimate[N];
#pragma unroll
        for (int e = 0; e < N; ++e) estimate[e] = e < count ? race.estimate(x[e], noise[e], q[e]) : 0.f;
        race.template run<N>(x, noise, q, estimate, [&](int e) { return begin + e; });
      } else {
#pragma unroll 1
        for (int e = 0; e < count; ++e)
          race.compute(as_float(target[(r0 + stop) * p.target_stride + begin + e]), p.noise[s * p.noise_stride + begin + e],
                       dense && round == 0 ? p.draft_probs[(r0 + stop) * p.draft_stride + begin + e] : 0.f, begin + e);
      }
      unsigned long long key = warp_best(race.key);
      if (lane == 0) s_key[warp] = key;
      __syncthreads();
      key = warp_best(lane < FUSED_WARPS ? s_key[lane] : 0);
      if (ctas > 1) {
        if (tid < ctas) store_remote(remote_smem(&s_keys[round][rank], tid), key);
        cluster_sync();
        key = warp_best(lane < ctas ? s_keys[round][lane] : 0);
      } else {
        __syncthreads();
      }
      next = place_of(key);
      gone = -1;
#pragma unroll
      for (int e = 0; e < N; ++e) q[e] = 0.f;
    }
  }
  const int acc = max(stop, 0);
  int32_t* out_tokens = p.out_tokens ? p.out_tokens + (size_t)s * p.out_stride : nullptr;
  float* out_logprobs = p.out_logprobs ? p.out_logprobs + (size_t)s * p.out_stride : nullptr;
  // written by the thread that holds the token, or the first
  if (next >= 0 ? next >= begin && next < begin + count : rank == 0 && tid == 0) {
    int status = rows_ok ? 0 : EFIM_DEV_BAD_POSITION;
    if (last.ok < 0) status |= EFIM_DEV_BAD_TOKEN;
    float logprob = 0.f;
    if (next >= 0) {
      float v = x[0];
#pragma unroll
      for (int e = 1; e < N; ++e)
        if (next == begin + e) v = x[e];
      logprob = Row<KIND>{last.m, last.l, sc.c}.log_of(v);
    } else if (n > 0) {
      status |= EFIM_DEV_NO_TOKEN;
    }
    p.accepted[s] = acc;
    p.next_token[s] = next;
    if (acc < p.out_stride) {
      if (out_tokens) out_tokens[acc] = next;
      if (out_logprobs) out_logprobs[acc] = logprob;
    }
    if (status && p.status) atomicOr(p.status, status);
  }
  if (rank == 0) {
    for (long long i = tid; i < p.out_stride; i += FUSED_THREADS) {
      if (i < stop) {
        if (out_tokens) out_tokens[i] = *(p.tokens + r0 + i + 1);
      } else if (i > acc) {
        if (out_tokens) out_tokens[i] = -1;
        if (out_logprobs) out_logprobs[i] = 0.f;
      }
    }
  }
}

static unsigned fused_ctas(long long vocab, int kind) {
  const int places = FUSED_THREADS * (kind == TARGET_BF16 ? 8 : 4);
  unsigned ctas = 1;
  while (ctas * places < vocab) ctas *= 2;
  return ctas;
}

// As long as all CTAs are resident at once, two an SM.  GPU microseconds, one kernel against two, five rows each: bf16 logits, 1 x 1,000 5.4 / 5.7,
// 1 x 32,768 7.4 / 7.2 (and 4 us of host time less), 8 x 32,768 7.5 / 9.5, 128 x 4,096 6.5 / 10.6, 256 x 4,096 9.4 / 13.7, 32 x 32,768 11.9 / 11.7,
// 128 x 32,768 45 / 25; probabilities, 1 x 16,384 3.5 / 5.0, 32 x 16,384 4.8 / 6.0, 128 x 16,384 15.8 / 8.1.  With more rows, all accepted,
// two kernels are ahead (bf16, 1 x 32,768 places: 9 rows 10.7 / 7.6, 17 15.7 / 9.7, 40 28 / 14, 128 84 / 32; 8 sequences 10.9 / 9.9, 16 / 12, 29 / 19,
// 87 / 46), but calls of these sizes are promised to need no workspace, however many rows they have.
bool verify_is_fused(long long batch, long long vocab, int kind) {
  return vocab * (kind == TARGET_BF16 ? 2 : 4) <= FUSED_MOST_BYTES && batch * fused_ctas(vocab, kind) <= 2 * sm_count();
}

cudaError_t verify_fused_launch(const VerifyParams& p, int kind, cudaStream_t stream) {
  const unsigned ctas = fused_ctas(p.vocab, kind), grid = p.batch * ctas;
  auto launch = [&](auto kernel) { return launch_clusters(kernel, ctas, dim3(grid), dim3(FUSED_THREADS), stream, p); };
  // with an SM to itself a CTA may keep more of its slice on the way (256 CTAs of bf16 rows as two waves of these: 10.7 instead of 7.4 us)
  const bool alone = grid <= (unsigned)sm_count();
  if (kind == TARGET_BF16) return launch(alone ? verify_fused_kernel<TARGET_BF16, 1> : verify_fused_kernel<TARGET_BF16, 2>);
  if (kind == TARGET_F32) return launch(alone ? verify_fused_kernel<TARGET_F32, 1> : verify_fused_kernel<TARGET_F32, 2>);
  return launch(verify_fused_kernel<TARGET_PROBS, 2>);
}

}  // namespace efim
