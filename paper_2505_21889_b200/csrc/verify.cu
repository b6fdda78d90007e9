// efim_verify_drafts: which of a step's drafted tokens the target model's distributions accept, and the token that follows them.
//
// Row i of a sequence holds the target's distribution p_i after the step's token i; the draft it judges is token i + 1, drawn from
// q_i (or with certainty).  With u_i uniform in [0, 1) and e exponential, all given:
//   draft x is accepted  iff  u_i q_i(x) < p_i(x)
//   at the first row that accepts nothing, or the last one: next = argmax_j r_j / e_j,  r = (p - q)^+ or, behind the last draft, p
// (argmax_j r_j / e_j is a draw from r / sum r: the first of exponential times with rates r_j).  Together the emitted tokens are
// distributed as if the target had been sampled token by token.  At temperature 0: accepted while the draft is the row's argmax.
//
// Two kernels.  The first takes every row's maximum and sum (its mass), a piece of a row per CTA.  The second has CTAs for pieces of the
// vocabulary of every sequence: each joins the masses, finds the row at which its sequence stops and runs its piece of the race
// for the next token there; the last of them to finish writes the result.  (Few sequences of small vocabularies: verify_fused.cu.)
//
// Bound, 256 sequences x 5 rows x 131,072 bf16 with dense drafts, 120 us in all: the masses 66-70 us for 336 MB (5 TB/s; the exponentials keep
// the special function units at 72 %, without them it is 58), the race 45 us for 274 MB (6 TB/s).  16 sequences, 14.9 us: 1.5 us of
// dependent loads to the stop, 1.2 to count the race's CTAs, launches.
// Not kept: every fourth exponential on the FMA pipe (the same, every second 12 us longer); copies through shared memory, four groups
// on their way (the same; 16 sequences 1 us longer); rows taken first rows first, so that those behind a refusal are left out, which halves
// the bytes here: with a count behind each piece 117 us, as a persistent kernel of 16 KB pieces 115-193, of whole rows 127; a cluster per
// sequence that walks its rows 160-212.
#include "verify.cuh"
#include <algorithm>

namespace efim {

constexpr int VERIFY_THREADS = 256;
constexpr int VERIFY_WARPS = VERIFY_THREADS / 32;
constexpr int VERIFY_MOST = 1 << 30;                    // places, rows, and those a piece or a step further on, are counted in 32 bits

// A thread's share of a piece of a row: up to MASS_VECTORS vectors of 16 bytes, a CTA's threads apart, and one value before and behind
// the vectors of a piece that is not aligned.  All of it is on its way before anything is computed.
constexpr int MASS_VECTORS = 8;
template <typename T>
struct Share {
  static constexpr int EPV = 16 / sizeof(T);
  uint4 w[MASS_VECTORS];
  const T* values;
  float head, tail;
  int first, n_vec, begin, n;                         // first value of the vectors, vectors, place of the first value, values
  __device__ __forceinline__ void fetch(const T* row, int begin_, int end) {
    begin = begin_;
    n = end - begin;
    const T* p = values = row + begin;
    first = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(T));
    n_vec = (n - first) / EPV;
    const uint4* vec = reinterpret_cast<const uint4*>(p + first);
    const uint32_t low = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;       // -inf
#pragma unroll
    for (int u = 0; u < MASS_VECTORS; ++u) {
      const int v = threadIdx.x + u * VERIFY_THREADS;
      w[u] = make_uint4(low, low, low, low);
      if (v < n_vec) w[u] = ldg_stream(vec + v);
    }
    head = (int)threadIdx.x < first ? as_float(p[threadIdx.x]) : -INFINITY;
    const int rest = first + n_vec * EPV + threadIdx.x;
    tail = rest < n ? as_float(p[rest]) : -INFINITY;
  }
  __device__ __forceinline__ Mass mass(float c, bool want_at) const {
    Mass s = no_mass();
    s.m = top_of<T, MASS_VECTORS>(w);
    s.m = fmaxf(fmaxf(s.m, -INFINITY), fmaxf(head, tail));                 // (not NaN where all values are)
    if (want_at) {
      // from the last place to the first
      if (tail == s.m) s.at = begin + first + n_vec * EPV + threadIdx.x;
#pragma unroll
      for (int u = MASS_VECTORS - 1; u >= 0; --u)
#pragma unroll
        for (int e = EPV / 2 - 1; e >= 0; --e) {
          const float2 x = pair_of<T>(w[u], e);
          const int at = begin + first + (threadIdx.x + u * VERIFY_THREADS) * EPV + 2 * e;
          if (x.y == s.m) s.at = at + 1;
          if (x.x == s.m) s.at = at;
        }
      if (head == s.m) s.at = begin + threadIdx.x;
    }
    if (has_ref(s.m, c)) {
      const float2 cc = make_float2(c, c), ref = make_float2(-rintf(s.m * c), -rintf(s.m * c));
      float2 l = make_float2(exp2_fast(fmaf(head, c, ref.x)), exp2_fast(fmaf(tail, c, ref.x)));
#pragma unroll
      for (int u = 0; u < MASS_VECTORS; ++u) {
        if (u * VERIFY_THREADS >= n_vec) break;                            // the whole CTA
#pragma unroll
        for (int e = 0; e < EPV / 2; ++e) {
          const float2 y = fma2(pair_of<T>(w[u], e), cc, ref);
          l = add2(l, make_float2(exp2_fast(y.x), exp2_fast(y.y)));
        }
      }
      s.l = l.x + l.y;
    } else {
      // one value after the other, read again.  By the thread's own maximum: all of its values are -inf, or the largest is +inf or times c
      // beyond 2^30.  Rows masked but for 50 places, by -inf or the type's lowest values, send nearly every thread here: 256 sequences x
      // 5 rows x 131,072 bf16 with certain drafts 115 -> 237 us, 16 13.4 -> 23.1, 37 x 1-8 x 100,003 fp32 20.6 -> 34.1.
      s.l = exp2_fast(below_ref(head, s.m, c)) + exp2_fast(below_ref(tail, s.m, c));
#pragma unroll 1
      for (int v = threadIdx.x; v < n_vec; v += VERIFY_THREADS)
#pragma unroll 1
        for (int e = 0; e < EPV; ++e) s.l += exp2_fast(below_ref(as_float(values[first + v * EPV + e]), s.m, c));
    }
    return s;
  }
};

// The race over places [begin, end) of a row.  VEC: the operands are 16-byte aligned there (8 for bf16 logits) and end - begin is a
// multiple of 4.
template <int KIND, bool VEC>
__device__ __forceinline__ void race_over(Race<KIND>& race, const typename TargetOf<KIND>::type* row, const float* noise, const float* q,
                                          int begin, int end) {
  constexpr int N = 8;                                // places of a thread in flight: two groups of four, or eight apart
  using T = typename TargetOf<KIND>::type;
  const int tid = threadIdx.x;
  auto place = [&](int a0, int i) { return VEC ? a0 + (i / 4) * 4 * VERIFY_THREADS + i % 4 : a0 + i * VERIFY_THREADS; };
  // whole warps stay together: the first lane's place decides; places past the end take forever (e infinite)
#pragma unroll 1
  for (int a0 = begin + (VEC ? 4 * tid : tid); a0 - (VEC ? 4 : 1) * (tid & 31) < end; a0 += N * VERIFY_THREADS) {
    __align__(16) float x[N], e[N], qx[N], estimate[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = qx[i] = 0.f;
      e[i] = INFINITY;
    }
    if constexpr (VEC) {
#pragma unroll
      for (int g = 0; g < N; g += 4) {
        const int at = place(a0, g);
        if (at < end) {
          if constexpr (sizeof(T) == 2) {
            const uint2 w = *reinterpret_cast<const uint2*>(row + at);
            x[g] = bf16lo(w.x);
            x[g + 1] = bf16hi(w.x);
            x[g + 2] = bf16lo(w.y);
            x[g + 3] = bf16hi(w.y);
          } else {
            *reinterpret_cast<float4*>(x + g) = *reinterpret_cast<const float4*>(row + at);
          }
          *reinterpret_cast<uint4*>(e + g) = ldg_stream(noise + at);
          if (q) *reinterpret_cast<uint4*>(qx + g) = ldg_stream(q + at);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int at = place(a0, i);
        if (at < end) {
          x[i] = as_float(row[at]);
          e[i] = noise[at];
          if (q) qx[i] = q[at];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) estimate[i] = race.estimate(x[i], e[i], qx[i]);
    race.template run<N>(x, e, qx, estimate, [&](int i) { return place(a0, i); });
  }
}

// Row r's judgement by a warp, from the masses of the row's pieces.
template <int KIND>
__device__ __forceinline__ RowResult judge_row(const VerifyParams& p, int r, const Draft& d, const Scale& sc) {
  Mass sum = no_mass();
  if (KIND != TARGET_PROBS) {
    for (int k = threadIdx.x & 31; k < p.pieces; k += 32) {
      const uint4 w = __ldcg(p.part + (size_t)r * p.pieces + k);
      const Mass o{__uint_as_float(w.x), __uint_as_float(w.y), (int)w.z};
      const float m = fmaxf(sum.m, o.m);
      sum.l = sum.l * shift(sum.m, m, sc.c) + o.l * shift(o.m, m, sc.c);
      if (o.m > sum.m) sum.at = o.at;                  // (a lane's places rise)
      sum.m = m;
    }
    sum = warp_join(sum, sc.c, sc.greedy);
  }
  return judge<KIND>(sum, d, sc);
}

// What the CTAs of the second kernel meet in, cleared by all of a grid's threads together.  In 64 bits: a grid of rows and pieces may
// have more than 2^31 threads.
__device__ __forceinline__ void clear_meetings(const VerifyParams& p) {
  for (long long s = (long long)blockIdx.x * VERIFY_THREADS + threadIdx.x; s < p.batch; s += (long long)gridDim.x * VERIFY_THREADS) {
    p.key[s] = 0;
    p.done[s] = 0;
  }
}
__global__ void __launch_bounds__(VERIFY_THREADS) verify_init_kernel(const VerifyParams p) {
  pdl_wait();
  pdl_launch();
  clear_meetings(p);
}

// The masses of all rows, a CTA a piece.
template <int KIND>
__device__ __forceinline__ Mass piece_mass(const Share<typename TargetOf<KIND>::type>& share, const Scale& sc, Mass* s_warp) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Mass mass = warp_join(share.mass(sc.c, sc.greedy), sc.c, sc.greedy);
  if (lane == 0) s_warp[warp] = mass;
  __syncthreads();
  return warp == 0 ? warp_join(lane < VERIFY_WARPS ? s_warp[lane] : no_mass(), sc.c, sc.greedy) : mass;      // (of the first warp)
}
__device__ __forceinline__ uint4 packed(const Mass& s) { return make_uint4(__float_as_uint(s.m), __float_as_uint(s.l), s.at, 0); }

template <int KIND>
__global__ void __launch_bounds__(VERIFY_THREADS, 4) verify_mass_kernel(const VerifyParams p) {
  using T = typename TargetOf<KIND>::type;
  __shared__ Mass s_warp[VERIFY_WARPS];
  const int tid = threadIdx.x, lane = tid & 31;
  const int r = blockIdx.x / p.pieces, piece = blockIdx.x % p.pieces;
  pdl_wait();
  pdl_launch();
  clear_meetings(p);
  Share<T> share;
  share.fetch(static_cast<const T*>(p.target) + r * p.target_stride, piece * p.piece, min(p.vocab, (piece + 1) * p.piece));
  // the row's sequence: the last that starts at or before it
  int lo = 0, n = p.batch;
  while (n > 32) {
    const int step = (n + 31) / 32;
    const bool le = lane * step < n && *(p.row_indptr + lo + lane * step) <= r;
    const int i = 31 - __clz((int)(__ballot_sync(0xffffffffu, le) | 1u));
    n = min(step, n - i * step);
    lo += i * step;
  }
  lo += 31 - __clz((int)(__ballot_sync(0xffffffffu, lane < n && *(p.row_indptr + lo + lane) <= r) | 1u));
  const Mass sum = piece_mass<KIND>(share, scale_of(p, lo), s_warp);
  if (tid == 0) p.part[blockIdx.x] = packed(sum);
}

// The end of every sequence: the row it stops at, and the race.
template <int KIND>
__global__ void __launch_bounds__(VERIFY_THREADS, 4) verify_pick_kernel(const VerifyParams p) {
  using T = typename TargetOf<KIND>::type;
  __shared__ RowResult s_row[VERIFY_WARPS];
  __shared__ unsigned long long s_key[VERIFY_WARPS];
  __shared__ bool s_last, s_empty;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int s = blockIdx.x / p.race_pieces, piece = blockIdx.x % p.race_pieces;
  const T* target = static_cast<const T*>(p.target);
  // (the kernel before this one wrote none of the inputs, and whatever came before that one is complete)
  const int r0 = *(p.row_indptr + s), r1 = *(p.row_indptr + s + 1);
  const bool rows_ok = r0 >= 0 && r1 <= p.total_rows && r0 <= r1;
  const int n = rows_ok ? r1 - r0 : 0;
  const Scale sc = KIND == TARGET_PROBS ? Scale{1.f, false} : scale_of(p, s);
  const bool first = piece == 0;
  const int begin = piece * p.race_piece, end = min(p.vocab, begin + p.race_piece);
  int32_t* out_tokens = p.out_tokens ? p.out_tokens + (size_t)s * p.out_stride : nullptr;
  float* out_logprobs = p.out_logprobs ? p.out_logprobs + (size_t)s * p.out_stride : nullptr;
  if (tid == 0 && n > 0 && !sc.greedy) prefetch_l2(p.noise + s * p.noise_stride + begin, (end - begin) * 4LL);

  int stop = -1, status = rows_ok ? 0 : EFIM_DEV_BAD_POSITION;
  RowResult last{};
  bool waited = false;
  // rows until one accepts nothing: a warp a row
  for (int i0 = 0; i0 < n && stop < 0; i0 += VERIFY_WARPS) {
    const int i = i0 + warp;
    const Draft d = draft_of<KIND>(p, r0 + i, i < n - 1 ? *(p.tokens + r0 + i + 1) : -1, i < n - 1, sc);
    if (!waited) pdl_wait();
    waited = true;
    if (i < n) {
      const RowResult row = judge_row<KIND>(p, r0 + i, d, sc);
      if (lane == 0) s_row[warp] = row;
    }
    __syncthreads();
    const int count = min(VERIFY_WARPS, n - i0);
    int good = 0;
    while (good < count && s_row[good].ok > 0) ++good;
    if (good < count) {
      stop = i0 + good;
      last = s_row[good];
    }
    if (first && out_logprobs && tid < good && i0 + tid < p.out_stride) out_logprobs[i0 + tid] = s_row[tid].logprob;
    __syncthreads();
  }
  if (last.ok < 0) status |= EFIM_DEV_BAD_TOKEN;
  if (!waited) pdl_wait();
  pdl_launch();
  if (first) {
    for (long long i = tid; i < p.out_stride; i += VERIFY_THREADS) {
      if (i < stop) {
        if (out_tokens) out_tokens[i] = *(p.tokens + r0 + i + 1);
      } else if (i > max(stop, 0)) {
        if (out_tokens) out_tokens[i] = -1;
        if (out_logprobs) out_logprobs[i] = 0.f;
      }
    }
  }

  // ---- the next token
  const bool judged = stop < n - 1;                    // the row refused a draft
  const bool sound = n > 0 && (KIND == TARGET_PROBS || last.l > 0.f);
  const bool runs = sound && !sc.greedy;
  unsigned long long key = 0;
  if (!runs) {
    if (!first) return;
  } else {
    const T* row = target + (r0 + stop) * p.target_stride;
    const float* noise = p.noise + s * p.noise_stride;
    const float* q = judged && p.draft_probs ? p.draft_probs + (r0 + stop) * p.draft_stride : nullptr;
    int gone = judged && !p.draft_probs ? last.draft : -1;
    if (tid == 0) {
      prefetch_l2(row + begin, (end - begin) * (long long)sizeof(T));
      if (q) prefetch_l2(q + begin, (end - begin) * 4LL);
    }
    const Row<KIND> of{last.m, last.l, sc.c};
    const bool aligned = !((reinterpret_cast<uintptr_t>(row) & (4 * sizeof(T) - 1)) | (reinterpret_cast<uintptr_t>(noise) & 15) |
                           (reinterpret_cast<uintptr_t>(q) & 15));
    auto run = [&](int a, int b, float known) {        // the whole CTA's best, in thread 0
      Race<KIND> r(of, gone, known);
      int rest = a;                                    // what is left to be computed place by place
      if (r.estimates()) {
        rest = aligned ? a + ((b - a) & ~3) : b;
        if (aligned) race_over<KIND, true>(r, row, noise, q, a, rest);
        else race_over<KIND, false>(r, row, noise, q, a, b);
      }
      for (int at = rest + tid; at < b; at += VERIFY_THREADS) r.compute(as_float(row[at]), noise[at], q ? q[at] : 0.f, at);
      unsigned long long k = warp_best(r.key);
      if (lane == 0) s_key[warp] = k;
      __syncthreads();
      return warp == 0 ? warp_best(lane < VERIFY_WARPS ? s_key[lane] : 0) : k;
    };
    // Other CTAs raise the key meanwhile, and the race's loops are a warp's together: one lane looks, for all of its warp.
    float known = 0.f;
    if (lane == 0) known = __uint_as_float((uint32_t)(*(volatile unsigned long long*)(p.key + s) >> 32));
    key = run(begin, end, __shfl_sync(0xffffffffu, known, 0));
    // the CTAs of a sequence meet: the last one through has the best of all
    if (p.race_pieces > 1) {
      if (tid == 0) {
        if (key) atomicMax(p.key + s, key);
        int before;                                    // the keys of those before are seen with it
        asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(before) : "l"(p.done + s) : "memory");
        s_last = before == p.race_pieces - 1;
        if (s_last) key = *(volatile unsigned long long*)(p.key + s);
      }
      __syncthreads();
      if (!s_last) return;
    }
    // where the draft's distribution leaves nothing (rounding alone refused it): the target's own
    if (tid == 0) s_empty = key == 0 && (q || gone >= 0);
    __syncthreads();
    if (s_empty) {
      q = nullptr;
      gone = -1;
      key = run(0, p.vocab, 0.f);
    }
  }
  if (tid != 0) return;
  int next = -1;
  if (sound && sc.greedy) next = last.at;
  if (key) next = place_of(key);
  float logprob = 0.f;
  if (next >= 0) {
    const float x = as_float(target[(r0 + stop) * p.target_stride + next]);
    logprob = Row<KIND>{last.m, last.l, sc.c}.log_of(x);
  } else if (n > 0) {
    status |= EFIM_DEV_NO_TOKEN;
  }
  const int acc = max(stop, 0);
  p.accepted[s] = acc;
  p.next_token[s] = next;
  if (acc < p.out_stride) {
    if (out_tokens) out_tokens[acc] = next;
    if (out_logprobs) out_logprobs[acc] = logprob;
  }
  if (status && p.status) atomicOr(p.status, status);
}

// Pieces of the race of at most 16,384 places: 256 sequences x 131,072 118 us, 8,192 125, 32,768 127 (every CTA looks for the stop itself).
// Places of a piece and pieces of a row (or a sequence) of `vocab` places, where there are `rows` of them: as many as fill the GPU once
// (4 CTAs an SM), of 2,048 to `most` places.
struct Pieces {
  int size, count;
};
static Pieces pieces_of(long long rows, int vocab, int most) {
  const long long wave = 4LL * sm_count(), want = std::max<long long>(1, wave / std::max<long long>(rows, 1));
  long long size = (vocab + want - 1) / want;
  size = std::min<long long>(most, std::max<long long>(2048, size));
  size = (size + 63) / 64 * 64;
  return {(int)size, (int)((vocab + size - 1) / size)};
}
constexpr int MASS_MOST_BYTES = MASS_VECTORS * VERIFY_THREADS * 16, RACE_MOST = 16384;

// The workspace, laid out one array behind the other.  Masses: the most that a call of at most these rows over at most this vocabulary
// cuts them into is one wave, or the largest pieces.
static size_t verify_layout(long long batch, long long rows, int vocab, char* ws, VerifyParams* p) {
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* x = ws + at;
    at += (bytes + 255) / 256 * 256;
    return x;
  };
  const long long least = (vocab + MASS_MOST_BYTES / 4 - 1) / (MASS_MOST_BYTES / 4);
  uint4* part = reinterpret_cast<uint4*>(take(std::max(4LL * sm_count() + rows, rows * least) * sizeof(uint4)));
  unsigned long long* key = reinterpret_cast<unsigned long long*>(take(batch * 8));
  int* done = reinterpret_cast<int*>(take(batch * 4));
  if (p) {
    p->part = part;
    p->key = key;
    p->done = done;
  }
  return at;
}

}  // namespace efim

extern "C" size_t efim_verify_workspace_bytes(int32_t batch, int32_t total_rows, int32_t vocab, int32_t target_kind) {
  if (batch <= 0 || total_rows < 0 || vocab <= 0 || efim::verify_is_fused(batch, vocab, target_kind)) return 0;
  return efim::verify_layout(batch, total_rows, vocab, nullptr, nullptr);
}

extern "C" efim_status efim_verify_drafts(const efim_verify_desc* d, int32_t* d_accepted, int32_t* d_next_token,
                                          int32_t* d_out_tokens, float* d_out_logprobs, int32_t out_stride, void* d_workspace,
                                          size_t workspace_bytes, int32_t* d_status, void* stream) {
  using namespace efim;
  if (!d || d->batch < 0 || d->total_rows < 0 || d->vocab <= 0) return EFIM_ERR_INVALID_ARG;
  if (d->vocab > VERIFY_MOST || d->total_rows > VERIFY_MOST) return EFIM_ERR_UNSUPPORTED;
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
  const size_t need = efim_verify_workspace_bytes(d->batch, d->total_rows, d->vocab, d->target_kind);
  if (need > 0 && (!d_workspace || workspace_bytes < need)) return EFIM_ERR_WORKSPACE;
  if (need > 0 && reinterpret_cast<uintptr_t>(d_workspace) & 255) return EFIM_ERR_INVALID_ARG;
  VerifyParams p{};
  p.target = d->d_target;
  p.row_indptr = d->d_row_indptr;
  p.tokens = d->d_tokens;
  p.draft_probs = d->d_draft_probs;
  p.uniform = d->d_uniform;
  p.noise = d->total_rows > 0 ? d->d_noise : nullptr;   // (without rows nothing of it was checked, and nothing is read)
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
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (need == 0) {
    if (d->batch > 0x7fffffff / 8) return EFIM_ERR_UNSUPPORTED;
    EFIM_CUDA_TRY(verify_fused_launch(p, d->target_kind, s));
    return EFIM_OK;
  }
  verify_layout(d->batch, d->total_rows, d->vocab, static_cast<char*>(d_workspace), &p);
  const Pieces mass = pieces_of(d->total_rows, d->vocab, d->target_kind == EFIM_TARGET_LOGITS_BF16 ? MASS_MOST_BYTES / 2 : MASS_MOST_BYTES / 4);
  const bool logits = d->target_kind != EFIM_TARGET_PROBS_F32 && d->total_rows > 0;
  const bool bf16 = d->target_kind == EFIM_TARGET_LOGITS_BF16;
  const Pieces race = pieces_of(d->batch, d->vocab, RACE_MOST);
  p.piece = mass.size;
  p.pieces = mass.count;
  p.race_piece = race.size;
  p.race_pieces = race.count;
  const long long ctas = (long long)mass.count * d->total_rows;
  if (ctas > 0x7fffffffLL || (long long)race.count * d->batch > 0x7fffffffLL) return EFIM_ERR_UNSUPPORTED;
  const dim3 block(VERIFY_THREADS), pick((unsigned)(race.count * d->batch));
  if (logits) {
    EFIM_CUDA_TRY(launch_pdl(bf16 ? verify_mass_kernel<TARGET_BF16> : verify_mass_kernel<TARGET_F32>, dim3((unsigned)ctas), block, 0, s, p));
  } else {
    EFIM_CUDA_TRY(launch_pdl(verify_init_kernel, dim3((unsigned)((d->batch + (long long)VERIFY_THREADS - 1) / VERIFY_THREADS)), block, 0, s, p));
  }
  EFIM_CUDA_TRY(launch_pdl(!logits ? verify_pick_kernel<TARGET_PROBS> : bf16 ? verify_pick_kernel<TARGET_BF16> : verify_pick_kernel<TARGET_F32>,
                           pick, block, 0, s, p));
  return EFIM_OK;
}
