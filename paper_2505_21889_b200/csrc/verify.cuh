// What the kernels of efim_verify_drafts share: a row's mass, its probabilities, the judgement of a draft, the race for the next token.
#pragma once
#include "common.cuh"
#include <float.h>

namespace efim {

struct RowResult {
  float m, l, logprob;      // maximum and sum of the row, log-probability of its draft
  int at, ok;               // place of the maximum; draft accepted: 1, refused: 0, refused for what it is: -1
  int draft;
};

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
  uint4* part;              // [total_rows][pieces]: maximum, sum, place of the maximum
  unsigned long long* key;  // [batch] best of the race so far
  int* done;                // [batch] pieces of the race that are through
  long long target_stride, draft_stride, noise_stride;
  int batch, total_rows, vocab, out_stride;
  int piece, pieces;        // places of a CTA of the first kernel, CTAs of a row
  int race_piece, race_pieces;   // places of a CTA of the second, CTAs of a sequence
};

enum { TARGET_BF16 = EFIM_TARGET_LOGITS_BF16, TARGET_F32 = EFIM_TARGET_LOGITS_F32, TARGET_PROBS = EFIM_TARGET_PROBS_F32 };
template <int KIND> struct TargetOf { using type = float; };
template <> struct TargetOf<TARGET_BF16> { using type = uint16_t; };

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_fast(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// maximum over the warp; NaN lanes do not count
__device__ __forceinline__ float warp_max(float x) {
  float y;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}
// Mass of a row's values: the largest, m; the sum l of 2^(x c - ref(m)); and the first place of the largest (where asked for).
// ref(m) is the whole number next to m c: x c - ref is then one fused product with one rounding, of what is left, and masses of
// different m are joined by exact powers of two.  Where m c passes 2^30 (no fp32 logits there are closer than 2^6 in x c) it is m c
// itself, by way of (x - m) c; so it is for infinite m.  A NaN among the values makes the sum NaN; values of -inf have no mass; at
// +inf those values share all of it.
struct Mass {
  float m, l;
  int at;
};
__device__ __forceinline__ Mass no_mass() { return {-INFINITY, 0.f, 0x7fffffff}; }
__device__ __forceinline__ bool has_ref(float m, float c) { return fabsf(m * c) < 1073741824.f; }
// x c - ref(m), x <= m
__device__ __forceinline__ float below_ref(float x, float m, float c) {
  if (has_ref(m, c)) return fmaf(x, c, -rintf(m * c));
  if (x == m) return m == -INFINITY ? -INFINITY : 0.f;
  return (x - m) * c;
}
// what a sum at `from` is worth at `to` >= from
__device__ __forceinline__ float shift(float from, float to, float c) {
  if (has_ref(from, c) && has_ref(to, c)) return exp2_fast(rintf(from * c) - rintf(to * c));
  if (from == to) return 1.f;
  return exp2_fast((from - to) * c);
}
// The lanes' masses together, in every lane.
__device__ __forceinline__ Mass warp_join(Mass s, float c, bool want_at) {
  Mass r{warp_max(s.m), 0.f, 0x7fffffff};
  r.l = s.l * shift(s.m, r.m, c);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) r.l += __shfl_xor_sync(0xffffffffu, r.l, d);
  if (want_at) r.at = (int)__reduce_min_sync(0xffffffffu, s.m == r.m ? (unsigned)s.at : 0x7fffffffu);
  return r;
}

__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// Values 2 e and 2 e + 1 of the 16 bytes of a vector
template <typename T>
__device__ __forceinline__ float2 pair_of(const uint4& w, int e) {
  const uint32_t q[4] = {w.x, w.y, w.z, w.w};
  if constexpr (sizeof(T) == 2) return make_float2(bf16lo(q[e]), bf16hi(q[e]));
  else return make_float2(__uint_as_float(q[2 * e]), __uint_as_float(q[2 * e + 1]));
}

// The largest of N vectors' values; NaN does not count.
template <typename T, int N>
__device__ __forceinline__ float top_of(const uint4* w) {
  if constexpr (sizeof(T) == 2) {
    uint32_t m = w[0].x;
#pragma unroll
    for (int u = 0; u < N; ++u) m = max_bf16x2(max_bf16x2(max_bf16x2(m, w[u].x), w[u].y), max_bf16x2(w[u].z, w[u].w));
    return fmaxf(bf16lo(m), bf16hi(m));
  } else {
    float m = __uint_as_float(w[0].x);
#pragma unroll
    for (int u = 0; u < N; ++u)
      m = fmaxf(fmaxf(fmaxf(m, __uint_as_float(w[u].x)), __uint_as_float(w[u].y)), fmaxf(__uint_as_float(w[u].z), __uint_as_float(w[u].w)));
    return m;
  }
}

// Probabilities of one row, from its logits or as they are: m, and l = sum of 2^((x - m) c).
template <int KIND>
struct Row {
  float m, l, c;
  // (x - m) c, where it is not 0 times or less infinity
  __device__ __forceinline__ float below(float x) const { return x == m ? 0.f : (x - m) * c; }
  __device__ __forceinline__ float exact(float x) const { return KIND == TARGET_PROBS ? x : exp2f(below(x)) / l; }
  __device__ __forceinline__ float log_of(float x) const {
    return KIND == TARGET_PROBS ? logf(x) : below(x) * 0.6931471805599453f - logf(l);
  }
};

// The race for the next token: the largest r / e, r = (p - q)^+ or p, the lowest place among equals.
//
// An exact result costs two divisions and an exponential.  So every place gets an estimate first, by the fast instructions, and only places
// whose estimate, a little increased, reaches the best result known so far are computed: a few a warp.  What an estimate has to make up
// for, in a probability of 2^-126 and more (smaller ones are taken for 0 here), whose exponents are below 128 and half an ulp of them at
// most 2^-18: its own exponent's rounding, 2^-18, and those of the computed one's difference and product, 126 * 2^-24 + 2^-18, together
// 254 * 2^-24 ln 2 = 1.05e-5; ex2 2^-22 in either and in the sum's reference, the exponential's and the division's few 2^-24: below 1.5e-6.
// `scale` is 1.52e-5 more (before q is taken off); rcp and the last product are 2^-22, for which RACE_ABOVE comes in again.
constexpr float RACE_ABOVE = 1.f + 1.f / 65536;
template <int KIND>
struct Race {
  Row<KIND> of;
  float scale, ref;
  int gone;                                           // a place that does not take part
  float best;                                         // of the warp (the same in its lanes), or known to be reached by others: what it leaves out cannot win
  unsigned long long key;                             // of this lane: result and place as one number to be compared, 0 for none
  __device__ __forceinline__ Race(const Row<KIND>& of_, int gone_, float known) : of(of_), gone(gone_), best(known), key(0) {
    const bool logits = KIND != TARGET_PROBS;
    scale = logits ? RACE_ABOVE / (of.l * exp2_fast(below_ref(of.m, of.m, of.c))) : RACE_ABOVE;
    ref = logits && has_ref(of.m, of.c) ? -rintf(of.m * of.c) : 0.f;
  }
  // Whether estimates can be made; else (logits beyond 2^30 or infinite) every place is computed.
  __device__ __forceinline__ bool estimates() const { return KIND == TARGET_PROBS || has_ref(of.m, of.c); }
  __device__ __forceinline__ float estimate(float x, float e, float q) const {
    return fmaf(KIND == TARGET_PROBS ? x : exp2_fast(fmaf(x, of.c, ref)), scale, -q) * rcp_fast(e);
  }
  // The result of one place, computed.
  __device__ __forceinline__ float compute(float x, float e, float q, int at) {
    const float r = of.exact(x) - q, t = r > 0.f && at != gone ? r / e : 0.f;
    if (t > 0.f) key = max(key, (unsigned long long)__float_as_uint(t) << 32 | (0xffffffffu - (uint32_t)at));
    return t;
  }
  // N places of every lane of the warp with their estimates; places with an estimate of 0 do not run.
  template <int N, typename Place>
  __device__ __forceinline__ void run(const float* x, const float* e, const float* q, float* estimate, Place place) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmaxf(top, estimate[i]);
    // from the highest estimate down, as long as they reach the best result
    for (float highest; (highest = warp_max(top)) > 0.f && highest * RACE_ABOVE >= best;) {
      float t = 0.f;
      if (top == highest) {
        int at = 0;
        float px = 0.f, ex = 1.f, qx = 0.f;
        bool found = false;
        top = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          if (!found && estimate[i] == highest) {
            found = true;
            at = place(i);
            px = x[i];
            ex = e[i];
            qx = q[i];
            estimate[i] = 0.f;
          }
          top = fmaxf(top, estimate[i]);
        }
        t = compute(px, ex, qx, at);
      }
      best = fmaxf(best, warp_max(t));
    }
  }
};
__device__ __forceinline__ int place_of(unsigned long long key) { return key ? (int)(0xffffffffu - (uint32_t)key) : -1; }
__device__ __forceinline__ unsigned long long warp_best(unsigned long long key) {
  const unsigned top = __reduce_max_sync(0xffffffffu, (unsigned)(key >> 32));
  const unsigned at = __reduce_max_sync(0xffffffffu, (unsigned)(key >> 32) == top ? (unsigned)key : 0u);
  return (unsigned long long)top << 32 | at;
}

// Temperature of a sequence, as a factor of its logits; greedy sequences take 1.
struct Scale {
  float c;                  // log2(e) / T
  bool greedy;
};
__device__ __forceinline__ Scale scale_of(const VerifyParams& p, int s) {
  Scale r{1.4426950408889634f, !p.noise};
  if (p.noise && p.temperature) {
    const float t = *(p.temperature + s);
    r.greedy = !(t > 0.f);
    if (!r.greedy) r.c = fminf(fmaxf(1.4426950408889634f / t, FLT_MIN), FLT_MAX);   // (0 times -inf would be NaN)
  }
  return r;
}

// The draft that a row judges (`token`), and what it is judged by: inputs alone.
struct Draft {
  int x;
  bool any, inside;         // the row has a draft; it is one of the vocabulary
  float value, q, u;        // of the target's row, of its own distribution, uniform
};
template <int KIND>
__device__ __forceinline__ Draft draft_of(const VerifyParams& p, int r, int token, bool any, const Scale& sc) {
  Draft d{token, any, false, -INFINITY, 1.f, 0.f};
  if (!any) return d;
  d.inside = d.x >= 0 && d.x < p.vocab;
  if (d.inside) {
    d.value = as_float(static_cast<const typename TargetOf<KIND>::type*>(p.target)[r * p.target_stride + d.x]);
    if (!sc.greedy) {
      d.u = *(p.uniform + r);
      if (p.draft_probs) d.q = p.draft_probs[r * p.draft_stride + d.x];
    }
  }
  return d;
}
// What a row makes of it, the same in all lanes that ask: from its mass, or its probabilities as they are.
template <int KIND>
__device__ __forceinline__ RowResult judge(const Mass& sum, const Draft& d, const Scale& sc) {
  RowResult row{0.f, 1.f, 0.f, 0, 0, d.x};
  if (KIND == TARGET_PROBS) {
    row.ok = d.inside && d.u * d.q < d.value;
    row.logprob = logf(d.value);
  } else {
    row.m = sum.m;
    row.l = sum.l / exp2_fast(below_ref(sum.m, sum.m, sc.c));    // (exactly 1 where there is one token)
    row.at = sum.at;
    const bool some = row.l > 0.f;                     // (and not NaN)
    const Row<KIND> of{row.m, row.l, sc.c};
    const float px = some ? of.exact(d.value) : 0.f;
    row.ok = some && d.inside && (sc.greedy ? sum.at == d.x : d.u * d.q < px);
    row.logprob = of.log_of(d.value);
  }
  if (d.any && !d.inside) row.ok = -1;
  return row;
}

// efim_verify_drafts in one kernel (verify_fused.cu): whether it is the way for these sizes, and the launch.
constexpr int FUSED_MOST_BYTES = 65536;        // of a row
bool verify_is_fused(long long batch, long long vocab, int kind);
cudaError_t verify_fused_launch(const VerifyParams& p, int kind, cudaStream_t stream);

}  // namespace efim
