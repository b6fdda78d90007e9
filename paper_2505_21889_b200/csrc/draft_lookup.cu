// efim_draft_lookup: drafts from a sequence's own history (infilled code repeats its prefix and suffix).  The place e of the
// history whose preceding tokens agree longest with the history's last ones - up to max_ngram tokens, the latest such place - is
// taken as what comes next:
//   e* = argmax over 1 <= e < len of (min(max_ngram, |common suffix of T[0, e) and T[0, len)|), e),   draft_i = T[e* + i mod (len - e*)]
// (the draft goes on with itself where it reaches the end of the history, as a repetition does).
//
// A cluster per sequence; the scan is for the last token, 16 bytes a load, and only places behind it look further back: at the token
// before, which a lane has in registers, and from there on in memory.  Bound: latency - launch, length, last tokens, scan, join - and with
// many long histories L2.  Histories that agree with themselves everywhere cost the looks back (256 x 32,768, 32 tokens a look: one token
// repeated 15 us, two at random 46; random tokens 5.8).
#include "cluster.cuh"

namespace efim {

constexpr int LOOKUP_THREADS = 512;
constexpr int LOOKUP_MAX_CTAS = 8;
constexpr int LOOKUP_MAX_NGRAM = 32;

struct LookupParams {
  const int32_t* history;   // rows of [max_len], stride elements apart
  const int32_t* len;       // [batch]
  int32_t* drafts;          // [batch][num_drafts]
  int32_t* draft_len;       // [batch]
  int32_t* status;
  long long stride;
  int batch, max_len, min_ngram, max_ngram, num_drafts;
};

__global__ void __launch_bounds__(LOOKUP_THREADS) draft_lookup_kernel(const LookupParams p) {
  __shared__ int s_tail[LOOKUP_MAX_NGRAM];
  __shared__ unsigned long long s_key[LOOKUP_THREADS / 32];
  __shared__ unsigned long long s_keys[LOOKUP_MAX_CTAS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)cluster_rank(), ctas = (int)cluster_size();
  const int s = blockIdx.x / ctas;
  cluster_arrive();
  pdl_wait();
  pdl_launch();
  const int32_t* T = p.history + s * p.stride;
  int len = *(p.len + s);
  if (len < 0 || len > p.max_len) {
    if (rank == 0 && tid == 0 && p.status) atomicOr(p.status, EFIM_DEV_BAD_POSITION);
    len = len < 0 ? 0 : p.max_len;
  }
  if (tid < LOOKUP_MAX_NGRAM) s_tail[tid] = tid < len ? T[len - 1 - tid] : 0;
  cluster_wait();
  __syncthreads();
  // key: agreeing tokens, then the place.  A thread's places come from the last to the first, so that only more agreeing tokens than
  // any of its later places had are of interest, and none once all of them agreed.
  unsigned long long key = 0;
  int best = p.min_ngram - 1;
  const int n = len - 1;                               // tokens that something comes after
  if (n > 0) {
    const int last = s_tail[0], second = s_tail[1];
    auto agreeing = [&](int before, int at) {          // of a place behind the last token; `before`: the token at - 1, if there is one
      int m = 1;
      if (m < p.max_ngram && at > 0 && before == second)
        for (m = 2; m < p.max_ngram && m <= at && T[at - m] == s_tail[m];) ++m;
      return m;
    };
    auto look = [&](int token, int before, int at) {
      if (token != last || best >= p.max_ngram) return;
      const int m = agreeing(before, at);
      if (m <= best) return;
      best = m;
      key = (unsigned long long)m << 32 | (uint32_t)(at + 1);
    };
    const int lead = min(n, (int)(((16 - (reinterpret_cast<uintptr_t>(T) & 15)) & 15) / 4));
    const int n_vec = (n - lead) / 4, tail = lead + n_vec * 4;
    const int id = rank * LOOKUP_THREADS + tid, lanes = ctas * LOOKUP_THREADS;
    auto look_at = [&](int at) { look(T[at], at > 0 ? T[at - 1] : 0, at); };
    if (id < n - tail) look_at(tail + id);             // (tail + id may pass 2^31)
    const int4* vec = reinterpret_cast<const int4*>(T + lead);
    constexpr int U = 8;                               // vectors of four tokens in flight
    for (int v0 = n_vec - 1 - id; v0 + lane >= 0; v0 -= U * lanes) {       // (the same for a warp's lanes)
      int4 w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        w[u] = make_int4(~last, ~last, ~last, ~last);
        if (v0 - u * lanes >= 0) w[u] = vec[v0 - u * lanes];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (v0 + lane - u * lanes < 0) break;
        const bool hit = w[u].x == last || w[u].y == last || w[u].z == last || w[u].w == last;
        if (!__any_sync(0xffffffffu, hit)) continue;
        int before = __shfl_down_sync(0xffffffffu, w[u].w, 1);             // the lane before has the vector behind this one
        if (!hit) continue;
        const int v = v0 - u * lanes, at = lead + v * 4;
        if (w[u].x == last && at > 0 && (lane == 31 || v == 0)) before = T[at - 1];
        look(w[u].w, w[u].z, at + 3);
        look(w[u].z, w[u].y, at + 2);
        look(w[u].y, w[u].x, at + 1);
        look(w[u].x, before, at);
      }
    }
    if (id < lead) look_at(id);
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) key = max(key, __shfl_xor_sync(0xffffffffu, key, d));
  if (lane == 0) s_key[warp] = key;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < LOOKUP_THREADS / 32; ++w) key = max(key, s_key[w]);
    store_remote(remote_smem(&s_keys[rank], 0), key);
  }
  cluster_sync();
  if (rank != 0) return;
  key = s_keys[0];
  for (int k = 1; k < ctas; ++k) key = max(key, s_keys[k]);
  const int e = (int)(uint32_t)key;
  const unsigned period = max(1, len - e);             // (len - e >= 1 where there is a key)
  for (unsigned i = tid; i < (unsigned)p.num_drafts; i += LOOKUP_THREADS)
    p.drafts[(size_t)s * p.num_drafts + i] = key ? T[e + (int)(i % period)] : -1;
  if (tid == 0) p.draft_len[s] = key ? p.num_drafts : 0;
}

}  // namespace efim

extern "C" efim_status efim_draft_lookup(int32_t batch, const int32_t* d_history, int64_t history_stride, int32_t max_len,
                                         const int32_t* d_len, int32_t min_ngram, int32_t max_ngram, int32_t num_drafts,
                                         int32_t* d_drafts, int32_t* d_draft_len, int32_t* d_status, void* stream) {
  using namespace efim;
  if (batch < 0 || max_len <= 0 || history_stride < max_len || num_drafts <= 0) return EFIM_ERR_INVALID_ARG;
  if (min_ngram < 1 || max_ngram < min_ngram) return EFIM_ERR_INVALID_ARG;
  if (max_ngram > LOOKUP_MAX_NGRAM) return EFIM_ERR_UNSUPPORTED;
  if (batch == 0) return EFIM_OK;
  if (!d_history || !d_len || !d_drafts || !d_draft_len || (reinterpret_cast<uintptr_t>(d_history) & 3)) return EFIM_ERR_INVALID_ARG;
  LookupParams p{d_history, d_len, d_drafts, d_draft_len, d_status, history_stride, batch, max_len, min_ngram, max_ngram, num_drafts};
  // at most two CTAs an SM, of 2,048 places and more.  1 x 2,300 tokens 3.1 us, 64 x 1-16k 4.0, 256 x 4-32k 6.3 (3.0 TB/s out of L2; with up to four
  // CTAs an SM 9.2, four vectors on the way 7.4; 1,024 threads a CTA 9.6, 256 7.3, with four of those an SM 6.5)
  unsigned ctas = LOOKUP_MAX_CTAS;
  while (ctas > 1 && ((long long)batch * ctas > 2LL * sm_count() || max_len / (int)ctas < 2048)) ctas /= 2;
  if ((long long)batch * ctas > 0x7fffffffLL) return EFIM_ERR_UNSUPPORTED;
  EFIM_CUDA_TRY(launch_clusters(draft_lookup_kernel, ctas, dim3(batch * ctas), dim3(LOOKUP_THREADS),
                                static_cast<cudaStream_t>(stream), p));
  return EFIM_OK;
}
