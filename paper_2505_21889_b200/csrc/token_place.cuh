// Which sequence a new token of a ragged batch belongs to, looked up by the lanes of a warp together.
#pragma once
#include "common.cuh"

namespace efim {

struct TokenPlace {
  int seq, pos;            // the sequence, and the token's position cached_len[seq] + i
};

// Sequence of token t: the last of `batch` that starts at or before it.  Called by whole warps, `wl` the lane: 32 candidates a
// trip, and the last trip brings the lengths along.
__device__ __forceinline__ TokenPlace find_token(const int32_t* q_indptr, const int32_t* cached_len, int batch, int t, int wl) {
  int lo = 0, n = batch;
  while (n > 32) {
    const int step = (n + 31) / 32;
    const bool le = wl * step < n && *(q_indptr + lo + wl * step) <= t;
    const int i = 31 - __clz((int)(__ballot_sync(0xffffffffu, le) | 1u));
    n = min(step, n - i * step);
    lo += i * step;
  }
  int first = 0, cached = 0;
  if (wl < n) {
    first = *(q_indptr + lo + wl);
    cached = *(cached_len + lo + wl);
  }
  const int i_seq = 31 - __clz((int)(__ballot_sync(0xffffffffu, wl < n && first <= t) | 1u));
  return {lo + i_seq, __shfl_sync(0xffffffffu, cached, i_seq) + t - __shfl_sync(0xffffffffu, first, i_seq)};
}

}  // namespace efim
