// efim_adjust_logits: penalties for tokens that occurred, biases and grammar masks on the rows of a step, before they are judged or sampled.
//
// A CTA has one sequence's slice of the vocabulary in shared memory, a word per token: how often it was generated, whether the prompt
// holds it, and which entry of the bias list it has.  Few tokens are touched by any of that, so the rows are copied first (with the
// mask, in place only where it takes something away); then the touched tokens, listed, are computed over it, a thread a token, walking
// the sequence's rows and counting each row's own draft before it (a row's distribution comes after that token).
//
// Bound: 256 users x 1-5 rows x 131,072 places in bf16 125 us with cold caches (the copy 82, all but the copy 80: two CTAs an SM overlap them in part; the histories,
// which each slice reads, 33); 16 users x 5 rows 22.5: the phases' latencies, one wave.  Every logit through fp32: 189.  Not kept: clusters that read a history once and
// count in each other's shared memory (165: remote atomics, CTAs that wait for each other), half of the warps copying while the others count (198),
// 1,024 threads (188), three CTAs by 40 registers (141).
#include "common.cuh"
#include <algorithm>
#include <atomic>

namespace efim {

struct AdjustParams {
  const void* logits;           // rows of [vocab], stride elements apart
  void* out;
  long long stride, out_stride, history_stride, mask_stride;
  const int32_t* row_indptr;
  const int32_t* tokens;        // [total_rows] or null
  const int32_t* history;       // or null
  const int32_t *len, *prompt_len;
  const float *repetition, *presence, *frequency;
  const int32_t *bias_indptr, *bias_tokens;
  const float* bias;
  const uint32_t* mask;
  int32_t* status;
  int batch, total_rows, vocab, max_len, bias_entries, entry_shift, slice, slice_bits, slices, vector;
};

constexpr int ADJUST_THREADS = 512;

// A word of the counts, W: the prompt's bit on top, then the bias entry + 1, from bit p.entry_shift on, then the count.
template <typename W> constexpr int PROMPT_BIT = sizeof(W) * 8 - 1;

struct Penalties {
  float repetition, presence, frequency;
  const float* bias;
  int entry_shift;
};
// a logit of a token whose word is not 0
template <typename W>
__device__ __forceinline__ float adjusted(float x, W w, const Penalties& q) {
  const W n = w & (((W)1 << q.entry_shift) - 1);
  if (n || (w >> PROMPT_BIT<W>)) x = x > 0.f ? __fdiv_rn(x, q.repetition) : x * q.repetition;
  if (n) x = x - q.frequency * (float)n - q.presence;
  const W entry = (w & (((W)1 << PROMPT_BIT<W>) - 1)) >> q.entry_shift;
  if (entry) x += *(q.bias + (entry - 1));
  return x;
}

__device__ __forceinline__ float value_of(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ float value_of(float x) { return x; }
__device__ __forceinline__ void round_to(float x, uint16_t* y) { *y = (uint16_t)pack_bf16x2(x, 0.f); }
__device__ __forceinline__ void round_to(float x, float* y) { *y = x; }

// Eight logits of neighbouring tokens, as they lie: 16 bytes of bf16 or 32 of fp32.
template <typename T> struct Eight;
template <> struct Eight<uint16_t> {
  uint32_t x[4];
  __device__ __forceinline__ void mask(uint32_t allowed) {                    // -inf where the bit is 0
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // bits 2i and 2i + 1 as the signs of two bytes, and those signs over two halves
      uint32_t keep;
      asm("prmt.b32 %0, %1, 0, 0x9988;" : "=r"(keep) : "r"((allowed >> (2 * i) & 3u) * (1u << 7 | 1u << 14)));
      x[i] = (x[i] & keep) | (0xff80ff80u & ~keep);
    }
  }
  __device__ __forceinline__ void load(const uint16_t* p) {
    const uint4 u = ldg_stream(p);
    x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w;
  }
  __device__ __forceinline__ void store(uint16_t* p) const { *reinterpret_cast<uint4*>(p) = make_uint4(x[0], x[1], x[2], x[3]); }
  __device__ __forceinline__ void load(const uint16_t* p, int n) {            // the first n, one by one
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (2 * i < n ? p[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)p[2 * i + 1] << 16 : 0u);
  }
  __device__ __forceinline__ void store(uint16_t* p, int n) const {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = (uint16_t)(x[e / 2] >> (16 * (e & 1)));
  }
};
template <> struct Eight<float> {
  float x[8];
  __device__ __forceinline__ void mask(uint32_t allowed) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = allowed >> e & 1 ? x[e] : -INFINITY;
  }
  __device__ __forceinline__ void load(const float* p) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint4 u = ldg_stream(p + 4 * i);
      x[4 * i] = __uint_as_float(u.x), x[4 * i + 1] = __uint_as_float(u.y), x[4 * i + 2] = __uint_as_float(u.z), x[4 * i + 3] = __uint_as_float(u.w);
    }
  }
  __device__ __forceinline__ void store(float* p) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) *reinterpret_cast<float4*>(p + 4 * i) = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
  }
  __device__ __forceinline__ void load(const float* p, int n) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = e < n ? p[e] : 0.f;
  }
  __device__ __forceinline__ void store(float* p, int n) const {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = x[e];
  }
};

// most tokens of a slice, and places of the list of the touched ones
constexpr int ADJUST_SLICE = 16384, ADJUST_LIST = 4096;

template <typename T, typename W>
__global__ void __launch_bounds__(ADJUST_THREADS) adjust_logits_kernel(const AdjustParams p) {
  constexpr int AHEAD = 4;                               // loads on their way
  extern __shared__ __align__(16) uint8_t adjust_smem[];
  W* slot = reinterpret_cast<W*>(adjust_smem);
  __shared__ uint16_t s_list[ADJUST_LIST];
  __shared__ int s_listed;
  const int tid = threadIdx.x, s = blockIdx.x / p.slices, part = blockIdx.x % p.slices;
  const int v0 = part * p.slice, n_slot = min(p.slice, p.vocab - v0);
  const bool tells = part == 0 && p.status;              // one slice reports what is wrong with the sequence
  for (int i = tid * 16 / (int)sizeof(W); i < p.slice; i += ADJUST_THREADS * 16 / (int)sizeof(W))
    *reinterpret_cast<uint4*>(slot + i) = make_uint4(0, 0, 0, 0);
  if (tid == 0) s_listed = 0;
  pdl_wait();
  pdl_launch();
  int row0 = *(p.row_indptr + s), row1 = *(p.row_indptr + s + 1), err = 0;
  int len = p.history ? *(p.len + s) : 0, prompt = p.history && p.prompt_len ? *(p.prompt_len + s) : 0;
  Penalties q{p.repetition ? *(p.repetition + s) : 1.f, p.presence ? *(p.presence + s) : 0.f, p.frequency ? *(p.frequency + s) : 0.f, nullptr,
              p.entry_shift};
  if (row0 < 0 || row1 > p.total_rows || row1 < row0) {
    if (row0 < 0 || row0 > p.total_rows || row1 < row0) row1 = row0 = 0;
    row1 = min(row1, p.total_rows);
    err = EFIM_DEV_BAD_POSITION;
  }
  if (len < 0 || len > p.max_len || prompt < 0 || prompt > len) err |= EFIM_DEV_BAD_POSITION;
  len = min(max(len, 0), p.max_len);
  prompt = min(max(prompt, 0), len);
  __syncthreads();
  // ---- every logit: copied, or -inf where the mask says so; in place only the latter
  {
    const bool in_place = p.logits == p.out;
    const int groups = (n_slot + 7) / 8, whole = p.vector ? n_slot / 8 : 0;
    // A pass of the CTA is AHEAD groups of eight a thread: a row or a part of it, or several rows of a small slice
    const int bits = p.slice_bits - 3, rows = max(1, AHEAD * ADJUST_THREADS >> bits);
    const T* from[AHEAD];
    T* to[AHEAD];
    const uint8_t* mask[AHEAD];
    int row_of[AHEAD], at[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int i = tid + k * ADJUST_THREADS;
      at[k] = i & ((1 << bits) - 1);
      row_of[k] = at[k] < groups ? i >> bits : 1 << 30;   // (past every row)
      from[k] = static_cast<const T*>(p.logits) + (i >> bits) * p.stride + v0 + 8 * at[k];
      to[k] = static_cast<T*>(p.out) + (i >> bits) * p.out_stride + v0 + 8 * at[k];
      mask[k] = reinterpret_cast<const uint8_t*>(p.mask) + (i >> bits) * 4 * p.mask_stride + v0 / 8 + at[k];
    }
    for (int row = row0; row < row1 && !(in_place && !p.mask); row += rows) {
      Eight<T> x[AHEAD];
      uint32_t allowed[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
        if (row_of[k] < row1 - row) {
          allowed[k] = p.mask ? *(mask[k] + 4LL * row * p.mask_stride) : 0xffu;
          if (at[k] < whole) x[k].load(from[k] + row * p.stride);
          else x[k].load(from[k] + row * p.stride, n_slot - 8 * at[k]);
        }
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
        if (row_of[k] < row1 - row) {
          if (allowed[k] != 0xffu) x[k].mask(allowed[k]);
          else if (in_place) continue;
          if (at[k] < whole) x[k].store(to[k] + row * p.out_stride);
          else x[k].store(to[k] + row * p.out_stride, n_slot - 8 * at[k]);
        }
    }
  }
  if (p.bias) {
    int b0 = *(p.bias_indptr + s), b1 = *(p.bias_indptr + s + 1);
    if (b0 < 0 || b1 > p.bias_entries || b1 < b0) {
      err |= EFIM_DEV_BAD_POSITION;
      b0 = b1 = 0;
    }
    q.bias = p.bias + b0;
    for (int i = tid; i < b1 - b0; i += ADJUST_THREADS) {
      const int x = *(p.bias_tokens + b0 + i);
      if ((uint32_t)(x - v0) < (uint32_t)n_slot) atomicMax(&slot[x - v0], (W)(i + 1) << p.entry_shift);   // the last entry of a token counts
      if ((uint32_t)x >= (uint32_t)p.vocab) err |= EFIM_DEV_BAD_TOKEN;
    }
    __syncthreads();
  }
  {
    const int32_t* history = p.history + s * p.history_stride;
    auto count = [&](int i, int x) {
      if ((uint32_t)(x - v0) < (uint32_t)n_slot) {
        if (i < prompt) atomicOr(&slot[x - v0], (W)1 << PROMPT_BIT<W>);
        else atomicAdd(&slot[x - v0], (W)1);
      }
      if (tells && (uint32_t)x >= (uint32_t)p.vocab) err |= EFIM_DEV_BAD_TOKEN;
    };
    // four tokens at a time from where the row is 16-byte aligned on, four such vectors on their way
    const int head = min(len, (int)((16 - (reinterpret_cast<uintptr_t>(history) & 15)) & 15) / 4), vectors = (len - head) / 4;
    for (int i0 = tid; i0 < vectors; i0 += 4 * ADJUST_THREADS) {
      int4 x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i0 + k * ADJUST_THREADS < vectors) x[k] = *reinterpret_cast<const int4*>(history + head + 4 * (i0 + k * ADJUST_THREADS));
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = i0 + k * ADJUST_THREADS, at = head + 4 * i;
        if (i < vectors) {
          count(at, x[k].x);
          count(at + 1, x[k].y);
          count(at + 2, x[k].z);
          count(at + 3, x[k].w);
        }
      }
    }
    const int rest = len - head - 4 * vectors;           // before and behind them
    if (tid < head + rest) {
      const int i = tid < head ? tid : len - rest + (tid - head);
      count(i, *(history + i));
    }
  }
  __syncthreads();
  const bool drafts = p.history && p.tokens;
  if (drafts) {
    // drafts may touch tokens that nothing else does
    for (int row = row0 + 1 + tid; row < row1; row += ADJUST_THREADS) {
      const int x = *(p.tokens + row);
      if ((uint32_t)(x - v0) < (uint32_t)n_slot && slot[x - v0] == 0) {
        int before = row0 + 1;                            // once only: where it is drafted first
        while (before < row && *(p.tokens + before) != x) ++before;
        if (before == row) {
          const int at = atomicAdd(&s_listed, 1);
          if (at < ADJUST_LIST) s_list[at] = (uint16_t)(x - v0);
        }
      }
      if ((uint32_t)x >= (uint32_t)p.vocab) err |= EFIM_DEV_BAD_TOKEN;
    }
  }
  {
    // a thread's touched tokens as bits, 16 bytes of words at a time; a warp's take their places together
    constexpr int PER = 16 / sizeof(W);
    uint32_t mine = 0;
    for (int k = 0; k * ADJUST_THREADS * PER < p.slice; ++k) {
      const int i = (k * ADJUST_THREADS + tid) * PER;
      if (i >= p.slice) break;
      W w[PER];
      *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(slot + i);
#pragma unroll
      for (int e = 0; e < PER; ++e) mine |= (w[e] != 0 ? 1u : 0u) << (k * PER + e);
    }
    int upto = __popc(mine);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, upto, d);
      if ((tid & 31) >= d) upto += y;
    }
    int at = 0;
    if ((tid & 31) == 31 && upto) at = atomicAdd(&s_listed, upto);
    at = __shfl_sync(0xffffffffu, at, 31) + upto - __popc(mine);
    for (; mine; mine &= mine - 1, ++at) {
      const int bit = __ffs(mine) - 1;
      if (at < ADJUST_LIST) s_list[at] = (uint16_t)((bit / PER * ADJUST_THREADS + tid) * PER + bit % PER);
    }
  }
  __syncthreads();
  // ---- the touched tokens, over what the copy has left; a thread has a token and walks the sequence's rows
  const T* in = static_cast<const T*>(p.logits) + v0;
  T* out = static_cast<T*>(p.out) + v0;
  const bool listed = s_listed <= ADJUST_LIST;
  const int hits = listed ? s_listed : n_slot;
  for (int h = tid; h < hits; h += ADJUST_THREADS) {
    const int i = listed ? s_list[h] : h;
    W w = slot[i];
    if (!listed && w == 0 && !drafts) continue;
    const uint32_t* mask = p.mask ? p.mask + (v0 + i) / 32 : nullptr;
    for (int r0 = row0; r0 < row1; r0 += AHEAD) {
      T x[AHEAD];
      uint32_t word[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
        if (r0 + k < row1) {
          x[k] = *(in + (r0 + k) * p.stride + i);
          word[k] = mask ? *(mask + (r0 + k) * p.mask_stride) : 0xffffffffu;
        }
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
        if (r0 + k < row1) {
          if (drafts && r0 + k > row0) w += *(p.tokens + r0 + k) == v0 + i;   // the row's own token comes before it
          if (w && (word[k] >> ((v0 + i) & 31) & 1)) round_to(adjusted<W>(value_of(x[k]), w, q), out + (r0 + k) * p.out_stride + i);
        }
    }
  }
  if (err && tells) atomicOr(p.status, err);
}

template <typename T, typename W>
static efim_status adjust_launch(const AdjustParams& p, cudaStream_t stream) {
  constexpr int kMaxDevices = 64, kMost = ADJUST_SLICE * (int)sizeof(W);
  static std::atomic<bool> done[kMaxDevices];
  int dev = 0;
  EFIM_CUDA_TRY(cudaGetDevice(&dev));
  if (dev < 0 || dev >= kMaxDevices || !done[dev].load(std::memory_order_acquire)) {
    EFIM_CUDA_TRY(cudaFuncSetAttribute(adjust_logits_kernel<T, W>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost));
    if (dev >= 0 && dev < kMaxDevices) done[dev].store(true, std::memory_order_release);
  }
  EFIM_CUDA_TRY(launch_pdl(adjust_logits_kernel<T, W>, dim3((unsigned)((long long)p.batch * p.slices)), dim3(ADJUST_THREADS),
                           p.slice * sizeof(W), stream, p));
  return EFIM_OK;
}

}  // namespace efim

extern "C" efim_status efim_adjust_logits(const efim_adjust_desc* d, void* d_out, int64_t out_stride, int32_t* d_status, void* stream) {
  using namespace efim;
  if (!d || d->batch < 0 || d->total_rows < 0 || d->vocab <= 0 || (d->logits_f32 != 0 && d->logits_f32 != 1)) return EFIM_ERR_INVALID_ARG;
  if (d->batch == 0 || d->total_rows == 0) return EFIM_OK;
  if (d->vocab > 1 << 30 || d->total_rows > 1 << 30) return EFIM_ERR_UNSUPPORTED;
  auto address = [](const void* x) { return reinterpret_cast<uintptr_t>(x); };
  const int size = d->logits_f32 ? 4 : 2;
  if (!d->d_row_indptr || !d->d_logits || !d_out || d->logits_stride < d->vocab || out_stride < d->vocab ||
      ((address(d->d_logits) | address(d_out)) & (size - 1)))
    return EFIM_ERR_INVALID_ARG;
  if (d->d_history && (!d->d_len || d->max_len <= 0 || d->history_stride < d->max_len)) return EFIM_ERR_INVALID_ARG;
  if (!d->d_history && (d->d_repetition || d->d_presence || d->d_frequency)) return EFIM_ERR_INVALID_ARG;
  if (d->d_bias && (!d->d_bias_indptr || !d->d_bias_tokens || d->bias_entries < 0)) return EFIM_ERR_INVALID_ARG;
  if (d->d_mask && d->mask_stride < ((long long)d->vocab + 31) / 32) return EFIM_ERR_INVALID_ARG;
  if ((address(d->d_row_indptr) | address(d->d_tokens) | address(d->d_history) | address(d->d_len) | address(d->d_prompt_len) |
       address(d->d_repetition) | address(d->d_presence) | address(d->d_frequency) | address(d->d_bias_indptr) |
       address(d->d_bias_tokens) | address(d->d_bias) | address(d->d_mask)) & 3)
    return EFIM_ERR_INVALID_ARG;
  // in place, or apart: a row of the result must not lie where another one is still to be read
  const bool in_place = d_out == d->d_logits && out_stride == d->logits_stride;
  auto span = [&](long long stride) { return (uintptr_t)(((d->total_rows - 1LL) * stride + d->vocab) * size); };
  if (!in_place && address(d_out) < address(d->d_logits) + span(d->logits_stride) && address(d->d_logits) < address(d_out) + span(out_stride))
    return EFIM_ERR_INVALID_ARG;
  AdjustParams p{};
  p.logits = d->d_logits;
  p.out = d_out;
  p.stride = d->logits_stride;
  p.out_stride = out_stride;
  p.row_indptr = d->d_row_indptr;
  p.tokens = d->d_tokens;
  p.history = d->d_history;
  p.history_stride = d->history_stride;
  p.len = d->d_len;
  p.prompt_len = d->d_prompt_len;
  p.repetition = d->d_repetition;
  p.presence = d->d_presence;
  p.frequency = d->d_frequency;
  p.bias_indptr = d->d_bias_indptr;
  p.bias_tokens = d->d_bias_tokens;
  p.bias = d->d_bias;
  p.bias_entries = d->bias_entries;
  p.mask = static_cast<const uint32_t*>(d->d_mask);
  p.mask_stride = d->mask_stride;
  p.status = d_status;
  p.batch = d->batch;
  p.total_rows = d->total_rows;
  p.vocab = d->vocab;
  p.max_len = d->max_len;
  // whole 16-byte vectors where every row starts on one
  p.vector = ((address(d->d_logits) | address(d_out) | (uintptr_t)(d->logits_stride * size) | (uintptr_t)(out_stride * size)) & 15) == 0;
  // 32 bits a word where they hold the largest count, the longest bias list and the prompt's bit, else 64
  auto bits = [](long long most) { int n = 0; while (most >> n) ++n; return n; };
  p.entry_shift = bits((long long)d->max_len + d->total_rows);
  const bool narrow = p.entry_shift + bits(d->d_bias ? d->bias_entries : 0) <= 31;
  if (!narrow) p.entry_shift = 32;
  p.slice = narrow ? ADJUST_SLICE : ADJUST_SLICE / 2;
  // Slices as long as they come (each reads the history) while that gives one and a half CTAs an SM: 16 users x 5 rows x 131,072 places 22.5 us with 256
  // CTAs, 28.7 with 512, 256 users x 1-5 rows 125 us with slices of 16,384 and 179 of 8,192.
  while (p.slice > 2048 && (long long)d->batch * ((d->vocab + p.slice - 1) / p.slice) < sm_count() * 3LL / 2) p.slice /= 2;
  while (1 << p.slice_bits < p.slice) ++p.slice_bits;
  p.slices = (d->vocab + p.slice - 1) / p.slice;
  if ((long long)p.batch * p.slices > 0x7fffffffLL) return EFIM_ERR_UNSUPPORTED;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (d->logits_f32) return narrow ? adjust_launch<float, uint32_t>(p, s) : adjust_launch<float, unsigned long long>(p, s);
  return narrow ? adjust_launch<uint16_t, uint32_t>(p, s) : adjust_launch<uint16_t, unsigned long long>(p, s);
}
