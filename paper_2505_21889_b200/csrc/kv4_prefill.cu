// efim_kv4_append_prefill_attn: a turn's increments over a 4-bit cache.  Few rows a sequence take the kernel of efim_kv4_decode_attn; more
// rows make the products the larger part, and those belong on the tensor cores of efim_append_prefill_attn: the batch's pages are
// unpacked to bf16 (exactly) into the workspace, sequence after sequence, and attended there.
#include "kv4_attn.cuh"
#include <algorithm>

namespace efim {

struct Kv4StageParams {
  const uint8_t *k_codes, *v_codes, *k_scales, *v_scales;
  uint16_t *k_out, *v_out;          // [n][Hkv][16][D] bf16
  const int32_t *cached_len, *new_len, *block_table;
  int32_t* table;                   // [batch][width]: where each page went, -1 for bad ones
  float k_scale, v_scale;
  int n, batch, max_pages_per_seq, width, num_pages, Hkv;
};

constexpr int KV4_STAGE_THREADS = 256;

// One page of one sequence a CTA.  Bound: HBM (4.5 bits in, 16 out a value): 16 x 2-8k tokens at 8 heads x 128 70 us; 16 bytes of codes a thread 111.
template <int D>
__global__ void __launch_bounds__(KV4_STAGE_THREADS) kv4_stage_kernel(const Kv4StageParams p) {
  __shared__ int s_before[KV4_STAGE_THREADS / 32];
  const int s = blockIdx.y, i = blockIdx.x, tid = threadIdx.x;
  pdl_wait();
  pdl_launch();
  // sequences without new tokens have no pages here
  auto pages_of = [&](int x) {
    const int c = *(p.cached_len + x), n = *(p.new_len + x);
    return n > 0 ? (int)min((c + (long long)n + 15) / 16, (long long)p.width) : 0;
  };
  if (i >= pages_of(s)) return;
  int before = 0;
  for (int x = tid; x < s; x += KV4_STAGE_THREADS) before += pages_of(x);
  before = __reduce_add_sync(0xffffffffu, before);
  if ((tid & 31) == 0) s_before[tid >> 5] = before;
  __syncthreads();
  int to = i;
#pragma unroll
  for (int w = 0; w < KV4_STAGE_THREADS / 32; ++w) to += s_before[w];
  const int page = i < p.max_pages_per_seq ? *(p.block_table + (size_t)s * p.max_pages_per_seq + i) : -1;
  const bool ok = page >= 0 && page < p.num_pages && to < p.n;
  if (tid == 0) p.table[(size_t)s * p.width + i] = ok ? to : -1;      // (the attention reports what is bad)
  if (!ok) return;
  kv4_page_to_bf16<D, KV4_STAGE_THREADS>(p.k_codes, p.v_codes, p.k_scales, p.v_scales, p.k_scale, p.v_scale, page, to, p.Hkv, p.k_out, p.v_out);
}

namespace {
// Where a call's parts stand in its workspace.
struct StagePlan {
  long long pages;        // of sequences with new tokens
  int width;              // of the widest of all
  size_t table, pool, total;   // bytes: the table, one pool, everything before the attention's own workspace
};
StagePlan stage_plan(const efim_cache4_desc* cache, const efim_batch_desc* batch) {
  StagePlan pl{};
  for (int s = 0; s < batch->batch; ++s) {
    const long long n = ((long long)batch->h_cached_len[s] + batch->h_new_len[s] + 15) / 16;
    if (batch->h_new_len[s] > 0) pl.pages += n;
    pl.width = (int)std::max<long long>(pl.width, n);
  }
  auto round = [](size_t n) { return (n + 255) / 256 * 256; };
  pl.table = round((size_t)batch->batch * pl.width * 4);
  pl.pool = (size_t)pl.pages * cache->num_kv_heads * 16 * cache->head_dim * 2;
  pl.total = pl.table + 2 * round(pl.pool);
  return pl;
}
// the cache and the batch as the attention sees them, in workspace `ws` (or as sizes alone, at a place that is never read)
void staged(const efim_cache4_desc* cache, const efim_batch_desc* batch, const StagePlan& pl, char* ws, efim_cache_desc* c, efim_batch_desc* b) {
  *c = efim_cache_desc{ws + pl.table, ws + pl.table + (pl.total - pl.table) / 2, (int32_t)pl.pages, 16, cache->num_q_heads, cache->num_kv_heads,
                       cache->head_dim};
  *b = *batch;
  b->max_pages_per_seq = pl.width;
  b->d_block_table = reinterpret_cast<const int32_t*>(ws);
}
struct Lengths {
  int new_len, ctx;       // the largest
};
Lengths longest(const efim_batch_desc* b) {
  Lengths r{0, 0};
  for (int s = 0; s < b->batch; ++s) {
    if (b->h_new_len[s] == 0) continue;
    r.new_len = std::max(r.new_len, b->h_new_len[s]);
    r.ctx = std::max(r.ctx, b->h_cached_len[s] + b->h_new_len[s]);
  }
  return r;
}
// Rows a (sequence, kv head) up to which the keys are taken from the codes by the decode kernel: its time grows with the rows, the other way's first
// with the pages that are unpacked.  Microseconds, direct / unpacked: 16 x 5k keys at 32/8 heads 32 rows 83 / 155, 64 134 / 158, 80 175 / 160; at 28/4
// 63 rows 81 / 86, 77 99 / 86; 8 x 4k at 32/32 64 rows 191 / 222, 80 247 / 220; 64 x 2k at 32/8 64 rows 224 / 220, 80 292 / 222; 16 x 5k at 8/8 x 64
// 64 rows 101 / 102, 80 128 / 103.  With few pages, where both are latencies: 1 x 4k at 32/8 8 rows 21.6 / 26.7, 16 25.6 / 27.1, 24 35.8 / 26.7; 4 x 4k
// 16 rows 29.7 / 42, 48 50 / 45.  At 65 to 80 rows the direct way is 10 to 31 % longer; it is taken up to 80 for its weights of 11
// bits, where the bf16 kernel's have 8.
bool goes_direct(const efim_cache4_desc* cache, const efim_batch_desc* batch, const Lengths& most) {
  long long page_heads = 0;
  for (int s = 0; s < batch->batch; ++s)
    if (batch->h_new_len[s] > 0) page_heads += ((long long)batch->h_cached_len[s] + batch->h_new_len[s] + 15) / 16 * cache->num_kv_heads;
  const long long rows = (long long)most.new_len * (cache->num_q_heads / cache->num_kv_heads);
  return rows <= (page_heads < 64LL * sm_count() ? 16 : 80);
}
efim_status check(const efim_cache4_desc* cache, const efim_batch_desc* batch) {
  const efim_status st = check_cache4(cache);
  if (st != EFIM_OK) return st;
  const efim_cache_desc shape{nullptr, nullptr, 0, cache->page_size};
  return check_batch(&shape, batch, true);
}
}  // namespace
}  // namespace efim

extern "C" size_t efim_kv4_prefill_workspace_bytes(const efim_cache4_desc* cache, const efim_batch_desc* batch) {
  using namespace efim;
  if (check(cache, batch) != EFIM_OK || batch->batch == 0 || batch->total_new_tokens == 0) return 0;
  const Lengths most = longest(batch);
  if (goes_direct(cache, batch, most)) return kv4_plan(cache, batch->batch, most.new_len, most.ctx).bytes;
  const StagePlan pl = stage_plan(cache, batch);
  if (pl.pages * cache->num_kv_heads > 0x7fffffffLL) return 0;
  efim_cache_desc c;
  efim_batch_desc b;
  staged(cache, batch, pl, reinterpret_cast<char*>(4096), &c, &b);
  return pl.total + efim_prefill_workspace_bytes(&c, &b);
}

extern "C" efim_status efim_kv4_append_prefill_attn(const efim_cache4_desc* cache, const efim_batch_desc* batch, const void* d_q, void* d_out,
                                                    float* d_lse, float sm_scale, void* d_workspace, size_t workspace_bytes,
                                                    int32_t* d_status, void* stream) {
  using namespace efim;
  const efim_status st = check(cache, batch);
  if (st != EFIM_OK) return st;
  if (batch->batch == 0 || batch->total_new_tokens == 0) return EFIM_OK;
  if (!d_q || !d_out || ((reinterpret_cast<uintptr_t>(d_q) | reinterpret_cast<uintptr_t>(d_out)) & 15)) return EFIM_ERR_INVALID_ARG;
  const Lengths most = longest(batch);
  if (goes_direct(cache, batch, most)) {
    Kv4AttnParams p{};
    p.q = static_cast<const uint16_t*>(d_q);
    p.len = batch->d_cached_len;
    p.len_is_cached = 1;
    p.q_indptr = batch->d_q_indptr;
    p.block_table = batch->d_block_table;
    p.out = static_cast<uint16_t*>(d_out);
    p.lse = d_lse;
    p.status = d_status;
    p.batch = batch->batch;
    p.total_rows = batch->total_new_tokens;
    p.max_new = most.new_len;
    p.Hq = cache->num_q_heads;
    p.max_pages_per_seq = batch->max_pages_per_seq;
    return kv4_attn_run(cache, p, most.ctx, sm_scale, d_workspace, workspace_bytes, stream);
  }
  const StagePlan pl = stage_plan(cache, batch);
  if (pl.pages * cache->num_kv_heads > 0x7fffffffLL || batch->batch > 65535) return EFIM_ERR_UNSUPPORTED;
  char* ws = static_cast<char*>(d_workspace);
  efim_cache_desc c;
  efim_batch_desc b;
  staged(cache, batch, pl, reinterpret_cast<char*>(4096), &c, &b);
  if (!ws || workspace_bytes < pl.total + efim_prefill_workspace_bytes(&c, &b)) return EFIM_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(ws) & 255) return EFIM_ERR_INVALID_ARG;
  staged(cache, batch, pl, ws, &c, &b);
  Kv4StageParams p{};
  p.k_codes = static_cast<const uint8_t*>(cache->d_k_codes);
  p.v_codes = static_cast<const uint8_t*>(cache->d_v_codes);
  p.k_scales = static_cast<const uint8_t*>(cache->d_k_scales);
  p.v_scales = static_cast<const uint8_t*>(cache->d_v_scales);
  p.k_out = static_cast<uint16_t*>(c.d_k_pool);
  p.v_out = static_cast<uint16_t*>(c.d_v_pool);
  p.cached_len = batch->d_cached_len;
  p.new_len = batch->d_new_len;
  p.block_table = batch->d_block_table;
  p.table = reinterpret_cast<int32_t*>(ws);
  p.k_scale = cache->k_scale;
  p.v_scale = cache->v_scale;
  p.n = (int)pl.pages;
  p.batch = batch->batch;
  p.max_pages_per_seq = batch->max_pages_per_seq;
  p.width = pl.width;
  p.num_pages = cache->num_pages;
  p.Hkv = cache->num_kv_heads;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const dim3 grid(pl.width, batch->batch);
  EFIM_CUDA_TRY(cache->head_dim == 128 ? launch_pdl(kv4_stage_kernel<128>, grid, dim3(KV4_STAGE_THREADS), 0, s, p)
                                       : launch_pdl(kv4_stage_kernel<64>, grid, dim3(KV4_STAGE_THREADS), 0, s, p));
  return efim_append_prefill_attn(&c, &b, d_q, d_out, d_lse, sm_scale, ws + pl.total, workspace_bytes - pl.total, d_status, stream);
}
