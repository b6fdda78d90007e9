// efim_step_tables: a step's rows, positions, slots and pages from the lengths that the device holds; efim_release_pages: pages that
// sequences no longer need.  Sequences without a host copy of their lengths (a drafted step's accepted tokens) go on from step to step.
//
// Both hand pages out or take them back in the order of sequences and places, so each row needs the number of pages that the rows before
// it take: one kernel counts row by row, the second adds up what stands before its row (all CTAs read the counts, a few KB) and writes.  Bound: launches and
// dependent loads; 512 prompts of up to 512 tokens with tables of 1,024 6.4 us on the GPU (6.6 MB).
#include "common.cuh"
#include <limits.h>

namespace efim {

struct TablesParams {
  const int32_t *cached_len, *new_len;      // release: cached_len holds the lengths that are kept
  const int32_t* table_in;
  int32_t* table_out;
  int32_t* free_pages;
  const int32_t* num_free;
  int32_t* num_free_out;
  int32_t* q_indptr;
  int32_t* positions;                       // these three: [rows] or null
  int64_t* slots;
  int32_t* sequences;
  int32_t* counts;                          // workspace: [0] free pages at the start, [1 + s] pages that row s takes or gives
  int32_t* status;
  int batch, width, capacity, rows;
};

constexpr int TABLES_THREADS = 128;

// A row's lengths as they count: none for a sequence with a negative one.
struct RowSpan {
  int cached, fresh;        // tokens before, new tokens
  int first, last;          // places of the table that the new tokens may add: [first, last)
  bool bad;
};
__device__ __forceinline__ RowSpan row_span(const TablesParams& p, int s) {
  RowSpan r;
  r.cached = *(p.cached_len + s);
  r.fresh = *(p.new_len + s);
  const long long end = (long long)r.cached + r.fresh;
  r.bad = r.cached < 0 || r.fresh < 0 || end > (long long)p.width * 16;
  if (r.cached < 0 || r.fresh < 0 || end > INT_MAX) r.cached = r.fresh = 0;
  r.first = (int)(((long long)r.cached + 15) / 16);
  r.last = (int)min((long long)p.width, ((long long)r.cached + r.fresh + 15) / 16);
  return r;
}

// sum over the CTA of N values a thread; the result is every thread's
template <int N>
__device__ __forceinline__ void block_sum(long long* v) {
  __shared__ long long s[TABLES_THREADS / 32][N];
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], d);
  __syncthreads();
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) s[threadIdx.x >> 5][i] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = 0;
#pragma unroll
    for (int w = 0; w < TABLES_THREADS / 32; ++w) v[i] += s[w][i];
  }
}

// pages that a row takes (places without one), or gives back; a warp a row
template <bool RELEASE>
__global__ void __launch_bounds__(TABLES_THREADS) tables_count_kernel(const TablesParams p) {
  pdl_wait();
  pdl_launch();
  const int s = blockIdx.x * (TABLES_THREADS / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (s == 0 && lane == 0) {
    const int n = *p.num_free;
    p.counts[0] = min(max(n, 0), p.capacity);
    if ((n < 0 || n > p.capacity) && p.status) atomicOr(p.status, EFIM_DEV_BAD_POSITION);
  }
  if (s >= p.batch) return;
  int first, last;
  if (RELEASE) {
    const int keep = *(p.cached_len + s);
    first = keep < 0 ? p.width : (int)(((long long)keep + 15) / 16);
    last = p.width;
    if (keep < 0 && lane == 0 && p.status) atomicOr(p.status, EFIM_DEV_BAD_POSITION);
  } else {
    const RowSpan r = row_span(p, s);
    first = r.first;
    last = r.last;
    if (r.bad && lane == 0 && p.status) atomicOr(p.status, EFIM_DEV_BAD_POSITION);
  }
  const int32_t* row = p.table_in + (size_t)s * p.width;
  int n = 0;
  for (int e = first + lane; e < last; e += 32) n += (*(row + e) < 0) != RELEASE;
  n = __reduce_add_sync(0xffffffffu, n);
  if (lane == 0) p.counts[1 + s] = n;
}

__global__ void __launch_bounds__(TABLES_THREADS) tables_write_kernel(const TablesParams p) {
  pdl_wait();
  pdl_launch();
  const int s = blockIdx.x, tid = threadIdx.x, lane = tid & 31;
  long long sum[4] = {0, 0, 0, 0};                  // before this row: pages, tokens; in all: pages, tokens
  for (int i = tid; i < p.batch; i += TABLES_THREADS) {
    const int pages = *(p.counts + 1 + i), fresh = row_span(p, i).fresh;
    sum[2] += pages;
    sum[3] += fresh;
    if (i < s) {
      sum[0] += pages;
      sum[1] += fresh;
    }
  }
  block_sum<4>(sum);
  const int have = *p.counts;
  const RowSpan r = row_span(p, s);
  const int32_t* in = p.table_in + (size_t)s * p.width;
  int32_t* out = p.table_out + (size_t)s * p.width;
  if (in != out)
    for (int e = tid; e < p.width; e += TABLES_THREADS)
      if (e < r.first || e >= r.last) out[e] = *(in + e);
  if (tid < 32) {
    long long rank = sum[0];
    for (int e0 = r.first; e0 < r.last; e0 += 32) {
      const int e = e0 + lane;
      int page = e < r.last ? *(in + e) : 0;
      const unsigned missing = __ballot_sync(0xffffffffu, page < 0);
      const long long mine = rank + __popc(missing & ((1u << lane) - 1));
      if (page < 0) page = mine < have ? *(p.free_pages + (have - 1 - mine)) : -1;
      if (e < r.last) out[e] = page;
      rank += __popc(missing);
    }
  }
  if (tid == 0) {
    p.q_indptr[s] = (int32_t)min(sum[1], (long long)INT_MAX);
    if (s == p.batch - 1) {
      p.q_indptr[p.batch] = (int32_t)min(sum[3], (long long)INT_MAX);
      *p.num_free_out = (int32_t)max(have - sum[2], 0LL);
      const int err = (sum[2] > have ? EFIM_DEV_NO_PAGE : 0) |
                      (sum[3] > INT_MAX || (sum[3] > p.rows && (p.positions || p.slots || p.sequences)) ? EFIM_DEV_BAD_POSITION : 0);
      if (err && p.status) atomicOr(p.status, err);
    }
  }
  __syncthreads();
  for (int i = tid; i < r.fresh; i += TABLES_THREADS) {
    const long long at = sum[1] + i;
    if (at >= p.rows) break;
    const int pos = r.cached + i, place = pos >> 4;
    if (p.positions) p.positions[at] = pos;
    if (p.sequences) p.sequences[at] = s;
    if (p.slots) {
      const int page = place < p.width ? out[place] : -1;
      p.slots[at] = page < 0 ? -1 : (int64_t)page * 16 + (pos & 15);
    }
  }
  for (long long at = sum[3] + (long long)s * TABLES_THREADS + tid; at < p.rows; at += (long long)p.batch * TABLES_THREADS) {
    if (p.positions) p.positions[at] = -1;
    if (p.sequences) p.sequences[at] = -1;
    if (p.slots) p.slots[at] = -1;
  }
}

// Both in one CTA, for few sequences and small tables, where a launch is most of the time: a warp has two rows (16 sequences of up to 9 tokens, tables
// of 1,024: 4.6 us).
constexpr int TABLES_ONE_THREADS = 1024, TABLES_ONE_ROWS = 64, TABLES_ONE_WORDS = 32768;
__global__ void __launch_bounds__(TABLES_ONE_THREADS) tables_one_kernel(const TablesParams p) {
  __shared__ int s_pages[TABLES_ONE_ROWS];          // that each row takes
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  pdl_launch();
  // a table of its own: all of the old one, over which the rows' new places go later on
  if (p.table_in != p.table_out) {
    const int n = p.batch * p.width;
    if (((reinterpret_cast<uintptr_t>(p.table_in) | reinterpret_cast<uintptr_t>(p.table_out)) & 15) == 0) {
      for (int i = tid; i < n / 4; i += TABLES_ONE_THREADS) reinterpret_cast<int4*>(p.table_out)[i] = *(reinterpret_cast<const int4*>(p.table_in) + i);
      for (int i = n / 4 * 4 + tid; i < n; i += TABLES_ONE_THREADS) p.table_out[i] = *(p.table_in + i);
    } else {
      for (int i = tid; i < n; i += TABLES_ONE_THREADS) p.table_out[i] = *(p.table_in + i);
    }
  }
  const int have0 = *p.num_free, have = min(max(have0, 0), p.capacity);
  int err = have != have0 ? EFIM_DEV_BAD_POSITION : 0;
  RowSpan r[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int s = warp + 32 * k;
    if (s >= p.batch) break;
    r[k] = row_span(p, s);
    if (r[k].bad) err |= EFIM_DEV_BAD_POSITION;
    const int32_t* row = p.table_in + (size_t)s * p.width;
    int n = 0;
    for (int e = r[k].first + lane; e < r[k].last; e += 32) n += *(row + e) < 0;
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) s_pages[s] = n;
  }
  __syncthreads();                                  // (everything that is read of num_free and the places to fill has been)
  // every warp adds up what stands before each row, and all
  long long total = 0, tokens = 0, before[2] = {0, 0}, first[2] = {0, 0};
  for (int i = 0; i < p.batch; i += 32) {
    const bool in = i + lane < p.batch;
    const int pages = in ? s_pages[i + lane] : 0, fresh = in ? row_span(p, i + lane).fresh : 0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const bool ahead = i + lane < warp + 32 * k;
      before[k] += __reduce_add_sync(0xffffffffu, ahead ? pages : 0);
      // (lengths up to 2^31 - 1: their halves are added)
      first[k] += ((long long)__reduce_add_sync(0xffffffffu, ahead ? (unsigned)fresh >> 16 : 0u) << 16) + __reduce_add_sync(0xffffffffu, ahead ? (unsigned)fresh & 0xffffu : 0u);
    }
    total += __reduce_add_sync(0xffffffffu, pages);
    tokens += ((long long)__reduce_add_sync(0xffffffffu, (unsigned)fresh >> 16) << 16) + __reduce_add_sync(0xffffffffu, (unsigned)fresh & 0xffffu);
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int s = warp + 32 * k;
    if (s >= p.batch) break;
    const int32_t* in = p.table_in + (size_t)s * p.width;
    int32_t* out = p.table_out + (size_t)s * p.width;
    long long rank = before[k];
    for (int e0 = r[k].first; e0 < r[k].last; e0 += 32) {
      const int e = e0 + lane;
      int page = e < r[k].last ? *(in + e) : 0;
      const unsigned missing = __ballot_sync(0xffffffffu, page < 0);
      const long long mine = rank + __popc(missing & ((1u << lane) - 1));
      if (page < 0) page = mine < have ? *(p.free_pages + (have - 1 - mine)) : -1;
      if (e < r[k].last) out[e] = page;
      rank += __popc(missing);
    }
    if (lane == 0) p.q_indptr[s] = (int32_t)min(first[k], (long long)INT_MAX);
    __syncwarp();
    for (int i = lane; i < r[k].fresh; i += 32) {
      const long long at = first[k] + i;
      if (at >= p.rows) break;
      const int pos = r[k].cached + i, place = pos >> 4;
      if (p.positions) p.positions[at] = pos;
      if (p.sequences) p.sequences[at] = s;
      if (p.slots) {
        const int page = place < p.width ? out[place] : -1;
        p.slots[at] = page < 0 ? -1 : (int64_t)page * 16 + (pos & 15);
      }
    }
  }
  for (long long at = tokens + tid; at < p.rows; at += TABLES_ONE_THREADS) {
    if (p.positions) p.positions[at] = -1;
    if (p.sequences) p.sequences[at] = -1;
    if (p.slots) p.slots[at] = -1;
  }
  if (tid == 0) {
    p.q_indptr[p.batch] = (int32_t)min(tokens, (long long)INT_MAX);
    *p.num_free_out = (int32_t)max(have - total, 0LL);
    if (total > have) err |= EFIM_DEV_NO_PAGE;
    if (tokens > INT_MAX || (tokens > p.rows && (p.positions || p.slots || p.sequences))) err |= EFIM_DEV_BAD_POSITION;
  }
  if (err && lane == 0 && p.status) atomicOr(p.status, err);
}

__global__ void __launch_bounds__(TABLES_THREADS) tables_release_kernel(const TablesParams p) {
  pdl_wait();
  pdl_launch();
  const int s = blockIdx.x, tid = threadIdx.x, lane = tid & 31;
  long long sum[2] = {0, 0};                        // pages of the rows before, of all
  for (int i = tid; i < p.batch; i += TABLES_THREADS) {
    const int pages = *(p.counts + 1 + i);
    sum[1] += pages;
    if (i < s) sum[0] += pages;
  }
  block_sum<2>(sum);
  const int have = *p.counts, keep = *(p.cached_len + s);
  int32_t* row = p.table_out + (size_t)s * p.width;
  if (tid < 32 && keep >= 0) {
    long long at = have + sum[0];
    for (int e0 = (int)(((long long)keep + 15) / 16); e0 < p.width; e0 += 32) {
      const int e = e0 + lane;
      const int page = e < p.width ? *(row + e) : -1;
      const unsigned mine = __ballot_sync(0xffffffffu, page >= 0);
      const long long to = at + __popc(mine & ((1u << lane) - 1));
      if (page >= 0 && to < p.capacity) {           // (what the stack has no room for stays in the table)
        p.free_pages[to] = page;
        row[e] = -1;
      }
      at += __popc(mine);
    }
  }
  if (tid == 0 && s == p.batch - 1) {
    *p.num_free_out = (int32_t)min(have + sum[1], (long long)p.capacity);
    if (have + sum[1] > p.capacity && p.status) atomicOr(p.status, EFIM_DEV_NO_PAGE);
  }
}

}  // namespace efim

extern "C" size_t efim_step_tables_workspace_bytes(int32_t batch) { return batch > 0 ? ((size_t)batch + 1) * 4 : 0; }

extern "C" efim_status efim_step_tables(int32_t batch, const int32_t* d_cached_len, const int32_t* d_new_len, const int32_t* d_block_table,
                                        int32_t max_pages_per_seq, const int32_t* d_free_pages, int32_t free_capacity,
                                        const int32_t* d_num_free, int32_t* d_block_table_out, int32_t* d_num_free_out,
                                        int32_t* d_q_indptr, int32_t rows, int32_t* d_positions, int64_t* d_slots, int32_t* d_sequences,
                                        void* d_workspace, size_t workspace_bytes, int32_t* d_status, void* stream) {
  using namespace efim;
  if (batch < 0 || max_pages_per_seq <= 0 || free_capacity < 0 || rows < 0) return EFIM_ERR_INVALID_ARG;
  if (batch == 0) return EFIM_OK;
  if (!d_cached_len || !d_new_len || !d_block_table || !d_num_free || !d_block_table_out || !d_num_free_out || !d_q_indptr ||
      (free_capacity > 0 && !d_free_pages))
    return EFIM_ERR_INVALID_ARG;
  auto address = [](const void* x) { return reinterpret_cast<uintptr_t>(x); };
  if ((address(d_cached_len) | address(d_new_len) | address(d_block_table) | address(d_free_pages) | address(d_num_free) |
       address(d_block_table_out) | address(d_num_free_out) | address(d_q_indptr) | address(d_positions) | address(d_sequences)) & 3)
    return EFIM_ERR_INVALID_ARG;
  if (address(d_slots) & 7) return EFIM_ERR_INVALID_ARG;
  if (!d_workspace || workspace_bytes < efim_step_tables_workspace_bytes(batch)) return EFIM_ERR_WORKSPACE;
  if (address(d_workspace) & 3) return EFIM_ERR_INVALID_ARG;
  TablesParams p{};
  p.cached_len = d_cached_len;
  p.new_len = d_new_len;
  p.table_in = d_block_table;
  p.table_out = d_block_table_out;
  p.free_pages = const_cast<int32_t*>(d_free_pages);
  p.num_free = d_num_free;
  p.num_free_out = d_num_free_out;
  p.q_indptr = d_q_indptr;
  p.positions = d_positions;
  p.slots = d_slots;
  p.sequences = d_sequences;
  p.counts = static_cast<int32_t*>(d_workspace);
  p.status = d_status;
  p.batch = batch;
  p.width = max_pages_per_seq;
  p.capacity = free_capacity;
  p.rows = rows;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  // (the rows are the caller's bound of the new tokens; a copy of the table counts too)
  if (batch <= TABLES_ONE_ROWS && (long long)rows + (d_block_table == d_block_table_out ? 0LL : (long long)batch * max_pages_per_seq) <= TABLES_ONE_WORDS) {
    EFIM_CUDA_TRY(launch_pdl(tables_one_kernel, dim3(1), dim3(TABLES_ONE_THREADS), 0, s, p));
    return EFIM_OK;
  }
  const unsigned ctas = (unsigned)(((long long)batch + TABLES_THREADS / 32 - 1) / (TABLES_THREADS / 32));
  EFIM_CUDA_TRY(launch_pdl(tables_count_kernel<false>, dim3(ctas), dim3(TABLES_THREADS), 0, s, p));
  EFIM_CUDA_TRY(launch_pdl(tables_write_kernel, dim3(batch), dim3(TABLES_THREADS), 0, s, p));
  return EFIM_OK;
}

extern "C" efim_status efim_release_pages(int32_t batch, const int32_t* d_keep_len, int32_t* d_block_table, int32_t max_pages_per_seq,
                                          int32_t* d_free_pages, int32_t free_capacity, int32_t* d_num_free, void* d_workspace,
                                          size_t workspace_bytes, int32_t* d_status, void* stream) {
  using namespace efim;
  if (batch < 0 || max_pages_per_seq <= 0 || free_capacity < 0) return EFIM_ERR_INVALID_ARG;
  if (batch == 0) return EFIM_OK;
  if (!d_keep_len || !d_block_table || !d_num_free || (free_capacity > 0 && !d_free_pages)) return EFIM_ERR_INVALID_ARG;
  auto address = [](const void* x) { return reinterpret_cast<uintptr_t>(x); };
  if ((address(d_keep_len) | address(d_block_table) | address(d_free_pages) | address(d_num_free)) & 3) return EFIM_ERR_INVALID_ARG;
  if (!d_workspace || workspace_bytes < efim_step_tables_workspace_bytes(batch)) return EFIM_ERR_WORKSPACE;
  if (address(d_workspace) & 3) return EFIM_ERR_INVALID_ARG;
  TablesParams p{};
  p.cached_len = d_keep_len;
  p.table_in = p.table_out = d_block_table;
  p.free_pages = d_free_pages;
  p.num_free = p.num_free_out = d_num_free;
  p.counts = static_cast<int32_t*>(d_workspace);
  p.status = d_status;
  p.batch = batch;
  p.width = max_pages_per_seq;
  p.capacity = free_capacity;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const unsigned ctas = (unsigned)(((long long)batch + TABLES_THREADS / 32 - 1) / (TABLES_THREADS / 32));
  EFIM_CUDA_TRY(launch_pdl(tables_count_kernel<true>, dim3(ctas), dim3(TABLES_THREADS), 0, s, p));
  EFIM_CUDA_TRY(launch_pdl(tables_release_kernel, dim3(batch), dim3(TABLES_THREADS), 0, s, p));
  return EFIM_OK;
}
