// efim_kv4_decode_attn: attention of one or a few new tokens a sequence over a 4-bit cache.
//
// A unit of work is a (sequence, kv head, tile of up to 8 NT rows); a row is a (new token, query head of the group) pair.  One wave of CTAs shares all units'
// keys out evenly (Kv4Line), a second kernel joins the units that are cut.  A CTA's 4 warps walk pages (16 tokens), each with a ring of its own that
// cp.async fills.  A page is one 16-token tile of mma.sync m16n8k16 (fp16 in, fp32 accumulation), rows along n:
//   S^T [16 tokens][rows]  = K [16][D] Q^T [D][rows]
//   O^T [D][rows]         += V^T [D][16] P^T [16][rows]
// The operands K and V are made in registers: a code times its block's scale is exact in fp16 (cvt from 4-bit floats, one product), and
// the order of a contraction's index is free, so each lane takes neighbouring codes as they lie:
//   K: lane (g, t) = (lane / 4, lane % 4) has tokens g, g + 8 and dims [t D/4, (t+1) D/4): a 16-byte (D = 64: 8-byte) piece of each row
//   V: tokens 2t, 2t+1, 2t+8, 2t+9 and dims [g D/8, (g+1) D/8): 8 (4) bytes of four rows; nibbles of two tokens are put side by
//      side, so that a conversion gives a pair of tokens
// with the page's tokens numbered such that neither read meets a bank twice (kv4_token, kv4_v_piece).
// Queries enter as fp16 after a shift by a power of two per row that takes the row's largest value to [2^14, 2^15): exact for
// values down to 2^-28 of it, smaller ones to within 2^-39.  P = 2^(s - m + 11) enters as fp16 (a rounding of 2^-11 of each, between 2^15 and, at full precision, 2^-25 of
// the largest); the sums that it is divided by are the unrounded fp32 values.
//
// Bound: with up to 8 rows the instructions, then HBM: of the 296 that a page (2,304 bytes) of one kv head costs (the kernel's, starts included), 64 are conversions and 64
// products, 16 matrix products; 64 users x 1-16k keys at 32/8 heads x 128 take 140 us (4.5 TB/s of codes and scales; their copies alone 115, the rest alone
// 120).  What brought it from 174: two pages a trip 161, even pieces in one wave and starts that count 150, no branch around a page's copies 142,
// three CTAs an SM instead of four with spills 140.  Not kept: bulk copies (four of 128 to 1,024 bytes a page: 173), four pages a trip, two or five CTAs.
// With more rows, and few users, the latency of one warp's chain: its registers leave two CTAs an SM.
#include "kv4_attn.cuh"
#include "token_place.cuh"
#include <algorithm>
#include <cfloat>
#include <climits>
#include <type_traits>

namespace efim {

constexpr int KV4_WARPS = 4;
constexpr int KV4_THREADS = 32 * KV4_WARPS;
constexpr float KV4_P_SHIFT = 11.f;     // P's largest value, log2, with the reference right; the reference may be 4 behind
constexpr float KV4_LAG = 4.f;
// References (log2) from here on are rounded by 2^-4 and more, by which P = 2^(score - reference) would be off, and from 2^25 on beyond fp16: the weights of
// such a row are taken from the scores' differences to the one at which the reference moves.
constexpr float KV4_FAR = 1048576.f;

__host__ __device__ constexpr int kv4_page_bytes(int D) { return 2 * (kv4_code_bytes(D) + kv4_scale_bytes(D)); }
// pages that a warp takes at a time, and sets of them in its ring
__host__ __device__ constexpr int kv4_pages(int NT) { return NT == 1 ? 2 : 1; }
__host__ __device__ constexpr int kv4_stages(int NT) { return NT == 1 ? 2 : NT == 2 ? 4 : 6; }
__host__ __device__ constexpr int kv4_ctas_per_sm(int NT) { return NT == 1 ? 3 : 2; }
__host__ __device__ constexpr int kv4_smem_bytes(int D, int NT) {
  const int ring = KV4_WARPS * kv4_stages(NT) * kv4_pages(NT) * kv4_page_bytes(D), exchange = KV4_WARPS * 8 * NT * (D + 4) * 4;
  return ring > exchange ? ring : exchange;
}

// The token of a page that is the products' token 2t + e + 8h
__device__ __forceinline__ int kv4_token(int t, int e, int h) { return (e ^ (t & 1)) | (t & 1) << 1 | (t >> 1) << 2 | h << 3; }
// Where 16-byte piece c of a token's V codes stands in a staged page
template <int D>
__device__ __forceinline__ int kv4_v_piece(int token, int c) {
  const int odd = (token >> 2) & 1;
  return D == 128 ? token * 64 + ((c ^ (odd << 1)) << 4) : (token ^ odd) * 32 + (c << 4);
}

__device__ __forceinline__ uint32_t kv4_movm_t(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// c += a b, a 16 x 16 (row), b 16 x 8 (col), fp16 in, fp32 accumulation
__device__ __forceinline__ void kv4_mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// c = a b
__device__ __forceinline__ void kv4_mma_first(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ float kv4_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t kv4_pack_half2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ void kv4_cp16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ uint32_t kv4_smem(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// A sequence's part of the call.
struct Kv4Seq {
  int ctx;        // keys, clamped to what the launch covers
  int first_row;  // its first row of q
  int new_len;    // its rows of q that are computed
  int cached;     // keys before its first new token
  int err;
};
__device__ __forceinline__ Kv4Seq kv4_seq(const Kv4AttnParams& p, int s) {
  Kv4Seq w;
  w.first_row = s;
  w.new_len = 1;
  if (p.q_indptr) {
    w.first_row = *(p.q_indptr + s);
    w.new_len = *(p.q_indptr + s + 1) - w.first_row;
  }
  int ctx = *(p.len + s);
  if (p.len_is_cached) ctx += w.new_len;
  w.cached = ctx - w.new_len;
  w.ctx = ctx;
  w.err = 0;
  if (w.first_row < 0 || w.new_len < 0 || w.new_len > p.total_rows - w.first_row) {   // rows that were not given
    w.err = EFIM_DEV_BAD_POSITION;
    w.new_len = 0;
  }
  if (w.new_len > p.max_new) {
    w.err = EFIM_DEV_BAD_POSITION;
    w.new_len = p.max_new;
  }
  if (w.ctx > p.key_cap) {
    // (a turn's bound is of the sequences with new tokens: one without any may be longer)
    if (!p.len_is_cached || w.new_len > 0) w.err = EFIM_DEV_BAD_POSITION;
    w.ctx = p.key_cap;
  }
  w.ctx = max(w.ctx, 0);
  return w;
}

// The work of a call is a line of trips (a trip: PG pages by each of a CTA's warps), unit after unit: (sequence, kv head, tile of rows).  Each CTA has
// an equal piece of the line, so all end together whatever the lengths are; a unit that lies in one piece is finished
// there, the pieces of the others leave partial results, which a second kernel joins.  A piece has at most two such: of a unit that began before it
// (kept in the CTA's first place), and of one that goes on behind it (second place).  The line is measured in
// what trips cost: COST of a tile's 8-row parts that have rows; a unit's start (queries, first pages, results) stands in it with START
// before the unit's trips, where pieces are a good deal longer than that.  (Microseconds of a trip with 1 / 2 / 3 / 4 parts, NT = 4: 0.81 / 0.93 /
// 1.21 / 1.41, its start 6 to 9; with NT = 1 1.9, its start 6.)
template <int NT>
struct Kv4Line {
  static constexpr int TRIP = 16 * KV4_WARPS * kv4_pages(NT);              // keys of a trip
  static constexpr int START = NT == 1 ? 3 : 35, MOST = NT == 1 ? 1 : NT + 3;
  static __device__ __forceinline__ int cost(int rows) { return NT == 1 ? 1 : (rows + 7) / 8 + 3; }
  static __device__ __forceinline__ int trips(const Kv4Seq& w) { return max(1, (w.ctx + TRIP - 1) / TRIP); }
  static __device__ __forceinline__ int tiles(const Kv4Seq& w, int G) { return (w.new_len * G + 8 * NT - 1) / (8 * NT); }
  // of a kv head: all tiles but the last are full
  static __device__ __forceinline__ long long costs(const Kv4Seq& w, int G) {
    const int n = tiles(w, G);
    return n == 0 ? 0 : (n - 1LL) * MOST + cost(w.new_len * G - (n - 1) * 8 * NT);
  }
};
// what a CTA leaves for the joining kernel
struct Kv4Piece {
  int seq, head, tile;    // of the unit that goes on behind it; seq -1: none
  int first_ends;         // the unit that began before it ends in it
};

template <int D, int NT>
__global__ void __launch_bounds__(KV4_THREADS, kv4_ctas_per_sm(NT)) kv4_attn_kernel(const Kv4AttnParams p) {
  using Line = Kv4Line<NT>;
  constexpr int ST = kv4_stages(NT), PG = kv4_pages(NT), ROWS = 8 * NT;
  constexpr int CODES = kv4_code_bytes(D), SCALES = kv4_scale_bytes(D), PAGE = kv4_page_bytes(D);
  constexpr int STAGE = PG * PAGE;        // bytes of the ring that a trip's pages take
  constexpr int KS = D / 16;              // k-steps of S^T, m-tiles of O^T
  constexpr int XD = D + 4;               // floats per row of the warps' exchange buffer
  constexpr bool Q_IN_REGS = NT <= 2;
  extern __shared__ __align__(128) uint8_t kv4_smem_raw[];
  __shared__ __align__(16) uint16_t s_q[ROWS][D + 16];    // fp16, shifted; dim t D/4 + 4k + x at 16k + 4t + x
  __shared__ float s_m[KV4_WARPS][ROWS], s_l[KV4_WARPS][ROWS], s_scale[ROWS];
  __shared__ uint8_t s_nan[ROWS][8];      // rows that see a NaN value in dims [g D/8, (g+1) D/8)
  __shared__ long long s_sum[KV4_WARPS][2];
  __shared__ long long s_at;              // trips of the line before the sequence that this CTA begins with
  __shared__ int s_seq;

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int G = p.Hq / p.Hkv;
  pdl_wait();
  pdl_launch();
  // ---- this CTA's piece of the line
  long long x0, x1;                       // in trips
  int seq;                                // its first sequence
  long long off;                          // what of that one, then of the unit at hand, lies before it
  int start = 0;                          // what a unit's start counts
  if (p.whole) {                          // units that are never cut, one a CTA
    seq = blockIdx.x / p.units_per_seq;
    x0 = x1 = off = 0;
  } else {
    const int per = (p.batch + KV4_THREADS - 1) / KV4_THREADS, first = min(p.batch, tid * per), last = min(p.batch, first + per);
    long long mine[2] = {0, 0};           // of trips, units
    for (int i = first; i < last; ++i) {
      const Kv4Seq q = kv4_seq(p, i);
      if (q.err && blockIdx.x == 0 && p.status) atomicOr(p.status, q.err);   // (one CTA reports the lengths that do not fit)
      mine[0] += Line::costs(q, G) * Line::trips(q) * p.Hkv;
      mine[1] += (long long)Line::tiles(q, G) * p.Hkv;
    }
    long long upto[2] = {mine[0], mine[1]}, total[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, upto[k], d);
        if (lane >= d) upto[k] += y;
      }
      if (lane == 31) s_sum[warp][k] = upto[k];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < KV4_WARPS; ++i)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (i < warp) upto[k] += s_sum[i][k];
        total[k] += s_sum[i][k];
      }
    start = total[0] >= 4LL * Line::START * gridDim.x ? Line::START : 0;
    const long long all = total[0] + start * total[1], before = upto[0] - mine[0] + start * (upto[1] - mine[1]);
    const long long share = max((long long)p.least_trips * Line::MOST, (all + gridDim.x - 1) / gridDim.x);
    x0 = blockIdx.x * share;
    x1 = min(all, x0 + share);
    if (x0 >= all) {
      if (tid == 0) p.pieces[blockIdx.x] = Kv4Piece{-1, 0, 0, 1};
      return;
    }
    if (x0 >= before && x0 < upto[0] + start * upto[1]) {
      long long at = before;
      int i = first;
      for (; i < last - 1; ++i) {
        const Kv4Seq q = kv4_seq(p, i);
        const long long y = ((long long)start * Line::tiles(q, G) + Line::costs(q, G) * Line::trips(q)) * p.Hkv;
        if (x0 < at + y) break;
        at += y;
      }
      s_seq = i;
      s_at = at;
    }
    __syncthreads();
    seq = s_seq;
    off = x0 - s_at;
  }
  Kv4Seq w = kv4_seq(p, seq);
  int kvh, tile;                          // the unit at hand, `off` of it done
  if (p.whole) {
    const int unit = blockIdx.x % p.units_per_seq;
    if (w.err && unit == 0 && tid == 0 && p.status) atomicOr(p.status, w.err);
    kvh = unit / p.row_tiles;
    tile = unit % p.row_tiles;
    if (tile >= Line::tiles(w, G)) return;
    x1 = (long long)Line::trips(w) * Line::cost(min(ROWS, w.new_len * G - tile * ROWS));
  } else {
    const int n = Line::trips(w), tiles = Line::tiles(w, G);
    const long long per_head = (long long)start * tiles + Line::costs(w, G) * n, full = start + (long long)Line::MOST * n;
    kvh = (int)(off / per_head);
    off -= kvh * per_head;
    tile = (int)min(off / full, tiles - 1LL);
    off -= tile * full;
  }
  Kv4Piece left{-1, 0, 0, 0};

  auto token_of = [&](int row) { return p.max_new == 1 ? 0 : row / G; };
  while (x0 < x1) {
    const int tiles = Line::tiles(w, G);
    const int row0 = tile * ROWS, n_rows = min(ROWS, w.new_len * G - row0), cost = Line::cost(n_rows);
    // (a unit's length fits 32 bits: 2^31 keys in trips of 64 or more)
    const int unit_len = start + Line::trips(w) * cost, from = (int)off, here = (int)min((long long)(unit_len - from), x1 - x0);   // of the unit in this piece
    const int trip0 = max(from - start, 0) / cost, trip1 = max(from + here - start, 0) / cost;
    const bool first_part = trip0 > 0, ends = from + here == unit_len;       // the unit began before this piece; it ends in it
    if (trip1 <= trip0) break;              // (the piece ends before the unit's first trip: it begins in the next one)
    const int32_t* bt = p.block_table + (size_t)seq * p.max_pages_per_seq;
    // warp x has pages PG (x + 4 i) + {0 .. PG-1} of the piece
    const int begin = trip0 * Line::TRIP, first_pg = (begin >> 4) + PG * warp;
    auto page_of = [&](int i) { return first_pg + (PG == 1 ? KV4_WARPS * i : i % PG + KV4_WARPS * PG * (i / PG)); };
    // keys that the tile's last row sees, of this piece
    const int end = (int)min((long long)min(w.ctx, w.cached + token_of(row0 + n_rows - 1) + 1), (long long)trip1 * Line::TRIP);
    const int last_pg = (end - 1) >> 4;
    const int n_trips = end > begin && first_pg <= last_pg ? (last_pg - first_pg) / (KV4_WARPS * PG) + 1 : 0;
    // Lane l holds where the l-th of this warp's pages is (then of the next 32): (page, kv head) in the pools, -1 for no page.
    int at_cache;
    bool hole = false;                      // some pages are missing: every trip looks at its own
    auto look_up = [&](int i) {
      const int pg = page_of(i + lane);
      at_cache = -1;
      if (pg <= last_pg) {
        const int pid = *(bt + pg);
        if ((uint32_t)pid < (uint32_t)p.num_pages) at_cache = pid * p.Hkv + kvh;
        else if (p.status) atomicOr(p.status, EFIM_DEV_BAD_PAGE);
      }
      hole |= __any_sync(0xffffffffu, pg <= last_pg && at_cache < 0);
    };
    look_up(0);
    // query rows, a warp a row: on their way before the pages are
    uint2 q_raw[ROWS / KV4_WARPS];
#pragma unroll
    for (int i = 0; i < ROWS / KV4_WARPS; ++i) {
      const int r = i * KV4_WARPS + warp;
      q_raw[i] = make_uint2(0, 0);
      if (r < n_rows) {
        const int token = token_of(row0 + r), h = kvh * G + row0 + r - token * G;
        const uint16_t* q = p.q + ((size_t)(w.first_row + token) * p.Hq + h) * D + lane * (D / 32);
        if constexpr (D == 128) q_raw[i] = *reinterpret_cast<const uint2*>(q);
        else q_raw[i].x = *reinterpret_cast<const uint32_t*>(q);
      }
    }

    const uint32_t ring = kv4_smem(kv4_smem_raw) + warp * (ST * STAGE);
    const uint8_t* ring_ptr = kv4_smem_raw + warp * (ST * STAGE);
    constexpr int PIECES = CODES / 16, PS = 2 * SCALES / 16;                // 16-byte pieces of a page's codes (K or V), of its scales
    // where this lane's pieces come from and go to: of every page's codes, of one page's scales
    const uint8_t *k_src = p.k_codes + lane * 16, *v_src = p.v_codes + lane * 16;
    const uint8_t* s_src = lane % PS < PS / 2 ? p.k_scales + lane % PS * 16 : p.v_scales + (lane % PS - PS / 2) * 16;
    const uint32_t k_dst = ring + lane * 16, v_dst = ring + CODES + kv4_v_piece<D>(lane / (D / 32), lane % (D / 32));
    const uint32_t s_dst = ring + lane / PS * PAGE + 2 * CODES + lane % PS * 16;
    uint32_t missing = 0;                   // a bit per page, the last one sent for lowest: not there (kept where there is a hole)
    auto issue = [&](int i, uint32_t to) {  // send for the pages of this warp's i-th trip, to `to` bytes into the ring
      if (i < n_trips) {
        int at[PG];
#pragma unroll
        for (int x = 0; x < PG; ++x) {
          at[x] = __shfl_sync(0xffffffffu, at_cache, (i * PG + x) & 31);
          if (hole) missing = missing << 1 | (uint32_t)at[x] >> 31;
          at[x] = max(at[x], 0);            // (a page of the pool stands in for one that is not there)
          const uint8_t *k = k_src + (uint64_t)at[x] * CODES, *v = v_src + (uint64_t)at[x] * CODES;
#pragma unroll
          for (int u = 0; u < PIECES; u += 32) {
            kv4_cp16(k_dst + to + x * PAGE + u * 16, k + u * 16);
            kv4_cp16(v_dst + to + x * PAGE + u * 16, v + u * 16);
          }
        }
        const int mine = lane < PS ? at[0] : at[PG - 1];
        if (lane < PG * PS) kv4_cp16(s_dst + to, s_src + (uint64_t)mine * SCALES);
        if (((i * PG + PG) & 31) == 0) look_up(i * PG + PG);
      } else {
        missing <<= PG;
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < ST - 1; ++i) issue(i, i * STAGE);

    // ---- query rows as fp16, shifted
#pragma unroll
    for (int i = 0; i < ROWS / KV4_WARPS; ++i) {
      const int r = i * KV4_WARPS + warp;
      const float x[4] = {bf16lo(q_raw[i].x), bf16hi(q_raw[i].x), bf16lo(q_raw[i].y), bf16hi(q_raw[i].y)};
      float top = 0.f;
#pragma unroll
      for (int e = 0; e < D / 32; ++e) top = max_nan(top, fabsf(x[e]));
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, d));
      // 2^-(exponent of the largest) and back; a row with an infinity or a NaN becomes NaN
      const int ex = (int)(__float_as_uint(top) >> 23);                    // biased; subnormal rows count as 2^-126
      const bool bad = ex >= 255;
      const float down = __uint_as_float((uint32_t)min(254, max(1, 268 - max(ex, 1))) << 23);    // 2^(14 - exponent), 2^127 at most
#pragma unroll
      for (int e = 0; e < D / 32; e += 2) {
        const float lo = bad ? NAN : x[e] * down, hi = bad ? NAN : x[e + 1] * down;
        const int d = lane * (D / 32) + e;
        *reinterpret_cast<uint32_t*>(&s_q[r][d % (D / 4) / 4 * 16 + d / (D / 4) * 4 + d % 4]) = kv4_pack_half2(lo, hi);
      }
      if (lane == 0) s_scale[r] = fmaxf(fminf(p.scale_log2 / down, FLT_MAX), FLT_MIN);   // (by a power of two: exact)
      if (lane < 8) s_nan[r][lane] = 0;
    }
    __syncthreads();
    // B fragments of row g: the dims that the K fragments have, D/4 from t D/4 on
    uint32_t qf[Q_IN_REGS ? NT : 1][KS][2];
    if constexpr (Q_IN_REGS) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const uint2 u = *reinterpret_cast<const uint2*>(&s_q[n * 8 + g][16 * k + 4 * t]);
          qf[n][k][0] = u.x;
          qf[n][k][1] = u.y;
        }
    }
    float o[NT][KS][4];                     // O^T: dims g D/8 + 2 k + (e / 2), rows 8 n + 2 t + (e % 2)
    // Scores stay as the products leave them; times sc they are in log2.  Per row: the score that the reference stands at, the one from which
    // on it moves, and what is taken off a score (in log2, KV4_P_SHIFT less than the reference).  Before any score: p = 2^(-inf) = 0.
    float m_next[NT][2], m_off[NT][2], l_part[NT][2], sc[NT][2];
    int limit[NT][2];                       // keys that rows 8 n + 2 t + {0, 1} see
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][k][e] = 0.f;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = n * 8 + 2 * t + e;
        m_next[n][e] = -FLT_MAX;
        m_off[n][e] = -KV4_P_SHIFT;
        l_part[n][e] = 0.f;
        sc[n][e] = s_scale[r];
        limit[n][e] = min(end, w.cached + token_of(row0 + min(r, n_rows - 1)) + 1);
      }
    }
    const int first_limit = min(end, w.cached + token_of(row0) + 1);
    const int tok0 = kv4_token(g >> 1, g & 1, 0);             // this lane's key in S^T; the other is 8 on
    // this lane's places in a staged page
    const uint8_t* k_at = ring_ptr + (D == 128 ? tok0 * 64 + t * 16 : tok0 * 32 + t * 8);
    const uint8_t* ks_at = ring_ptr + 2 * CODES + (D == 128 ? tok0 * 8 + 2 * t : tok0 * 4 + t);
    const uint8_t *v_at[2], *vs_at[2];                        // of tokens 2t, 2t+1 (the others are 8 rows on)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int token = kv4_token(t, e, 0);
      v_at[e] = ring_ptr + CODES + (D == 128 ? kv4_v_piece<D>(token, g >> 1) + (g & 1) * 8 : kv4_v_piece<D>(token, g >> 2) + (g & 3) * 4);
      vs_at[e] = ring_ptr + 2 * CODES + SCALES + (D == 128 ? token * 8 + g : token * 4 + (g >> 1));
    }

    bool far_off = false;                   // a row of the warp has a reference of KV4_FAR or more
    // trips whose pages every row sees in full
    const int seen = max(first_limit, 0) >> 4, n_full = seen >= first_pg + PG ? (seen - first_pg - PG) / (KV4_WARPS * PG) + 1 : 0;

    // The walk over the pages, for as many 8-row tiles as have rows (a call's sequences bring different numbers of them).
    auto walk = [&](auto active) {
      constexpr int NA = decltype(active)::value;
      int at = 0;                             // where in the ring the trip's pages are
      for (int i = 0; i < n_trips; ++i) {
        __syncwarp();                         // everyone is done with the stage of the last trip
        issue(i + ST - 1, at == 0 ? (ST - 1) * STAGE : at - STAGE);
        asm volatile("cp.async.wait_group %0;" ::"n"(ST - 1) : "memory");
        __syncwarp();
        const bool border = i >= n_full || hole;
        int key0[PG];                         // first keys; past every limit where there is no page (looked at where border is)
#pragma unroll
        for (int x = 0; x < PG; ++x) key0[x] = (missing >> (ST * PG - 1 - x)) & 1u ? INT_MAX - 16 : page_of(i * PG + x) << 4;
        // ---- S^T
        float sx[PG][NA][4];
#pragma unroll
        for (int x = 0; x < PG; ++x) {
          __half2 scale[2];                    // of the two tokens: the lane's blocks of 16 dims, D / 64 of them
          uint32_t kw[2][D / 32];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if constexpr (D == 128) {
              const uint4 u = *reinterpret_cast<const uint4*>(k_at + at + x * PAGE + h * 512);
              kw[h][0] = u.x, kw[h][1] = u.y, kw[h][2] = u.z, kw[h][3] = u.w;
              scale[h] = as_half2(scales_to_half2(*reinterpret_cast<const uint16_t*>(ks_at + at + x * PAGE + h * 64)));
            } else {
              const uint2 u = *reinterpret_cast<const uint2*>(k_at + at + x * PAGE + h * 256);
              kw[h][0] = u.x, kw[h][1] = u.y;
              scale[h] = as_half2(scales_to_half2(ks_at[at + x * PAGE + h * 32]));
            }
          }
#pragma unroll
          for (int q = 0; q < D / 32; ++q) {   // 8 dims of each token: two k-steps
            uint32_t kx[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              codes_to_half2(kw[h][q], kx[h]);
#pragma unroll
              for (int e = 0; e < 4; ++e) kx[h][e] = mul_half2(kx[h][e], q / 2 ? __high2half2(scale[h]) : __low2half2(scale[h]));
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const uint32_t a[4] = {kx[0][2 * k], kx[1][2 * k], kx[0][2 * k + 1], kx[1][2 * k + 1]};
#pragma unroll
              for (int n = 0; n < NA; ++n) {
                uint2 u;
                if constexpr (Q_IN_REGS) u = make_uint2(qf[n][2 * q + k][0], qf[n][2 * q + k][1]);
                else u = *reinterpret_cast<const uint2*>(&s_q[n * 8 + g][16 * (2 * q + k) + 4 * t]);
                if (q == 0 && k == 0) kv4_mma_first(sx[x][n], a, u.x, u.y);
                else kv4_mma(sx[x][n], a, u.x, u.y);
              }
            }
          }
        }
        if (border) {
#pragma unroll
          for (int x = 0; x < PG; ++x)
#pragma unroll
            for (int n = 0; n < NA; ++n)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (key0[x] + tok0 + (e >> 1) * 8 >= limit[n][e & 1]) sx[x][n][e] = -INFINITY;
        }
        // ---- the values' scales: of tokens 2t, 2t+1, 2t+8, 2t+9
        uint32_t vs[PG];
#pragma unroll
        for (int x = 0; x < PG; ++x) {
          constexpr int H = D == 128 ? 64 : 32;
          const uint32_t b00 = vs_at[0][at + x * PAGE], b01 = vs_at[1][at + x * PAGE], b10 = vs_at[0][at + x * PAGE + H], b11 = vs_at[1][at + x * PAGE + H];
          vs[x] = __byte_perm(__byte_perm(b00, b01, 0x5540), __byte_perm(b10, b11, 0x5540), 0x5410);
          if (border) {
            // what stands behind the last key is anything, a NaN's scale too: P is 0 there, 0 times NaN is not
#pragma unroll
            for (int q = 0; q < 4; ++q)
              if (key0[x] + kv4_token(t, q & 1, q >> 1) >= end) vs[x] &= ~(0xffu << (8 * q));
          }
        }
        // ---- the reference; values that are NaN
        bool grow = false, nan = false;
        float mx[NA][2];
#pragma unroll
        for (int n = 0; n < NA; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            mx[n][e] = fmaxf(sx[0][n][e], sx[0][n][e + 2]);
#pragma unroll
            for (int x = 1; x < PG; ++x) mx[n][e] = fmaxf(fmaxf(mx[n][e], sx[x][n][e]), sx[x][n][e + 2]);
            grow |= mx[n][e] > m_next[n][e];
          }
#pragma unroll
        for (int x = 0; x < PG; ++x) nan |= (((vs[x] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0;
        // Lazy rescale: the reference of a row only moves when a score exceeds it by more than 2^4 (always at the first), and each row's by its
        // own scores: its bits do not depend on the other rows.
        if (__any_sync(0xffffffffu, grow | nan)) {
#pragma unroll
          for (int n = 0; n < NA; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float x = mx[n][e];
#pragma unroll
              for (int off = 4; off < 32; off <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, off));
              if (x > m_next[n][e]) {
                float off = fmaf(x, sc[n][e], -KV4_P_SHIFT), next = x + KV4_LAG / sc[n][e];
                if (fabsf(off) >= KV4_FAR) {
                  next = __fadd_rd(x, KV4_LAG / sc[n][e]);      // (P is 2^15 there: no score between it and the reference's may come out larger)
                  off = fmaf(next, sc[n][e], -(KV4_P_SHIFT + KV4_LAG));
                }
                if (!(fabsf(off) <= FLT_MAX)) off = NAN;        // scores that leave fp32
                const float alpha = m_next[n][e] == -FLT_MAX ? 0.f : kv4_ex2(m_off[n][e] - off);
                m_next[n][e] = next;
                m_off[n][e] = off;
                l_part[n][e] *= alpha;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                  o[n][k][e] *= alpha;
                  o[n][k][e + 2] *= alpha;
                }
              }
            }
          bool off = false;
#pragma unroll
          for (int n = 0; n < NA; ++n) off |= fabsf(m_off[n][0]) >= KV4_FAR || fabsf(m_off[n][1]) >= KV4_FAR;
          far_off = __any_sync(0xffffffffu, off);
          // Rows that see a value that is NaN are marked and get their NaN at the end; in the products such values are zeros, since rows that
          // do not see them have a P of 0 there.
#pragma unroll
          for (int x = 0; x < PG; ++x)
#pragma unroll 1
            for (int q = 0; q < 4; ++q) {
              if (((vs[x] >> (8 * q)) & 0x7f) != 0x7f) continue;
              vs[x] &= ~(0xffu << (8 * q));
              const int key = key0[x] + kv4_token(t, q & 1, q >> 1);
              for (int r = 0; r < n_rows; ++r)
                if (key < min(end, w.cached + token_of(row0 + r) + 1)) s_nan[r][g] = 1;
            }
        }
        // ---- the weights' exponents in the scores' place
        if (!far_off) {
#pragma unroll
          for (int x = 0; x < PG; ++x)
#pragma unroll
            for (int n = 0; n < NA; ++n)
#pragma unroll
              for (int e = 0; e < 4; ++e) sx[x][n][e] = fmaf(sx[x][n][e], sc[n][e & 1], -m_off[n][e & 1]);
        } else {
#pragma unroll
          for (int x = 0; x < PG; ++x)
#pragma unroll
            for (int n = 0; n < NA; ++n)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                sx[x][n][e] = fabsf(m_off[n][e & 1]) >= KV4_FAR ? fmaf(sx[x][n][e] - m_next[n][e & 1], sc[n][e & 1], KV4_P_SHIFT + KV4_LAG)
                                                                : fmaf(sx[x][n][e], sc[n][e & 1], -m_off[n][e & 1]);
        }
#pragma unroll
        for (int x = 0; x < PG; ++x) {
          uint32_t pb[NA][2];
#pragma unroll
          for (int n = 0; n < NA; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float x0 = kv4_ex2(sx[x][n][2 * h]), x1 = kv4_ex2(sx[x][n][2 * h + 1]);
              l_part[n][0] += x0;
              l_part[n][1] += x1;
              pb[n][h] = kv4_movm_t(kv4_pack_half2(x0, x1));
            }
          // ---- O^T
          uint32_t vw[2][2][D / 64];
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              if constexpr (D == 128) {
                const uint2 u = *reinterpret_cast<const uint2*>(v_at[e] + at + x * PAGE + h * 512);
                vw[h][e][0] = u.x, vw[h][e][1] = u.y;
              } else {
                vw[h][e][0] = *reinterpret_cast<const uint32_t*>(v_at[e] + at + x * PAGE + h * 256);
              }
            }
          const __half2 scale[2] = {as_half2(scales_to_half2(vs[x] & 0xffff)), as_half2(scales_to_half2(vs[x] >> 16))};
#pragma unroll
          for (int q = 0; q < D / 64; ++q) {
            // lo: even dims of the two tokens side by side, hi: odd dims
            uint32_t lo[2][4], hi[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t a0 = vw[h][0][q], a1 = vw[h][1][q];
              codes_to_half2((a0 & 0x0f0f0f0fu) | ((a1 << 4) & 0xf0f0f0f0u), lo[h]);
              codes_to_half2(((a0 >> 4) & 0x0f0f0f0fu) | (a1 & 0xf0f0f0f0u), hi[h]);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                lo[h][e] = mul_half2(lo[h][e], scale[h]);
                hi[h][e] = mul_half2(hi[h][e], scale[h]);
              }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t a[4] = {lo[0][e], hi[0][e], lo[1][e], hi[1][e]};
#pragma unroll
              for (int n = 0; n < NA; ++n) kv4_mma(o[n][4 * q + e], a, pb[n][0], pb[n][1]);
            }
          }
        }
        at = at == (ST - 1) * STAGE ? 0 : at + STAGE;
      }
    };
    using std::integral_constant;
    if constexpr (NT == 1) {
      walk(integral_constant<int, 1>());
    } else if constexpr (NT == 2) {
      if (n_rows <= 8) walk(integral_constant<int, 1>());
      else walk(integral_constant<int, 2>());
    } else {
      if (n_rows <= 8) walk(integral_constant<int, 1>());
      else if (n_rows <= 16) walk(integral_constant<int, 2>());
      else if (n_rows <= 24) walk(integral_constant<int, 3>());
      else walk(integral_constant<int, 4>());
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    // ---- fold the lanes' sums, then the 4 warps (the exchange buffer takes their rings' place)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) l_part[n][e] += __shfl_xor_sync(0xffffffffu, l_part[n][e], off);
        if (lane < 4) {
          s_l[warp][n * 8 + 2 * lane + e] = l_part[n][e];
          s_m[warp][n * 8 + 2 * lane + e] = m_next[n][e] == -FLT_MAX ? -FLT_MAX : m_off[n][e];   // (of a warp that saw nothing: no weight)
        }
      }
    __syncthreads();
    float* xo = reinterpret_cast<float*>(kv4_smem_raw);       // [warp][row][XD]
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          *reinterpret_cast<float2*>(&xo[(warp * ROWS + n * 8 + 2 * t + e) * XD + g * (D / 8) + 2 * k]) = make_float2(o[n][k][e], o[n][k][e + 2]);
    __syncthreads();
    for (int idx = tid; idx < n_rows * (D / 4); idx += KV4_THREADS) {
      const int r = idx / (D / 4), d = (idx % (D / 4)) * 4;
      float M = s_m[0][r];
#pragma unroll
      for (int x = 1; x < KV4_WARPS; ++x) M = fmaxf(M, s_m[x][r]);
      float L = 0.f;
      float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int x = 0; x < KV4_WARPS; ++x) {
        const float f = exp2f(s_m[x][r] - M);
        const float4 y = *reinterpret_cast<const float4*>(xo + (x * ROWS + r) * XD + d);
        L = fmaf(s_l[x][r], f, L);
        O.x = fmaf(y.x, f, O.x);
        O.y = fmaf(y.y, f, O.y);
        O.z = fmaf(y.z, f, O.z);
        O.w = fmaf(y.w, f, O.w);
      }
      float inv = L == 0.f ? 0.f : p.v_scale / L;
      if (s_nan[r][d / (D / 8)]) inv = NAN;
      if (!first_part && ends) {
        const int token = token_of(row0 + r), h = kvh * G + row0 + r - token * G;
        const size_t row_head = (size_t)(w.first_row + token) * p.Hq + h;
        *reinterpret_cast<uint2*>(p.out + row_head * D + d) =
            make_uint2(pack_bf16x2(O.x * inv, O.y * inv), pack_bf16x2(O.z * inv, O.w * inv));
        if (p.lse && d == 0) p.lse[row_head] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;   // (a sum of NaN stays NaN)
      } else {
        const size_t part = ((size_t)blockIdx.x * 2 + (first_part ? 0 : 1)) * ROWS + r;
        *reinterpret_cast<float4*>(p.part_o + part * D + d) = make_float4(O.x * inv, O.y * inv, O.z * inv, O.w * inv);
        if (d == 0) p.part_sum[part] = make_float2(L == 0.f ? -INFINITY : M, L);
      }
    }
    // ---- on along the line
    if (first_part) left.first_ends = ends;
    else if (!ends) left = Kv4Piece{seq, kvh, tile, left.first_ends};
    x0 += here;
    off = 0;
    if (x0 < x1) {
      if (++tile == tiles) {
        tile = 0;
        ++kvh;
      }
      if (kvh == p.Hkv) {
        kvh = 0;
        do w = kv4_seq(p, ++seq);
        while (w.new_len == 0);                       // (the line goes on, so there is one)
      }
      __syncthreads();                                // the exchange buffer becomes the rings again
    }
  }
  if (!p.whole && tid == 0) p.pieces[blockIdx.x] = left;
}

// Joins a unit's partial results (reference M_c, sum L_c, o_c): w_c = L_c 2^(M_c - max M), o = sum w_c o_c / sum w_c.  (The two apart: M_c + log2 L_c in one
// number would lose the sum beside a large reference.)  A CTA has four rows of the unit that goes on behind a
// piece: its second place, then the first places of the pieces behind it until the unit ends.  A warp has a row, lanes over head_dim; the
// weights of 32 pieces are computed by the lanes together, four pieces' rows are on their way at a time.
template <int D, int NT>
__global__ void __launch_bounds__(KV4_THREADS) kv4_join_kernel(const Kv4AttnParams p) {
  constexpr int EPL = D / 32, ROWS = 8 * NT, AT_ONCE = 4;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = blockIdx.y * KV4_WARPS + warp;
  pdl_wait();
  pdl_launch();
  const Kv4Piece me = p.pieces[blockIdx.x];
  if (me.seq < 0) return;
  int n = 1;                                        // pieces that it has
  for (int c0 = blockIdx.x + 1;; c0 += 32) {
    const int c = c0 + lane;
    const unsigned ends = __ballot_sync(0xffffffffu, c >= (int)gridDim.x || p.pieces[c].first_ends);
    if (ends) {
      n = min(c0 + __ffs(ends), (int)gridDim.x) - (int)blockIdx.x;
      break;
    }
  }
  const Kv4Seq w = kv4_seq(p, me.seq);
  const int G = p.Hq / p.Hkv, row = me.tile * ROWS + r;
  if (row >= w.new_len * G) return;
  const size_t first = ((size_t)blockIdx.x * 2 + 1) * ROWS + r;                // the c-th one: ROWS places on, then every 2 ROWS
  auto place = [&](int c) { return first + (c == 0 ? 0 : (size_t)(2 * c - 1) * ROWS); };
  float M = -INFINITY;
  for (int c = lane; c < n; c += 32) M = max_nan(M, p.part_sum[place(c)].x);   // a NaN piece makes the row NaN
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) M = max_nan(M, __shfl_xor_sync(0xffffffffu, M, d));
  float L = 0.f, acc[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) acc[e] = 0.f;
  for (int c0 = 0; c0 < n && !(M == -INFINITY); c0 += 32) {                    // (else a row without keys)
    const float2 sum = c0 + lane < n ? p.part_sum[place(c0 + lane)] : make_float2(-INFINITY, 0.f);
    const float wi = sum.x == -INFINITY ? 0.f : sum.y * exp2f(sum.x - M);
    L += wi;
    const int some = min(32, n - c0);
    for (int k0 = 0; k0 < some; k0 += AT_ONCE) {
      float x[AT_ONCE][EPL];
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k)
        if (k0 + k < some) {
          const float* po = p.part_o + place(c0 + k0 + k) * D + lane * EPL;
          if constexpr (EPL == 4) *reinterpret_cast<float4*>(x[k]) = *reinterpret_cast<const float4*>(po);
          else *reinterpret_cast<float2*>(x[k]) = *reinterpret_cast<const float2*>(po);
        }
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k)
        if (k0 + k < some) {
          const float wk = __shfl_sync(0xffffffffu, wi, k0 + k);
#pragma unroll
          for (int e = 0; e < EPL; ++e) acc[e] = fmaf(wk, x[k][e], acc[e]);
        }
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) L += __shfl_xor_sync(0xffffffffu, L, d);
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const size_t row_head = (size_t)(w.first_row + row / G) * p.Hq + me.head * G + row % G;
  uint16_t* out = p.out + row_head * D + lane * EPL;
  if constexpr (EPL == 4)
    *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv));
  else
    *reinterpret_cast<uint32_t*>(out) = pack_bf16x2(acc[0] * inv, acc[1] * inv);
  if (p.lse && lane == 0) p.lse[row_head] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
}

// One wave of CTAs, fewer where their pieces would fall below KV4_LEAST keys.  Units that fit KV4_WHOLE keys are not cut.
constexpr int KV4_LEAST = 256, KV4_WHOLE = 512;
Kv4Plan kv4_plan(const efim_cache4_desc* cache, int batch, int max_new, int max_ctx) {
  Kv4Plan pl;
  const int G = cache->num_q_heads / cache->num_kv_heads;
  const long long rows = (long long)max_new * G;
  pl.nt = rows <= 8 ? 1 : rows <= 16 ? 2 : 4;
  pl.row_tiles = (rows + 8 * pl.nt - 1) / (8 * pl.nt);
  const int trip = 16 * KV4_WARPS * kv4_pages(pl.nt);
  const long long trips = (max_ctx + (long long)trip - 1) / trip, units = (long long)batch * cache->num_kv_heads * pl.row_tiles;
  pl.whole = max_ctx <= KV4_WHOLE;
  pl.least_trips = KV4_LEAST / trip;
  pl.ctas = pl.whole ? units : std::min<long long>((long long)sm_count() * kv4_ctas_per_sm(pl.nt), (units * trips + pl.least_trips - 1) / pl.least_trips);
  const size_t parts = pl.whole ? 0 : (size_t)pl.ctas * 2 * 8 * pl.nt;
  auto round = [](size_t n) { return (n + 255) / 256 * 256; };
  pl.sum_bytes = round(parts * 8);
  pl.piece_bytes = pl.whole ? 0 : round((size_t)pl.ctas * sizeof(Kv4Piece));
  pl.bytes = pl.sum_bytes + pl.piece_bytes + parts * cache->head_dim * 4;
  return pl;
}

template <int D, int NT>
static efim_status kv4_launch_nt(const Kv4AttnParams& p, const Kv4Plan& pl, cudaStream_t s) {
  constexpr int kMaxDevices = 64;
  static std::atomic<bool> done[kMaxDevices];
  constexpr int smem = kv4_smem_bytes(D, NT);
  int dev = 0;
  EFIM_CUDA_TRY(cudaGetDevice(&dev));
  if (dev < 0 || dev >= kMaxDevices || !done[dev].load(std::memory_order_acquire)) {
    EFIM_CUDA_TRY(cudaFuncSetAttribute(kv4_attn_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    if (dev >= 0 && dev < kMaxDevices) done[dev].store(true, std::memory_order_release);
  }
  EFIM_CUDA_TRY(launch_pdl(kv4_attn_kernel<D, NT>, dim3((unsigned)pl.ctas), dim3(KV4_THREADS), smem, s, p));
  if (!pl.whole) EFIM_CUDA_TRY(launch_pdl(kv4_join_kernel<D, NT>, dim3((unsigned)pl.ctas, 8 * NT / KV4_WARPS), dim3(KV4_THREADS), 0, s, p));
  return EFIM_OK;
}
template <int D>
static efim_status kv4_launch(const Kv4AttnParams& p, const Kv4Plan& pl, cudaStream_t s) {
  return pl.nt == 1 ? kv4_launch_nt<D, 1>(p, pl, s) : pl.nt == 2 ? kv4_launch_nt<D, 2>(p, pl, s) : kv4_launch_nt<D, 4>(p, pl, s);
}

efim_status kv4_attn_run(const efim_cache4_desc* cache, Kv4AttnParams p, int max_ctx, float sm_scale, void* ws, size_t ws_bytes, void* stream) {
  const long long cap = (long long)p.max_pages_per_seq * cache->page_size;
  constexpr int MOST = INT_MAX - 1023;      // keys, and those of a trip that ends behind them, count in 32 bits
  if (max_ctx <= 0) max_ctx = (int)std::min<long long>(cap, MOST);
  if (max_ctx > cap) return EFIM_ERR_OUT_OF_RANGE;
  if (max_ctx > MOST) return EFIM_ERR_UNSUPPORTED;
  const long long G = cache->num_q_heads / cache->num_kv_heads;
  if ((long long)p.max_new * G > 0x3fffffff || (long long)p.batch * p.max_new * p.Hq > 0x7fffffff) return EFIM_ERR_UNSUPPORTED;
  const Kv4Plan pl = kv4_plan(cache, p.batch, p.max_new, max_ctx);
  if (pl.ctas > 0x7fffffff || pl.row_tiles * cache->num_kv_heads > 0x7fffffff) return EFIM_ERR_UNSUPPORTED;
  if (pl.bytes > 0) {
    if (!ws || ws_bytes < pl.bytes) return EFIM_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(ws) & 255) return EFIM_ERR_INVALID_ARG;
    p.part_sum = static_cast<float2*>(ws);
    p.pieces = reinterpret_cast<Kv4Piece*>(static_cast<char*>(ws) + pl.sum_bytes);
    p.part_o = reinterpret_cast<float*>(static_cast<char*>(ws) + pl.sum_bytes + pl.piece_bytes);
  }
  p.k_codes = static_cast<const uint8_t*>(cache->d_k_codes);
  p.v_codes = static_cast<const uint8_t*>(cache->d_v_codes);
  p.k_scales = static_cast<const uint8_t*>(cache->d_k_scales);
  p.v_scales = static_cast<const uint8_t*>(cache->d_v_scales);
  p.v_scale = cache->v_scale;
  const float scale = sm_scale > 0.f ? sm_scale : 1.0f / sqrtf((float)cache->head_dim);
  p.scale_log2 = scale * 1.4426950408889634f * cache->k_scale;
  p.Hkv = cache->num_kv_heads;
  p.num_pages = cache->num_pages;
  p.row_tiles = (int)pl.row_tiles;
  p.units_per_seq = (int)(pl.row_tiles * cache->num_kv_heads);
  p.whole = pl.whole;
  p.least_trips = pl.least_trips;
  p.key_cap = max_ctx;
  return cache->head_dim == 128 ? kv4_launch<128>(p, pl, static_cast<cudaStream_t>(stream)) : kv4_launch<64>(p, pl, static_cast<cudaStream_t>(stream));
}

}  // namespace efim

extern "C" size_t efim_kv4_decode_workspace_bytes(const efim_cache4_desc* cache, int32_t batch, int32_t max_new_len, int32_t max_ctx_len) {
  if (efim::check_cache4(cache) != EFIM_OK || batch <= 0 || max_new_len <= 0) return 0;
  // (a plan's size does not fall with the keys: the longest context's is enough for every table's capacity)
  return efim::kv4_plan(cache, batch, max_new_len, max_ctx_len <= 0 ? INT_MAX : max_ctx_len).bytes;
}

extern "C" efim_status efim_kv4_decode_attn(const efim_cache4_desc* cache, int32_t batch, const int32_t* d_ctx_len, int32_t max_ctx_len,
                                            const int32_t* d_block_table, int32_t max_pages_per_seq, const int32_t* d_q_indptr,
                                            int32_t total_rows, int32_t max_new_len, const void* d_q, void* d_out, float* d_lse,
                                            float sm_scale, void* d_workspace, size_t workspace_bytes, int32_t* d_status, void* stream) {
  using namespace efim;
  const efim_status st = check_cache4(cache);
  if (st != EFIM_OK) return st;
  if (batch < 0 || max_pages_per_seq <= 0 || total_rows < 0 || max_new_len <= 0) return EFIM_ERR_INVALID_ARG;
  if (!d_q_indptr && (max_new_len != 1 || total_rows != batch)) return EFIM_ERR_INVALID_ARG;
  if (batch == 0 || total_rows == 0) return EFIM_OK;
  if (!d_ctx_len || !d_block_table || !d_q || !d_out) return EFIM_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(d_q) | reinterpret_cast<uintptr_t>(d_out)) & 15) return EFIM_ERR_INVALID_ARG;
  Kv4AttnParams p{};
  p.q = static_cast<const uint16_t*>(d_q);
  p.len = d_ctx_len;
  p.q_indptr = d_q_indptr;
  p.block_table = d_block_table;
  p.out = static_cast<uint16_t*>(d_out);
  p.lse = d_lse;
  p.status = d_status;
  p.batch = batch;
  p.total_rows = total_rows;
  p.max_new = max_new_len;
  p.Hq = cache->num_q_heads;
  p.max_pages_per_seq = max_pages_per_seq;
  return kv4_attn_run(cache, p, max_ctx_len, sm_scale, d_workspace, workspace_bytes, stream);
}
