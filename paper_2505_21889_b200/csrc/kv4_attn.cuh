// Internal interface of the attention over a 4-bit cache.
#pragma once
#include "kv4.cuh"
#include <atomic>

namespace efim {

struct Kv4AttnParams {
  const uint16_t* q;          // rows of [Hq][D] bf16
  const int32_t* len;         // [batch] keys of each sequence, its new tokens included, or (len_is_cached) those before them
  const int32_t* q_indptr;    // [batch + 1], or null: one row a sequence
  const int32_t* block_table; // [batch][max_pages_per_seq]
  const uint8_t *k_codes, *v_codes, *k_scales, *v_scales;
  uint16_t* out;
  float* lse;                 // natural log, or null
  float* part_o;              // [CTAs][2][rows of a tile][D]
  float2* part_sum;           // [CTAs][2][rows of a tile]: reference (base-2 log), sum of weights relative to it
  struct Kv4Piece* pieces;    // [CTAs]
  int32_t* status;
  int batch, total_rows, max_new, Hq, Hkv, max_pages_per_seq, num_pages, row_tiles, units_per_seq, whole, least_trips, len_is_cached;
  int key_cap;                // keys the launch can cover
  float scale_log2;           // sm_scale * log2(e) * the key pool's scale
  float v_scale;
};

struct Kv4Plan {
  int nt;                     // 8-row tiles of a CTA
  long long row_tiles;        // tiles of a sequence's (new token, head of the group) rows
  long long ctas;
  int whole, least_trips;
  size_t sum_bytes, piece_bytes, bytes;
};
Kv4Plan kv4_plan(const efim_cache4_desc* cache, int batch, int max_new, int max_ctx);

// Plans, checks the workspace and launches; `p` holds what the caller's arguments say.
efim_status kv4_attn_run(const efim_cache4_desc* cache, Kv4AttnParams p, int max_ctx, float sm_scale, void* ws, size_t ws_bytes, void* stream);

}  // namespace efim
