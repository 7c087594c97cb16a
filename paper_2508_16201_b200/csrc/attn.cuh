// Parameters shared by the attention kernels and their launchers.
#pragma once
#include "common.cuh"

namespace specvlm {

struct AttnParams {
  const __nv_bfloat16* q;     // [L][B][n_q][Hq][D]
  __nv_bfloat16* out;         // same shape
  float* lse;                 // [L][B][n_q][Hq] or null
  const int32_t* block_table; // [B][max_blocks] or null
  const int32_t* seq_lens;    // [B]
  int32_t* d_status;
  int32_t batch, n_q, n_q_heads, n_kv_heads, group, rows;   // rows = group * n_q
  int32_t max_blocks, block_tokens, max_seq_len;
  float scale_log2;           // sm_scale * log2(e)
  int32_t lost_cta;           // test hook: the CTA that gives up as if a wait had expired; -1 as a rule
  int32_t window, n_sinks;    // specvlm_window_attn: the last keys and the first keys that a query sees
  int32_t n_blocks;           // pages of the cache
  int32_t row_groups;         // with a window, and more than 16 rows per KV head: groups of 16 rows, an item each
  int32_t sliced;             // with a window: tiles are copied in slices, without those that no query sees
};

__device__ __forceinline__ int clamp_len(int n, int max_len) { return n < 0 ? 0 : (n > max_len ? max_len : n); }

// The keys of a sequence as the kernels walk them.  With a window and sinks (WIN) the tiles that no query of the call sees are
// left out: positions from gap_at on stand for keys `gap` further on, both multiples of a tile.  Key j is visible to the
// query that sees the keys below `lim` when j < lim and (j >= lim - window or j < sinks), in positions as in keys,
// since a gap lies between the two kinds.  Positions sinks .. lo - 1 are visible to no query.
struct KeyView {
  int len;                    // positions
  int gap_at, gap, lo;
};
template <bool WIN, typename P>
__device__ __forceinline__ KeyView key_view(const P& p, int n_q, int b) {
  KeyView v;
  v.len = clamp_len(p.seq_lens[b], p.max_seq_len);
  if constexpr (WIN) {
    const int behind = v.len - p.window;                   // (the host has clamped the window to the cache's length)
    v.lo = (behind > -kTileTokens ? behind : -kTileTokens) - (n_q - 1);       // no lower than it takes to say "all"
    v.gap_at = (p.n_sinks + kTileTokens - 1) & ~(kTileTokens - 1);
    v.gap = v.lo > v.gap_at ? (v.lo & ~(kTileTokens - 1)) - v.gap_at : 0;
    v.len -= v.gap;
    v.lo -= v.gap;
  }
  return v;
}
// Where the tile (of kTileTokens) at a tile's position lies in the sequence
template <bool WIN>
__device__ __forceinline__ int key_tile(const KeyView& v, int tile) {
  if constexpr (WIN) return tile * kTileTokens >= v.gap_at ? tile + v.gap / kTileTokens : tile;
  return tile;
}

}  // namespace specvlm
