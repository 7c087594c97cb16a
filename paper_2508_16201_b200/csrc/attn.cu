// Attention entry points (draft decode and verification) and the kernels for up to 16 query rows
// per KV head, i.e. draft decode: the GQA group's heads of one query token.
//
// With so few rows the step is a pure K/V stream (3.5 flop per cache byte at group 7): 64-token K
// and V tiles go HBM -> shared memory by 128-byte-swizzled tensor-map bulk copies
// (cp.async.bulk.tensor) through an mbarrier ring, four warps each score 16 tokens of a tile on
// m16n8k16 bf16 tiles with a private online softmax, and are merged once per item, i.e. per (layer, sequence, KV
// head).  An item has a CTA of its own where that is the fastest; else the CTAs work on slices of the list
// of all tiles.  Windows of more than 16 rows (verification) run on the tcgen05 kernels; with a sliding window also here, in groups
// of 16 rows (window_rows_form).
#include "attn_tc.cuh"

namespace specvlm {

// ---------------------------------------------------------------------------------------------
// One consumer warp's share of an item: 16 of a tile's 64 tokens, with a private running (max, sum, O).
// ---------------------------------------------------------------------------------------------
template <int D>
struct Rows16 {
  static constexpr int KSTEPS = D / 16;
  static constexpr int NT_O = D / 8;
  static constexpr int OPITCH = D + 8;            // fp32 pitch of the merge buffer
  uint32_t qf[KSTEPS][4];
  float o[NT_O][4];
  float m0, m1, l0, l1;
  int lim0, lim1;                                 // visible keys of the two rows this thread holds

  // P: AttnParams or AttnTcParams (n_q: query tokens of the window, lb: layer * batch + sequence; the rows base .. rows - 1)
  template <typename P>
  __device__ __forceinline__ void start(const P& p, int n_q, int rows, size_t lb, int g, int kv_len, int lane, int base = 0) {
    const int row0 = base + (lane >> 2), row1 = row0 + 8, col = (lane & 3) * 2;
    const __nv_bfloat16* q0 = nullptr;
    const __nv_bfloat16* q1 = nullptr;
    lim0 = lim1 = 0;
    if (row0 < rows) {
      const int t = row0 / p.group, h = g * p.group + (row0 - t * p.group);
      q0 = p.q + ((lb * n_q + t) * p.n_q_heads + h) * D;
      lim0 = kv_len - n_q + t + 1;
    }
    if (row1 < rows) {
      const int t = row1 / p.group, h = g * p.group + (row1 - t * p.group);
      q1 = p.q + ((lb * n_q + t) * p.n_q_heads + h) * D;
      lim1 = kv_len - n_q + t + 1;
    }
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) {
      qf[ks][0] = q0 ? *reinterpret_cast<const uint32_t*>(q0 + ks * 16 + col) : 0u;
      qf[ks][1] = q1 ? *reinterpret_cast<const uint32_t*>(q1 + ks * 16 + col) : 0u;
      qf[ks][2] = q0 ? *reinterpret_cast<const uint32_t*>(q0 + ks * 16 + 8 + col) : 0u;
      qf[ks][3] = q1 ? *reinterpret_cast<const uint32_t*>(q1 + ks * 16 + 8 + col) : 0u;
    }
#pragma unroll
    for (int nt = 0; nt < NT_O; ++nt) o[nt][0] = o[nt][1] = o[nt][2] = o[nt][3] = 0.f;
    m0 = m1 = -INFINITY;
    l0 = l1 = 0.f;
  }

  // tile0: position of the tile's first token; vt: the V tile (generic address); cw: this warp's slice of 16 U tokens
  template <bool WIN, int U = 1, typename P>
  __device__ __forceinline__ void tile(const P& p, int n_q, uint32_t k_base, uint32_t v_base, uint8_t* vt, int tile0, const KeyView& view,
                                       int cw, int lane) {
    constexpr int SLICE = 16 * U;
    const int kv_len = view.len;
    const float scale_log2 = p.scale_log2;
    const int col = (lane & 3) * 2;
    // per-lane ldmatrix row/chunk selectors
    const int mi = lane >> 3, r8 = lane & 7;
    const int k_tok = cw * SLICE + (mi >> 1) * 8 + r8, k_chunk = mi & 1;   // K: non-transposed
    const int v_tok = cw * SLICE + (mi & 1) * 8 + r8, v_chunk = mi >> 1;   // V: transposed
    const int tb = tile0 + cw * SLICE;                                      // first token of this warp's slice
    if (tb >= kv_len) return;
    // positions that no query sees, between the sinks and the window, hold whatever the page holds, as those past the end do
    const bool hidden = WIN && tb < view.lo && tb + SLICE > p.n_sinks;
    if (hidden) {
      if (tb >= p.n_sinks && tb + SLICE <= view.lo) return;
      const int first = (p.n_sinks > tb ? p.n_sinks : tb) - tile0, last = (view.lo < tb + SLICE ? view.lo : tb + SLICE) - tile0;
      for (int t = first + (lane >> 3); t < last; t += 4) {
#pragma unroll
        for (int h = 0; h < D / 64; ++h)
          *reinterpret_cast<uint4*>(vt + h * (kTileTokens * 128) + t * 128 + (lane & 7) * 16) =
              make_uint4(0, 0, 0, 0);
      }
      fence_proxy_async();
      __syncwarp();
    }
    if (tb + SLICE > kv_len) {
      // rows past the end of the sequence hold whatever the page held: clear V there so that
      // a zero probability times a stale non-finite value cannot reach the accumulator
      const int first = kv_len - tile0;                                  // first invalid local row
      for (int t = first + (lane >> 3); t < (cw + 1) * SLICE; t += 4) {
#pragma unroll
        for (int h = 0; h < D / 64; ++h)
          *reinterpret_cast<uint4*>(vt + h * (kTileTokens * 128) + t * 128 + (lane & 7) * 16) =
              make_uint4(0, 0, 0, 0);
      }
      fence_proxy_async();                                               // a copy may refill the slot later
      __syncwarp();
    }
    float sc[2 * U][4];
#pragma unroll
    for (int nt = 0; nt < 2 * U; ++nt) sc[nt][0] = sc[nt][1] = sc[nt][2] = sc[nt][3] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        uint32_t b0, b1, b2, b3;
        ldmatrix_x4(k_base + tile_offset<D>(k_tok + 16 * u, 2 * ks + k_chunk), b0, b1, b2, b3);
        mma_bf16_16816(sc[2 * u], qf[ks], b0, b1);
        mma_bf16_16816(sc[2 * u + 1], qf[ks], b2, b3);
      }
    }
    // scale, causal / length mask, running max
    float mx0 = -INFINITY, mx1 = -INFINITY;
    // (WIN: most slices lie inside every query's window; rows out of use may then hold anything)
    if (WIN && tb + SLICE <= view.len - n_q + 1 && (tb >= view.lo + n_q - 1 || tb + SLICE <= p.n_sinks)) {
#pragma unroll
      for (int nt = 0; nt < 2 * U; ++nt) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sc[nt][e] *= scale_log2;
          if (e < 2) mx0 = fmaxf(mx0, sc[nt][e]); else mx1 = fmaxf(mx1, sc[nt][e]);
        }
      }
    } else {
#pragma unroll
      for (int nt = 0; nt < 2 * U; ++nt) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int tok = tb + nt * 8 + col + (e & 1);
          const int lim = (e < 2) ? lim0 : lim1;
          const bool seen = tok < lim && (!WIN || tok >= lim - p.window || tok < p.n_sinks);
          const float v = seen ? sc[nt][e] * scale_log2 : -INFINITY;
          sc[nt][e] = v;
          if (e < 2) mx0 = fmaxf(mx0, v); else mx1 = fmaxf(mx1, v);
        }
      }
    }
    mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, 1));
    mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, 2));
    mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, 1));
    mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, 2));
    const float mn0 = fmaxf(m0, mx0), mn1 = fmaxf(m1, mx1);
    const float mu0 = mn0 == -INFINITY ? 0.f : mn0, mu1 = mn1 == -INFINITY ? 0.f : mn1;
    const float a0 = fast_exp2(m0 - mu0), a1 = fast_exp2(m1 - mu1);
    m0 = mn0;
    m1 = mn1;
    float ps0 = 0.f, ps1 = 0.f;
#pragma unroll
    for (int nt = 0; nt < 2 * U; ++nt) {
      sc[nt][0] = fast_exp2(sc[nt][0] - mu0);
      sc[nt][1] = fast_exp2(sc[nt][1] - mu0);
      sc[nt][2] = fast_exp2(sc[nt][2] - mu1);
      sc[nt][3] = fast_exp2(sc[nt][3] - mu1);
      ps0 += sc[nt][0] + sc[nt][1];
      ps1 += sc[nt][2] + sc[nt][3];
    }
    l0 = l0 * a0 + ps0;
    l1 = l1 * a1 + ps1;
    // P goes into the product with V as bf16, the type that the tensor cores take beside V's: off by 2^-8 of each probability at most,
    // independently of one another, so that an output, itself rounded to bf16, differs from 64 bits by 2.0e-3 to 2.3e-3 of its size
    // instead of 1.7e-3.  The sum that divides it takes them unrounded, in fp32.  A second product for the rest of each P would double
    // the tensor work and the conversions of a tile.
    uint32_t pa[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      pa[u][0] = pack_bf16x2(sc[2 * u][0], sc[2 * u][1]);
      pa[u][1] = pack_bf16x2(sc[2 * u][2], sc[2 * u][3]);
      pa[u][2] = pack_bf16x2(sc[2 * u + 1][0], sc[2 * u + 1][1]);
      pa[u][3] = pack_bf16x2(sc[2 * u + 1][2], sc[2 * u + 1][3]);
    }
#pragma unroll
    for (int nt = 0; nt < NT_O; ++nt) {
      o[nt][0] *= a0;
      o[nt][1] *= a0;
      o[nt][2] *= a1;
      o[nt][3] *= a1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < D / 16; ++j) {
        uint32_t b0, b1, b2, b3;
        ldmatrix_x4_trans(v_base + tile_offset<D>(v_tok + 16 * u, 2 * j + v_chunk), b0, b1, b2, b3);
        mma_bf16_16816(o[2 * j], pa[u], b0, b1);
        mma_bf16_16816(o[2 * j + 1], pa[u], b2, b3);
      }
  }

  // the rows of a warp that has seen all of their keys: normalised, to the output
  __device__ __forceinline__ void store(const AttnParams& p, int base, int rows, int lb, int g, int lane) {
    l0 += __shfl_xor_sync(0xffffffffu, l0, 1);
    l0 += __shfl_xor_sync(0xffffffffu, l0, 2);
    l1 += __shfl_xor_sync(0xffffffffu, l1, 1);
    l1 += __shfl_xor_sync(0xffffffffu, l1, 2);
    const int col = (lane & 3) * 2;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = (lane >> 2) + 8 * e;
      if (r >= rows) continue;
      const float l = e ? l1 : l0, m = e ? m1 : m0, inv = l > 0.f ? 1.f / l : 0.f;
      const int t = (base + r) / p.group, h = g * p.group + (base + r - t * p.group);
      const size_t orow = ((size_t)lb * p.n_q + t) * p.n_q_heads + h;
#pragma unroll
      for (int nt = 0; nt < NT_O; ++nt)
        *reinterpret_cast<uint32_t*>(p.out + orow * D + nt * 8 + col) = pack_bf16x2(o[nt][2 * e] * inv, o[nt][2 * e + 1] * inv);
      if (p.lse && (lane & 3) == 0) p.lse[orow] = l > 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
    }
  }

  // this warp's partial to the merge buffer: o_sm [NW][16][OPITCH], m_sm and l_sm [NW][16]
  __device__ __forceinline__ void publish(float* o_sm, float* m_sm, float* l_sm, int rows, int warp, int lane) {
    const int row0 = lane >> 2, row1 = row0 + 8, col = (lane & 3) * 2;
    l0 += __shfl_xor_sync(0xffffffffu, l0, 1);
    l0 += __shfl_xor_sync(0xffffffffu, l0, 2);
    l1 += __shfl_xor_sync(0xffffffffu, l1, 1);
    l1 += __shfl_xor_sync(0xffffffffu, l1, 2);
    float* ow = o_sm + warp * 16 * OPITCH;
    // only the rows in use (7 of the 16 for the 7-head group of a decode step)
    if (row0 < rows) {
#pragma unroll
      for (int nt = 0; nt < NT_O; ++nt)
        *reinterpret_cast<float2*>(ow + row0 * OPITCH + nt * 8 + col) = make_float2(o[nt][0], o[nt][1]);
    }
    if (row1 < rows) {
#pragma unroll
      for (int nt = 0; nt < NT_O; ++nt)
        *reinterpret_cast<float2*>(ow + row1 * OPITCH + nt * 8 + col) = make_float2(o[nt][2], o[nt][3]);
    }
    if ((lane & 3) == 0) {
      m_sm[warp * 16 + row0] = m0;
      m_sm[warp * 16 + row1] = m1;
      l_sm[warp * 16 + row0] = l0;
      l_sm[warp * 16 + row1] = l1;
    }
  }
};

// The consumer warps' partials of row r, channels c .. c + 3, merged and normalised; returns the row's
// log-sum-exp (log2 units).  Every thread of the final pass derives its row's weights 2^(m_w - M) / den itself
// (16 shared loads and NW exponentials): cheaper than a separate weight phase behind two more barriers.
template <int D, int NW>
__device__ __forceinline__ float rows16_merge(const float* o_sm, const float* m_sm, const float* l_sm, int r, int c, float4& acc) {
  constexpr int OPITCH = Rows16<D>::OPITCH;
  float M = -INFINITY;
#pragma unroll
  for (int w = 0; w < NW; ++w) M = fmaxf(M, m_sm[w * 16 + r]);
  float den = 0.f;
  float wt[NW];
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    wt[w] = M != -INFINITY ? fast_exp2(m_sm[w * 16 + r] - M) : 0.f;
    den += l_sm[w * 16 + r] * wt[w];
  }
  const float inv = den > 0.f ? 1.f / den : 0.f;
  acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const float f = wt[w] * inv;
    const float4 x = *reinterpret_cast<const float4*>(o_sm + (w * 16 + r) * OPITCH + c);
    acc.x += x.x * f;
    acc.y += x.y * f;
    acc.z += x.z * f;
    acc.w += x.w * f;
  }
  return den > 0.f ? M + log2f(den) : -INFINITY;
}

__device__ __forceinline__ void store_bf16x4(__nv_bfloat16* dst, const float4& v) {
  uint2 packed;
  packed.x = pack_bf16x2(v.x, v.y);
  packed.y = pack_bf16x2(v.z, v.w);
  *reinterpret_cast<uint2*>(dst) = packed;
}

constexpr int kMaxRows16Cluster = 8;       // the portable cluster size
constexpr int kSliceTokens = 16;           // of a tile that is copied in slices (load_seen)
constexpr int kSlicedTiles = 3;            // in windows of at most so many

// By a consumer thread of a CTA that gives up (a wait expired): it stays, bounded, until the producer has gone and the last
// copies that it asked for have landed, since the CTA must not end under copies to its shared memory.  flags[0] is the abort
// flag, flags[1] the copies asked for once the producer has gone, -1 before.
template <int STAGES>
__device__ __forceinline__ void await_copies(uint32_t bar_full, volatile int* flags) {
  const uint64_t t0 = global_timer_ns();
  while (flags[1] < 0 && global_timer_ns() - t0 < kWaitLimitNs) {
  }
  const int issued = flags[1];
  for (int i = issued > STAGES ? issued - STAGES : 0; i < issued; ++i)
    while (!mbar_try_wait(bar_full + 8 * (i % STAGES), (i / STAGES) & 1) && global_timer_ns() - t0 < kWaitLimitNs) {
    }
}

// The copies of a window's tile at position tile0 in slices of 16 tokens (kSliceTokens), those that no query sees left out.
template <int D>
__device__ __forceinline__ void load_seen(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const KeyView& view, int n_sinks, int tile0, uint32_t dst,
                                          uint32_t full, int tok, int g, int blk, int layer, uint64_t policy) {
  constexpr int TILE_BYTES = kTileTokens * D * 2, N = kTileTokens / kSliceTokens;
  auto seen = [&](int u) {
    const int at = tile0 + u * kSliceTokens;
    return at < view.len && (at < n_sinks || at + kSliceTokens > view.lo);
  };
  int n = 0;
#pragma unroll
  for (int u = 0; u < N; ++u) n += seen(u);
  mbar_arrive_expect_tx(full, n * (2 * TILE_BYTES / N));
#pragma unroll
  for (int u = 0; u < N; ++u)
    if (seen(u)) {
#pragma unroll
      for (int h = 0; h < D / 64; ++h) {
        const uint32_t at = dst + h * (kTileTokens * 128) + u * (kSliceTokens * 128);
        tma_load_5d(at, &tm_k, full, h * 64, tok + u * kSliceTokens, g, blk, layer, policy);
        tma_load_5d(at + TILE_BYTES, &tm_v, full, h * 64, tok + u * kSliceTokens, g, blk, layer, policy);
      }
    }
}

// ---------------------------------------------------------------------------------------------
// One CTA per item.  4 consumer warps each own 16 of a tile's 64 tokens; they are merged once at the end.
// The last warp is the TMA producer.
// ---------------------------------------------------------------------------------------------
// NG consumer groups of 4 warps take alternate tiles (NG = 2 where an SM holds a single CTA, so
// that eight warps hide each other's latencies as two resident CTAs would).
// SPLIT: a cluster of n_cta CTAs per item, CTA r on tiles r, r + n_cta, ..; their results meet over distributed
// shared memory, each CTA folding its share of the output positions.  For a few short items, whose tiles one CTA would
// work through one after the other at 0.35 us each.
//
// The consumer warps of an item, or of a cluster's CTA.
template <int D, int STAGES, int NG, bool SPLIT, bool WIN>
__device__ __forceinline__ void rows16_consume(const AttnParams& p, uint8_t* smem, uint32_t base, volatile int* abort_flag,
                                               const KeyView& view, int n_my, int rank, int n_cta) {
  constexpr int TILE_BYTES = kTileTokens * D * 2, STAGE_BYTES = 2 * TILE_BYTES;
  constexpr int OPITCH = Rows16<D>::OPITCH;
  const uint32_t bar_full = base + STAGES * STAGE_BYTES, bar_empty = bar_full + 8 * STAGES;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g = WIN ? (int)blockIdx.y / p.row_groups : (int)blockIdx.y, lb = blockIdx.z;
  // this item's rows: all, or a group of 16
  const int base_row = WIN ? 16 * ((int)blockIdx.y - g * p.row_groups) : 0;
  const int rows = WIN && p.rows - base_row > 16 ? 16 : p.rows - base_row;
  const bool spec = !WIN && p.block_table == nullptr;
  const int kv_len = view.len;
  const int n_all = (kv_len + kTileTokens - 1) / kTileTokens;

  if (n_all == 0) {
    // An empty sequence: its outputs are zero, its LSE -inf.  The ring stays untouched: the tile that the producer
    // asked for before it knew the length may still be landing there, with whatever the cache rows hold.
    for (int idx = tid; idx < rows * (D / 8); idx += 128 * NG) {
      const int r = base_row + idx / (D / 8), c8 = idx % (D / 8);
      const int t = r / p.group, h = g * p.group + (r - t * p.group);
      const size_t orow = ((size_t)lb * p.n_q + t) * p.n_q_heads + h;
      *reinterpret_cast<uint4*>(p.out + orow * D + c8 * 8) = make_uint4(0, 0, 0, 0);
      if (p.lse && c8 == 0) p.lse[orow] = -INFINITY;
    }
    return;
  }
  const int cw = warp & 3, grp = warp >> 2;                           // token slice, consumer group
  Rows16<D> st;
  // (positions of the newest keys are as far apart as the keys)
  st.start(p, p.n_q, base_row + rows, lb, g, kv_len, lane, base_row);
  bool alive = true;
  // a CTA without a tile of its own: the one asked for before the length was known lands where the merge buffer will be
  if (SPLIT && n_my == 0 && spec && !mbar_wait(bar_full, 0, abort_flag)) alive = false;
  for (int i = grp; i < n_my; i += NG) {
    const int s = i % STAGES;
    if (!mbar_wait(bar_full + 8 * s, (i / STAGES) & 1, abort_flag)) {
      alive = false;
      break;
    }
    const uint32_t k_base = base + s * STAGE_BYTES;
    st.template tile<WIN>(p, p.n_q, k_base, k_base + TILE_BYTES, smem + s * STAGE_BYTES + TILE_BYTES, (i * n_cta + rank) * kTileTokens, view,
                          cw, lane);
    __syncwarp();
    if (lane == 0) mbar_arrive(bar_empty + 8 * s);
  }

  // test hook: the CTA that gives up although it has seen its tiles
  if (p.lost_cta == (int)((blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x)) *abort_flag = 1;
  // ------------------------------------------------------------ merge the consumer warps' partials
  // (named barrier over the consumer threads; the producer warp has no part in it)
  asm volatile("bar.sync 1, %0;" ::"n"(128 * NG) : "memory");
  const bool gave_up = !alive || *abort_flag;   // a wait expired somewhere in this CTA (the flag tells all of it)
  // (the producer reports only the waits of its own, and it has none where the tiles fit the ring)
  if (gave_up && tid == 0 && p.d_status) *p.d_status = SPECVLM_ERR_TIMEOUT;
  if (!SPLIT && gave_up) {             // leave outputs alone
    if (tid == 0) await_copies<STAGES>(bar_full, abort_flag);
    return;
  }
  constexpr int NW = 4 * NG;                                           // consumer warps
  float* const o_sm = reinterpret_cast<float*>(smem);                  // [NW][16][OPITCH]
  float* const m_sm = o_sm + NW * 16 * OPITCH;                         // [NW][16]
  float* const l_sm = m_sm + NW * 16;                                  // [NW][16]
  st.publish(o_sm, m_sm, l_sm, rows, warp, lane);
  asm volatile("bar.sync 1, %0;" ::"n"(128 * NG) : "memory");
  if constexpr (SPLIT) {
    // This CTA's result, normalised, behind the merge buffer, and its log-sum-exps, for the whole cluster to read.  The
    // latter say whether the CTA gave up, and lie behind the ring, where no copy that was asked for before lands on them.
    float* const part_o = l_sm + NW * 16;                              // [16][D]
    float* const part_lse = reinterpret_cast<float*>(smem + STAGES * STAGE_BYTES + 16 * STAGES + 16);   // [16]
    for (int idx = tid; idx < rows * (D / 4); idx += 128 * NG) {
      const int r = idx / (D / 4), c = (idx - r * (D / 4)) * 4;
      float4 acc;
      const float lse2 = rows16_merge<D, NW>(o_sm, m_sm, l_sm, r, c, acc);
      *reinterpret_cast<float4*>(part_o + r * D + c) = acc;
      if (c == 0) part_lse[r] = gave_up ? __uint_as_float(kUnwritten) : lse2;
    }
    cluster_barrier();
    for (int idx = rank * 128 * NG + tid; idx < rows * (D / 4); idx += n_cta * 128 * NG) {
      const int r = idx / (D / 4), c = (idx - r * (D / 4)) * 4;
      float lse[kMaxRows16Cluster];
      float4 x[kMaxRows16Cluster];
#pragma unroll
      for (int k = 0; k < kMaxRows16Cluster; ++k) {
        lse[k] = -INFINITY;
        x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (k < n_cta) {
          lse[k] = ld_cluster_f32(cluster_map(smem_u32(part_lse + r), k));
          x[k] = ld_cluster_f32x4(cluster_map(smem_u32(part_o + r * D + c), k));
        }
      }
      float mm = -INFINITY, den = 0.f;
      bool lost = false;
#pragma unroll
      for (int k = 0; k < kMaxRows16Cluster; ++k) {
        lost |= unwritten(lse[k]);
        mm = fmaxf(mm, lse[k]);
      }
      if (lost) continue;                                              // a part is missing: leave the row alone
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < kMaxRows16Cluster; ++k) {
        const float w = lse[k] == -INFINITY ? 0.f : fast_exp2(lse[k] - mm);
        acc.x += w * x[k].x;
        acc.y += w * x[k].y;
        acc.z += w * x[k].z;
        acc.w += w * x[k].w;
        den += w;
      }
      const float inv = den > 0.f ? 1.f / den : 0.f;
      const int t = (base_row + r) / p.group, h = g * p.group + (base_row + r - t * p.group);
      const size_t orow = ((size_t)lb * p.n_q + t) * p.n_q_heads + h;
      store_bf16x4(p.out + orow * D + c, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
      if (p.lse && c == 0) p.lse[orow] = den > 0.f ? (mm + log2f(den)) * kLn2 : -INFINITY;
    }
    cluster_barrier();                                                 // nobody reads this CTA's shared memory any more
    if (gave_up && tid == 0) await_copies<STAGES>(bar_full, abort_flag);
    return;
  }
  for (int idx = tid; idx < rows * (D / 4); idx += 128 * NG) {
    const int r = idx / (D / 4), c = (idx - r * (D / 4)) * 4;
    float4 acc;
    const float lse2 = rows16_merge<D, NW>(o_sm, m_sm, l_sm, r, c, acc);
    const int t = (base_row + r) / p.group, h = g * p.group + (base_row + r - t * p.group);
    const size_t orow = ((size_t)lb * p.n_q + t) * p.n_q_heads + h;
    store_bf16x4(p.out + orow * D + c, acc);
    if (p.lse && c == 0) p.lse[orow] = lse2 * kLn2;
  }
}

// SPLIT: launched in clusters of gridDim.x CTAs per item, a number that the host's bound on the lengths gives.  A sequence of
// a few tiles is left to the first of them, since the hand-over would take longer (one layer, 4 items of d = 128 in a cache of
// 800 tokens, alone / by eight: 40 tokens 2.9 / 4.1 us, 200 3.9 / 4.1, 400 4.8 / 4.1; d = 64: 200 tokens 3.0 / 3.3, 400
// 3.8 / 3.3; by two, 36 items of d = 128: 200 tokens 4.1 / 4.5, 320 4.5 / 4.9, 400 5.2 / 5.1).  The producer serves both
// forms in one loop and the consumers have code of their own for each: the other ways round cost a cluster's full lengths
// 1 to 5 %.
constexpr int kSoloTiles = 4, kSoloTilesPair = 6;
// (CTAs per SM are as many as the ring allows; without that the compiler held d = 64 to 96 registers and spilled: 6 layers of
// 800 tokens, 24 items, 4.4 -> 4.2 us, 112 items of d = 128 and 755 tokens 9.83 -> 9.65)
constexpr int kHalfRing = 4;      // stages of a CTA with two groups that shares an SM with another (d = 64)
constexpr int kShortRing = 2;     // stages of a CTA that shares an SM with two others (d = 128)
constexpr int kShortTiles = 8;
// WIN: queries see a window and sinks (KeyView); the first tile is not known before the length then.
template <int D, int STAGES, int NG, bool SPLIT, bool WIN = false>
__global__ void __launch_bounds__(32 * (4 * NG + 1), NG == 2 ? (STAGES == kHalfRing ? 2 : 1) : D == 64 ? 4 : STAGES == kShortRing ? 3 : 2)
attn_rows16_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                   const AttnParams p) {
  constexpr int TILE_BYTES = kTileTokens * D * 2;
  constexpr int STAGE_BYTES = 2 * TILE_BYTES;
  // A consumer group must see every phase of the ring slots it waits on: with the groups on
  // alternate tiles that holds only when a slot always belongs to the same group.  (A wait on a
  // phase two behind the barrier returns at once, the group then releases a slot it never read,
  // and the surplus arrival on the barrier is undefined behaviour: it faulted the kernel.)
  static_assert(STAGES % NG == 0, "ring depth must be a multiple of the number of consumer groups");

  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = smem_u32(smem_raw);
  const uint32_t base = (raw_addr + 1023u) & ~1023u;
  uint8_t* const smem = smem_raw + (base - raw_addr);
  const uint32_t bar_full = base + STAGES * STAGE_BYTES;
  const uint32_t bar_empty = bar_full + 8 * STAGES;
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(smem + STAGES * STAGE_BYTES + 16 * STAGES);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g = WIN ? (int)blockIdx.y / p.row_groups : (int)blockIdx.y, lb = blockIdx.z;
  const int layer = lb / p.batch, b = lb - layer * p.batch;
  const int rank = SPLIT ? (int)blockIdx.x : 0, n_cta = SPLIT ? (int)gridDim.x : 1;

  if (tid == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(bar_full + 8 * s, 1);
      mbar_init(bar_empty + 8 * s, 4);
    }
    abort_flag[0] = 0;
    abort_flag[1] = -1;                  // see await_copies
    mbar_fence_init();
  }
  if (tid == 32 * 4 * NG) {              // the producer's lane: descriptors are kernel parameters
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  __syncthreads();                       // the barriers are initialised
  pdl_launch_next();
  pdl_wait();

  // The first tile of a contiguous cache sits at a known place whatever the sequence's
  // length (rows past the cache's end are zero-filled by the copy): the producer asks for it
  // before the length has even been read, which takes a global-memory round trip off the start.
  const bool spec = !WIN && p.block_table == nullptr;
  if (spec && tid == 32 * 4 * NG) {
    const uint64_t policy = l2_policy_evict_first();
    mbar_arrive_expect_tx(bar_full, STAGE_BYTES);
#pragma unroll
    for (int h = 0; h < D / 64; ++h) {
      tma_load_5d(base + h * (kTileTokens * 128), &tm_k, bar_full, h * 64, rank * kTileTokens, g, b, layer, policy);
      tma_load_5d(base + TILE_BYTES + h * (kTileTokens * 128), &tm_v, bar_full, h * 64, rank * kTileTokens, g, b, layer, policy);
    }
  }

  const KeyView view = key_view<WIN>(p, p.n_q, b);
  const int n_all = (view.len + kTileTokens - 1) / kTileTokens;
  const bool solo = SPLIT && n_all <= (n_cta == 2 ? kSoloTilesPair : kSoloTiles);
  const int n_split = SPLIT ? (n_all + n_cta - 1 - rank) / n_cta : n_all;
  const int n_my = !solo ? n_split : rank == 0 ? n_all : 0;

  if (warp == 4 * NG) {
    // ------------------------------------------------------------------ producer
    if (lane == 0 && n_my == 0) {
      // an empty sequence, or a CTA without a part: nobody will consume the tile asked for above; stay until it has landed
      const uint64_t t0 = global_timer_ns();
      while (spec && !mbar_try_wait(bar_full, 0) && global_timer_ns() - t0 < kWaitLimitNs) {
      }
      abort_flag[1] = 0;
    }
    if (lane == 0 && n_my > 0) {
      const uint64_t policy = l2_policy_evict_first();
      const int tiles_per_block = p.block_tokens / kTileTokens;   // used only when paged
      int issued = spec ? 1 : 0;
      bool ok = true;
      for (int i = issued; i < n_my && ok; ++i) {
        const int s = i % STAGES;
        if (i >= STAGES) ok = mbar_wait(bar_empty + 8 * s, ((i / STAGES) - 1) & 1, abort_flag);
        if (!ok) break;
        const int t = key_tile<WIN>(view, solo ? i : i * n_cta + rank);
        int blk, tok;
        if (p.block_table) {
          blk = p.block_table[(size_t)b * p.max_blocks + t / tiles_per_block];
          if (WIN && (blk < 0 || blk >= p.n_blocks) && p.d_status) *p.d_status = SPECVLM_ERR_INVALID_ARG;   // the copy gives zeros
          tok = (t % tiles_per_block) * kTileTokens;
        } else {
          blk = b;
          tok = t * kTileTokens;
        }
        const uint32_t full = bar_full + 8 * s;
        const uint32_t dst = base + s * STAGE_BYTES;
        if (WIN && !SPLIT && p.sliced) {
          load_seen<D>(tm_k, tm_v, view, p.n_sinks, i * kTileTokens, dst, full, tok, g, blk, layer, policy);
          issued = i + 1;
          continue;
        }
        mbar_arrive_expect_tx(full, STAGE_BYTES);
#pragma unroll
        for (int h = 0; h < D / 64; ++h) {
          tma_load_5d(dst + h * (kTileTokens * 128), &tm_k, full, h * 64, tok, g, blk, layer, policy);
          tma_load_5d(dst + TILE_BYTES + h * (kTileTokens * 128), &tm_v, full, h * 64, tok, g, blk,
                      layer, policy);
        }
        issued = i + 1;
      }
      if (!ok) {
        // a wait expired: report, then stay until this CTA's copies in flight have landed
        if (p.d_status) *p.d_status = SPECVLM_ERR_TIMEOUT;
        const int first = issued > STAGES ? issued - STAGES : 0;
        for (int i = first; i < issued; ++i) {
          const uint64_t t0 = global_timer_ns();
          while (!mbar_try_wait(bar_full + 8 * (i % STAGES), (i / STAGES) & 1) &&
                 global_timer_ns() - t0 < kWaitLimitNs) {
          }
        }
      }
      abort_flag[1] = issued;
    }
    return;
  }

  if constexpr (SPLIT) {
    if (solo) {
      if (rank == 0) rows16_consume<D, STAGES, NG, false, WIN>(p, smem, base, abort_flag, view, n_my, 0, 1);
      return;
    }
  }
  rows16_consume<D, STAGES, NG, SPLIT, WIN>(p, smem, base, abort_flag, view, n_my, rank, n_cta);
}

// ---------------------------------------------------------------------------------------------
// More than 16 rows per KV head and a window: one CTA per item, in which each consumer warp has 16 of the rows and goes through
// whole tiles.  Nothing is merged at the end, and a tile is read once for all rows.  For many items of short windows, whose
// time is what is around the tiles: an SM holds as many items as it holds of the 16-row kernel's groups (window_rows_form).
// NW: warps at most; U: 16-token slices that a warp scores together, as many as the registers that PER_SM CTAs leave it allow: a
// tile takes a warp that is alone 2.3 us with one slice at a time, 1.5 to 1.9 with all four (d = 128), 1.3 with two (d = 64).  Two CTAs an SM
// of four slices for three of one: 42 rows, 2000 items of 64 / 256 / 512 keys 35 / 80 / 141 -> 40 / 83 / 133 us.
// ---------------------------------------------------------------------------------------------
template <int D, int NW, int STAGES, int PER_SM, int U>
__global__ void __launch_bounds__(32 * (NW + 1), PER_SM)
attn_row_groups_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const AttnParams p) {
  constexpr int TILE_BYTES = kTileTokens * D * 2, STAGE_BYTES = 2 * TILE_BYTES;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = smem_u32(smem_raw);
  const uint32_t base = (raw_addr + 1023u) & ~1023u;
  uint8_t* const smem = smem_raw + (base - raw_addr);
  const uint32_t bar_full = base + STAGES * STAGE_BYTES, bar_empty = bar_full + 8 * STAGES;
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(smem + STAGES * STAGE_BYTES + 16 * STAGES);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g = blockIdx.y, lb = blockIdx.z, layer = lb / p.batch, b = lb - layer * p.batch;
  const int n_warps = p.row_groups;      // the producer's warp is behind them

  if (tid == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(bar_full + 8 * s, 1);
      mbar_init(bar_empty + 8 * s, n_warps);
    }
    abort_flag[0] = 0;
    abort_flag[1] = -1;                  // see await_copies
    mbar_fence_init();
  }
  if (tid == 32 * n_warps) {
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  __syncthreads();                       // the barriers are initialised
  pdl_launch_next();
  pdl_wait();
  const KeyView view = key_view<true>(p, p.n_q, b);
  const int n_tiles = (view.len + kTileTokens - 1) / kTileTokens;

  if (warp == n_warps) {
    // ------------------------------------------------------------------ producer
    if (lane != 0) return;
    const uint64_t policy = l2_policy_evict_first();
    const int tiles_per_block = p.block_tokens / kTileTokens;     // used only when paged
    bool ok = true;
    int issued = 0;
    for (int i = 0; i < n_tiles && ok; ++i) {
      const int s = i % STAGES;
      if (i >= STAGES) ok = mbar_wait(bar_empty + 8 * s, ((i / STAGES) - 1) & 1, abort_flag);
      if (!ok) break;
      const int t = key_tile<true>(view, i);
      int blk = b, tok = t * kTileTokens;
      if (p.block_table) {
        blk = p.block_table[(size_t)b * p.max_blocks + t / tiles_per_block];
        if ((blk < 0 || blk >= p.n_blocks) && p.d_status) *p.d_status = SPECVLM_ERR_INVALID_ARG;   // the copy gives zeros
        tok = (t % tiles_per_block) * kTileTokens;
      }
      const uint32_t full = bar_full + 8 * s, dst = base + s * STAGE_BYTES;
      if (p.sliced) {
        load_seen<D>(tm_k, tm_v, view, p.n_sinks, i * kTileTokens, dst, full, tok, g, blk, layer, policy);
        issued = i + 1;
        continue;
      }
      mbar_arrive_expect_tx(full, STAGE_BYTES);
#pragma unroll
      for (int h = 0; h < D / 64; ++h) {
        tma_load_5d(dst + h * (kTileTokens * 128), &tm_k, full, h * 64, tok, g, blk, layer, policy);
        tma_load_5d(dst + TILE_BYTES + h * (kTileTokens * 128), &tm_v, full, h * 64, tok, g, blk, layer, policy);
      }
      issued = i + 1;
    }
    abort_flag[1] = issued;
    if (!ok) {                           // a wait expired: stay until the copies in flight have landed
      if (p.d_status) *p.d_status = SPECVLM_ERR_TIMEOUT;
      await_copies<STAGES>(bar_full, abort_flag);
    }
    return;
  }

  const int base_row = 16 * warp, rows = p.rows - base_row > 16 ? 16 : p.rows - base_row;
  Rows16<D> st;
  st.start(p, p.n_q, base_row + rows, lb, g, view.len, lane, base_row);
  bool alive = true;
  for (int i = 0; i < n_tiles; ++i) {
    const int s = i % STAGES;
    if (!warp_wait(bar_full + 8 * s, (i / STAGES) & 1, abort_flag)) {
      alive = false;
      break;
    }
    const uint32_t k_base = base + s * STAGE_BYTES;
#pragma unroll 1
    for (int cw = 0; cw < kTileTokens / (16 * U); ++cw)
      st.template tile<true, U>(p, p.n_q, k_base, k_base + TILE_BYTES, smem + s * STAGE_BYTES + TILE_BYTES, i * kTileTokens, view, cw, lane);
    __syncwarp();
    if (lane == 0) mbar_arrive(bar_empty + 8 * s);
  }
  // test hook: the CTA that gives up although it has seen its tiles
  if (p.lost_cta == (int)(blockIdx.z * gridDim.y + blockIdx.y)) alive = false;
  if (!alive) {                          // leave the rows alone
    if (lane == 0) {
      if (p.d_status) *p.d_status = SPECVLM_ERR_TIMEOUT;
      await_copies<STAGES>(bar_full, abort_flag);
    }
    return;
  }
  st.store(p, base_row, rows, lb, g, lane);
}

// bar.sync 1 over n threads (whole warps) that also answers whether the predicate holds for all of them
__device__ __forceinline__ bool bar_and(bool pred, int n) {
  uint32_t all;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "bar.red.and.pred q, 1, %2, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(all) : "r"((uint32_t)pred), "r"(n) : "memory");
  return all != 0;
}

// ---------------------------------------------------------------------------------------------
// The same on slices: a persistent CTA per SM streams a contiguous slice of the flat (layer, sequence, KV
// head, 64-token tile) list (attn_sched.h), whatever the items' number and lengths, so that every SM moves the
// same bytes; the producer runs ahead over item boundaries while the consumers merge and store an item, and
// items that a slice boundary cuts leave partial results for the merge kernel (attn_tc.cu).  It replaces a split
// of every item over the same number of CTAs with arrival counters (a memset, fences and a merge by one CTA):
// 1 layer of 6400 / 50 000 tokens 26.1 / 33.0 -> 8.6 / 21.4 us, 4 layers x 4 sequences of up to 12 800 tokens
// 99 -> 46.5 us (39 at the copy rate).
// ---------------------------------------------------------------------------------------------
template <int D>
struct SliceCfg {
  static constexpr int NG = 2;
  static constexpr int STAGES = D == 128 ? 4 : 8;
  static constexpr int TILE_BYTES = kTileTokens * D * 2;
  static constexpr int OFF_O = STAGES * 2 * TILE_BYTES;                          // merge buffer
  static constexpr int OFF_ML = OFF_O + 4 * NG * 16 * Rows16<D>::OPITCH * 4;
  static constexpr int OFF_BAR = OFF_ML + 2 * 4 * NG * 16 * 4;
  static constexpr int OFF_MISC = OFF_BAR + 16 * STAGES;
  static constexpr int OFF_PLAN = OFF_MISC + 16;
  static constexpr int OFF_PREFIX = OFF_PLAN + (kPlanBytes + 7) / 8 * 8;
  static constexpr int SMEM = OFF_PREFIX + (kSchedMaxBatch + 1) * 4 + 1024;
  static_assert(STAGES % NG == 0, "ring depth must be a multiple of the number of consumer groups");
  static_assert(SMEM <= 232448, "shared-memory plan does not fit");
};

template <int D, bool WIN = false>
__global__ void __launch_bounds__(32 * (4 * SliceCfg<D>::NG + 1), 1)
attn_rows16_slices_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                          const __grid_constant__ AttnTcParams p) {
  using C = SliceCfg<D>;
  constexpr int NG = C::NG, STAGES = C::STAGES, TILE_BYTES = C::TILE_BYTES, STAGE_BYTES = 2 * TILE_BYTES, NW = 4 * NG;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = smem_u32(smem_raw);
  const uint32_t base = (raw_addr + 1023u) & ~1023u;
  uint8_t* const smem = smem_raw + (base - raw_addr);
  const uint32_t bar_full = base + C::OFF_BAR, bar_empty = bar_full + 8 * STAGES;
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(smem + C::OFF_MISC);
  CtaSlice* const slice = reinterpret_cast<CtaSlice*>(smem + C::OFF_PLAN);
  int* const prefix = reinterpret_cast<int*>(smem + C::OFF_PREFIX);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(bar_full + 8 * s, 1);
      mbar_init(bar_empty + 8 * s, 4);
    }
    abort_flag[0] = 0;
    abort_flag[1] = -1;                  // see await_copies
    mbar_fence_init();
  }
  if (tid == 32 * NW) {
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  pdl_launch_next();
  pdl_wait();
  if (warp == 0) plan_slice<kTileTokens, WIN>(p, prefix, slice, blockIdx.x, gridDim.x, lane);
  if (warp > 0 && warp < NW) unwritten_parts(p, blockIdx.x, D, tid - 32, 32 * (NW - 1));
  __syncthreads();
  const int hkv = p.n_kv_heads, cta = blockIdx.x;
  const int64_t T0 = slice->begin, T1 = slice->end;

  if (warp == NW) {
    // ------------------------------------------------------------------ producer
    {
      const bool leader = elect_one();
      SliceCursor c;
      c.start(T0, T1, slice->first);
      const uint64_t policy = l2_policy_evict_first();
      const int tiles_per_block = p.block_table ? p.block_tokens / kTileTokens : 1;
      bool ok = true, told = false;
      int i = 0;
      KeyView view = {};
      for (; !c.done() && ok; ++i) {
        const int s = i % STAGES;
        if (i >= STAGES) ok = warp_wait(bar_empty + 8 * s, ((i / STAGES) - 1) & 1, abort_flag);
        if (!ok) break;
        if (WIN && (i == 0 || c.j == 0)) view = key_view<WIN>(p, p.n_win, c.sg.b);
        const int t = key_tile<WIN>(view, c.sg.tile0 + c.j);
        int blk = c.sg.b, tok = t * kTileTokens;
        if (p.block_table) {
          blk = p.block_table[(size_t)c.sg.b * p.max_blocks + t / tiles_per_block];
          if (WIN && (blk < 0 || blk >= p.n_blocks) && p.d_status) *p.d_status = SPECVLM_ERR_INVALID_ARG;   // the copy gives zeros
          tok = (t % tiles_per_block) * kTileTokens;
        }
        const uint32_t full = bar_full + 8 * s, dst = base + s * STAGE_BYTES;
        if (leader) {
          mbar_arrive_expect_tx(full, STAGE_BYTES);
#pragma unroll
          for (int h = 0; h < D / 64; ++h) {
            tma_load_5d(dst + h * (kTileTokens * 128), &tm_k, full, h * 64, tok, c.sg.g, blk, c.sg.layer, policy);
            tma_load_5d(dst + TILE_BYTES + h * (kTileTokens * 128), &tm_v, full, h * 64, tok, c.sg.g, blk, c.sg.layer, policy);
          }
        }
        if (!told && i == STAGES - 1) {                     // the ring is full: time for the hand-over of a cut item
          if (leader) publish_cut_item(p, *slice, cta, cta, prefix);
          told = true;
        }
        c.next_tile(prefix, p.batch, hkv);
      }
      if (!told && leader) publish_cut_item(p, *slice, cta, cta, prefix);
      if (!ok) {
        // a wait expired: report, then stay until this CTA's copies in flight have landed
        if (p.d_status && leader) *p.d_status = SPECVLM_ERR_TIMEOUT;
        const uint64_t t0 = global_timer_ns();
        for (int k = i > STAGES ? i - STAGES : 0; k < i; ++k)
          while (!mbar_test_wait(bar_full + 8 * (k % STAGES), (k / STAGES) & 1) && global_timer_ns() - t0 < kWaitLimitNs) {
          }
      }
      if (leader) abort_flag[1] = i;
    }
    return;
  }

  // -------------------------------------------------------------------- consumers
  const int cw = warp & 3, grp = warp >> 2;                           // token slice, consumer group
  float* const o_sm = reinterpret_cast<float*>(smem + C::OFF_O);      // [NW][16][OPITCH]
  float* const m_sm = reinterpret_cast<float*>(smem + C::OFF_ML);     // [NW][16]
  float* const l_sm = m_sm + NW * 16;                                  // [NW][16]
  // sequences without any token: their outputs are zero, their LSE -inf
  if (slice->any_empty) {
    const int n_items = p.n_layers * p.batch * hkv;
    for (int item = cta; item < n_items; item += (int)gridDim.x) {
      const int lb = item / hkv, g = item - lb * hkv, b = lb % p.batch;
      if (prefix[b + 1] != prefix[b]) continue;
      for (int idx = tid; idx < p.rows * (D / 8); idx += 128 * NG) {
        const int r = idx / (D / 8), c8 = idx - r * (D / 8);
        const int t = r / p.group, h = g * p.group + (r - t * p.group);
        const size_t orow = ((size_t)lb * p.n_win + t) * p.n_q_heads + h;
        *reinterpret_cast<uint4*>(p.out + orow * D + c8 * 8) = make_uint4(0, 0, 0, 0);
        if (p.lse && c8 == 0) p.lse[orow] = -INFINITY;
      }
    }
  }
  SliceCursor c;
  c.start(T0, T1, slice->first);
  bool alive = true;
  int i0 = 0;                                                          // slice index of the item's first tile
  while (!c.done()) {
    const Segment sg = c.sg;
    const KeyView view = key_view<WIN>(p, p.n_win, sg.b);
    const size_t lb = (size_t)sg.layer * p.batch + sg.b;
    Rows16<D> st;
    st.start(p, p.n_win, p.rows, lb, sg.g, view.len, lane);
    for (int j = (grp + NG - i0 % NG) % NG; alive && j < sg.n_tiles; j += NG) {
      const int i = i0 + j, s = i % STAGES;
      if (!mbar_wait(bar_full + 8 * s, (i / STAGES) & 1, abort_flag)) {
        alive = false;
        break;
      }
      const uint32_t k_base = base + s * STAGE_BYTES;
      st.template tile<WIN>(p, p.n_win, k_base, k_base + TILE_BYTES, smem + s * STAGE_BYTES + TILE_BYTES, (sg.tile0 + j) * kTileTokens, view,
                            cw, lane);
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_empty + 8 * s);
    }
    // merge the consumer warps' partials; the first barrier also says that the previous item's have been read
    const bool complete = sg.tile0 == 0 && sg.n_tiles == sg.item_tiles;
    const int slot = partial_slot(cta, T0, sg.item_begin);
    // and whether every consumer has seen all its tiles: one answer for all threads, so that a row is stored whole or not at all
    const bool whole = bar_and(alive && cta != p.lost_cta, 128 * NG);
    if (!whole && tid == 0 && p.d_status) *p.d_status = SPECVLM_ERR_TIMEOUT;
    st.publish(o_sm, m_sm, l_sm, p.rows, warp, lane);
    asm volatile("bar.sync 1, %0;" ::"n"(128 * NG) : "memory");
    if (whole) {
      for (int idx = tid; idx < p.rows * (D / 4); idx += 128 * NG) {
        const int r = idx / (D / 4), ch = (idx - r * (D / 4)) * 4;
        float4 acc;
        const float lse2 = rows16_merge<D, NW>(o_sm, m_sm, l_sm, r, ch, acc);
        if (complete) {
          const int t = r / p.group, h = sg.g * p.group + (r - t * p.group);
          const size_t orow = (lb * p.n_win + t) * p.n_q_heads + h;
          store_bf16x4(p.out + orow * D + ch, acc);
          if (p.lse && ch == 0) p.lse[orow] = lse2 * kLn2;
        } else {
          const size_t prow = (size_t)slot * p.rows + r;
          *reinterpret_cast<float4*>(p.ws_o + prow * D + ch) = acc;
          if (ch % 64 == 0) p.ws_lse[(size_t)(ch / 64) * p.lse_block + prow] = lse2;
        }
      }
    }
    i0 += sg.n_tiles;
    c.next_segment(prefix, p.batch, hkv);
  }
  if (!alive && lane == 0) await_copies<STAGES>(bar_full, abort_flag);
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
// Test hook (specvlm_debug_set_attn_splits): 1 forces a CTA per item, n > 1 slices of about an n-th of a
// sequence each; 0 leaves the choice to the rule below.
static std::atomic<int> g_forced_splits{0};
// Test hook (specvlm_debug_set_window_kernel): 1 the tcgen05 kernel, 2 groups of 16 rows, 3 a warp for each, 0 the rule below
static std::atomic<int> g_forced_rows_form{0};

constexpr int kRows16Max = 16;     // windows up to this many rows run on the 16-row kernels
constexpr int kTcMaxRows = 128;    // what one CTA of the tcgen05 kernel takes
constexpr int32_t kWindowMaxKeys = 0x7fffff00;     // positions and tiles of a call with a window stay within 31 bits, rounded up too

// Time that one CTA takes for a tile, us.
static double rows16_tile_us(const specvlm_kv_t* kv) {
  return (kv->head_dim == 128 ? 0.35 : 0.25) * (kv->block_table ? 1.25 : 1.0);
}

// CTAs per item of a launch without slices: the number that is the fastest where every CTA has an SM of its own.  The
// hand-over costs 1.3 us: one layer of 4 items of 200 tokens 3.7 us with a CTA each, 4.3 with two; of 800 / 1600 / 3200
// tokens 7.0 / 11.3 / 20.1 with one (7.4 / 8.5 on slices from 1600) and 4.4 / 5.0 / 6.3 with eight.  Clusters do not use
// every SM of a GPC: 16 of eight CTAs no longer run side by side (4 layers of 800 tokens 7.3 -> 8.4), 24 of four do (2 layers
// x 3 sequences of 800 tokens 8.0 -> 5.4).
// window: a call with a window, whose items are all as long as the host's bound.  There 32 clusters of four and 12 of eight, which
// do run side by side, are used too: 32 items, d = 128, window 512 / 1024 6.53 / 8.45 -> 6.01 / 7.35 us, 12 of 1024 6.56 -> 5.85.
static int rows16_cluster(const specvlm_kv_t* kv, int64_t items, int64_t tiles, bool window = false) {
  if (g_forced_splits.load(std::memory_order_relaxed) == 1) return 1;
  int best = 1;
  double best_us = rows16_tile_us(kv) * tiles;
  for (int n = 2; n <= kMaxRows16Cluster; n *= 2) {
    const double us = 1.3 + rows16_tile_us(kv) * ((tiles + n - 1) / n);
    if (items * n <= (n == 2 ? 144 : n == 4 ? (window ? 128 : 96) : (window ? 96 : 64)) && us < best_us) {
      best = n;
      best_us = us;
    }
  }
  return best;
}

// Whether slices are worth a workspace: estimated times in us, from the host's bound on the lengths, against a CTA per item.
static bool rows16_slices_beat_ctas(const specvlm_kv_t* kv, int32_t batch, int64_t items, int64_t tiles, bool window) {
  // A CTA per item: about 3 us around the tiles; while the items fit the SMs the longest one counts (one CTA takes 0.35 us
  // a tile at d = 128, a quarter more with a block table) or HBM does; beyond, rounds of two CTAs per SM at 0.75 us a tile,
  // or HBM with a last round that is partly empty.  Slices: 4.5 us with the merge kernel, the bytes, 2 us for every
  // item boundary of a CTA.  A batch is taken as ragged (slices balance it; so do many rounds): 0.85 of the bytes.
  // Slices have to win by 1.5 us: they cost a second launch.  Measured, 4 KV heads of d = 128, CTA per item / slices:
  // 1 layer of 1600 / 3200 / 6400 / 12 800 tokens 11.3 / 20.1 / 38.0 / 73.7 against 7.4 / 8.5 / 10.3 / 11.2; 20 layers of
  // 2560 / 5120 / 10 240 tokens 20.7 / 37.7 / 72.7 against 23.8 / 37.9 / 65.9; 28 layers of 640 / 1280 / 5120 tokens
  // 6.3 / 11.9 / 46.4 against 12.9 / 16.2 / 50.0; 28 layers x 4 ragged paged sequences of up to 640 / 1280 tokens
  // 18.1 / 34.0 against 28.1 / 41.4.
  const int64_t sms = sm_count();
  const double hbm = (double)items * tiles * (256.0 * kv->head_dim) / 6.65e6;
  const double ragged = batch > 1 && !window ? 0.85 : 1.0;
  double per_item;
  if (items <= sms) {
    const double longest = rows16_tile_us(kv) * tiles;
    per_item = 3.0 + (longest > hbm ? longest : hbm);
  } else {
    const double rounds = (double)((items + 2 * sms - 1) / (2 * sms));
    const double stream = (1.0 + 0.2 / rounds) * ragged * hbm, serial = rounds * tiles * 0.75 * kv->head_dim / 128;
    per_item = 3.0 + (stream > serial ? stream : serial);
  }
  return 4.5 + ragged * hbm + 2.0 * (1.0 + (double)items / sms) + 1.5 < per_item;
}

// CTAs of a launch on slices, or 0 for a CTA (or a cluster) per item.  *scratch_ctas: the CTAs that the workspace has to
// have room for, 0 for none.  It does not depend on whether a cluster takes the slices' place: the choice between the two
// turns back and forth with the length, and a workspace sized for the longest sequences has to serve the shorter ones.
static int rows16_slices(const specvlm_kv_t* kv, int32_t batch, int* scratch_ctas, bool window = false) {
  const int64_t items = (int64_t)kv->n_layers * batch * kv->n_kv_heads;
  const int64_t tiles = (kv->max_seq_len + kTileTokens - 1) / kTileTokens, sms = sm_count();
  const int forced = g_forced_splits.load(std::memory_order_relaxed);
  *scratch_ctas = 0;
  if (batch > kSchedMaxBatch || forced == 1) return 0;
  if (forced > 1) {
    const int64_t n = items * (forced < tiles ? forced : tiles);
    return *scratch_ctas = (int)(n < 4 * sms ? n : 4 * sms);
  }
  if (!rows16_slices_beat_ctas(kv, batch, items, tiles, window)) return 0;
  *scratch_ctas = sched_scratch_ctas(items * tiles, (int)sms);
  const int n = rows16_cluster(kv, items, tiles, window);
  if (n > 1) {
    // A cluster per item, 3.9 us around its CTAs' tiles or the bytes, which half the SMs do not stream as well, against
    // slices, 6.5 us around the bytes (in pages 6) and more for many parts an item.  Measured, cluster / slices: 1 item
    // (d = 64) of 10 240 tokens 8.5 / 11.6; 12 items of 640 / 2560 / 10 240 4.9 / 7.3 / 18.5 against 7.0 / 8.3 / 16.4; 16 paged ones of 2560 / 5120 /
    // 10 240 8.3 / 13.4 / 23.9 against 9.0 / 10.8 / 15.7; 40 of 2560 / 10 240 / 20 480 11.3 / 38.8 / 75.5 against 14.2 / 37.3 /
    // 64.7; 64 of 1280 / 2560 / 5120 / 10 240 7.5 / 15.3 / 28.4 / 52.6 against 11.0 / 20.5 / 31.8 / 55.0; 72 ragged ones of up to
    // 1280 / 2560 / 10 240 7.5 / 11.3 / 47.2 against 12.9 / 16.1 / 48.3.
    const double hbm = (double)items * tiles * (256.0 * kv->head_dim) / 6.65e6, ragged = batch > 1 && !window ? 0.85 : 1.0;
    const double longest = 1.08 * rows16_tile_us(kv) * ((tiles + n - 1) / n);
    const double parts = (double)(items * tiles < sms ? items * tiles : sms) / items;
    if ((kv->block_table ? 6.0 : 6.5) + ragged * hbm + 0.04 * parts >= 3.9 + (longest > 1.09 * hbm ? longest : 1.09 * hbm)) return 0;
  }
  const int even = sched_active_ctas(items * tiles, (int)sms);
  // slices that keep to item boundaries may use more CTAs: every item rounds its own up
  const int64_t aligned = items * sched_active_ctas(tiles, (int)sms);
  return aligned > even && items <= sms ? (int)(aligned < sms ? aligned : sms) : even;
}

static size_t rows16_scratch_bytes(const specvlm_kv_t* kv, int scratch_ctas, int rows) {
  return scratch_ctas == 0 ? 256 : SliceScratch(scratch_ctas, rows, kv->head_dim).bytes();
}
static size_t rows16_ws_bytes(const specvlm_kv_t* kv, int32_t batch, int rows, bool window = false) {
  int scratch_ctas;
  rows16_slices(kv, batch, &scratch_ctas, window);
  return rows16_scratch_bytes(kv, scratch_ctas, rows);
}

// tcgen05 path (attn_tc.cu)
size_t attn_tc_ws_bytes(const specvlm_kv_t* kv, int32_t batch, int rows, int group);
double attn_tc_window_us(const specvlm_kv_t* kv, int32_t batch, int rows);      // estimate for a call with a window
int32_t attn_tc_launch(const specvlm_kv_t* kv, const void* q, int32_t batch, int32_t n_q_heads, int32_t n_q,
                       float sm_scale, void* out, float* lse, void* ws, size_t ws_bytes, int32_t* d_status,
                       cudaStream_t st, const int32_t* tree_parents, const KeyWindow* win = nullptr, int lost_cta = -1, int32_t* n_ctas = nullptr);

template <int D, int STAGES, int NG, bool SPLIT, bool WIN>
static int32_t launch_rows16_s(const CUtensorMap& tk, const CUtensorMap& tv, const AttnParams& p,
                               dim3 grid, cudaStream_t st) {
  constexpr int SMEM = STAGES * 2 * kTileTokens * D * 2 + 1024 + 16 * STAGES + 16 + (SPLIT ? 16 * 4 : 0);
  auto kern = attn_rows16_kernel<D, STAGES, NG, SPLIT, WIN>;
  static std::atomic<uint64_t> attr_done{0};
  if (!smem_attr_once(attr_done, reinterpret_cast<const void*>(kern), SMEM)) return SPECVLM_ERR_CUDA;
  return launch_clusters_after(kern, grid, (int)grid.x, dim3(32 * (4 * NG + 1)), (size_t)SMEM, st, tk, tv, p);
}

// Ring depth: 3 stages let two CTAs share an SM; a launch with no more CTAs than SMs would leave
// every SM with one CTA and 96 KB of copies in flight, too little to cover the HBM latency, so it
// takes 6 stages and two consumer groups instead.
template <int D, bool WIN>
static int32_t launch_rows16(const CUtensorMap& tk, const CUtensorMap& tv, const AttnParams& p,
                             dim3 grid, int64_t tiles, cudaStream_t st) {
  const int64_t ctas = (int64_t)grid.x * grid.y * grid.z;
  constexpr int kDeep = D == 128 ? 6 : 12;
  if (grid.x > 1) return launch_rows16_s<D, kDeep, 2, true, WIN>(tk, tv, p, grid, st);
  // Short windows, two CTAs an SM: their tiles, one after the other, are the time, and two groups halve them.
  if constexpr (WIN && D == 64)
    if (ctas > sm_count() && ctas <= 2 * sm_count()) return launch_rows16_s<D, kHalfRing, 2, false, WIN>(tk, tv, p, grid, st);
  // More CTAs than two an SM: where they are short their time is what is around their tiles, and three an SM with shorter rings
  // overlap more of it.  d = 128, two / three: 384 items, which run at once then, of 64 / 256 / 512 / 1024 keys 6.2 / 12.9 / 20.8 / 36.1 against
  // 4.4 / 10.8 / 18.1 / 32.4 us, 1088 of 64 / 256 / 512 / 1024 14.9 / 28.0 / 46.3 / 84.3 against 13.8 / 26.7 / 46.6 / 86.1, 896 of 2112 156 against
  // 164.  (d = 64, five of two stages for four of three: 1088 of 64 / 512 keys 6.3 / 25.3 -> 7.3 / 28.3.)
  if constexpr (WIN && D == 128)
    if (ctas > 2 * sm_count() && (ctas <= 3 * sm_count() || tiles <= kShortTiles))
      return launch_rows16_s<D, kShortRing, 1, false, WIN>(tk, tv, p, grid, st);
  return ctas <= sm_count() ? launch_rows16_s<D, kDeep, 2, false, WIN>(tk, tv, p, grid, st)
                            : launch_rows16_s<D, 3, 1, false, WIN>(tk, tv, p, grid, st);
}

template <int D, int NW, int STAGES, int PER_SM, int U>
static int32_t launch_row_groups_s(const CUtensorMap& tk, const CUtensorMap& tv, const AttnParams& p, dim3 grid, cudaStream_t st) {
  constexpr int SMEM = STAGES * 2 * kTileTokens * D * 2 + 1024 + 16 * STAGES + 16;
  auto kern = attn_row_groups_kernel<D, NW, STAGES, PER_SM, U>;
  static std::atomic<uint64_t> attr_done{0};
  if (!smem_attr_once(attr_done, reinterpret_cast<const void*>(kern), SMEM)) return SPECVLM_ERR_CUDA;
  return launch_after(kern, grid, dim3(32 * (p.row_groups + 1)), (size_t)SMEM, st, tk, tv, p);
}
template <int D>
static int32_t launch_row_groups(const CUtensorMap& tk, const CUtensorMap& tv, const AttnParams& p, dim3 grid, cudaStream_t st) {
  if constexpr (D == 128)
    return p.row_groups <= 4 ? launch_row_groups_s<D, 4, 2, 3, 1>(tk, tv, p, grid, st) : launch_row_groups_s<D, 9, 3, 1, 4>(tk, tv, p, grid, st);
  else
    return p.row_groups <= 4 ? launch_row_groups_s<D, 4, 3, 4, 2>(tk, tv, p, grid, st) : launch_row_groups_s<D, 9, 3, 2, 2>(tk, tv, p, grid, st);
}

template <int D, bool WIN>
static int32_t launch_slices(const CUtensorMap& tk, const CUtensorMap& tv, const AttnTcParams& p, int ctas, cudaStream_t st) {
  using C = SliceCfg<D>;
  auto kern = attn_rows16_slices_kernel<D, WIN>;
  static std::atomic<uint64_t> attr_done{0};
  if (!smem_attr_once(attr_done, reinterpret_cast<const void*>(kern), C::SMEM)) return SPECVLM_ERR_CUDA;
  return launch_after(kern, dim3((unsigned)ctas), dim3(32 * (4 * C::NG + 1)), (size_t)C::SMEM, st, tk, tv, p);
}

// Test hook (specvlm_debug_attn_merge): one CTA's partial results as if it had given up, without a wait that expires.
__global__ void give_up_kernel(const __grid_constant__ AttnTcParams p, int gcta, int head_dim) {
  pdl_wait();
  unwritten_parts(p, gcta, head_dim, threadIdx.x, blockDim.x);
}

// How a call with a window and more than 16 rows runs: on the tcgen05 kernel, which takes kTcMaxRows rows of a window at most and
// refuses more; as groups of 16 rows on the kernels above, each with CTAs of its own that read the same tiles (all but the first
// from the L2 cache); or on a CTA per item with a warp for each group.  For short windows the time is what is around the tiles: 4
// us an item here, which the CTAs of an SM overlap, against 8 to 12 there, or 3 to 4 an item of a CTA's list; a tile takes a warp
// that goes through it alone 1.2 to 3.6 us, four warps 0.35 and the tcgen05 kernel about 1 for all rows.  So groups where the items
// are few, warps where they are many and short, tcgen05 where they are long.  Measured, tcgen05 / groups / warps, us: d = 128, 42 rows,
// 50 items of 64 / 512 keys 6.6 / 4.5 / 5.0 and 10.4 / 9.2 / 21.2, 200 of 512 23.2 / 23.1 / 30.1, 2000 of 512 115 / 171 / 144; 24 rows, 440
// of 64 / 256 16.2 / 10.5 / 6.2 and 25.4 / 17.8 / 16.6, 2000 of 64 / 256 61 / 41 / 30 and 74 / 70 / 72; 96 rows, 400 of 64 25.4 / 27.6 / 16.4;
// d = 64, 36 rows, 2000 of 64 / 512 50 / 36 / 21 and 86 / 95 / 75.  The estimates below choose the fastest of the three or one that
// takes 0.9 % more on average (geometric mean; 6 % of the calls more than 5 %, none more than 25 %) in 594 calls: d = 128 with 24, 42,
// 64, 72, 96 and 128 rows and d = 64 with 24, 36, 64, 72 and 128, 50 to 2000 items, windows of 64 to 512 keys.
enum class RowsForm { kTc, kGroups, kWarps };
// (kv: the positions that size the launch, of which `seen` are keys that some query sees)
static RowsForm window_rows_form(const specvlm_kv_t* kv, int64_t seen, int32_t batch, int rows) {
  const int groups = (rows + kRows16Max - 1) / kRows16Max, forced = g_forced_rows_form.load(std::memory_order_relaxed);
  const int64_t items = (int64_t)kv->n_layers * batch * kv->n_kv_heads, n_groups = items * groups, sms = sm_count();
  const int64_t tiles = (kv->max_seq_len + kTileTokens - 1) / kTileTokens;
  const bool wide = kv->head_dim == 128;
  if ((int64_t)kv->n_layers * batch > 65535 || (int64_t)kv->n_kv_heads * groups > 65535) return RowsForm::kTc;
  if (forced == 1 && rows <= kTcMaxRows) return RowsForm::kTc;
  if (forced > 1) return forced == 2 ? RowsForm::kGroups : RowsForm::kWarps;
  const double floor_us = 3.9 + (double)items * kv->max_seq_len * (4.0 * kv->head_dim) / 6.5e6;
  // rounds of `at_once` pieces of work: whole ones while they are few
  auto rounds = [](int64_t n, int64_t at_once) { return n > 4 * at_once ? (double)n / at_once : (double)((n + at_once - 1) / at_once); };
  double groups_us;
  if (n_groups <= sms) {
    const int n = rows16_cluster(kv, n_groups, tiles, true);
    groups_us = 3.9 + (n > 1 ? 1.0 : 0.0) + 1.08 * rows16_tile_us(kv) * (double)((tiles + n - 1) / n);
  } else if (n_groups <= 2 * sms) {
    groups_us = wide ? 4.4 + 0.68 * tiles : 4.2 + 0.5 * tiles;
  } else {
    groups_us = rounds(n_groups, (wide ? 3 : 4) * sms) * (wide ? 4.0 + 0.98 * tiles : 3.0 + 0.74 * tiles);
  }
  // items on an SM at once (attn_row_groups_kernel), and a tile of an item that is alone there, or not
  const int most = wide ? (groups <= 4 ? 3 : groups == 5 ? 2 : 1) : groups <= 4 ? 4 : groups == 5 ? 3 : 2;
  double tile_us = wide ? 2.1 : groups <= 4 ? 1.2 : 1.5;
  if (items > sms) tile_us = wide ? (groups <= 4 ? 2.0 + 0.4 * groups : groups == 5 ? 2.4 : 2.1) : groups <= 4 ? 0.8 + 0.35 * groups : 2.0;
  // (up to four warps take a tile in parts, of which they leave out those that no query sees)
  const double seen_tiles = groups <= 4 ? (double)(seen + (wide ? 16 : 32)) / kTileTokens : (double)tiles;
  double warps_us = rounds(items, most * sms) * (4.0 + tile_us * (seen_tiles < tiles ? seen_tiles : (double)tiles));
  if (groups_us < floor_us) groups_us = floor_us;
  if (warps_us < floor_us) warps_us = floor_us;
  if (rows <= kTcMaxRows && attn_tc_window_us(kv, batch, rows) <= (groups_us < warps_us ? groups_us : warps_us)) return RowsForm::kTc;
  return groups_us <= warps_us ? RowsForm::kGroups : RowsForm::kWarps;
}

static int32_t attn_common(const specvlm_kv_t* kv, const void* q, int32_t batch, int32_t n_q_heads,
                           int32_t n_q, float sm_scale, void* out, float* lse, void* ws,
                           size_t ws_bytes, int32_t* d_status, void* stream, int lost_cta = -1, int32_t* n_ctas = nullptr,
                           const KeyWindow* win = nullptr) {
  int32_t rc = validate_kv(kv, batch, true);
  if (rc != SPECVLM_OK) return rc;
  if (!q || !out || n_q_heads < 1 || n_q < 1 || !(sm_scale > 0.f)) return SPECVLM_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(out)) return SPECVLM_ERR_INVALID_ARG;
  if (n_q_heads % kv->n_kv_heads != 0) return SPECVLM_ERR_INVALID_ARG;
  const int group = n_q_heads / kv->n_kv_heads;
  if (group > 16 || n_q > 9) return SPECVLM_ERR_UNSUPPORTED_SHAPE;
  const int rows = group * n_q;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const specvlm_kv_t sched = win ? win->view(kv, n_q) : *kv;
  if (win && rows > kRows16Max) {          // what the tcgen05 kernel asks for, whichever is chosen
    if (batch > kSchedMaxBatch) return SPECVLM_ERR_UNSUPPORTED_SHAPE;
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u)) return SPECVLM_ERR_INVALID_ARG;
    if (ws_bytes < attn_tc_ws_bytes(&sched, batch, rows, group)) return SPECVLM_ERR_WORKSPACE_TOO_SMALL;
  }
  const RowsForm form = win && rows > kRows16Max ? window_rows_form(&sched, (int64_t)win->window + win->n_sinks + n_q - 1, batch, rows) : RowsForm::kTc;
  const int row_groups = form != RowsForm::kTc ? (rows + kRows16Max - 1) / kRows16Max : 1;
  if (rows > kRows16Max && form == RowsForm::kTc)
    return attn_tc_launch(kv, q, batch, n_q_heads, n_q, sm_scale, out, lse, ws, ws_bytes, d_status, st, nullptr, win, lost_cta, n_ctas);

  const int64_t lb64 = (int64_t)kv->n_layers * batch;
  if (lb64 > 65535 || kv->n_kv_heads * row_groups > 65535) return SPECVLM_ERR_UNSUPPORTED_SHAPE;
  int scratch_ctas = 0;
  const int ctas = row_groups > 1 ? 0 : rows16_slices(&sched, batch, &scratch_ctas, win != nullptr);
  if (scratch_ctas > 0) {
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u)) return SPECVLM_ERR_INVALID_ARG;
    if (ws_bytes < rows16_scratch_bytes(kv, scratch_ctas, rows)) return SPECVLM_ERR_WORKSPACE_TOO_SMALL;
  }
  const int64_t tiles = (sched.max_seq_len + kTileTokens - 1) / kTileTokens, items = lb64 * kv->n_kv_heads * (form == RowsForm::kWarps ? 1 : row_groups);
  const int n = ctas > 0 || form == RowsForm::kWarps ? 1 : rows16_cluster(&sched, items, tiles, win != nullptr);
  // The tiles of short windows are mostly rows that no query sees.  Where there are more CTAs than SMs these need not be read: copies of
  // 16 rows.  A wait for twelve of them takes longer than for four of 64 where the CTAs are few.  Windows of 16 / 100 / 400 keys, whole
  // tiles / slices, us, d = 128: 48 items 3.4 / 4.3 / - against 3.3 / 5.0 / -, 200 4.0 / 6.7 / - against 3.6 / 5.7 / -, 1088 12.8 / 22.5 / 41.8
  // against 10.6 / 20.5 / 42.4, of 50 keys and 4 sinks 22.6 against 18.5; 24 rows, a warp for 16, 18.6 / 27.7 / 67.3 against 15.4 / 26.5 / 65.4.
  const bool sliced = win && ctas == 0 && n == 1 && tiles <= kSlicedTiles && sched.max_seq_len < kv->max_seq_len &&
                      2 * items > (kv->head_dim == 128 ? 2 : 3) * (int64_t)sm_count();
  CUtensorMap tk, tv;
  rc = encode_kv_map(&tk, kv, kv->k, sliced ? kSliceTokens : kTileTokens);
  if (rc != SPECVLM_OK) return rc;
  rc = encode_kv_map(&tv, kv, kv->v, sliced ? kSliceTokens : kTileTokens);
  if (rc != SPECVLM_OK) return rc;

  if (ctas > 0) {
    const SliceScratch sc(ctas, rows, kv->head_dim);
    AttnTcParams p = slice_params(kv, q, batch, n_q_heads, n_q, sm_scale, out, lse, d_status, 1, n_q, ws, sc);
    p.lost_cta = lost_cta;
    if (n_ctas) *n_ctas = ctas;
    if (win) {
      p.window = win->window;
      p.n_sinks = win->n_sinks;
      rc = kv->head_dim == 128 ? launch_slices<128, true>(tk, tv, p, ctas, st) : launch_slices<64, true>(tk, tv, p, ctas, st);
    } else {
      rc = kv->head_dim == 128 ? launch_slices<128, false>(tk, tv, p, ctas, st) : launch_slices<64, false>(tk, tv, p, ctas, st);
    }
    return rc != SPECVLM_OK ? rc : attn_merge_launch(p, kv->head_dim, ctas, st);
  }

  AttnParams p;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.out = static_cast<__nv_bfloat16*>(out);
  p.lse = lse;
  p.block_table = kv->block_table;
  p.seq_lens = kv->seq_lens;
  p.d_status = d_status;
  p.batch = batch;
  p.n_q = n_q;
  p.n_q_heads = n_q_heads;
  p.n_kv_heads = kv->n_kv_heads;
  p.group = group;
  p.rows = rows;
  p.max_blocks = kv->max_blocks;
  p.block_tokens = kv->block_tokens;
  p.max_seq_len = kv->max_seq_len;
  p.scale_log2 = sm_scale * kLog2e;
  p.lost_cta = lost_cta;
  p.window = win ? win->window : 0;
  p.n_sinks = win ? win->n_sinks : 0;
  p.n_blocks = kv->n_blocks;
  p.row_groups = row_groups;
  p.sliced = sliced ? 1 : 0;

  if (form == RowsForm::kWarps) {
    const dim3 grid(1, (unsigned)kv->n_kv_heads, (unsigned)lb64);
    if (n_ctas) *n_ctas = (int32_t)(grid.y * grid.z);
    return kv->head_dim == 128 ? launch_row_groups<128>(tk, tv, p, grid, st) : launch_row_groups<64>(tk, tv, p, grid, st);
  }
  dim3 grid((unsigned)n, (unsigned)(kv->n_kv_heads * row_groups), (unsigned)lb64);
  if (n_ctas) *n_ctas = (int32_t)(grid.x * grid.y * grid.z);
  if (win) return kv->head_dim == 128 ? launch_rows16<128, true>(tk, tv, p, grid, tiles, st) : launch_rows16<64, true>(tk, tv, p, grid, tiles, st);
  return kv->head_dim == 128 ? launch_rows16<128, false>(tk, tv, p, grid, tiles, st) : launch_rows16<64, false>(tk, tv, p, grid, tiles, st);
}

}  // namespace specvlm

using namespace specvlm;

extern "C" void specvlm_debug_set_attn_splits(int32_t n_splits) {
  g_forced_splits.store(n_splits > 0 ? n_splits : 0, std::memory_order_relaxed);
}

extern "C" void specvlm_debug_set_window_kernel(int32_t mode) {
  g_forced_rows_form.store(mode >= 1 && mode <= 3 ? mode : 0, std::memory_order_relaxed);
}

extern "C" int32_t specvlm_debug_attn_merge(const specvlm_kv_t* kv, int32_t batch, int32_t n_q_heads, int32_t n_q,
                                            void* out, float* lse_or_null, void* ws, size_t ws_bytes, int32_t lost_cta,
                                            int32_t* n_ctas, void* stream) {
  const int32_t rc = validate_kv(kv, batch, true);
  if (rc != SPECVLM_OK) return rc;
  if (!out || !ws || !n_ctas || n_q_heads < 1 || n_q < 1 || n_q_heads % kv->n_kv_heads != 0) return SPECVLM_ERR_INVALID_ARG;
  const int group = n_q_heads / kv->n_kv_heads;
  if (group > 16 || n_q > 9 || batch > kSchedMaxBatch) return SPECVLM_ERR_UNSUPPORTED_SHAPE;
  int room;
  const SlicePlan pl = group * n_q > kRows16Max ? attn_tc_plan(kv, batch, group, n_q) : SlicePlan{rows16_slices(kv, batch, &room), 1, n_q};
  const int grid = pl.n_parts * pl.ctas;
  *n_ctas = grid;
  if (grid == 0) return SPECVLM_ERR_UNSUPPORTED_SHAPE;
  const SliceScratch sc(grid, pl.q_per * group, kv->head_dim);
  if (ws_bytes < sc.bytes()) return SPECVLM_ERR_WORKSPACE_TOO_SMALL;
  if (lost_cta >= grid) return SPECVLM_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const AttnTcParams p = slice_params(kv, nullptr, batch, n_q_heads, n_q, 1.f, out, lse_or_null, nullptr, pl.n_parts, pl.q_per, ws, sc);
  if (lost_cta >= 0) {
    const int32_t marked = launch_after(give_up_kernel, dim3(1), dim3(128), 0, st, p, lost_cta, kv->head_dim);
    if (marked != SPECVLM_OK) return marked;
  }
  return attn_merge_launch(p, kv->head_dim, pl.ctas, st);
}

extern "C" int32_t specvlm_debug_attn_give_up(const specvlm_kv_t* kv, const void* q, int32_t batch, int32_t n_q_heads, float sm_scale,
                                              void* out, float* lse_or_null, void* ws, size_t ws_bytes, int32_t lost_cta,
                                              int32_t* n_ctas, int32_t* d_status, void* stream) {
  if (!n_ctas) return SPECVLM_ERR_INVALID_ARG;
  return attn_common(kv, q, batch, n_q_heads, 1, sm_scale, out, lse_or_null, ws, ws_bytes, d_status, stream, lost_cta, n_ctas);
}

extern "C" size_t specvlm_attn_workspace_bytes(const specvlm_kv_t* kv, int32_t batch,
                                               int32_t n_q_heads, int32_t gamma) {
  if (!kv || batch < 1 || n_q_heads < 1 || gamma < 0 || kv->n_kv_heads < 1 ||
      n_q_heads % kv->n_kv_heads != 0 || kv->n_layers < 1 || kv->max_seq_len < 1)
    return 0;
  const int rows = (n_q_heads / kv->n_kv_heads) * (gamma + 1);
  if (n_q_heads / kv->n_kv_heads > 16 || gamma > 8) return 0;
  if (rows > kRows16Max) return batch <= kSchedMaxBatch ? attn_tc_ws_bytes(kv, batch, rows, n_q_heads / kv->n_kv_heads) : 0;
  return rows16_ws_bytes(kv, batch, rows);
}

extern "C" int32_t specvlm_draft_decode_attn(const specvlm_kv_t* kv, const void* q, int32_t batch,
                                             int32_t n_q_heads, float sm_scale, void* out,
                                             float* lse_or_null, void* ws, size_t ws_bytes,
                                             int32_t* d_status, void* stream) {
  NvtxRange nvtx_range(__func__);
  return attn_common(kv, q, batch, n_q_heads, 1, sm_scale, out, lse_or_null, ws, ws_bytes, d_status,
                     stream);
}

extern "C" int32_t specvlm_verify_attn(const specvlm_kv_t* kv, const void* q, int32_t batch,
                                       int32_t n_q_heads, int32_t gamma, float sm_scale, void* out,
                                       float* lse_or_null, void* ws, size_t ws_bytes,
                                       int32_t* d_status, void* stream) {
  NvtxRange nvtx_range(__func__);
  if (gamma < 0 || gamma > 8) return SPECVLM_ERR_UNSUPPORTED_SHAPE;
  return attn_common(kv, q, batch, n_q_heads, gamma + 1, sm_scale, out, lse_or_null, ws, ws_bytes,
                     d_status, stream);
}

extern "C" size_t specvlm_window_attn_workspace_bytes(const specvlm_kv_t* kv, int32_t batch, int32_t n_q_heads, int32_t n_q,
                                                      int32_t window, int32_t n_sinks) {
  if (!kv || n_q < 1 || window < 1 || n_sinks < 0 || kv->n_kv_heads < 1 || kv->max_seq_len < 1 || kv->max_seq_len > kWindowMaxKeys)
    return 0;
  const specvlm_kv_t view = KeyWindow(kv, window, n_sinks).view(kv, n_q);
  const size_t bytes = specvlm_attn_workspace_bytes(&view, batch, n_q_heads, n_q - 1);      // 0: refused
  const int rows = bytes > 0 ? n_q_heads / kv->n_kv_heads * n_q : 0;
  return rows > 0 && rows <= kRows16Max ? rows16_ws_bytes(&view, batch, rows, true) : bytes;
}

extern "C" int32_t specvlm_window_attn(const specvlm_kv_t* kv, const void* q, int32_t batch, int32_t n_q_heads, int32_t n_q,
                                       int32_t window, int32_t n_sinks, float sm_scale, void* out, float* lse_or_null,
                                       void* ws, size_t ws_bytes, int32_t* d_status, void* stream) {
  NvtxRange nvtx_range(__func__);
  if (!kv || window < 1 || n_sinks < 0 || n_q < 1 || kv->n_kv_heads < 1) return SPECVLM_ERR_INVALID_ARG;
  if (n_q > 9 || kv->max_seq_len > kWindowMaxKeys) return SPECVLM_ERR_UNSUPPORTED_SHAPE;
  const KeyWindow win(kv, window, n_sinks);
  return attn_common(kv, q, batch, n_q_heads, n_q, sm_scale, out, lse_or_null, ws, ws_bytes, d_status, stream, -1, nullptr, &win);
}

extern "C" int32_t specvlm_debug_window_give_up(const specvlm_kv_t* kv, const void* q, int32_t batch, int32_t n_q_heads, int32_t n_q,
                                                int32_t window, int32_t n_sinks, float sm_scale, void* out, float* lse_or_null,
                                                void* ws, size_t ws_bytes, int32_t lost_cta, int32_t* n_ctas, int32_t* d_status,
                                                void* stream) {
  if (!kv || !n_ctas || window < 1 || n_sinks < 0 || n_q < 1 || kv->n_kv_heads < 1) return SPECVLM_ERR_INVALID_ARG;
  if (n_q > 9 || kv->max_seq_len > kWindowMaxKeys) return SPECVLM_ERR_UNSUPPORTED_SHAPE;
  const KeyWindow win(kv, window, n_sinks);
  return attn_common(kv, q, batch, n_q_heads, n_q, sm_scale, out, lse_or_null, ws, ws_bytes, d_status, stream, lost_cta, n_ctas, &win);
}

extern "C" size_t specvlm_verify_tree_workspace_bytes(const specvlm_kv_t* kv, int32_t batch, int32_t n_q_heads,
                                                      int32_t n_nodes) {
  if (!kv || batch < 1 || batch > kSchedMaxBatch || n_q_heads < 1 || n_nodes < 1 || n_nodes > 64 ||
      kv->n_kv_heads < 1 || n_q_heads % kv->n_kv_heads != 0 || kv->n_layers < 1 || kv->max_seq_len < 1)
    return 0;
  const int rows = (n_q_heads / kv->n_kv_heads) * n_nodes;
  if (n_q_heads / kv->n_kv_heads > 16) return 0;
  return attn_tc_ws_bytes(kv, batch, rows, n_q_heads / kv->n_kv_heads);
}

extern "C" int32_t specvlm_verify_tree_attn(const specvlm_kv_t* kv, const void* q, const int32_t* parents,
                                            int32_t batch, int32_t n_q_heads, int32_t n_nodes, float sm_scale,
                                            void* out, float* lse_or_null, void* ws, size_t ws_bytes,
                                            int32_t* d_status, void* stream) {
  NvtxRange nvtx_range(__func__);
  int32_t rc = validate_kv(kv, batch, true);
  if (rc != SPECVLM_OK) return rc;
  if (!q || !out || !parents || n_q_heads < 1 || n_nodes < 1 || !(sm_scale > 0.f)) return SPECVLM_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(out) || n_q_heads % kv->n_kv_heads != 0) return SPECVLM_ERR_INVALID_ARG;
  const int group = n_q_heads / kv->n_kv_heads;
  if (group > 16 || n_nodes > 64) return SPECVLM_ERR_UNSUPPORTED_SHAPE;
  return attn_tc_launch(kv, q, batch, n_q_heads, n_nodes, sm_scale, out, lse_or_null, ws, ws_bytes, d_status,
                        static_cast<cudaStream_t>(stream), parents);
}
