// Rotary positions of new tokens' queries and keys, fused with the append of keys and values to the cache.
//
// Every row is read once and written once: a long prompt is bound by HBM (one layer of 4 x 6528 tokens, 64 + 8 heads of d = 128,
// 744 MB in 122 us, 6.1 TB/s).  A warp works on one token of one layer and walks its rows (query heads, then key and
// value heads), a thread on the same 16 channels of each, so that the 8 sines and cosines of a thread serve all of them.  A
// short call is bound by the chain of a warp -- lengths, angles, then a round trip to memory for every two rounds of rows
// -- so a token's rounds are dealt out to several warps, and each angle is computed by one lane of a warp and handed on through
// shared memory: 28 layers x 16 sequences x 6 tokens (50 MB) 19.7 us with a warp a token and every thread its own angles, 12.8 now,
// the counting kernel (1.3) included.
//
// Angles: a position times a frequency in radians loses the angle's digits to the whole turns (position 50 000 in fp32: 2e-3
// radians).  Here frequencies are fractions of a turn in 64-bit fixed point, and position * fraction modulo 2^64 is the exact
// fraction of the angle, of which the upper 32 bits are used.
//
// Lengths and block tables are device data: checked before they become part of an address (see cache.cu).
#include <math.h>

#include "common.cuh"
#include "host_util.h"
#include "rope_turn.h"

namespace specvlm {

struct RopeParams {
  const uint4* q;                                  // rows in 16-byte units
  uint4* q_out;
  const uint4* new_k;
  const uint4* new_v;
  uint4* k;
  uint4* v;
  const uint64_t* turns;
  const int32_t* positions;                        // [n_axes][B][n_new] or null
  const int32_t* new_lens;                         // [B] or null
  int32_t* seq_lens;
  const int32_t* table;
  int32_t* d_status;
  int64_t q_layer, q_batch, q_token, q_head;       // strides in 16-byte units
  int64_t o_layer, o_batch, o_token, o_head;
  int64_t k_layer, k_batch, k_token, k_head;
  int64_t v_layer, v_batch, v_token, v_head;
  int64_t s_layer, s_block, s_head, s_token;       // cache
  int32_t block_tokens, max_blocks, max_seq_len, n_blocks;
  int32_t n_layers, batch, n_new, n_q_heads, n_kv_heads;
  int32_t n_rot;                                   // rotated channels / 16
  int32_t n_axes, axis1, axis2;                    // first pair of axis 1 and of axis 2
  int32_t counted, share;                          // share: warps that a token's rows are dealt out to
  int32_t per_warp;                                // layers that a warp goes through (rope_layers), 0: rope_rows
  float factor;
};

// First cache position of the n new tokens of a sequence of length `len`; false if it is to be left alone.
__device__ __forceinline__ bool rope_range(const RopeParams& p, int n, int len, int& start) {
  if (n < 0 || n > p.n_new || len < 0 || len > p.max_seq_len) return false;
  start = p.counted ? len - n : len;
  return start >= 0 && n <= p.max_seq_len - start;
}
__device__ __forceinline__ void rope_count(const RopeParams& p, int b) {       // (the append has reported the others)
  const int n = p.new_lens ? p.new_lens[b] : p.n_new, len = p.seq_lens[b];
  int start;
  if (rope_range(p, n, len, start)) p.seq_lens[b] = start + n;
}

__device__ __forceinline__ uint64_t bf16x2_to_f2(uint32_t x) {
  return f2_pack(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}
__device__ __forceinline__ uint32_t f2_to_bf16x2(uint64_t v) {
  float lo, hi;
  f2_unpack(v, lo, hi);
  return pack_bf16x2(lo, hi);
}
__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t f2_swap(uint64_t v) {
  float lo, hi;
  f2_unpack(v, lo, hi);
  return f2_pack(hi, lo);
}

// The 8 pairs of two 16-byte vectors, two at a time.  Half layout: the e-th channels of both; c and s hold the cosines and sines of
// pairs 2 w and 2 w + 1.  Interleaved: neighbours; c and s hold those of pair w twice, the first sine negated.
template <bool INTER>
__device__ __forceinline__ void turn_pairs(uint4& x, uint4& y, const uint64_t (&c)[INTER ? 8 : 4], const uint64_t (&s)[INTER ? 8 : 4]) {
  uint32_t* const xw = reinterpret_cast<uint32_t*>(&x);
  uint32_t* const yw = reinterpret_cast<uint32_t*>(&y);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const uint64_t a = bf16x2_to_f2(xw[w]), b = bf16x2_to_f2(yw[w]);
    if constexpr (INTER) {
      xw[w] = f2_to_bf16x2(f2_fma(a, c[w], f2_mul(f2_swap(a), s[w])));
      yw[w] = f2_to_bf16x2(f2_fma(b, c[w + 4], f2_mul(f2_swap(b), s[w + 4])));
    } else {
      const uint64_t minus_b = b ^ 0x8000000080000000ull;
      xw[w] = f2_to_bf16x2(f2_fma(a, c[w], f2_mul(minus_b, s[w])));
      yw[w] = f2_to_bf16x2(f2_fma(b, c[w], f2_mul(a, s[w])));
    }
  }
}

constexpr int kRopeThreads = 128, kRopeOneThreads = 512, kRopeOneTokens = 8, kRopeOneCtas = 8;
constexpr int kRopeOneWarps = kRopeOneCtas * kRopeOneThreads / 32, kRopeOneRounds = 4;
constexpr int kRopeCtas = 8;                       // on an SM: 64 registers a thread
constexpr int kRopeWarps = 48;                     // on an SM: with fewer tokens several warps share one
constexpr int kRopeManyWarps = 128;                // on an SM, that are left where a warp takes several layers
constexpr int kRopeLayerRounds = 4, kRopeLayerBatch = 2;
constexpr int kRopeBatch = 2;         // rounds whose loads are in flight together

// What a warp has to know of its token before it turns rows: loads that depend on nothing (ask), and what follows from them.
template <int D, bool INTER>
struct RopeToken {
  static constexpr int kPerLane = D / 64;            // pairs of a lane: each angle is computed once a warp
  int b, t, u;                                       // sequence, token, this thread's unit: 16 channels of a row
  bool rotates;
  int v0, dv;                                        // its vectors: v0, v0 + dv
  int n_asked, len, pos[3];
  uint64_t turns[kPerLane];
  int blk, off;                                      // where the token's key and value go
  bool stored;
  uint64_t c[INTER ? 8 : 4], s[INTER ? 8 : 4];

  __device__ __forceinline__ void ask(const RopeParams& p, int lane) {
    constexpr int UNITS = D / 16;
    u = lane % UNITS;
    rotates = u < p.n_rot;
    v0 = !INTER && rotates ? u : 2 * u;
    dv = !INTER && rotates ? p.n_rot : 1;
    n_asked = p.new_lens ? p.new_lens[b] : p.n_new;
    len = p.seq_lens[b];
    pos[0] = pos[1] = pos[2] = 0;
    if (p.positions) {
      const int32_t* const where = p.positions + (size_t)b * p.n_new + t;
      const size_t axis = (size_t)p.batch * p.n_new;
#pragma unroll
      for (int a = 0; a < 3; ++a)
        if (a < p.n_axes) pos[a] = where[a * axis];
    }
#pragma unroll
    for (int e = 0; e < kPerLane; ++e) turns[e] = lane + 32 * e < 8 * p.n_rot ? p.turns[lane + 32 * e] : 0;
  }

  // false: the token's rows are padding, or its sequence is left alone
  __device__ __forceinline__ bool find(const RopeParams& p, float* cs_sm, int lane) {
    int start;
    if (!rope_range(p, n_asked, len, start)) {
      if (lane == 0 && p.d_status) *p.d_status = SPECVLM_ERR_INVALID_ARG;
      return false;
    }
    if (t >= n_asked) return false;
    const int at = start + t;
    blk = b;
    off = at;
    stored = true;
    if (p.table) {
      const int nth = (int)((uint32_t)at / (uint32_t)p.block_tokens);
      blk = p.table[(size_t)b * p.max_blocks + nth];
      off = at - nth * p.block_tokens;
      stored = blk >= 0 && blk < p.n_blocks;
      if (!stored && lane == 0 && p.d_status) *p.d_status = SPECVLM_ERR_INVALID_ARG;
    }
    if (!p.positions) pos[0] = pos[1] = pos[2] = at;
#pragma unroll
    for (int e = 0; e < kPerLane; ++e) {
      const int i = lane + 32 * e, where = i < p.axis1 ? pos[0] : i < p.axis2 ? pos[1] : pos[2];
      float sn, cs;
      turn_sincos((uint32_t)(((uint64_t)(int64_t)where * turns[e]) >> 32), sn, cs);
      cs_sm[i] = cs * p.factor;
      cs_sm[D / 2 + i] = sn * p.factor;
    }
    __syncwarp();
    if (rotates) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float4 cs = reinterpret_cast<const float4*>(cs_sm)[2 * u + e], sn = reinterpret_cast<const float4*>(cs_sm + D / 2)[2 * u + e];
        if constexpr (INTER) {
          c[4 * e] = f2_pack(cs.x, cs.x), c[4 * e + 1] = f2_pack(cs.y, cs.y), c[4 * e + 2] = f2_pack(cs.z, cs.z), c[4 * e + 3] = f2_pack(cs.w, cs.w);
          s[4 * e] = f2_pack(-sn.x, sn.x), s[4 * e + 1] = f2_pack(-sn.y, sn.y), s[4 * e + 2] = f2_pack(-sn.z, sn.z), s[4 * e + 3] = f2_pack(-sn.w, sn.w);
        } else {
          c[2 * e] = f2_pack(cs.x, cs.y), c[2 * e + 1] = f2_pack(cs.z, cs.w);
          s[2 * e] = f2_pack(sn.x, sn.y), s[2 * e + 1] = f2_pack(sn.z, sn.w);
        }
      }
    }
    return true;
  }
};

// A warp's rounds are the query rows first and then the key and value rows; those of a token are dealt out to `share` warps.
template <int D, bool INTER>
__device__ __forceinline__ void rope_rows(const RopeParams& p, float* cs_sm, uint32_t warp, int lane) {
  constexpr int UNITS = D / 16, ROWS = 32 / UNITS;  // threads of a row, rows of a round
  const uint32_t token = warp / (uint32_t)p.share, lb = token / (uint32_t)p.n_new;
  const int part = (int)(warp - token * p.share), t = (int)(token - lb * p.n_new);
  const int layer = (int)(lb / (uint32_t)p.batch), b = (int)(lb - (uint32_t)layer * p.batch);
  const int sub = lane / UNITS, step = ROWS * p.share;
  // All loads that depend on nothing are asked for together: the launch is one or two waves of short warps, whose time
  // is the number of round trips to memory one after the other.
  RopeToken<D, INTER> tok;
  tok.b = b;
  tok.t = t;
  tok.ask(p, lane);
  const bool rotates = tok.rotates;
  const int v0 = tok.v0, dv = tok.dv;
  const uint4* q = p.q + layer * p.q_layer + b * p.q_batch + t * p.q_token + v0;
  uint4 x[kRopeBatch], y[kRopeBatch];
  int row = part * ROWS + sub;
  const int64_t q_step = step * p.q_head;
  const uint4* src = q + row * p.q_head;
#pragma unroll
  for (int i = 0; i < kRopeBatch; ++i) {            // (the rows of padding are dropped)
    if (row + i * step < p.n_q_heads) {
      x[i] = src[0];
      y[i] = src[dv];
    }
    src += q_step;
  }
  if (!tok.find(p, cs_sm, lane)) return;
  // queries
  const int64_t o_step = step * p.o_head;
  uint4* to = p.q_out + layer * p.o_layer + b * p.o_batch + t * p.o_token + row * p.o_head + v0;
  while (row < p.n_q_heads) {
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      if (row + i * step < p.n_q_heads) {
        if (rotates) turn_pairs<INTER>(x[i], y[i], tok.c, tok.s);
        to[0] = x[i];
        to[dv] = y[i];
      }
      to += o_step;
    }
    row += kRopeBatch * step;
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      if (row + i * step < p.n_q_heads) {
        x[i] = src[0];
        y[i] = src[dv];
      }
      src += q_step;
    }
  }
  // keys and values, to the cache: their rounds go on where those of the queries end
  if (!tok.stored) return;
  const int q_rounds = (p.n_q_heads + ROWS - 1) / ROWS;
  int first = part - q_rounds % p.share;
  if (first < 0) first += p.share;
  const int64_t dst = layer * p.s_layer + tok.blk * p.s_block + tok.off * p.s_token + v0;
  const uint4* const nk = p.new_k + layer * p.k_layer + b * p.k_batch + t * p.k_token + v0;
  const uint4* const nv = p.new_v + layer * p.v_layer + b * p.v_batch + t * p.v_token + v0;
  for (row = first * ROWS + sub; row < 2 * p.n_kv_heads; row += kRopeBatch * step) {
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      const int h = row + i * step, g = h - p.n_kv_heads;
      if (g < p.n_kv_heads) {
        const uint4* const from = g < 0 ? nk + h * p.k_head : nv + g * p.v_head;
        x[i] = from[0];
        y[i] = from[dv];
      }
    }
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      const int h = row + i * step, g = h - p.n_kv_heads;
      if (g < p.n_kv_heads) {
        if (rotates && g < 0) turn_pairs<INTER>(x[i], y[i], tok.c, tok.s);
        uint4* const into = g < 0 ? p.k + dst + h * p.s_head : p.v + dst + g * p.s_head;
        into[0] = x[i];
        into[dv] = y[i];
      }
    }
  }
}

// The same for many tokens of few heads: a warp takes p.per_warp layers of its token, whose lengths and angles are most of the
// work then, and goes through the rows of all of them, eight or four at a time whichever layer they are of.
template <int D, bool INTER>
__device__ __forceinline__ void rope_layers(const RopeParams& p, float* cs_sm, uint32_t warp, int lane) {
  constexpr int UNITS = D / 16, ROWS = 32 / UNITS;
  const uint32_t lb = warp / (uint32_t)p.n_new;
  const int t = (int)(warp - lb * p.n_new), nth = (int)(lb / (uint32_t)p.batch), b = (int)(lb - (uint32_t)nth * p.batch);
  const int end = min((nth + 1) * p.per_warp, p.n_layers), n_rows = p.n_q_heads + 2 * p.n_kv_heads;
  RopeToken<D, INTER> tok;
  tok.b = b;
  tok.t = t;
  tok.ask(p, lane);
  const int v0 = tok.v0, dv = tok.dv;
  const uint4* const q = p.q + b * p.q_batch + t * p.q_token + v0;
  const uint4* const nk = p.new_k + b * p.k_batch + t * p.k_token + v0;
  const uint4* const nv = p.new_v + b * p.v_batch + t * p.v_token + v0;
  if (!tok.find(p, cs_sm, lane)) return;
  uint4* const o = p.q_out + b * p.o_batch + t * p.o_token + v0;
  const int64_t dst = tok.blk * p.s_block + tok.off * p.s_token + v0;
  int layer = nth * p.per_warp, row = lane / UNITS;
  auto wrap = [&]() {
    while (row >= n_rows) {
      row -= n_rows;
      ++layer;
    }
  };
  wrap();
  while (layer < end) {                             // (lanes of a warp may end a round apart)
    uint4 x[kRopeLayerBatch], y[kRopeLayerBatch];
    uint4* to[kRopeLayerBatch];
    bool turn[kRopeLayerBatch];
#pragma unroll
    for (int i = 0; i < kRopeLayerBatch; ++i) {
      to[i] = nullptr;
      if (layer < end) {
        const int h = row - p.n_q_heads, g = h - p.n_kv_heads;
        const uint4* const src = h < 0 ? q + layer * p.q_layer + row * p.q_head : g < 0 ? nk + layer * p.k_layer + h * p.k_head
                                                                                          : nv + layer * p.v_layer + g * p.v_head;
        x[i] = src[0];
        y[i] = src[dv];
        turn[i] = g < 0 && tok.rotates;
        if (h < 0) to[i] = o + layer * p.o_layer + row * p.o_head;
        else if (tok.stored) to[i] = (g < 0 ? p.k + h * p.s_head : p.v + g * p.s_head) + (dst + layer * p.s_layer);
      }
      row += ROWS;
      wrap();
    }
#pragma unroll
    for (int i = 0; i < kRopeLayerBatch; ++i) {
      if (to[i]) {
        if (turn[i]) turn_pairs<INTER>(x[i], y[i], tok.c, tok.s);
        to[i][0] = x[i];
        to[i][dv] = y[i];
      }
    }
  }
}

// ONE: the launch is one CTA, or one cluster, which also counts the new tokens
template <int D, bool INTER, bool ONE, bool LAYERS = false>
__global__ void __launch_bounds__(ONE ? kRopeOneThreads : kRopeThreads, ONE ? 1 : kRopeCtas) rope_append_kernel(const __grid_constant__ RopeParams p, uint32_t n_warps) {
  __shared__ __align__(16) float cs_sm[(ONE ? kRopeOneThreads : kRopeThreads) / 32][D];   // cosines and sines of a warp's token
  pdl_launch_next();
  pdl_wait();
  const uint32_t warp = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  if (warp < n_warps) {
    if constexpr (LAYERS) rope_layers<D, INTER>(p, cs_sm[threadIdx.x >> 5], warp, threadIdx.x & 31);
    else rope_rows<D, INTER>(p, cs_sm[threadIdx.x >> 5], warp, threadIdx.x & 31);
  }
  if constexpr (ONE) {
    if (gridDim.x > 1) cluster_barrier();          // every thread has read the lengths
    else __syncthreads();
    if (blockIdx.x == 0)
      for (int b = threadIdx.x; b < p.batch; b += blockDim.x) rope_count(p, b);
  }
}

__global__ void rope_count_kernel(const __grid_constant__ RopeParams p) {
  pdl_launch_next();
  pdl_wait();
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b < p.batch) rope_count(p, b);
}

static bool rows_ok(const specvlm_rows_t* r) {
  return aligned16(r->p) && r->stride_layer % 8 == 0 && r->stride_batch % 8 == 0 && r->stride_token % 8 == 0 && r->stride_head % 8 == 0;
}

template <int D, bool INTER>
static int32_t launch_rope(const RopeParams& p, uint32_t n_warps, int one_warps, cudaStream_t st) {
  if (n_warps <= (uint32_t)one_warps) {
    int ctas = 1;
    while (ctas * (kRopeOneThreads / 32) < (int)n_warps) ctas *= 2;
    return launch_clusters_after(rope_append_kernel<D, INTER, true>, dim3(ctas), ctas, dim3(ctas > 1 ? kRopeOneThreads : 32 * n_warps), 0, st, p,
                                 n_warps);
  }
  const uint32_t blocks = (n_warps + kRopeThreads / 32 - 1) / (kRopeThreads / 32);
  const int32_t rc = launch_after(p.per_warp > 0 ? rope_append_kernel<D, INTER, false, true> : rope_append_kernel<D, INTER, false>,
                                  dim3(blocks), dim3(kRopeThreads), 0, st, p, n_warps);
  if (rc != SPECVLM_OK || p.counted) return rc;
  return launch_after(rope_count_kernel, dim3((unsigned)((p.batch + 127) / 128)), dim3(128), 0, st, p);
}

}  // namespace specvlm

using namespace specvlm;

extern "C" int32_t specvlm_rope_turns(const double* frequencies, int32_t n, uint64_t* turns) {
  if (!frequencies || !turns || n < 1) return SPECVLM_ERR_INVALID_ARG;
  for (int32_t i = 0; i < n; ++i)
    if (!isfinite(frequencies[i])) return SPECVLM_ERR_INVALID_ARG;
  const long double two_pi = 6.283185307179586476925286766559005768L;
  for (int32_t i = 0; i < n; ++i) {
    long double x = (long double)frequencies[i] / two_pi;
    x = (x - floorl(x)) * 18446744073709551616.0L;           // 2^64
    turns[i] = x < 18446744073709551615.0L ? (uint64_t)(x + 0.5L) : 0;      // (rounded up to a whole turn)
  }
  return SPECVLM_OK;
}

extern "C" int32_t specvlm_rope_frequencies(int32_t scaling, int32_t rot_dim, double base, double scale, double context,
                                            double low, double high, double* frequencies) {
  if (!frequencies || rot_dim < 4 || rot_dim % 2 != 0 || !(base > 1.0) || !isfinite(base)) return SPECVLM_ERR_INVALID_ARG;
  if (scaling < SPECVLM_ROPE_PLAIN || scaling > SPECVLM_ROPE_BANDS) return SPECVLM_ERR_INVALID_ARG;
  if (scaling != SPECVLM_ROPE_PLAIN && !(scale > 0.0 && isfinite(scale))) return SPECVLM_ERR_INVALID_ARG;
  const bool bands = scaling == SPECVLM_ROPE_RAMP || scaling == SPECVLM_ROPE_BANDS;
  if (bands && !(context > 0.0 && low > 0.0 && high > low && isfinite(context) && isfinite(high))) return SPECVLM_ERR_INVALID_ARG;
  const double two_pi = 6.283185307179586477;
  if (scaling == SPECVLM_ROPE_BASE) base *= pow(scale, (double)rot_dim / (rot_dim - 2));
  // the pair, as a real number, that makes `turns` turns within the trained context
  auto pair_of = [&](double turns) { return rot_dim * log(context / (turns * two_pi)) / (2.0 * log(base)); };
  double from = 0.0, to = 0.0;
  if (scaling == SPECVLM_ROPE_RAMP) {
    from = fmax(floor(pair_of(high)), 0.0);
    to = fmin(ceil(pair_of(low)), rot_dim - 1.0);
    if (to <= from) to = from + 0.001;
  }
  for (int32_t i = 0; i < rot_dim / 2; ++i) {
    const double f = pow(base, -2.0 * i / rot_dim);
    double slow = 0.0;                                       // share of the divided frequency
    if (scaling == SPECVLM_ROPE_LINEAR) slow = 1.0;
    if (scaling == SPECVLM_ROPE_RAMP) slow = fmin(fmax((i - from) / (to - from), 0.0), 1.0);
    if (scaling == SPECVLM_ROPE_BANDS) slow = fmin(fmax((high - context * f / two_pi) / (high - low), 0.0), 1.0);
    frequencies[i] = slow > 0.0 ? f * (1.0 - slow) + f / scale * slow : f;
  }
  return SPECVLM_OK;
}

extern "C" int32_t specvlm_rope_append_kv(const specvlm_kv_t* kv, const specvlm_rope_t* rope, const specvlm_rows_t* q,
                                          const specvlm_rows_t* q_out, const specvlm_rows_t* new_k,
                                          const specvlm_rows_t* new_v, int32_t batch, int32_t n_new, int32_t n_q_heads,
                                          const int32_t* positions_or_null, const int32_t* new_lens_or_null,
                                          int32_t* seq_lens_inout, int32_t counted, int32_t* d_status, void* stream) {
  NvtxRange nvtx_range(__func__);
  if (!kv || !rope || !new_k || !new_v || !new_k->p || !new_v->p || !seq_lens_inout || n_new < 1 || n_q_heads < 0)
    return SPECVLM_ERR_INVALID_ARG;
  const bool has_q = q && q->p;
  if (has_q != (q_out && q_out->p) || has_q != (n_q_heads > 0)) return SPECVLM_ERR_INVALID_ARG;
  specvlm_kv_t c = *kv;
  c.seq_lens = seq_lens_inout;
  const int32_t rc = validate_kv(&c, batch, true);
  if (rc != SPECVLM_OK) return rc;
  if (n_new > c.max_seq_len || !rope->turns || !aligned16(rope->turns) || rope->n_axes < 1 || rope->n_axes > 3) return SPECVLM_ERR_INVALID_ARG;
  if (rope->rot_dim < 16 || rope->rot_dim > c.head_dim || rope->rot_dim % 16 != 0) return SPECVLM_ERR_UNSUPPORTED_SHAPE;
  if (!isfinite(rope->factor)) return SPECVLM_ERR_INVALID_ARG;
  int64_t pairs = 0;
  for (int a = 0; a < rope->n_axes && rope->n_axes > 1; ++a) {
    if (rope->sections[a] < 0) return SPECVLM_ERR_INVALID_ARG;
    pairs += rope->sections[a];
  }
  if (rope->n_axes > 1 && pairs != rope->rot_dim / 2) return SPECVLM_ERR_INVALID_ARG;
  if (!rows_ok(new_k) || !rows_ok(new_v) || (has_q && (!rows_ok(q) || !rows_ok(q_out)))) return SPECVLM_ERR_INVALID_ARG;
  const specvlm_rows_t none = {};
  const specvlm_rows_t& qr = has_q ? *q : none;
  const specvlm_rows_t& qo = has_q ? *q_out : none;
  RopeParams p;
  p.q = static_cast<const uint4*>(qr.p);
  p.q_out = static_cast<uint4*>(qo.p);
  p.new_k = static_cast<const uint4*>(new_k->p);
  p.new_v = static_cast<const uint4*>(new_v->p);
  p.k = static_cast<uint4*>(c.k);
  p.v = static_cast<uint4*>(c.v);
  p.turns = rope->turns;
  p.positions = positions_or_null;
  p.new_lens = new_lens_or_null;
  p.seq_lens = seq_lens_inout;
  p.table = c.block_table;
  p.d_status = d_status;
  p.q_layer = qr.stride_layer / 8; p.q_batch = qr.stride_batch / 8; p.q_token = qr.stride_token / 8; p.q_head = qr.stride_head / 8;
  p.o_layer = qo.stride_layer / 8; p.o_batch = qo.stride_batch / 8; p.o_token = qo.stride_token / 8; p.o_head = qo.stride_head / 8;
  p.k_layer = new_k->stride_layer / 8; p.k_batch = new_k->stride_batch / 8; p.k_token = new_k->stride_token / 8;
  p.k_head = new_k->stride_head / 8;
  p.v_layer = new_v->stride_layer / 8; p.v_batch = new_v->stride_batch / 8; p.v_token = new_v->stride_token / 8;
  p.v_head = new_v->stride_head / 8;
  p.s_layer = c.stride_layer / 8; p.s_block = c.stride_block / 8; p.s_head = c.stride_head / 8; p.s_token = c.stride_token / 8;
  p.block_tokens = c.block_tokens; p.max_blocks = c.max_blocks; p.max_seq_len = c.max_seq_len; p.n_blocks = c.n_blocks;
  p.n_layers = c.n_layers; p.batch = batch; p.n_new = n_new; p.n_q_heads = n_q_heads; p.n_kv_heads = c.n_kv_heads;
  p.n_rot = rope->rot_dim / 16;
  p.n_axes = rope->n_axes;
  p.axis1 = rope->n_axes > 1 ? rope->sections[0] : rope->rot_dim;
  p.axis2 = rope->n_axes > 1 ? rope->sections[0] + rope->sections[1] : rope->rot_dim;
  p.counted = counted ? 1 : 0;
  p.factor = rope->factor;
  const int64_t sequences = (int64_t)c.n_layers * batch;
  if (sequences > 0x3fffffff) return SPECVLM_ERR_UNSUPPORTED_SHAPE;      // (before the product, which may leave 64 bits)
  const int64_t tokens = sequences * n_new;
  const int64_t rows = 32 / (c.head_dim / 16);
  if (tokens > 0x3fffffff || n_q_heads > 65535 || c.n_kv_heads > 65535) return SPECVLM_ERR_UNSUPPORTED_SHAPE;
  // a token's rows go to as many warps as it takes to occupy the SMs, up to a round each
  const int64_t rounds = (n_q_heads + rows - 1) / rows + (2 * c.n_kv_heads + rows - 1) / rows, wanted = (int64_t)sm_count() * kRopeWarps;
  int64_t share = (wanted + tokens - 1) / tokens;
  p.share = (int32_t)(share < rounds ? share : rounds);
  // Few tokens that have to be counted: one CTA or one cluster, which spares the second launch.  17 layers x 6 tokens of 8 + 2 heads, passes
  // one after the other 11.4 -> 9.5 us, of which 4 are the call; on the device a cluster takes 0.5 us more than two launches, so in a graph,
  // whose launches cost the host nothing, it is one CTA or none.
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int one_warps = !counted && tokens <= kRopeOneTokens ? kRopeOneThreads / 32 : 0;
  if (!counted && one_warps == 0 && tokens <= kRopeOneWarps && rounds <= kRopeOneRounds * (kRopeOneWarps / tokens) && !being_captured(st))
    one_warps = kRopeOneWarps;
  if (one_warps > 0 && p.share > one_warps / tokens) p.share = (int32_t)(one_warps / tokens);
  // Many tokens of few rows: a warp takes as many layers as leave four times the warps that the SMs hold (rope_layers; with one
  // layer a warp it still gains, as key and value rows share the queries' rounds).  8 + 2 heads of d = 64, 25 layers of 8723
  // tokens 168 -> 135 us, one of 32 000 27.5 -> 25.6; 4 + 1 heads 28 layers of 8000 163 -> 70, one of 32 000 25.8 -> 21.3.
  const int64_t layers = rounds <= kRopeLayerRounds ? tokens / ((int64_t)sm_count() * kRopeManyWarps) : 0;
  p.per_warp = (int32_t)(layers < c.n_layers ? layers : c.n_layers);
  const uint32_t n_warps = p.per_warp > 0 ? (uint32_t)((c.n_layers + p.per_warp - 1) / p.per_warp * ((int64_t)batch * n_new))
                                          : (uint32_t)(tokens * p.share);   // < 2^31: more than a warp a token only for few tokens
  if (c.head_dim == 128)
    return rope->interleaved ? launch_rope<128, true>(p, n_warps, one_warps, st) : launch_rope<128, false>(p, n_warps, one_warps, st);
  return rope->interleaved ? launch_rope<64, true>(p, n_warps, one_warps, st) : launch_rope<64, false>(p, n_warps, one_warps, st);
}
