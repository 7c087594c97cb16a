// Rotary positions of new tokens' queries and keys, fused with the append of keys and values to the cache.
//
// Every row is read once and written once; per 16 channels there are 8 pairs to turn, 24 multiply-adds, against 64 bytes of
// traffic.  A warp works on one token of one layer and walks its rows (query heads, key heads, value heads), a thread on
// the same 16 channels of each, so that the 8 sines and cosines of a thread serve all of them.
//
// Angles: a position times a frequency in radians loses the angle's digits to the whole turns (position 50 000 in fp32: 2e-3
// radians).  Here frequencies are fractions of a turn in 64-bit fixed point, and position * fraction modulo 2^64 is the exact
// fraction of the angle; its upper 32 bits go to fp32 (2^-25 of a turn at most).
//
// Lengths and block tables are device data: checked before they become part of an address (see cache.cu).
#include <math.h>

#include "common.cuh"
#include "host_util.h"

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
  float factor;
};

// First cache position and number of a sequence's new tokens; false if it is to be left alone.
__device__ __forceinline__ bool rope_range(const RopeParams& p, int b, int& start, int& n) {
  n = p.new_lens ? p.new_lens[b] : p.n_new;
  const int len = p.seq_lens[b];
  if (n < 0 || n > p.n_new || len < 0 || len > p.max_seq_len) return false;
  start = p.counted ? len - n : len;
  return start >= 0 && n <= p.max_seq_len - start;
}

__device__ __forceinline__ float2 bf16x2_to_f2(uint32_t x) {
  return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}

// The 8 pairs of two 16-byte vectors: the e-th channels of both (half layout), or neighbours (interleaved).
template <bool INTER>
__device__ __forceinline__ void turn_pairs(uint4& x, uint4& y, const float (&c)[8], const float (&s)[8]) {
  uint32_t* const xw = reinterpret_cast<uint32_t*>(&x);
  uint32_t* const yw = reinterpret_cast<uint32_t*>(&y);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float2 a = bf16x2_to_f2(xw[w]), b = bf16x2_to_f2(yw[w]);
    if constexpr (INTER) {
      xw[w] = pack_bf16x2(a.x * c[w] - a.y * s[w], a.y * c[w] + a.x * s[w]);
      yw[w] = pack_bf16x2(b.x * c[w + 4] - b.y * s[w + 4], b.y * c[w + 4] + b.x * s[w + 4]);
    } else {
      xw[w] = pack_bf16x2(a.x * c[2 * w] - b.x * s[2 * w], a.y * c[2 * w + 1] - b.y * s[2 * w + 1]);
      yw[w] = pack_bf16x2(b.x * c[2 * w] + a.x * s[2 * w], b.y * c[2 * w + 1] + a.y * s[2 * w + 1]);
    }
  }
}

constexpr int kRopeThreads = 256, kRopeOneThreads = 1024, kRopeOneTokens = 8;

template <int D, bool INTER>
__device__ __forceinline__ void rope_rows(const RopeParams& p, uint32_t warp, int lane) {
  constexpr int UNITS = D / 16, ROWS = 32 / UNITS;  // threads of a row, rows of a warp's round
  const uint32_t token = warp / (uint32_t)p.share, lb = token / (uint32_t)p.n_new;
  const int part = (int)(warp - token * p.share), t = (int)(token - lb * p.n_new);
  const int layer = (int)(lb / (uint32_t)p.batch), b = (int)(lb - (uint32_t)layer * p.batch);
  const int u = lane % UNITS;
  const bool rotates = u < p.n_rot;
  const int v0 = !INTER && rotates ? u : 2 * u, v1 = !INTER && rotates ? u + p.n_rot : 2 * u + 1;   // this thread's vectors
  const int n_rows = p.n_q_heads + 2 * p.n_kv_heads, step = ROWS * p.share;

  int start, n;
  const bool ok = rope_range(p, b, start, n);
  if (!ok) {
    if (lane == 0 && p.d_status) *p.d_status = SPECVLM_ERR_INVALID_ARG;
    return;
  }
  if (t >= n) return;
  float c[8], s[8];
  if (rotates) {
    int pos[3] = {start + t, start + t, start + t};
    if (p.positions) {
#pragma unroll
      for (int a = 0; a < 3; ++a)
        if (a < p.n_axes) pos[a] = p.positions[((size_t)a * p.batch + b) * p.n_new + t];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = 8 * u + e;
      const int at = p.n_axes == 1 || i < p.axis1 ? pos[0] : i < p.axis2 ? pos[1] : pos[2];
      const uint64_t turn = (uint64_t)(int64_t)at * p.turns[i];
      sincospif((float)(int32_t)(turn >> 32) * 4.656612873077393e-10f, &s[e], &c[e]);    // 2^-31: half turns
      s[e] *= p.factor;
      c[e] *= p.factor;
    }
  }
  const int at = start + t;
  int blk = b, off = at;
  bool stored = true;
  if (p.table) {
    blk = p.table[(size_t)b * p.max_blocks + at / p.block_tokens];
    off = at % p.block_tokens;
    stored = blk >= 0 && blk < p.n_blocks;
    if (!stored && lane == 0 && p.d_status) *p.d_status = SPECVLM_ERR_INVALID_ARG;
  }
  const int64_t dst = layer * p.s_layer + blk * p.s_block + off * p.s_token;
  const uint4* const q = p.q + layer * p.q_layer + b * p.q_batch + t * p.q_token;
  uint4* const o = p.q_out + layer * p.o_layer + b * p.o_batch + t * p.o_token;
  const uint4* const nk = p.new_k + layer * p.k_layer + b * p.k_batch + t * p.k_token;
  const uint4* const nv = p.new_v + layer * p.v_layer + b * p.v_batch + t * p.v_token;
#pragma unroll 4
  for (int row = part * ROWS + lane / UNITS; row < n_rows; row += step) {
    const int h = row - p.n_q_heads, g = h - p.n_kv_heads;
    const uint4* src = h < 0 ? q + row * p.q_head : g < 0 ? nk + h * p.k_head : nv + g * p.v_head;
    uint4* to = h < 0 ? o + row * p.o_head : g < 0 ? p.k + dst + h * p.s_head : p.v + dst + g * p.s_head;
    uint4 x = src[v0], y = src[v1];
    if (rotates && g < 0) turn_pairs<INTER>(x, y, c, s);
    if (h < 0 || stored) {
      to[v0] = x;
      to[v1] = y;
    }
  }
}

// ONE: the only CTA of the launch, which also counts the new tokens
template <int D, bool INTER, bool ONE>
__global__ void __launch_bounds__(ONE ? kRopeOneThreads : kRopeThreads) rope_append_kernel(const __grid_constant__ RopeParams p, uint32_t n_warps) {
  pdl_launch_next();
  pdl_wait();
  const uint32_t warp = blockIdx.x * (kRopeThreads / 32) + (threadIdx.x >> 5);
  if (warp < n_warps) rope_rows<D, INTER>(p, warp, threadIdx.x & 31);
  if constexpr (ONE) {
    __syncthreads();                               // every thread has read the lengths
    for (int b = threadIdx.x; b < p.batch; b += blockDim.x) {
      int start, n;
      if (rope_range(p, b, start, n)) p.seq_lens[b] = start + n;
    }
  }
}

__global__ void rope_count_kernel(const __grid_constant__ RopeParams p) {
  pdl_launch_next();
  pdl_wait();
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  int start, n;
  if (b < p.batch && rope_range(p, b, start, n)) p.seq_lens[b] = start + n;   // the append has reported the others
}

static bool rows_ok(const specvlm_rows_t* r) {
  return aligned16(r->p) && r->stride_layer % 8 == 0 && r->stride_batch % 8 == 0 && r->stride_token % 8 == 0 && r->stride_head % 8 == 0;
}

template <int D, bool INTER>
static int32_t launch_rope(const RopeParams& p, uint32_t n_warps, cudaStream_t st) {
  if (!p.counted && n_warps <= kRopeOneThreads / 32)
    return launch_after(rope_append_kernel<D, INTER, true>, dim3(1), dim3(32 * n_warps), 0, st, p, n_warps);
  const uint32_t blocks = (n_warps + kRopeThreads / 32 - 1) / (kRopeThreads / 32);
  const int32_t rc = launch_after(rope_append_kernel<D, INTER, false>, dim3(blocks), dim3(kRopeThreads), 0, st, p, n_warps);
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
  if (n_new > c.max_seq_len || !rope->turns || rope->n_axes < 1 || rope->n_axes > 3) return SPECVLM_ERR_INVALID_ARG;
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
  p.axis1 = rope->n_axes > 1 ? rope->sections[0] : 0;
  p.axis2 = rope->n_axes > 1 ? rope->sections[0] + rope->sections[1] : 0;
  p.counted = counted ? 1 : 0;
  p.factor = rope->factor;
  const int64_t tokens = (int64_t)c.n_layers * batch * n_new;
  const int64_t n_rows = (int64_t)n_q_heads + 2 * (int64_t)c.n_kv_heads, rows = 32 / (c.head_dim / 16);
  if (tokens > 0x3fffffff || n_rows > 65535) return SPECVLM_ERR_UNSUPPORTED_SHAPE;
  // a token's rows go to as many warps as it takes to occupy the SMs, up to a round each
  const int64_t rounds = (n_rows + rows - 1) / rows, wanted = (int64_t)sm_count() * 32;
  int64_t share = (wanted + tokens - 1) / tokens;
  p.share = (int32_t)(share < rounds ? share : rounds);
  // few tokens that have to be counted: one CTA, which spares the second launch
  if (!counted && tokens <= kRopeOneTokens && p.share > kRopeOneThreads / 32 / tokens) p.share = (int32_t)(kRopeOneThreads / 32 / tokens);
  const uint32_t n_warps = (uint32_t)(tokens * p.share);   // < 2^31: more than a warp a token only for few tokens
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (c.head_dim == 128)
    return rope->interleaved ? launch_rope<128, true>(p, n_warps, st) : launch_rope<128, false>(p, n_warps, st);
  return rope->interleaved ? launch_rope<64, true>(p, n_warps, st) : launch_rope<64, false>(p, n_warps, st);
}
