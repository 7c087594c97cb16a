// Pages of a paged cache: reserving, releasing, forking, compacting.
//
// The pool's state is one count a page (0: free).  Planning is integer work on that array and the block tables: reserving
// and compacting need running sums over it in page order (so that the free pages are handed out lowest first, whatever the
// timing), which one CTA computes; releasing and forking change counts by atomic additions of integers, whose order
// does not matter.  The K/V rows move in a second kernel over the whole chip, from a list that the first one leaves.
// A plan is a chain of round trips to memory (lengths, entries, counts, the free pages) and of three or four running sums over
// 1024 threads, 4 to 5 us for pools of up to 16 384 pages; the launches around it cost the host more.
//
// Lengths and table entries are device data: checked before they become part of an address (see cache.cu).  An entry outside
// the pool is an unmapped one.
#include "common.cuh"
#include "host_util.h"

namespace specvlm {

constexpr int kPagesMaxBatch = 1024;
constexpr int kPlanThreads = 1024;
constexpr int kPagesPerThread = 16;                            // counts that a planning thread holds in a round
constexpr int32_t kPagesMost = 0x3fffffff;                     // pages of a pool: the rounds' ends stay within 32 bits

struct PagesParams {
  uint4* k;
  uint4* v;
  int32_t* table;              // [B][max_blocks]
  int32_t* ref;                // [n_blocks]
  const int32_t* seq_lens;
  const int32_t* new_lens;     // or null
  int32_t* d_status;
  int32_t* n_used;             // or null
  int32_t* n_copies;           // scratch: copies in the list
  int4* copies;                // scratch: (source page, destination page, rows, -)
  int32_t* list;               // scratch [n_blocks]: free pages to hand out; compaction: holes
  int32_t* dest;               // scratch [n_blocks]: new place of a page that moves
  int32_t* order;              // scratch [batch * max_blocks]: which of the fresh pages a slot gets, -1: none
  int64_t s_layer, s_block, s_head, s_token;                   // strides in 16-byte units
  int32_t block_tokens, max_blocks, max_seq_len, n_blocks;
  int32_t n_layers, n_kv_heads, chunk_bits;                    // 2^chunk_bits 16-byte chunks a row
  int32_t batch, n_new;
};

// Running sum over the CTA (kPlanThreads threads): the sum before this thread; total: of all.
__device__ __forceinline__ int block_scan(int v, int* warp_sums, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, x, off);
    if (lane >= off) x += o;
  }
  __syncthreads();                                             // the sums of the round before have been read
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  int s = warp_sums[lane];
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, s, off);
    if (lane >= off) s += o;
  }
  total = __shfl_sync(0xffffffffu, s, 31);
  const int before = __shfl_sync(0xffffffffu, s, warp > 0 ? warp - 1 : 0);
  return x - v + (warp > 0 ? before : 0);
}

__device__ __forceinline__ void load_counts(const int32_t* ref, int base, int n, int (&c)[kPagesPerThread], int beyond) {
  if (base + kPagesPerThread <= n && (reinterpret_cast<uintptr_t>(ref) & 15) == 0) {
#pragma unroll
    for (int i = 0; i < kPagesPerThread; i += 4) {
      const int4 x = *reinterpret_cast<const int4*>(ref + base + i);
      c[i] = x.x; c[i + 1] = x.y; c[i + 2] = x.z; c[i + 3] = x.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPagesPerThread; ++i) c[i] = base + i < n ? ref[base + i] : beyond;
  }
}

// ------------------------------------------------------------------------------ reserve
// A "slot" is an entry of a table's row that the new tokens fall on.
struct ReservePlan {
  int warp_sums[32];
  int begun[kPagesMaxBatch];          // the page that the sequence's next row falls on, if it has rows on it already; else -1
  int first[kPagesMaxBatch];          // its slot
  int before[kPagesMaxBatch + 1];     // slots of the sequences before
  uint8_t copied[kPagesMaxBatch];     // the begun page is replaced by a copy
  int list[kPlanThreads];             // the free pages to hand out, where a round of slots is all there is
};

// By one CTA; the number of copies that it leaves in the list.
__device__ __forceinline__ int reserve_plan(const PagesParams& p, ReservePlan& sm) {
  const int tid = threadIdx.x;
  int c[kPagesPerThread];                                      // the first round's counts, asked for before all else
  load_counts(p.ref, tid * kPagesPerThread, p.n_blocks, c, 1);
  // the sequences' slots
  int n_slots = 0, page = -1, rows = 0;
  if (tid < p.batch) {
    const int len = p.seq_lens[tid], n = p.new_lens ? p.new_lens[tid] : p.n_new;
    if (len < 0 || n < 0 || len > p.max_seq_len || n > p.max_seq_len - len) {
      if (p.d_status) *p.d_status = SPECVLM_ERR_INVALID_ARG;
    } else if (n > 0) {
      const int first = len / p.block_tokens;
      n_slots = (len + n - 1) / p.block_tokens - first + 1;
      rows = len - first * p.block_tokens;
      if (rows > 0) page = p.table[(size_t)tid * p.max_blocks + first];
      if (page < 0 || page >= p.n_blocks) page = -1;
      sm.first[tid] = first;
    }
    sm.begun[tid] = page;
  }
  int total_slots;
  const int before = block_scan(n_slots, sm.warp_sums, total_slots);
  if (tid < p.batch) sm.before[tid] = before;
  if (tid == 0) sm.before[p.batch] = total_slots;
  __syncthreads();
  // a begun page that somebody else holds too is copied, but by the last of its holders here
  bool copied = false;
  if (page >= 0) {
    int held = p.ref[page];
    for (int b = 0; held > 1 && b < tid; ++b) held -= sm.begun[b] == page;
    copied = held > 1;
  }
  if (tid < p.batch) sm.copied[tid] = copied;
  __syncthreads();

  // Slot i's sequence, entry and page (-1: none), and whether it needs a fresh one
  auto look = [&](int i, int& b, int& j, int& old) {
    int lo = 0, hi = p.batch - 1;                              // last b with before[b] <= i: sequences without slots share their
    while (lo < hi) {                                          // successor's number, so it is one that has some
      const int mid = (lo + hi + 1) >> 1;
      if (sm.before[mid] <= i) lo = mid; else hi = mid - 1;
    }
    b = lo;
    j = sm.first[lo] + i - sm.before[lo];
    old = p.table[(size_t)b * p.max_blocks + j];
    if (old < 0 || old >= p.n_blocks) old = -1;
  };
  const bool one_round = total_slots <= kPlanThreads;
  int32_t* const list = one_round ? sm.list : p.list;
  int total = 0, b = 0, j = 0, old = -1, nth = -1, copy_at = 0, n_copies = 0;
  for (int i0 = 0; i0 < total_slots; i0 += kPlanThreads) {
    const int i = i0 + tid;
    bool fresh = false;
    if (i < total_slots) {
      look(i, b, j, old);
      fresh = old < 0 || (j == sm.first[b] && sm.begun[b] >= 0 ? sm.copied[b] != 0 : p.ref[old] > 1);
    }
    // slots in the lower half; in the upper one the copies, whose list is in the order of the sequences
    int here;
    const int at = block_scan((fresh ? 1 : 0) + (i0 == 0 && copied ? 0x10000 : 0), sm.warp_sums, here);
    nth = fresh ? total + (at & 0xffff) : -1;
    if (!one_round && i < total_slots) p.order[i] = nth;
    total += here & 0xffff;
    if (i0 == 0) {
      copy_at = at >> 16;
      n_copies = here >> 16;
    }
  }
  // the lowest free pages, as many as are needed
  int found = 0;
  for (int base0 = 0; base0 < p.n_blocks && found < total; base0 += kPlanThreads * kPagesPerThread) {
    const int base = base0 + tid * kPagesPerThread;
    if (base0 > 0) load_counts(p.ref, base, p.n_blocks, c, 1);
    int n = 0;
#pragma unroll
    for (int i = 0; i < kPagesPerThread; ++i) n += c[i] == 0;
    int here;
    int at = found + block_scan(n, sm.warp_sums, here);
#pragma unroll
    for (int i = 0; i < kPagesPerThread; ++i)
      if (c[i] == 0) {
        if (at < total) list[at] = base + i;
        ++at;
      }
    found += here;
  }
  __syncthreads();                                             // the list is complete, and every count has been read
  if (found < total) {
    if (tid == 0 && p.d_status) *p.d_status = SPECVLM_ERR_NO_PAGES;
    return 0;
  }
  // hand them out, in the order of the slots
  for (int i0 = 0; i0 < total_slots; i0 += kPlanThreads) {
    const int i = i0 + tid;
    if (!one_round && i < total_slots) {
      look(i, b, j, old);
      nth = p.order[i];
    }
    if (i < total_slots && nth >= 0) {
      const int fresh = list[nth];
      p.table[(size_t)b * p.max_blocks + j] = fresh;
      p.ref[fresh] = 1;
      if (old >= 0) atomicSub(p.ref + old, 1);
      if (j == sm.first[b] && sm.begun[b] >= 0) sm.begun[b] = ~fresh;    // its copy's destination, for the thread of the sequence
    }
  }
  __syncthreads();
  if (copied) p.copies[copy_at] = make_int4(page, ~sm.begun[tid], rows, 0);
  return n_copies;
}

// The copies of a plan's list: a unit is a page of one layer and head, K and V.  The rows are read once and written once:
// eight 16-byte loads a thread in flight.
constexpr int kCopyThreads = 256;
template <int THREADS>
__device__ __forceinline__ void copy_pages(const PagesParams& p, int n_copies) {
  const int lh = p.n_layers * p.n_kv_heads;
  const int64_t n_units = (int64_t)n_copies * lh;
  // (a larger CTA is as many copying ones; its list is from another CTA of the same launch, and not read through the L1 cache)
  constexpr bool kSame = THREADS == kCopyThreads;
  const int cta = kSame ? blockIdx.x : blockIdx.x * (THREADS / kCopyThreads) + threadIdx.x / kCopyThreads;
  const int tid = kSame ? threadIdx.x : threadIdx.x % kCopyThreads;
  for (int64_t unit = cta; unit < n_units; unit += gridDim.x * (THREADS / kCopyThreads)) {
    const int nth = (int)(unit / lh), x = (int)(unit - (int64_t)nth * lh), layer = x / p.n_kv_heads, head = x - layer * p.n_kv_heads;
    const int4 c = kSame ? p.copies[nth] : __ldcg(p.copies + nth);
    const int64_t at = layer * p.s_layer + head * p.s_head, src = at + c.x * p.s_block, dst = at + c.y * p.s_block;
    const int n = c.z << p.chunk_bits, mask = (1 << p.chunk_bits) - 1;
    for (int i0 = tid; i0 < n; i0 += 4 * kCopyThreads) {
      uint4 k[4], v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * kCopyThreads;
        const int64_t off = (i >> p.chunk_bits) * p.s_token + (i & mask);
        if (i < n) {
          k[u] = p.k[src + off];
          v[u] = p.v[src + off];
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * kCopyThreads;
        const int64_t off = (i >> p.chunk_bits) * p.s_token + (i & mask);
        if (i < n) {
          p.k[dst + off] = k[u];
          p.v[dst + off] = v[u];
        }
      }
    }
  }
}

__global__ void __launch_bounds__(kCopyThreads) copy_pages_kernel(const __grid_constant__ PagesParams p) {
  pdl_launch_next();
  pdl_wait();
  copy_pages<kCopyThreads>(p, *p.n_copies);
}

__global__ void __launch_bounds__(kPlanThreads) reserve_plan_kernel(const __grid_constant__ PagesParams p) {
  __shared__ ReservePlan sm;
  pdl_launch_next();
  pdl_wait();
  const int n_copies = reserve_plan(p, sm);
  if (threadIdx.x == 0) *p.n_copies = n_copies;
}

// Plan and copies in one launch of a cluster, which spares the host 2 us: where the copies, of which there are seldom any, are
// small enough for the cluster's SMs.
// 64 sequences on 16 384 pages 6.1 -> 3.7 us of the host's time, as long on the device.
constexpr int kReserveCluster = 8;
constexpr double kReserveClusterBytes = 4 << 20;
__global__ void __launch_bounds__(kPlanThreads) reserve_cluster_kernel(const __grid_constant__ PagesParams p) {
  __shared__ ReservePlan sm;
  pdl_launch_next();
  pdl_wait();
  if (blockIdx.x == 0) {
    const int n_copies = reserve_plan(p, sm);
    if (threadIdx.x == 0) *p.n_copies = n_copies;
  }
  cluster_barrier();
  copy_pages<kPlanThreads>(p, __ldcg(p.n_copies));
}

// ------------------------------------------------------------------------------ release
__global__ void __launch_bounds__(256) release_pages_kernel(const __grid_constant__ PagesParams p, int window, int n_sinks) {
  pdl_launch_next();
  pdl_wait();
  const int b = blockIdx.y, j = blockIdx.x * 256 + threadIdx.x;
  if (j >= p.max_blocks) return;
  const int len = p.seq_lens[b];
  if (len < 0 || len > p.max_seq_len) {
    if (p.d_status) *p.d_status = SPECVLM_ERR_INVALID_ARG;
    return;
  }
  const int64_t begin = (int64_t)j * p.block_tokens, end = begin + p.block_tokens;
  if (begin < len && (begin < n_sinks || end > (int64_t)len - window)) return;
  int32_t* const entry = p.table + (size_t)b * p.max_blocks + j;
  const int page = *entry;
  if (page >= 0 && page < p.n_blocks) atomicSub(p.ref + page, 1);
  *entry = -1;
}

// ------------------------------------------------------------------------------ fork
// One CTA per old row, which changes the counts of its pages, and one per new row, which takes over the entries.
__global__ void __launch_bounds__(256) fork_pages_kernel(const __grid_constant__ PagesParams p, const int32_t* parents, int batch_out,
                                                         int32_t* table_out, int32_t* lens_out) {
  pdl_launch_next();
  pdl_wait();
  const bool is_new = (int)blockIdx.x >= p.batch;
  const int row = is_new ? blockIdx.x - p.batch : blockIdx.x;
  int from = row, change = -1;
  if (is_new) {
    from = parents[row];
    if (from < -1 || from >= p.batch) {
      if (threadIdx.x == 0 && p.d_status) *p.d_status = SPECVLM_ERR_INVALID_ARG;
      from = -1;
    }
  } else {
    for (int i0 = 0; i0 < batch_out; i0 += 256) {
      const int i = i0 + threadIdx.x;
      change += __syncthreads_count(i < batch_out && parents[i] == row);
    }
  }
  int len = from >= 0 ? p.seq_lens[from] : 0;
  if (len < 0 || len > p.max_seq_len) {                        // as if it had no token
    if (threadIdx.x == 0 && p.d_status) *p.d_status = SPECVLM_ERR_INVALID_ARG;
    len = 0;
  }
  const int kept = (int)(((int64_t)len + p.block_tokens - 1) / p.block_tokens);
  const int32_t* const entries = p.table + (size_t)(from >= 0 ? from : 0) * p.max_blocks;
  for (int j = threadIdx.x; j < p.max_blocks; j += 256) {
    const int page = from >= 0 ? entries[j] : -1;
    const bool mapped = page >= 0 && page < p.n_blocks;
    if (is_new) {
      table_out[(size_t)row * p.max_blocks + j] = mapped && j < kept ? page : -1;
    } else if (mapped) {
      const int by = j < kept ? change : -1;
      if (by != 0) atomicAdd(p.ref + page, by);
    }
  }
  if (is_new && threadIdx.x == 0) lens_out[row] = len;
}

// ------------------------------------------------------------------------------ compact
__global__ void __launch_bounds__(kPlanThreads) compact_plan_kernel(const __grid_constant__ PagesParams p) {
  __shared__ int warp_sums[32];
  pdl_launch_next();
  pdl_wait();
  const int tid = threadIdx.x, round = kPlanThreads * kPagesPerThread;
  const bool one_round = p.n_blocks <= round;
  int c[kPagesPerThread];
  int n_used = 0;
  for (int base0 = 0; base0 < p.n_blocks; base0 += round) {
    load_counts(p.ref, base0 + tid * kPagesPerThread, p.n_blocks, c, 0);
    int n = 0, here;
#pragma unroll
    for (int i = 0; i < kPagesPerThread; ++i) n += c[i] > 0;
    block_scan(n, warp_sums, here);
    n_used += here;
  }
  // holes before page n_used and used pages behind it, both in page order: there are as many of the one as of the other
  int holes = 0, movers = 0;
  for (int base0 = 0; base0 < p.n_blocks; base0 += round) {
    const int base = base0 + tid * kPagesPerThread;
    if (!one_round) load_counts(p.ref, base, p.n_blocks, c, 0);
    int n_h = 0, n_m = 0;
#pragma unroll
    for (int i = 0; i < kPagesPerThread; ++i) {
      n_h += base + i < n_used && c[i] <= 0;
      n_m += base + i >= n_used && c[i] > 0;
    }
    int here_h, here_m;
    int at_h = holes + block_scan(n_h, warp_sums, here_h), at_m = movers + block_scan(n_m, warp_sums, here_m);
#pragma unroll
    for (int i = 0; i < kPagesPerThread; ++i) {
      if (base + i < n_used && c[i] <= 0) p.list[at_h++] = base + i;
      if (base + i >= n_used && c[i] > 0) p.copies[at_m++] = make_int4(base + i, 0, p.block_tokens, c[i]);
      if (base + i >= n_used && c[i] <= 0 && base + i < p.n_blocks) p.dest[base + i] = -1;
    }
    holes += here_h;
    movers += here_m;
  }
  __syncthreads();                                             // both lists are complete
  for (int m = tid; m < movers; m += kPlanThreads) {
    const int4 move = p.copies[m];
    const int to = p.list[m];
    p.copies[m].y = to;
    p.dest[move.x] = to;
    p.ref[to] = move.w;
    p.ref[move.x] = 0;
  }
  if (tid == 0) {
    *p.n_copies = movers;
    p.n_copies[1] = n_used;
    if (p.n_used) *p.n_used = n_used;
  }
}

__global__ void __launch_bounds__(kCopyThreads) compact_move_kernel(const __grid_constant__ PagesParams p) {
  pdl_launch_next();
  pdl_wait();
  const int n_moves = p.n_copies[0], n_used = p.n_copies[1];
  if (n_moves > 0) {
    const int64_t n = (int64_t)p.batch * p.max_blocks;
    for (int64_t i = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kCopyThreads) {
      const int page = p.table[i];
      if (page >= n_used && page < p.n_blocks) {
        const int to = p.dest[page];
        if (to >= 0) p.table[i] = to;                          // (else an entry of a page that nobody counts)
      }
    }
  }
  copy_pages<kCopyThreads>(p, n_moves);
}

// ------------------------------------------------------------------------------ host side
struct PagesScratch {
  size_t copies, list, dest, order, bytes;
  PagesScratch(const specvlm_kv_t* kv, int32_t batch) {
    const size_t n = (size_t)kv->n_blocks;
    copies = 256;
    list = copies + round_up(sizeof(int4) * (n > (size_t)batch ? n : (size_t)batch), 256);
    dest = list + round_up(4 * n, 256);
    order = dest + round_up(4 * n, 256);
    bytes = order + round_up(4 * (size_t)batch * kv->max_blocks, 256);
  }
};

static int32_t pages_params(PagesParams& p, const specvlm_kv_t* kv, int32_t* table, int32_t* ref, int32_t batch, void* ws,
                            size_t ws_bytes, bool needs_ws, int32_t* d_status) {
  if (!kv || !table || !ref) return SPECVLM_ERR_INVALID_ARG;
  specvlm_kv_t c = *kv;
  c.block_table = table;
  const int32_t rc = validate_kv(&c, batch, true);
  if (rc != SPECVLM_OK) return rc;
  if (batch > kPagesMaxBatch || (int64_t)c.n_layers * c.n_kv_heads > 0x7fffffff) return SPECVLM_ERR_UNSUPPORTED_SHAPE;
  if (c.block_tokens > (1 << 24) || (int64_t)c.max_blocks * batch > 0x3fffffff || c.n_blocks > kPagesMost) return SPECVLM_ERR_UNSUPPORTED_SHAPE;
  if (needs_ws) {
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u)) return SPECVLM_ERR_INVALID_ARG;
    if (ws_bytes < PagesScratch(&c, batch).bytes) return SPECVLM_ERR_WORKSPACE_TOO_SMALL;
    const PagesScratch sc(&c, batch);
    uint8_t* const w = static_cast<uint8_t*>(ws);
    p.n_copies = reinterpret_cast<int32_t*>(w);
    p.copies = reinterpret_cast<int4*>(w + sc.copies);
    p.list = reinterpret_cast<int32_t*>(w + sc.list);
    p.dest = reinterpret_cast<int32_t*>(w + sc.dest);
    p.order = reinterpret_cast<int32_t*>(w + sc.order);
  }
  p.k = static_cast<uint4*>(c.k);
  p.v = static_cast<uint4*>(c.v);
  p.table = table;
  p.ref = ref;
  p.seq_lens = c.seq_lens;
  p.d_status = d_status;
  p.s_layer = c.stride_layer / 8; p.s_block = c.stride_block / 8; p.s_head = c.stride_head / 8; p.s_token = c.stride_token / 8;
  p.block_tokens = c.block_tokens; p.max_blocks = c.max_blocks; p.max_seq_len = c.max_seq_len; p.n_blocks = c.n_blocks;
  p.n_layers = c.n_layers; p.n_kv_heads = c.n_kv_heads; p.chunk_bits = c.head_dim == 128 ? 4 : 3;
  p.batch = batch;
  return SPECVLM_OK;
}

// CTAs of a launch that copies up to so many pages, for `units_each` units of them at least, but eight an SM, which run at once.
// Where most units are there (compaction) CTAs of a unit or a few each, more than run at once, copy faster than ones that walk the
// list, but those that find nothing to move cost a nanosecond each: 900 pages of 28 layers x 4 heads, a quarter of them moved, 8 /
// 16 / 32 / 64 an SM 258 / 253 / 248 / 246 us (6.4 TB/s of bytes moved in the kernel), 705 of 8 x 2 18.5 / 19.3 / 20.0 / 21.1, 30 of 117 pages of
// 22 x 8 64.8 / 62.8 / 61.8 / 61.9, none of them 7.2 / 8.2 / 10.8 / 15.9.  A reservation seldom copies anything, and its CTAs are few.
static unsigned copy_grid(const PagesParams& p, int64_t most_copies, int units_each, int most_per_sm) {
  const int64_t units = most_copies * p.n_layers * p.n_kv_heads, few = 8 * (int64_t)sm_count(), cap = (int64_t)sm_count() * most_per_sm;
  const int64_t n = units < few ? units : units / units_each > few ? units / units_each : few;
  return (unsigned)(n < cap ? n : cap);
}

static bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + b_bytes && y < x + a_bytes;
}

}  // namespace specvlm

using namespace specvlm;

extern "C" size_t specvlm_pages_workspace_bytes(const specvlm_kv_t* kv, int32_t batch) {
  if (!kv || batch < 1 || batch > kPagesMaxBatch || kv->n_blocks < 1 || kv->n_blocks > kPagesMost || kv->max_blocks < 1)
    return 0;
  return PagesScratch(kv, batch).bytes;
}

extern "C" int32_t specvlm_reserve_pages(const specvlm_kv_t* kv, int32_t* block_table_inout, int32_t* ref_count_inout,
                                         int32_t batch, int32_t n_new, const int32_t* new_lens_or_null, void* ws,
                                         size_t ws_bytes, int32_t* d_status, void* stream) {
  NvtxRange nvtx_range(__func__);
  PagesParams p = {};
  if (n_new < 0) return SPECVLM_ERR_INVALID_ARG;
  int32_t rc = pages_params(p, kv, block_table_inout, ref_count_inout, batch, ws, ws_bytes, true, d_status);
  if (rc != SPECVLM_OK) return rc;
  p.n_new = n_new;
  p.new_lens = new_lens_or_null;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const double most_bytes = (double)batch * p.n_layers * p.n_kv_heads * p.block_tokens * kv->head_dim * 4;   // K and V
  if (most_bytes <= kReserveClusterBytes)
    return launch_clusters_after(reserve_cluster_kernel, dim3(kReserveCluster), kReserveCluster, dim3(kPlanThreads), 0, st, p);
  rc = launch_after(reserve_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, p);
  if (rc != SPECVLM_OK) return rc;
  return launch_after(copy_pages_kernel, dim3(copy_grid(p, batch, 1, 8)), dim3(kCopyThreads), 0, st, p);
}

extern "C" int32_t specvlm_release_pages(const specvlm_kv_t* kv, int32_t* block_table_inout, int32_t* ref_count_inout,
                                         int32_t batch, int32_t window, int32_t n_sinks, int32_t* d_status, void* stream) {
  NvtxRange nvtx_range(__func__);
  PagesParams p = {};
  if (window < 1 || n_sinks < 0) return SPECVLM_ERR_INVALID_ARG;
  const int32_t rc = pages_params(p, kv, block_table_inout, ref_count_inout, batch, nullptr, 0, false, d_status);
  if (rc != SPECVLM_OK) return rc;
  return launch_after(release_pages_kernel, dim3((unsigned)((p.max_blocks + 255) / 256), (unsigned)batch), dim3(256), 0,
                      static_cast<cudaStream_t>(stream), p, window, n_sinks);
}

extern "C" int32_t specvlm_fork_pages(const specvlm_kv_t* kv, int32_t* ref_count_inout, int32_t batch, const int32_t* parents,
                                      int32_t batch_out, int32_t* block_table_out, int32_t* seq_lens_out, int32_t* d_status,
                                      void* stream) {
  NvtxRange nvtx_range(__func__);
  PagesParams p = {};
  if (!kv || !parents || !block_table_out || !seq_lens_out || batch_out < 1) return SPECVLM_ERR_INVALID_ARG;
  if (batch_out > kPagesMaxBatch) return SPECVLM_ERR_UNSUPPORTED_SHAPE;
  const int32_t rc = pages_params(p, kv, const_cast<int32_t*>(kv->block_table), ref_count_inout, batch, nullptr, 0, false, d_status);
  if (rc != SPECVLM_OK) return rc;
  const size_t row = (size_t)p.max_blocks * 4;
  if (overlap(block_table_out, row * batch_out, p.table, row * batch) || overlap(seq_lens_out, 4 * (size_t)batch_out, p.seq_lens, 4 * (size_t)batch))
    return SPECVLM_ERR_INVALID_ARG;
  return launch_after(fork_pages_kernel, dim3((unsigned)(batch + batch_out)), dim3(256), 0, static_cast<cudaStream_t>(stream), p, parents,
                      batch_out, block_table_out, seq_lens_out);
}

extern "C" int32_t specvlm_compact_pages(const specvlm_kv_t* kv, int32_t* block_table_inout, int32_t* ref_count_inout,
                                         int32_t batch, int32_t* n_used_or_null, void* ws, size_t ws_bytes, int32_t* d_status,
                                         void* stream) {
  NvtxRange nvtx_range(__func__);
  PagesParams p = {};
  int32_t rc = pages_params(p, kv, block_table_inout, ref_count_inout, batch, ws, ws_bytes, true, d_status);
  if (rc != SPECVLM_OK) return rc;
  p.n_used = n_used_or_null;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  rc = launch_after(compact_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, p);
  if (rc != SPECVLM_OK) return rc;
  return launch_after(compact_move_kernel, dim3(copy_grid(p, (p.n_blocks + 1) / 2, 3, 64)), dim3(kCopyThreads), 0, st, p);
}
