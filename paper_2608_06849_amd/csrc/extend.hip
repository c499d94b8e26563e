// Attention of new tokens over the caches and over themselves (paper Sec. 5,
// chunked-prefill stage: retrieval heads see the whole cached prefix, streaming heads what
// their sink + recent cache holds).
//
// Query t of sequence b stands at position start_pos[b] + t.  Its keys are the cached
// positions below start_pos[b] (paged cache, or the ring's slots) and the new tokens
// 0 .. t, whose K/V come from the call's tensors: the append runs after the attention, so
// the ring still holds what the first new queries see of the window.
//
// An item is a block of rows of one (sequence, KV head): row r is query head r % gs of
// token r / gs, so a tile of K/V is fetched once for the whole group.  The keys of an item
// are visited in tiles, first those of the cache, then the new ones; tiles that no row of
// the item sees are left out.  All items of a launch form one work space, of which every
// workgroup takes an equal range, whatever lengths and head types it crosses; an item that
// several workgroups share is merged by a second launch.
#include <algorithm>
#include <type_traits>

#include "aoh_device.h"
#include "aoh_internal.h"
#include "attn_tile.h"

namespace aoh {

// A sequence's new tokens: their number (0: the sequence is left out), its cached
// positions, and its first row in packed tensors.
struct ExtendSeq {
  int n, start, row0;
};

__device__ __forceinline__ ExtendSeq extend_seq(const ExtendArgs& a, int b) {
  ExtendSeq s = {a.T, a.start_pos ? a.start_pos[b] : 0, 0};
  if (a.cu_seqlens) {
    const int c0 = min(max(a.cu_seqlens[b], 0), a.total), c1 = min(max(a.cu_seqlens[b + 1], c0), a.total);
    s.n = min(c1 - c0, a.T);
    s.row0 = c0;
  }
  if (s.start < 0 || s.start > kMaxPos) s.n = 0;
  return s;
}

// Positions that a sequence's row of the block table has room for.
__device__ __forceinline__ int paged_cap(const ExtendArgs& a) { return min(a.max_pages, kMaxPos / kPage) * kPage; }

// Position that ring slot c holds when `start` tokens have been written, or -1.
__device__ __forceinline__ int ring_position(int c, int start, int n_sink, int window) {
  if (c < n_sink) return c < start ? c : -1;
  const int r = c - n_sink, last = start - 1 - n_sink;  // offsets behind the sinks
  if (r >= window || last < r) return -1;
  return n_sink + last - (last - r) % window;
}

// ---------------------------------------------------------------------------
// The work space.  An item's places: kUnit for each tile that its rows visit, about (a
// first number and a step from one block of rows to the next), and item_cost tiles for its
// start.  A range of places stands for the same share of the item's visits, so the numbers
// need not be exact.  A first launch writes the items and where every range starts, so that
// the others begin with a few scalar loads.
constexpr int kUnit = 16;
constexpr int kPlanSeqs = 1024;  // sequences of a launch; larger batches go in parts

struct ExtendHead {
  int64_t total, range;  // places of all items, of a range
  int32_t used, n_items; // ranges, items
};

struct ExtendItem {
  int64_t first, places;
  // element offsets of the sequence's first new token (query head: the group's first), of its
  // row of the block table, and of its ring
  int64_t q_off, k_off, v_off, o_off, table, ring;
  // Visits: tile = visit + (0 below c1, o1 below c2, o2) among the n_cached of the cache, then
  // counted from there + (0 below d1, e1) among the new ones; n in all.
  int32_t n, n_cached, c1, c2, o1, o2, d1, e1;
  int32_t start, cached, n_new, row0;   // tokens before, positions (slots) that the cache holds, new tokens, first row
  int32_t t_first, t_last;              // tokens of its rows
  // First key of token t's window: lo_off + t (far below where there is none).  Ring: offset r
  // behind the sinks holds position rbase + r, one window less behind r = rrem.
  int32_t lo_off, rbase, rrem;
  int32_t str, head, rank;              // streaming; KV head, and its rank in its cache

  __device__ __forceinline__ int tile(int it) const {
    if (it < n_cached) return it + (it < c1 ? 0 : it < c2 ? o1 : o2);
    const int j = it - n_cached;
    return j + (j < d1 ? 0 : e1);
  }
};

// A value that all lanes share, in scalar registers.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint64_t uniform(uint64_t x) {
  const uint32_t lo = (uint32_t)uniform((int)(uint32_t)x), hi = (uint32_t)uniform((int)(uint32_t)(x >> 32));
  return (uint64_t)hi << 32 | lo;
}
// A load from a uniform address into scalar registers: it is waited for with the LDS reads,
// not with the direct loads.
template <typename T>
__device__ __forceinline__ T scalar_load(const T* p) {
  static_assert(sizeof(T) % 4 == 0, "whole words");
  typedef const __attribute__((address_space(4))) uint32_t* words;
  const words w = (words)uniform((uint64_t)reinterpret_cast<uintptr_t>(p));
  uint32_t x[sizeof(T) / 4];
#pragma unroll
  for (size_t i = 0; i < sizeof(T) / 4; ++i) x[i] = w[i];
  return __builtin_bit_cast(T, x);
}

__device__ __forceinline__ int div_up(int a, int b) { return (a + b - 1) / b; }
// x / y of numbers below 2^53 (a 64-bit division is many times longer).
__device__ __forceinline__ int64_t div64(int64_t x, int64_t y) {
  int64_t q = (int64_t)((double)x / (double)y);
  const int64_t r = x - q * y;
  if (r < 0) --q;
  else if (r >= y) ++q;
  return q;
}
// x / gs for the rows of an item (x < 2^30): exact, as gs <= 16.
__device__ __forceinline__ int div_gs(const ExtendArgs& a, int x) { return (int)(((uint64_t)(uint32_t)x * a.gs_mul) >> 36); }

// Places of the first n of an item's blocks of rows.
__device__ __forceinline__ int64_t places_of(int64_t a, int c, int64_t n) { return n * a + c * (n * (n - 1) / 2); }

// Blocks of rows of a sequence, places of a block of rows of its retrieval and its streaming
// heads: first block, step.
struct SeqCost {
  int blocks;
  int64_t a[2];
  int c[2];
};

template <int ROWS, int TILE>
__device__ __forceinline__ SeqCost seq_cost(const ExtendArgs& a, const ExtendSeq& s) {
  SeqCost x;
  x.blocks = (int)(((int64_t)s.n * a.gs + ROWS - 1) / ROWS);
  const int n_new = div_up(s.n, TILE);
  const int paged = div_up(min(s.start, paged_cap(a)), TILE);
  const int ring = div_up(min(s.start, a.ring_cap), TILE);
  x.a[0] = (int64_t)kUnit * (a.item_cost + paged + min(n_new, a.block_tiles));
  x.c[0] = a.block_step;
  // Masked tiles of rings and windows take 2.5-3 us, those of a cached prefix 1.65.  (With
  // eviction the ring's tiles are not masked.  Counted like the prefix's, chunks of four
  // sequences took 196.5 us instead of 199.5, other calls the same within a run's noise of 1%.)
  x.a[1] = (int64_t)kUnit * a.item_cost + (kUnit * 3 / 2) * (int64_t)(a.evict ? ring + min(n_new, a.block_tiles) : min(ring + n_new, a.band_tiles));
  x.c[1] = a.evict ? a.block_step : 0;
  return x;
}

// Fills in the tiles that rows of tokens t_first .. t_last visit.
template <int TILE>
__device__ __forceinline__ void set_visits(const ExtendArgs& a, ExtendItem& x) {
  const int all = div_up(x.cached, TILE), n_new = x.t_last / TILE + 1;
  x.o1 = x.o2 = x.d1 = x.e1 = 0;
  x.lo_off = INT32_MIN / 2;
  x.rbase = x.rrem = 0;
  if (!x.str) {
    x.n_cached = x.c1 = x.c2 = all;
    x.n = all + n_new;
    return;
  }
  const int start = x.start;
  if (!a.evict) x.lo_off = start - a.window + 1;
  const int rlast = max(start - 1 - a.n_sink, 0);
  x.rrem = rlast % a.window;
  x.rbase = a.n_sink + rlast - x.rrem;
  const int lo = a.evict ? start - a.window : start + x.t_first - a.window + 1;
  const int w0 = max(lo, a.n_sink);  // first cached position of the window
  const int sinks = div_up(min(a.n_sink, x.cached), TILE);
  int f1 = sinks, l1 = sinks, f2 = 0, l2 = 0;  // runs of window tiles
  if (w0 < start) {
    const int back = start - 1 - w0;  // from the newest token's slot, offset rrem, to the oldest visible one's
    const int q = a.n_sink + x.rrem, p = a.n_sink + x.rrem - back;
    if (back + 1 >= a.window) {
      l1 = all;
    } else if (back <= x.rrem) {
      f1 = max(sinks, p / TILE);
      l1 = q / TILE + 1;
    } else {
      f1 = max(sinks, a.n_sink / TILE);
      l1 = q / TILE + 1;
      f2 = max(max(f1, l1), (p + a.window) / TILE);
      l2 = all;
    }
  }
  x.c1 = sinks;
  x.c2 = sinks + max(0, l1 - f1);
  x.n_cached = x.c2 + max(0, l2 - f2);
  x.o1 = f1 - x.c1;
  x.o2 = f2 - x.c2;
  const int d0 = max(0, lo - start) / TILE;  // first new tile of the window
  x.d1 = min(div_up(max(0, a.n_sink - start), TILE), d0);
  x.e1 = d0 - x.d1;
  x.n = x.n_cached + x.d1 + n_new - d0;
}

// Items go by head type, sequence, KV head and block of rows.  Every workgroup scans the
// sequences (consecutive ones a thread), each thread then writes items.  Bound: the chain of
// its loads and its own instructions' fetch, 5 us for one sequence, 7-8 for up to 24; in the
// tile kernel itself the same work took more registers than its loops have left.
template <int ROWS, int TILE>
__global__ __launch_bounds__(256) void extend_plan_kernel(ExtendArgs a) {
  __shared__ int64_t s_places[2][kPlanSeqs + 1];
  __shared__ int s_blocks[kPlanSeqs];
  __shared__ int64_t s_wave[3][4], s_all;
  __shared__ int64_t s_first[256];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n_kv[2] = {a.n_ret, a.n_str};
  const int b0 = div_up(a.B, 256) * tid, b1 = min(b0 + div_up(a.B, 256), a.B);  // this thread's sequences
  int64_t sum[3] = {0, 0, 0};
#pragma unroll 1
  for (int b = b0; b < b1; ++b) {
    const SeqCost k = seq_cost<ROWS, TILE>(a, extend_seq(a, b));
    for (int i = 0; i < 2; ++i) {
      s_places[i][b] = n_kv[i] * places_of(k.a[i], k.c[i], k.blocks);
      sum[i] += s_places[i][b];
    }
    s_blocks[b] = k.blocks;
    sum[2] += k.blocks;
  }
  int64_t inc[3] = {sum[0], sum[1], sum[2]};
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1)
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const int64_t y = __shfl_up(inc[i], o, kWave);
      if (lane >= o) inc[i] += y;
    }
  if (lane == kWave - 1)
#pragma unroll
    for (int i = 0; i < 3; ++i) s_wave[i][wave] = inc[i];
  __syncthreads();
  int64_t at[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    at[i] = inc[i] - sum[i];
    for (int w = 0; w < wave; ++w) at[i] += s_wave[i][w];
  }
#pragma unroll 1
  for (int b = b0; b < b1; ++b) {
    for (int i = 0; i < 2; ++i) {
      const int64_t own = s_places[i][b];
      s_places[i][b] = at[i];
      at[i] += own;
    }
    const int own = s_blocks[b];
    s_blocks[b] = (int)at[2];
    at[2] += own;
  }
  if (tid == 255) {
    for (int i = 0; i < 2; ++i) s_places[i][kPlanSeqs] = at[i];
    s_all = at[2];
  }
  __syncthreads();
  // Sequences whose packed rows overlap may need more items than there is room for: none then.
  const int blocks = (n_kv[0] + n_kv[1]) * s_all <= a.max_items ? (int)s_all : 0;
  const int n_items = (n_kv[0] + n_kv[1]) * blocks;
  const int64_t total = blocks ? s_places[0][kPlanSeqs] + s_places[1][kPlanSeqs] : 0;
  const int64_t range = max(div64(total + a.wgs - 1, a.wgs), (int64_t)a.min_tiles * kUnit);
  const int used = (int)div64(total + range - 1, range);
  if (blockIdx.x == 0 && tid == 0) *a.head = ExtendHead{total, range, used, n_items};
  if (blockIdx.x == 0) {  // the arguments for a function that takes them from memory, word by word
    static_assert(sizeof(ExtendArgs) % 4 == 0, "whole words");
    const auto args = (const __attribute__((address_space(4))) uint32_t*)__builtin_amdgcn_kernarg_segment_ptr();
    for (int i = tid; i < (int)(sizeof(ExtendArgs) / 4); i += 256) reinterpret_cast<uint32_t*>(a.copy)[i] = args[i];
  }
  const bool few = n_items <= 256;  // one item a thread of the first workgroup
  for (int idx = blockIdx.x * 256 + tid; idx < n_items; idx += gridDim.x * 256) {
    ExtendItem it;
    it.str = idx >= n_kv[0] * blocks;
    const int heads = n_kv[it.str], at = idx - (it.str ? n_kv[0] * blocks : 0);
    int b = 0;  // the last sequence whose items begin at or before this one
    for (int hi = a.B; hi - b > 1;) {
      const int mid = (b + hi) >> 1;
      if ((int64_t)heads * s_blocks[mid] <= at) b = mid;
      else hi = mid;
    }
    const ExtendSeq s = extend_seq(a, b);
    const SeqCost k = seq_cost<ROWS, TILE>(a, s);
    const int64_t ka = k.a[it.str];
    const int kc = k.c[it.str];
    const int in_seq = at - heads * s_blocks[b];
    it.rank = in_seq / k.blocks;
    const int rb = in_seq - it.rank * k.blocks;
    it.first = (it.str ? s_places[0][kPlanSeqs] : 0) + s_places[it.str][b] + it.rank * places_of(ka, kc, k.blocks) + places_of(ka, kc, rb);
    it.places = ka + (int64_t)kc * rb;
    it.head = a.kv_heads[it.str ? a.n_ret + it.rank : it.rank];
    const int64_t sb = a.cu_seqlens ? 0 : b, tok0 = a.cu_seqlens ? s.row0 : 0;
    it.q_off = sb * a.q_sb + tok0 * a.q_st + (int64_t)it.head * a.gs * a.q_sh;
    it.k_off = sb * a.k_sb + tok0 * a.k_st + it.head * a.k_sh;
    it.v_off = sb * a.v_sb + tok0 * a.v_st + it.head * a.v_sh;
    it.o_off = sb * a.o_sb + tok0 * a.o_st + (int64_t)it.head * a.gs * a.o_sh;
    it.table = (int64_t)b * a.max_pages;
    it.ring = ((int64_t)b * a.n_str + it.rank) * a.ring_blocks;
    it.start = s.start;
    it.n_new = s.n;
    it.cached = it.str ? min(s.start, a.ring_cap) : min(s.start, paged_cap(a));
    it.row0 = rb * ROWS;
    it.t_first = div_gs(a, it.row0);
    it.t_last = div_gs(a, min(it.row0 + ROWS, s.n * a.gs) - 1);
    set_visits<TILE>(a, it);
    a.items[idx] = it;
    if (few) {
      s_first[tid] = it.first;
      continue;
    }
    // ranges that start in this item
    const int w1 = min(used - 1, (int)div64(it.first + it.places - 1, range));
    for (int w = (int)div64(it.first + range - 1, range); w <= w1; ++w) a.first_item[w] = idx;
  }
  // few items have many ranges each, and each range looks for its item
  if (!few || blockIdx.x != 0) return;
  __syncthreads();
  for (int w = tid; w < used; w += 256) {
    int i = 0;  // the last item that begins at or before the range
    for (int hi = n_items; hi - i > 1;) {
      const int mid = (i + hi) >> 1;
      if (s_first[mid] <= w * range) i = mid;
      else hi = mid;
    }
    a.first_item[w] = i;
  }
}

// Ranges go to the 8 XCDs (each with its own L2) in eight consecutive parts, so that the
// blocks of rows that share K/V run on one.  Returns the range of workgroup w, or -1.
__device__ __forceinline__ int range_of(int w, int used) {
  const int per = (used + 7) >> 3, r = (w & 7) * per + (w >> 3);
  return (w >> 3) < per && r < used ? r : -1;
}

// x times a weight or a factor between weights: by the formula those are positive, so that an
// infinity stays one where they fall below fp32's range.
__device__ __forceinline__ float scaled(float x, float f) { return isinf(x) ? x : x * f; }

// Four output values at element `at`.
template <bool F32>
__device__ __forceinline__ void store4(const ExtendArgs& a, int64_t at, f32x4 o) {
  if (F32) {
    *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at) = o;
  } else {
    u32x2 w;
    w[0] = (uint32_t)f32_to_bf16_bits(o[0]) | ((uint32_t)f32_to_bf16_bits(o[1]) << 16);
    w[1] = (uint32_t)f32_to_bf16_bits(o[2]) | ((uint32_t)f32_to_bf16_bits(o[3]) << 16);
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + at) = w;
  }
}

// ---------------------------------------------------------------------------
// fp32: plain rows, kept exact; it has no performance role.
// A wave takes 64 keys at a time, one a lane, then the lanes take the output's dimensions.
template <int D>
__global__ __launch_bounds__(256) void extend_simple_kernel(ExtendArgs a) {
#pragma clang fp contract(off)
  constexpr int kDims = D / kWave;
  __shared__ float s_q[D];
  __shared__ int64_t s_at[4][kWave];
  __shared__ float s_p[4][kWave];
  __shared__ float s_o[4][D], s_m[4], s_l[4];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  auto value = [](const void* p, int64_t i) { return static_cast<const float*>(p)[i]; };
  const int64_t rows = (int64_t)a.B * a.T * a.Hq;
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const int h = (int)(row % a.Hq), t = (int)(row / a.Hq % a.T), b = (int)(row / a.Hq / a.T);
    const int g = h / a.gs, rank = a.rank[g];
    const bool str = (a.streaming_mask >> g) & 1ull;
    const ExtendSeq s = extend_seq(a, b);
    if (t >= s.n) continue;  // uniform
    __syncthreads();  // the row before has been stored
    const int64_t tok0 = a.cu_seqlens ? s.row0 : 0;
    const int64_t sb = a.cu_seqlens ? 0 : b;
    if (tid < D) s_q[tid] = value(a.q, sb * a.q_sb + (tok0 + t) * a.q_st + h * a.q_sh + tid);
    __syncthreads();
    const int n_cached = str ? min(s.start, a.ring_cap) : min(s.start, paged_cap(a));
    const int lo = a.evict ? s.start - a.window : s.start + t - a.window + 1;
    float m = -INFINITY, l = 0.f, o[kDims];
#pragma unroll
    for (int i = 0; i < kDims; ++i) o[i] = 0.f;
    const int n_keys = n_cached + t + 1;
    for (int k0 = 64 * wave; k0 < n_keys; k0 += 256) {
      const int j = k0 + lane;
      const void *kp = nullptr, *vp = nullptr;
      int64_t ka = 0, va = -1;  // K row, V's first value (step 16 in the caches, 1 in the tensors); -1: not visible
      if (j < n_cached) {
        int64_t unit = -1;
        if (str) {
          const int p = ring_position(j, s.start, a.n_sink, a.window);
          if (p >= 0 && (p < a.n_sink || p >= lo)) unit = ((int64_t)b * a.n_str + rank) * a.ring_blocks + j / kPage;
        } else {
          const int page = a.block_table[(int64_t)b * a.max_pages + j / kPage];
          if (page >= 0 && page < a.num_pages) unit = (int64_t)page * a.n_ret + rank;
        }
        if (unit >= 0) {
          kp = str ? a.rk : a.pk;
          ka = unit * (kPage * D) + j % kPage * D;
          va = unit * (kPage * D) + j % kPage;
        }
      } else if (j < n_keys) {
        const int p = s.start + j - n_cached;
        if (!str || p < a.n_sink || p >= lo) {
          kp = a.k;
          ka = sb * a.k_sb + (tok0 + j - n_cached) * a.k_st + g * a.k_sh;
          va = sb * a.v_sb + (tok0 + j - n_cached) * a.v_st + g * a.v_sh;
        }
      }
      float x = -INFINITY;
      if (va >= 0) {
        x = 0.f;
        for (int d = 0; d < D; ++d) x = fmaf(s_q[d], value(kp, ka + d), x);
        x *= a.scale;
        if (x == -INFINITY) va = -1;  // weight 0
      }
      float mx = x;
#pragma unroll
      for (int i = 1; i < kWave; i *= 2) mx = wave_xor_max(mx, i);
      const float m_new = fmaxf(m, mx);
      const float alpha = m == -INFINITY ? 0.f : expf(m - m_new);
      const float p = va < 0 ? 0.f : expf(x - m_new);
      float sum = p;
#pragma unroll
      for (int i = 1; i < kWave; i *= 2) sum = wave_xor_sum(sum, i);
      l = l * alpha + sum;
      m = m_new;
      s_at[wave][lane] = va;
      s_p[wave][lane] = p;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < kDims; ++i) o[i] = scaled(o[i], alpha);
      for (int i = 0; i < kWave; ++i) {
        const int64_t at = s_at[wave][i];
        if (at < 0) continue;
        const bool cached = k0 + i < n_cached;
        vp = cached ? (str ? a.rv : a.pv) : a.v;
#pragma unroll
        for (int u = 0; u < kDims; ++u) o[u] += scaled(value(vp, at + (int64_t)(lane + kWave * u) * (cached ? kPage : 1)), s_p[wave][i]);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int u = 0; u < kDims; ++u) s_o[wave][lane + kWave * u] = o[u];
    if (lane == 0) {
      s_m[wave] = m;
      s_l[wave] = l;
    }
    __syncthreads();
    if (tid < D) {
      float M = -INFINITY, L = 0.f, x = 0.f;
      for (int w = 0; w < 4; ++w) M = fmaxf(M, s_m[w]);
      for (int w = 0; w < 4; ++w) {
        if (s_m[w] == -INFINITY && s_l[w] == 0.f) continue;  // no key (keys with NaN scores leave a NaN sum)
        const float f = s_m[w] == -INFINITY ? 1.f : expf(s_m[w] - M);
        L += f * s_l[w];
        x += scaled(s_o[w][tid], f);
      }
      x /= L;
      const int64_t at = sb * a.o_sb + (tok0 + t) * a.o_st + h * a.o_sh + tid;
      static_cast<float*>(a.out)[at] = x;
    }
  }
}

template <int D>
static hipError_t launch_simple(const ExtendArgs& a, hipStream_t s) {
  const int64_t rows = (int64_t)a.B * a.T * a.Hq;
  hipLaunchKernelGGL((extend_simple_kernel<D>), dim3((unsigned)std::min<int64_t>(rows, 1 << 16)), dim3(256), 0, s, a);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// bf16, many rows: a workgroup of ROWS rows, 32 a wave, on the 32x32x16 bf16 MFMA, with
// 64-key tiles of K and V in LDS rings:
//   S^T[64 keys x 32 rows] = K . Q^T,  softmax in fp32,  O^T[D x 32 rows] += V^T . P^T.
// Bound: no unit alone.  The matrix cores are busy 0.57 of the SIMDs' cycles in the longest
// chunk measured and 0.50 in one of 2048 tokens, vector instructions (exponentials, masks,
// conversions) 0.44 and 0.40, and they overlap in part.  Three parts of a weight at width 64:
// vector instructions 0.53, matrix cores 0.31, with little overlap (no two waves of a block of
// 128 rows run a phase apart).  Measured at width 128: 4096 tokens after 126976 (groups of 4)
// 3.9-4.1 ms, 1060-1120 TFLOP/s; 2048 after 28672 (groups of 7) 440-470 us, about 1000 TFLOP/s;
// chunks of four sequences with eviction (groups of 4) 192-204 us, about 790 TFLOP/s.  Few rows:
// memory and the chain of one wave, 4 tokens of 8 sequences at 32700 (groups of 4) 134 us, 3.9 TB/s.
//  * Tiles move global -> LDS with direct loads, two or three tiles ahead.  K rows and new
//    V rows are token-major with swizzled 16-byte chunks (PPTile); pages keep V
//    dimension-major, [page][D][16 tokens], with the two halves of a dimension swapped in
//    every second group of eight dimensions, so that 16 lanes read 16 different bank
//    groups.
//  * K row i of a tile is MFMA row i with bits 2 and 3 swapped.  A lane's scores are then
//    those of 8 consecutive keys for each half, which is the B operand of the second
//    product as it stands, and its V^T operand is 8 consecutive tokens of a dimension: one
//    16-byte read of a page, two transpose reads of new rows.
//  * One barrier a tile.  With 256 rows waves 0-3 and 4-7 run one phase apart, so that a
//    SIMD's two waves alternate between the matrix cores and the vector phase.
//  * Exponentials are taken against a trailing reference max; a tile whose exponentials
//    sum to more than kSumHi moves it.
//  * PARTS = 3 (fp32 outputs): P as three bf16 numbers, whole; PARTS = 1 (bf16 outputs):
//    rounded, as in a prefill, for a third of the second product's time.
// V behind a cache's last token is zeroed in LDS by the wave that loaded it.  Where a row
// does not see a key that another row of the workgroup sees, V may be anything, and 0 V is
// not 0 if it is not finite: the waves look for such values in the tiles that are masked.
// An infinity that a row does see times a part of its weight, or a weight, below the types'
// range is NaN instead of infinite: the waves look for sums that are not finite.  A workgroup that
// has met either (or a page outside the cache) takes its range again in the careful loop, which
// sums the finite values and counts the others.
template <int D, int ROWS>
struct TileShape {
  static constexpr int kThreads = 2 * ROWS;
  static constexpr bool kPair = ROWS == 256;
  static constexpr int kAhead = kPair ? 3 : 2;
  static constexpr int kKSlots = kPair ? 4 : D == 128 ? 2 : 3;
  static constexpr int kVSlots = kPair ? 4 : 3;
  static constexpr int kLoads = kBN * (D / 8) / kThreads;  // loads per thread and tile, K or V
};

template <int D, int ROWS>
struct TileRing {
  uint16_t k[TileShape<D, ROWS>::kKSlots][kBN * D];
  uint16_t v[TileShape<D, ROWS>::kVSlots][kBN * D];
};

// Largest sum of a lane's 32 exponentials of one tile, taken against the trailing
// reference max, that is accepted as it is.
constexpr float kSumHi = 65536.f;

// Direct loads, 16 bytes a lane to lds_row + 16 lane (see lds_dma16): from a uniform address
// plus a lane's byte offset, and from a lane's address.  The hazards that the compiler does
// not see inside the assembly are waited for there: an address in scalar registers that a
// vector instruction has just written (five cycles), M0 just written (one).
__device__ __forceinline__ void lds_dma16_from(const void* base, uint32_t offset, const void* lds_row) {
  const uint32_t m0 = (uint32_t)uniform((int)reinterpret_cast<uintptr_t>(lds_row));
  asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(uniform((uint64_t)reinterpret_cast<uintptr_t>(base))), "{m0}"(m0) : "memory");
}

__device__ __forceinline__ void lds_dma16_at(const void* gptr, const void* lds_row) {
  const uint32_t m0 = (uint32_t)uniform((int)reinterpret_cast<uintptr_t>(lds_row));
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(gptr), "{m0}"(m0) : "memory");
}

__device__ __forceinline__ bool not_finite(u32x4 x) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) bad = bad || (x[i] & 0x7f80u) == 0x7f80u || (x[i] & 0x7f800000u) == 0x7f800000u;
  return bad;
}

// The tiles of one range.  CAREFUL: the second time, see above.  Returns whether it has to be
// taken again.
template <int D, int ROWS, int PARTS, bool CAREFUL>
__device__ __forceinline__ bool extend_range(const ExtendArgs& a, TileRing<D, ROWS>& ring) {
  using Tile = PPTile<D>;
  using Shape = TileShape<D, ROWS>;
  constexpr int kKSteps = D / 16;
  constexpr int kMBlocks = D / 32;
  constexpr std::integral_constant<bool, true> kCached{};
  constexpr std::integral_constant<bool, false> kNew{};

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = wave >> 2;
  const int lane = tid & 63;
  const int l32 = lane & 31;
  const int h2 = lane >> 5;
  const float c = a.scale_log2;

  // Per-lane LDS addresses.  K operand of step s, block blk: row 32 blk + (l32 with bits 2
  // and 3 swapped), logical chunk 2 s + h2.  V^T operand of key step ks, 32-dim block mb: in
  // pages the dimension's 16-byte half h2; of new rows transpose reads from row 16 ks + 8 h2
  // + i16 / 4 (+ 4 rows), logical chunk 4 mb + 2 (q16 & 1) + (i16 & 3) / 2, 4 more elements
  // for odd i16.
  const int q16 = lane >> 4;
  const int i16 = lane & 15;
  const uint32_t kring0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(&ring.k[0][0]));
  const uint32_t vring0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(&ring.v[0][0]));
  const int krow0 = (l32 & 19) | ((l32 & 4) << 1) | ((l32 & 8) >> 1);
  const uint32_t kaddr0 = kring0 + 2u * (uint32_t)Tile::koff(krow0, h2);
  const uint32_t vaddr0 = vring0 + 2u * (uint32_t)(Tile::voff(8 * h2 + (i16 >> 2), 2 * (q16 & 1) + ((i16 & 3) >> 1)) + 4 * (i16 & 1));
  const uint32_t paddr0 = vring0 + 32u * l32 + 16u * (h2 ^ ((l32 >> 3) & 1));
  // Direct loads of a tile: wave w fills kLoads blocks of 1 KB of K and of V, one instruction
  // each, which lie in one page of the tile (my_page): byte offsets in the page, and rows of
  // the tile.
  constexpr int kBlockRows = 512 / D;
  const int my_page = wave * Shape::kLoads * kBlockRows / kPage;
  uint32_t dma_k[Shape::kLoads];
#pragma unroll
  for (int jj = 0; jj < Shape::kLoads; ++jj) {
    const int r = kBlockRows * (Shape::kLoads * wave + jj) + lane / Tile::kChunks;
    dma_k[jj] = 2u * ((r % kPage) * D + 8 * ((lane % Tile::kChunks) ^ Tile::kx(r)));
  }
  const int dim0 = (32 * Shape::kLoads * wave + (lane >> 1)) % D, half0 = (lane & 1) ^ ((dim0 >> 3) & 1);
  const uint32_t dma_v = 2u * (dim0 * kPage + 8 * half0);
  auto k_operand = [&](uint32_t at, int blk) __attribute__((always_inline)) {
    typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
    return *reinterpret_cast<lds_bf16x8*>(at + 64u * D * blk);
  };
  // cached: a tile of pages, else of new rows
  auto v_operand = [&](auto cached, uint32_t at, int ks) __attribute__((always_inline)) {
    if constexpr (decltype(cached)::value) {
      typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
      return *reinterpret_cast<lds_bf16x8*>(at + 32u * D * ks);
    } else {
      typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
      const uint32_t x = at + 32u * D * ks;
      const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_i16x4*>(x));
      const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_i16x4*>(x + 8u * D));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  };
  auto barrier = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
  };

  const ExtendHead head = scalar_load(a.head);
  const int rng = range_of(blockIdx.x, head.used);
  if (rng < 0) return false;
  const int64_t g1 = min((rng + 1) * head.range, head.total);
  int64_t g0 = rng * head.range;
  bool again = false;
#pragma unroll 1
  for (int idx = scalar_load(a.first_item + rng); g0 < g1; ++idx) {
    const ExtendItem item = scalar_load(a.items + idx);
    // the share of the item's visits that this range stands for
    const int64_t s0 = g0 - item.first, s1 = min(g1 - item.first, item.places);
    const int v0 = uniform((int)div64(s0 * item.n, item.places)), v1 = uniform((int)div64(s1 * item.n, item.places));
    const bool whole = s0 == 0 && s1 == item.places;
    g0 = item.first + s1;
    const int64_t part = (int64_t)(2 * rng + (s0 == 0 ? 1 : 0)) * ROWS;
    if (v0 >= v1) {  // no tile of its own: an empty partial (an item has a visit, so not a whole one)
      if (tid < ROWS) {
        a.part_ml[(part + tid) * 2 + 0] = -INFINITY;
        a.part_ml[(part + tid) * 2 + 1] = 0.f;
      }
      continue;
    }
    const int start = item.start, n_new = item.n_new, cached = item.cached, lo_off = item.lo_off;
    const bool str = item.str, band = str && !a.evict;
    const int n_rows = n_new * a.gs;
    // This lane's row, and the wave's first and last tokens.
    const int my_r = min(item.row0 + wave * 32 + l32, n_rows - 1);
    const int my_t = div_gs(a, my_r);
    const int w_t0 = div_gs(a, min(item.row0 + wave * 32, n_rows - 1)), w_t1 = div_gs(a, min(item.row0 + wave * 32 + 31, n_rows - 1));
    const int64_t q_at = item.q_off + my_t * a.q_st + (my_r - my_t * a.gs) * a.q_sh;
    const uint16_t* kn = static_cast<const uint16_t*>(a.k) + item.k_off;
    const uint16_t* vn = static_cast<const uint16_t*>(a.v) + item.v_off;
    // cached tiles: units of 16 rows, unit_step elements from one page (block) to the next
    const int unit_step = (str ? 1 : a.n_ret) * (kPage * D);
    const int64_t unit0 = str ? item.ring : item.rank;
    const uint16_t* kc = static_cast<const uint16_t*>(str ? a.rk : a.pk) + unit0 * (kPage * D);
    const uint16_t* vc = static_cast<const uint16_t*>(str ? a.rv : a.pv) + unit0 * (kPage * D);
    const int32_t* item_table = a.block_table + item.table;
    const int last_page = max(div_up(cached, kPage) - 1, 0);
    const int end_page = str ? a.ring_blocks : a.num_pages;
    int64_t k_st = a.k_st, v_st = a.v_st;
    int n_sink = a.n_sink, window = a.window;
    // registers of their own, not those of the argument block's load
    if constexpr (!CAREFUL) asm("" : "+s"(k_st), "+s"(v_st), "+s"(n_sink), "+s"(window));
    // new tiles: byte offsets from the tile's first row, where they fit 32 bits
    const bool near = k_st < (1 << 24) && v_st < (1 << 24);
    uint32_t new_k[Shape::kLoads], new_v[Shape::kLoads];
#pragma unroll
    for (int jj = 0; jj < Shape::kLoads; ++jj) {
      const int r = kBlockRows * (Shape::kLoads * wave + jj) + lane / Tile::kChunks, pc = lane % Tile::kChunks;
      new_k[jj] = 2u * ((uint32_t)r * (uint32_t)k_st + 8 * (pc ^ Tile::kx(r)));
      new_v[jj] = 2u * ((uint32_t)r * (uint32_t)v_st + 8 * (pc ^ Tile::vx(r)));
    }
    bool bad = false;  // this wave has met a page outside the cache, or values that the fast loop cannot take
    auto issue_cached = [&](int slot_k, int slot_v, int entry_v) __attribute__((always_inline)) {
      int entry = uniform(entry_v);
      if (entry < 0 || entry >= end_page) {
        bad = true;
        entry = 0;
      }
      const int64_t unit = (int64_t)entry * unit_step;
      const uint16_t* ku = kc + unit;
      const uint16_t* vu = vc + unit;
#pragma unroll
      for (int jj = 0; jj < Shape::kLoads; ++jj) {
        const int j = Shape::kLoads * wave + jj;
        lds_dma16_from(ku, dma_k[jj], &ring.k[slot_k][512 * j]);
        lds_dma16_from(vu, dma_v + 1024 * jj, &ring.v[slot_v][512 * j]);
      }
    };
    auto issue_new = [&](int kb, int slot_k, int slot_v) __attribute__((always_inline)) {
      if (kb + kBN <= n_new && near) {
        const uint16_t* kt = kn + kb * k_st;
        const uint16_t* vt = vn + kb * v_st;
#pragma unroll
        for (int jj = 0; jj < Shape::kLoads; ++jj) {
          const int j = Shape::kLoads * wave + jj;
          lds_dma16_from(kt, new_k[jj], &ring.k[slot_k][512 * j]);
          lds_dma16_from(vt, new_v[jj], &ring.v[slot_v][512 * j]);
        }
        return;
      }
      int ln = lane;
      asm volatile("" : "+v"(ln));  // rare: its addresses are not to be kept in registers
#pragma unroll
      for (int jj = 0; jj < Shape::kLoads; ++jj) {
        const int j = Shape::kLoads * wave + jj;
        const int r = kBlockRows * j + ln / Tile::kChunks, pc = ln % Tile::kChunks;
        const int64_t row = min(kb + r, n_new - 1);  // rows behind the last repeat it; no query sees them
        lds_dma16_at(kn + row * k_st + 8 * (pc ^ Tile::kx(r)), &ring.k[slot_k][512 * j]);
        lds_dma16_at(vn + row * v_st + 8 * (pc ^ Tile::vx(r)), &ring.v[slot_v][512 * j]);
      }
    };
    // V of a tile that this wave's loads have brought: zeroes tokens behind the cache's last
    // one, and looks for values that are not finite where a row does not see all keys.
    auto clean = [&](int it, int kb, int slot_v) __attribute__((always_inline)) {
      const bool of_cache = it < item.n_cached;
      const bool tail = of_cache && kb + kBN > cached;
      const bool masked = of_cache ? band : kb + kBN - 1 > item.t_first || !(start + kb + kBN - 1 < n_sink || start + kb >= lo_off + item.t_last);
      if (!tail && !masked) return;
      int ln = lane;
      asm volatile("" : "+v"(ln));
#pragma unroll
      for (int jj = 0; jj < Shape::kLoads; ++jj) {
        const int j = Shape::kLoads * wave + jj;
        u32x4* at = reinterpret_cast<u32x4*>(&ring.v[slot_v][512 * j + 8 * ln]);
        u32x4 x = *at;
        if (tail) {
          const int half = (ln & 1) ^ ((((32 * j + (ln >> 1)) % D) >> 3) & 1);
          const int left = cached - (kb + (32 * j / D) * kPage + 8 * half);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = left >= 2 * e + 2 ? x[e] : left == 2 * e + 1 ? x[e] & 0xffffu : 0u;
          *at = x;
        }
        if (!CAREFUL && masked && __any(not_finite(x))) bad = true;
      }
    };

    bf16x8 qreg[kKSteps];
    f32x16 acc_o[kMBlocks];
#pragma unroll
    for (int mb = 0; mb < kMBlocks; ++mb)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc_o[mb][i] = 0.f;
    float m_run = -INFINITY;  // reference max (log2 units) of this lane's row
    float m_use = 0.f;        // m_run, or 0 while the row has seen no visible key
    float l_run = 0.f;        // this lane's part of the row sum (the partner lane has the rest)
    f32x16 sacc[2];           // S^T of the current tile, two 32-key blocks
    bf16x8 pop[PARTS][4];     // P^T operands of the previous tile's 4 key steps

    // Operands in the order of their products: V^T of each key step and 32-dim block, then K
    // of each step and block.  They are read kDepth products ahead; the barriers to the
    // scheduler keep that order (left to it, every product waited for its own read).
    constexpr int kNV = 4 * kMBlocks, kNK = 2 * kKSteps, kDepth = 6;
    auto products = [&](auto is_cached, auto with_v, auto with_k, int slot_k, int slot_v) __attribute__((always_inline)) {
      constexpr int kFirst = decltype(with_v)::value ? 0 : kNV, kLast = decltype(with_k)::value ? kNV + kNK : kNV;
      uint32_t ka[kKSteps], va[kMBlocks];
#pragma unroll
      for (int s = 0; s < kKSteps; ++s) ka[s] = (kaddr0 + (uint32_t)slot_k * Tile::kBytes) ^ (32u * s);
#pragma unroll
      for (int mb = 0; mb < kMBlocks; ++mb)
        va[mb] = decltype(is_cached)::value ? paddr0 + (uint32_t)slot_v * Tile::kBytes + 1024u * mb
                                            : (vaddr0 + (uint32_t)slot_v * Tile::kBytes) ^ (64u * mb);
      bf16x8 op[kDepth];
      auto read = [&](int o) __attribute__((always_inline)) {
        op[o % kDepth] = o < kNV ? v_operand(is_cached, va[o % kMBlocks], o / kMBlocks) : k_operand(ka[(o - kNV) / 2], o & 1);
      };
#pragma unroll
      for (int o = kFirst; o < kFirst + kDepth; ++o) read(o);
      if constexpr (decltype(with_k)::value) {
#pragma unroll
        for (int blk = 0; blk < 2; ++blk)
#pragma unroll
          for (int i = 0; i < 16; ++i) sacc[blk][i] = 0.f;
      }
#pragma unroll
      for (int o = kFirst; o < kLast; ++o) {
        __builtin_amdgcn_sched_barrier(0);
        const bf16x8 x = op[o % kDepth];
        if (o < kNV) {
#pragma unroll
          for (int i = PARTS - 1; i >= 0; --i) acc_o[o % kMBlocks] = mfma32(x, pop[i][o / kMBlocks], acc_o[o % kMBlocks]);
        } else {
          sacc[o & 1] = mfma32(x, qreg[(o - kNV) / 2], sacc[o & 1]);
        }
        if (o + kDepth < kLast) read(o + kDepth);
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    constexpr std::integral_constant<bool, true> kYes{};
    constexpr std::integral_constant<bool, false> kNo{};
    auto pv_part = [&](auto is_cached, int slot) __attribute__((always_inline)) { products(is_cached, kYes, kNo, 0, slot); };
    auto qk_part = [&](int slot) __attribute__((always_inline)) { products(kCached, kNo, kYes, slot, 0); };
    // Steady-state MFMA phase, at raised wave priority.
    auto mfma_phase = [&](auto is_cached, int slot_k, int slot_v) __attribute__((always_inline)) {
      __builtin_amdgcn_s_setprio(1);
      products(is_cached, kYes, kYes, slot_k, slot_v);
      __builtin_amdgcn_s_setprio(0);
    };

    // Whether this lane's row sees a key: with c the key's place in its run of 8 h2 .. (a
    // constant where it is used), comparisons with a few limits of the tile, of which a
    // register each is enough.
    struct Limits { int end, sinks, from, wrap, from2; };
    auto limits_of = [&](bool of_cache, int kb) __attribute__((always_inline)) {
      const int at = kb + 8 * h2;
      Limits x;
      if (of_cache) {  // c < end and (c < sinks or from <= c <= wrap or c >= from2)
        x.end = cached - at;
        x.sinks = n_sink - at;
        x.from = lo_off + my_t - item.rbase + n_sink - at;
        x.wrap = item.rrem + n_sink - at;
        x.from2 = x.from + window;
        if (!str) x.sinks = x.end;
      } else {  // c <= my_t and (c < sinks or c >= from)
        x.end = my_t + 1 - at;
        x.sinks = n_sink - start - at;
        x.from = lo_off + my_t - start - at;
        x.wrap = INT32_MAX;
        x.from2 = x.from;
      }
      return x;
    };
    // c of score i of block blk
    auto place_of = [&](int blk, int i) __attribute__((always_inline)) { return 32 * blk + 16 * (i >> 3) + (i & 7); };
    auto sees = [&](auto of_cache, const Limits& x, int c) __attribute__((always_inline)) {
      if constexpr (decltype(of_cache)::value)
        return (c < x.end) & ((c < x.sinks) | ((c >= x.from) & (c <= x.wrap)) | (c >= x.from2));
      else
        return (c < x.end) & ((c < x.sinks) | (c >= x.from));
    };
    auto apply_mask = [&](auto of_cache, int kb) __attribute__((always_inline)) {
      const Limits x = limits_of(decltype(of_cache)::value, kb);
#pragma unroll
      for (int blk = 0; blk < 2; ++blk)
#pragma unroll
        for (int i = 0; i < 16; ++i) sacc[blk][i] = sees(of_cache, x, place_of(blk, i)) ? sacc[blk][i] : -INFINITY;
    };
    // Exponentials against m_use into the P^T operands; their sum.
    auto exps = [&]() __attribute__((always_inline)) {
      float psum[4];
#pragma unroll
      for (int blk = 0; blk < 2; ++blk)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          float pf[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            pf[i] = fast_exp2(fmaf(sacc[blk][8 * hf + i], c, -m_use));
            const bf16 p0 = f32_to_bf16(pf[i]);
            pop[0][2 * blk + hf][i] = p0;
            if constexpr (PARTS == 3) {
              const float r1 = pf[i] - (float)p0;
              const bf16 p1 = f32_to_bf16(r1);
              pop[1][2 * blk + hf][i] = p1;
              pop[2][2 * blk + hf][i] = f32_to_bf16(r1 - (float)p1);
            }
          }
          if constexpr (PARTS == 1 && ROWS == 128) {
            // The rounded weights' sum, so that they sum to 1 as the product takes them: a
            // fifth less error in the output (relative 0.0019 instead of 0.0023, its own
            // rounding alone 0.0016).  In blocks of 256 rows the dot products cost 7 to 12%
            // (4096 tokens after 126976 3.99 -> 4.41 ms, 2048 after 28672 448 -> 480 us, packed
            // messages 267 -> 298), so those sum the weights as they were before the rounding.
            // In blocks of 128 they cost 1.3% at most, long chunks included (width 64: 2048 after
            // 28672 344 -> 348 us, 4096 after 60000 1412 -> 1417, chunks with eviction 138 -> 133;
            // width 128: 60 tokens of 8 sequences at 32700 211 -> 214).
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
            const bf16x2 one = {(__bf16)1.f, (__bf16)1.f};
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < 8; i += 2) s = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pop[0][2 * blk + hf][i], pop[0][2 * blk + hf][i + 1]}, one, s, false);
            psum[2 * blk + hf] = s;
          } else {
            psum[2 * blk + hf] = ((pf[0] + pf[1]) + (pf[2] + pf[3])) + ((pf[4] + pf[5]) + (pf[6] + pf[7]));
          }
        }
      return (psum[0] + psum[1]) + (psum[2] + psum[3]);
    };
    auto softmax_tile = [&]() __attribute__((always_inline)) {
      float tsum = exps();
      const bool off = !(tsum <= kSumHi) || m_run == -INFINITY;
      if (__any(off)) {
        // only the rows that need it move: a row's result is its own
        const bool moves = xor32_max(off ? 1.f : 0.f) > 0.f;
        float mx = -INFINITY;
#pragma unroll
        for (int blk = 0; blk < 2; ++blk)
#pragma unroll
          for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sacc[blk][i]);
        mx = xor32_max(mx) * c;
        const float m_new = moves ? fmaxf(m_run, mx) : m_run;
        const float alpha = (m_new == -INFINITY) ? 1.f : fast_exp2(m_run - m_new);
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int mb = 0; mb < kMBlocks; ++mb)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc_o[mb][i] = CAREFUL ? scaled(acc_o[mb][i], alpha) : acc_o[mb][i] * alpha;
        m_use = (m_run == -INFINITY) ? 0.f : m_run;
        tsum = exps();
      }
      l_run += tsum;
    };

    barrier();  // the ring's last use (the range's previous item) is over
    if constexpr (!CAREFUL) {
      auto valu_phase = [&](auto is_cached, int kb) __attribute__((always_inline)) {
        constexpr bool of_cache = decltype(is_cached)::value;
        bool dead = false, mask;
        if constexpr (of_cache) {
          mask = kb + kBN > cached || band;
        } else {
          dead = kb > w_t1 || (start + kb >= n_sink && start + kb + kBN - 1 < lo_off + w_t0);
          mask = kb + kBN - 1 > w_t0 || !(start + kb + kBN - 1 < n_sink || start + kb >= lo_off + w_t1);
        }
        if (dead) {  // no row of the wave sees a key
#pragma unroll
          for (int i = 0; i < PARTS; ++i)
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
#pragma unroll
              for (int e = 0; e < 8; ++e) pop[i][ks][e] = (bf16)0.f;
          return;
        }
        if (mask) apply_mask(is_cached, kb);
        softmax_tile();
      };
      // Slots of the tile that is loaded next, of the tile whose K and of the one whose V is
      // read next.
      int in_k = 0, in_v = 0, at_k = 0, at_v = 0;
      asm("" : "+s"(at_k));  // not known to be 0: no addresses of slot 0 are kept
      auto next_k = [&](int& x) __attribute__((always_inline)) { x = x + 1 == Shape::kKSlots ? 0 : x + 1; };
      auto next_v = [&](int& x) __attribute__((always_inline)) { x = x + 1 == Shape::kVSlots ? 0 : x + 1; };
      // First keys of the current tile and of the next ones, up to the one that is loaded next.
      int kbs[Shape::kAhead + 1];
#pragma unroll
      for (int u = 0; u <= Shape::kAhead; ++u) kbs[u] = item.tile(v0 + u) * kBN;
      // Block table entries of this wave's page in 64 tiles, one a lane: a load waits for the
      // direct loads before it, and a scalar one would make every LDS read behind it wait for
      // all of them.
      int entries = 0, entries0 = 0;
      auto read_entries = [&](int it) __attribute__((always_inline)) {
        entries0 = it;
        entries = item_table[min((it + lane) * (kBN / kPage) + my_page, last_page)];
        __builtin_amdgcn_s_waitcnt(kWaitVm0);  // here, not at every use
      };
      auto issue = [&](int it, int kb) __attribute__((always_inline)) {
        if (it < item.n_cached) {
          int page = min(kb / kPage + my_page, last_page);
          if (!str) {
            if (it - entries0 == kWave) read_entries(it);
            page = __builtin_amdgcn_readlane(entries, it - entries0);
          }
          issue_cached(in_k, in_v, page);
        } else {
          issue_new(kb, in_k, in_v);
        }
        next_k(in_k);
        next_v(in_v);
      };
      // The barrier of a tile follows each wave's wait for its loads of the next one (with
      // loads three tiles ahead those of the one after may stay in flight); after it, the
      // tile kAhead further goes into slots whose last reads every wave has completed.
      auto sync_tile = [&](int it) __attribute__((always_inline)) {
        if (Shape::kAhead > 2 && it + 2 < v1) __builtin_amdgcn_s_waitcnt(wait_vm(2 * Shape::kLoads));
        else __builtin_amdgcn_s_waitcnt(kWaitVm0);
        if (it + 1 < v1) {
          int s = in_v - (Shape::kAhead - 1);  // the next tile's slot
          if (it + Shape::kAhead > v1) s += it + Shape::kAhead - v1;
          clean(it + 1, kbs[1], s < 0 ? s + Shape::kVSlots : s);
        }
        __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
        barrier();
        if (it + Shape::kAhead < v1) issue(it + Shape::kAhead, kbs[Shape::kAhead]);
      };

      // Prologue: the first tiles and this wave's Q rows, then everything complete.
      if (!str && v0 < item.n_cached) read_entries(v0);
#pragma unroll
      for (int u = 0; u < Shape::kAhead; ++u)
        if (v0 + u < v1) issue(v0 + u, kbs[u]);
      {
        const uint16_t* qp = static_cast<const uint16_t*>(a.q) + q_at;
#pragma unroll
        for (int s = 0; s < kKSteps; ++s) qreg[s] = __builtin_bit_cast(bf16x8, ld16(qp + 8 * h2 + 16 * s));
      }
      __builtin_amdgcn_s_waitcnt(kWaitVm0);
      clean(v0, kbs[0], 0);
      __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
      barrier();

      auto next_kbs = [&](int it) __attribute__((always_inline)) {
        const int kb_next = item.tile(it + 1 + Shape::kAhead) * kBN;
#pragma unroll
        for (int u = 0; u < Shape::kAhead; ++u) kbs[u] = kbs[u + 1];
        kbs[Shape::kAhead] = kb_next;
      };
      // Every wave runs MFMA, vector phase, MFMA, ..: waves 0-3 take the barrier of a tile
      // after its vector phase, waves 4-7 after its MFMA phase.
      auto vector_phase = [&](auto is_cached, int it) __attribute__((always_inline)) {
        if (grp == 1) sync_tile(it);
        valu_phase(is_cached, kbs[0]);
        if (grp == 0) sync_tile(it);
        next_kbs(it);
      };
      auto run_tiles = [&](auto is_cached, int i0, int i1) __attribute__((always_inline)) {
        qk_part(at_k);
        next_k(at_k);
        vector_phase(is_cached, i0);
#pragma unroll 1
        for (int it = i0 + 1; it < i1; ++it) {
          mfma_phase(is_cached, at_k, at_v);
          next_k(at_k);
          next_v(at_v);
          vector_phase(is_cached, it);
        }
        pv_part(is_cached, at_v);
        next_v(at_v);
      };
      const int mid = min(max(item.n_cached, v0), v1);
      if (item.row0 + wave * 32 < n_rows) {
        if (v0 < mid) run_tiles(kCached, v0, mid);
        if (mid < v1) run_tiles(kNew, mid, v1);
        float zero = 0.f;  // NaN if a sum is not finite
#pragma unroll
        for (int mb = 0; mb < kMBlocks; ++mb)
#pragma unroll
          for (int i = 0; i < 16; i += 2) zero = fmaf(acc_o[mb][i], 0.f, fmaf(acc_o[mb][i + 1], 0.f, zero));
        bad = bad || __any(zero != zero);
      } else {  // a wave without rows takes part in the loads
#pragma unroll 1
        for (int it = v0; it < v1; ++it) {
          sync_tile(it);
          next_kbs(it);
        }
      }

      // Has a wave met what the loop above cannot take?  (The ring is free.)
      barrier();
      int* flags = reinterpret_cast<int*>(&ring.k[0][0]);
      if (lane == 0) flags[wave] = bad;
      __syncthreads();
      int any = 0;
#pragma unroll
      for (int w = 0; w < ROWS / 32; ++w) any |= flags[w];
      again = again || __builtin_amdgcn_readfirstlane(any);
    } else {
      const uint16_t* qp = static_cast<const uint16_t*>(a.q) + q_at;
#pragma unroll
      for (int s = 0; s < kKSteps; ++s) qreg[s] = __builtin_bit_cast(bf16x8, ld16(qp + 8 * h2 + 16 * s));
#pragma unroll 1
      for (int it = v0; it < v1; ++it) {
        const bool of_cache = it < item.n_cached;
        const int kb = item.tile(it) * kBN;
        __syncthreads();
        const int page = min(kb / kPage + my_page, last_page);
        if (of_cache) issue_cached(0, 0, str ? page : item_table[page]);
        else issue_new(kb, 0, 0);
        __builtin_amdgcn_s_waitcnt(kWaitVm0);
        clean(it, kb, 0);
        __syncthreads();
        uint32_t pages = 0;  // the tile's pages that are none
        if (of_cache && !str)
          for (int i = 0; i < kBN / kPage; ++i) {
            const int e = item_table[min(kb / kPage + i, last_page)];
            if (e < 0 || e >= end_page) pages |= 1u << i;
          }
        const Limits x = limits_of(of_cache, kb);
        auto seen = [&](int c) __attribute__((always_inline)) {
          return (of_cache ? sees(kCached, x, c) : sees(kNew, x, c)) && !((pages >> ((c + 8 * h2) / kPage)) & 1u);
        };
        qk_part(0);
#pragma unroll
        for (int blk = 0; blk < 2; ++blk)
#pragma unroll
          for (int i = 0; i < 16; ++i) sacc[blk][i] = seen(place_of(blk, i)) ? sacc[blk][i] : -INFINITY;
        softmax_tile();
        // P.V with the finite values; of the others that a row sees the infinities are counted in
        // units of 1 and 128, NaNs in units of 16384 (a tile has 64 keys, so the counts are exact
        // and keep apart).
#pragma unroll
        for (int mb = 0; mb < kMBlocks; ++mb) {
          f32x16 hits;
#pragma unroll
          for (int i = 0; i < 16; ++i) hits[i] = 0.f;
#pragma unroll
          for (int ks = 0; ks < 4; ++ks) {
            const bf16x8 v = of_cache ? v_operand(kCached, paddr0 + 1024u * mb, ks) : v_operand(kNew, vaddr0 ^ (64u * mb), ks);
            const i16x8 bits = __builtin_bit_cast(i16x8, v);
            i16x8 fin;
            bf16x8 ind, on;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const bool out = (bits[e] & 0x7f80) == 0x7f80;
              fin[e] = out ? (short)0 : bits[e];
              ind[e] = (bf16)(!out ? 0.f : (bits[e] & 0x7f) ? 16384.f : bits[e] < 0 ? 128.f : 1.f);
              on[e] = (bf16)(sacc[ks >> 1][8 * (ks & 1) + e] == -INFINITY ? 0.f : 1.f);  // hidden, or weight 0
            }
#pragma unroll
            for (int i = PARTS - 1; i >= 0; --i) acc_o[mb] = mfma32(__builtin_bit_cast(bf16x8, fin), pop[i][ks], acc_o[mb]);
            hits = mfma32(ind, on, hits);
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int n = (int)hits[i];
            float x = acc_o[mb][i];
            if (n & 0x7f) x += INFINITY;
            if (n & 0x3f80) x -= INFINITY;
            acc_o[mb][i] = n >> 14 ? __builtin_nanf("") : x;
          }
        }
      }
    }

    const float l_tot = xor32_sum(l_run);
    if (whole) {
      const float inv = 1.f / l_tot;
      if (item.row0 + wave * 32 + l32 < n_rows) {
        const int64_t at = item.o_off + my_t * a.o_st + (my_r - my_t * a.gs) * a.o_sh;
#pragma unroll
        for (int mb = 0; mb < kMBlocks; ++mb)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            f32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = acc_o[mb][4 * q4 + e] * inv;
            store4<PARTS == 3>(a, at + 32 * mb + 8 * q4 + 4 * h2, w);
          }
      }
    } else {
      const int64_t at = part + wave * 32 + l32;
#pragma unroll
      for (int mb = 0; mb < kMBlocks; ++mb)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          f32x4 w;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = acc_o[mb][4 * q4 + e];
          *reinterpret_cast<f32x4*>(a.part_acc + at * D + 32 * mb + 8 * q4 + 4 * h2) = w;
        }
      if (h2 == 0) {
        a.part_ml[at * 2 + 0] = m_run;
        a.part_ml[at * 2 + 1] = l_tot;
      }
    }
  }
  return again;
}

// The careful loop is a function of its own (with the arguments from memory): inlined, it
// would take registers from the fast one.
template <int D, int ROWS, int PARTS>
__device__ __attribute__((noinline)) void extend_again(const ExtendArgs* a, TileRing<D, ROWS>* ring) {
  extend_range<D, ROWS, PARTS, true>(*a, *ring);
}

template <int D, int ROWS, int PARTS>
__global__ __launch_bounds__(2 * ROWS, (D == 64 && PARTS == 1 ? 3 : 2)) void extend_tile_kernel(ExtendArgs a) {
  __shared__ __align__(1024) TileRing<D, ROWS> ring;
  if (extend_range<D, ROWS, PARTS, false>(a, ring)) extend_again<D, ROWS, PARTS>(a.copy, &ring);
}

// ---------------------------------------------------------------------------
// Items that several workgroups share: one row a wave, its lanes over groups of partials
// and the dimensions.  The workgroups' x is the range that an item starts in.  Bound: the
// partials' bytes (packed messages: 67 MB of 256-row blocks, 25-30 us), for few items the
// chain head -> item -> partials, 8.5 us; eight rows one after the other in a wave took 60.
template <int D, int ROWS>
__global__ __launch_bounds__(256) void extend_merge_kernel(ExtendArgs a) {
  constexpr int kLanes = D / 4, kGroups = kWave / kLanes;
  const int lane = threadIdx.x & 63;
  const int row = blockIdx.y * 4 + (threadIdx.x >> 6);
  const ExtendHead head = scalar_load(a.head);
  const int rng = blockIdx.x;
  if (rng + 1 >= head.used) return;
  // the item that goes on behind the range's end
  const int64_t g0 = rng * head.range, g1 = g0 + head.range;
  const ExtendItem item = scalar_load(a.items + scalar_load(a.first_item + rng + 1));
  if (item.first < g0 || item.first >= g1) return;  // starts before this range, or behind it
  const int r = item.row0 + row;
  if (r >= item.n_new * a.gs) return;
  const int last = (int)div64(item.first + item.places - 1, head.range);
  auto slot = [&](int w) { return (int64_t)(2 * w + (w == rng ? 1 : 0)) * ROWS + row; };
  // a partial without a key has m = -inf and l = 0 (keys with NaN scores leave a NaN sum)
  float M = -INFINITY;
  for (int w = rng + lane; w <= last; w += kWave) M = fmaxf(M, a.part_ml[slot(w) * 2]);
#pragma unroll
  for (int i = 1; i < kWave; i *= 2) M = wave_xor_max(M, i);
  float L;
  f32x4 o;
  // INF: an infinity stays one where its factor is below fp32's range
  auto join = [&](auto inf_c) __attribute__((always_inline)) {
    constexpr bool INF = decltype(inf_c)::value;
    constexpr int kUnroll = INF ? 1 : 8;
    L = 0.f;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll kUnroll
    for (int w = rng + lane / kLanes; w <= last; w += kGroups) {
      const int64_t at = slot(w);
      const float m = a.part_ml[at * 2], l = a.part_ml[at * 2 + 1];
      const f32x4 x = *reinterpret_cast<const f32x4*>(a.part_acc + at * D + 4 * (lane % kLanes));
      const bool none = m == -INFINITY && l == 0.f;
      const float f = none ? 0.f : m == -INFINITY ? 1.f : fast_exp2(m - M);
      L += f * l;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += none ? 0.f : INF ? scaled(x[e], f) : f * x[e];
    }
#pragma unroll
    for (int i = kLanes; i < kWave; i *= 2) {
      L = wave_xor_sum(L, i);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = wave_xor_sum(o[e], i);
    }
  };
  join(std::integral_constant<bool, false>{});
  if (__any(__builtin_isunordered(o[0], o[1]) || __builtin_isunordered(o[2], o[3]))) join(std::integral_constant<bool, true>{});
  if (lane >= kLanes) return;
  const float inv = 1.f / L;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] *= inv;
  const int t = div_gs(a, r);
  const int64_t at = item.o_off + t * a.o_st + (r - t * a.gs) * a.o_sh + 4 * lane;
  if (a.out_f32) store4<true>(a, at, o);
  else store4<false>(a, at, o);
}

template <int D, int ROWS>
static hipError_t launch_tiles(ExtendArgs a, hipStream_t s) {
  a.wgs = a.cus * (ROWS == 256 ? 1 : D == 64 && !a.out_f32 ? 3 : 2);
  // Smallest range: 17 tokens after 4093 29.9 us with 2 tiles, 32.5 with 1 (more partials to
  // merge), 34.9 with 4.
  a.min_tiles = 2;
  // An item's start costs as much as so many tiles (its first loads, its stores).  No number is
  // best for all calls, and these lie between.  Blocks of 256 rows with 8, 12, 14 and 20 tiles:
  // 2048 tokens after 28672 486, 459, 457 and 455 us, packed messages 264, 271, 273 and 275, chunks
  // of four sequences with eviction 194, 200, 202 and 209.  Blocks of 128 with 3, 8, 12 and 14:
  // packed chunks of width 64 with fp32 outputs 612, 635, 650 and 658, with bf16 ones 396, 364, 357
  // and 347, 4 tokens of 8 sequences at 32700 134 to 135 with each.
  a.item_cost = ROWS == 256 ? 12 : 8;
  a.block_step = std::max(1, kUnit * ROWS / (kBN * a.gs));
  a.block_tiles = ((ROWS + a.gs - 1) / a.gs + kBN - 1) / kBN;
  a.band_tiles = (a.n_sink + kBN - 1) / kBN + (a.window + kBN - 1) / kBN + a.block_tiles + 1;
  a.part_acc = static_cast<float*>(a.workspace);
  a.part_ml = a.part_acc + (int64_t)2 * a.wgs * ROWS * D;
  a.head = reinterpret_cast<ExtendHead*>(a.part_ml + (int64_t)2 * a.wgs * ROWS * 2);
  a.copy = reinterpret_cast<ExtendArgs*>(a.head + 1);
  a.items = reinterpret_cast<ExtendItem*>(a.copy + 1);
  const int64_t rows = (a.cu_seqlens ? std::min<int64_t>(a.total, (int64_t)a.B * a.T) : (int64_t)a.B * a.T) * a.gs;
  const int64_t n_items = (a.n_ret + a.n_str) * (rows / ROWS + a.B);  // at most
  a.max_items = (int)n_items;
  a.first_item = reinterpret_cast<int32_t*>(a.items + n_items);
  const int plan_wgs = (int)std::min<int64_t>((n_items + 255) / 256, a.cus);
  hipLaunchKernelGGL((extend_plan_kernel<ROWS, kBN>), dim3(plan_wgs), dim3(256), 0, s, a);
  if (hipError_t e = hipGetLastError()) return e;
  const dim3 grid((a.wgs + 7) / 8 * 8);
  if (a.out_f32) hipLaunchKernelGGL((extend_tile_kernel<D, ROWS, 3>), grid, dim3(2 * ROWS), 0, s, a);
  else hipLaunchKernelGGL((extend_tile_kernel<D, ROWS, 1>), grid, dim3(2 * ROWS), 0, s, a);
  if (hipError_t e = hipGetLastError()) return e;
  hipLaunchKernelGGL((extend_merge_kernel<D, ROWS>), dim3(a.wgs - 1, (unsigned)((std::min<int64_t>(ROWS, (int64_t)a.T * a.gs) + 3) / 4)), dim3(256), 0, s, a);
  return hipGetLastError();
}

// Bytes of the partials of the largest launch (two blocks of rows a workgroup), and of the
// plan of so many tokens in so many sequences.
size_t extend_workspace(int64_t batch, int64_t tokens, int hq, int hkv, int d, int cus) {
  const size_t rows = d == 64 ? 128 * 3 : 256;
  const size_t items = (size_t)hkv * (tokens * (hq / hkv) / 128 + batch);
  return (size_t)2 * cus * rows * (d + 2) * sizeof(float) + sizeof(ExtendHead) + sizeof(ExtendArgs) + items * sizeof(ExtendItem) + 3 * cus * sizeof(int32_t);
}

hipError_t launch_extend(const ExtendArgs& a, int dtype, int d, hipStream_t s) {
  if (dtype == 1) return d == 64 ? launch_simple<64>(a, s) : launch_simple<128>(a, s);
  for (int b0 = 0; b0 < a.B; b0 += kPlanSeqs) {
    ExtendArgs x = a;
    x.B = std::min(kPlanSeqs, a.B - b0);
    x.q = static_cast<const uint16_t*>(a.q) + b0 * a.q_sb;
    x.k = static_cast<const uint16_t*>(a.k) + b0 * a.k_sb;
    x.v = static_cast<const uint16_t*>(a.v) + b0 * a.v_sb;
    x.out = static_cast<char*>(a.out) + b0 * a.o_sb * (a.out_f32 ? 4 : 2);
    if (a.start_pos) x.start_pos += b0;
    if (a.cu_seqlens) x.cu_seqlens += b0;
    if (a.n_ret) x.block_table += (int64_t)b0 * a.max_pages;
    if (a.n_str) {
      const int64_t ring = (int64_t)b0 * a.n_str * a.ring_blocks * (kPage * d);
      x.rk = static_cast<const uint16_t*>(a.rk) + ring;
      x.rv = static_cast<const uint16_t*>(a.rv) + ring;
    }
    hipError_t e;
    // Blocks of 256 rows, one workgroup a CU, where a sequence can fill one: 2048 tokens after
    // 28672 448 us (534 in blocks of 128), 4096 after 126976 3.99 ms (4.48), 2048 after 28672
    // packed with 32 single tokens at 4000 860 us (884); 200 tokens after 4000 packed with 63 single
    // ones at 30000 721 (716).  Two workgroups of 128 rows a CU else: 4 tokens of 8 sequences at
    // 32700 135 us (138 in blocks of 256), 17 tokens after 4093 29.9 (31.2).
    if (d == 64) e = launch_tiles<64, 128>(x, s);
    else if ((int64_t)a.T * a.gs >= 256) e = launch_tiles<128, 256>(x, s);
    else e = launch_tiles<128, 128>(x, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace aoh
