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

// Position that ring slot c holds when `start` tokens have been written, or -1.
__device__ __forceinline__ int ring_position(int c, int start, int n_sink, int window) {
  if (c < n_sink) return c < start ? c : -1;
  const int r = c - n_sink, last = start - 1 - n_sink;  // offsets behind the sinks
  if (r >= window || last < r) return -1;
  return n_sink + last - (last - r) % window;
}

// ---------------------------------------------------------------------------
// The work space.  An item's places: kUnit for each tile that its rows visit, about (a
// first number and a step from one block of rows to the next), and kItemCost tiles for its
// start.  A range of places stands for the same share of the item's visits, so the numbers
// need not be exact.
constexpr int kUnit = 16;
constexpr int kItemCost = 1;
constexpr int kPlanSeqs = 64;  // sequences of a launch, one a lane; larger batches go in parts

struct ExtendPlan {
  int64_t n_ret_places, total;  // places of the retrieval items, of all items
  int64_t range;                // places of a workgroup
  int used;                     // workgroups with a range
  // this lane's sequence: first places of its retrieval and streaming items, places of one
  // head's items, of the first block of rows, and the step
  int64_t ret0, ret_head, ret_a, str0, str_head, str_a;
  int ret_c, str_c;
  int blocks;  // blocks of rows
};

__device__ __forceinline__ int64_t lane_scan(int64_t x) {
  const int lane = threadIdx.x & (kWave - 1);
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int64_t y = __shfl_up(x, o, kWave);
    if (lane >= o) x += y;
  }
  return x;
}
__device__ __forceinline__ int64_t from_lane(int64_t x, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)x, lane), hi = __builtin_amdgcn_readlane((uint32_t)(x >> 32), lane);
  return (int64_t)(((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ int div_up(int a, int b) { return (a + b - 1) / b; }
// Places of the first n of an item's blocks of rows.
__device__ __forceinline__ int64_t places_of(int64_t a, int c, int64_t n) { return n * a + c * (n * (n - 1) / 2); }

template <int ROWS, int TILE>
__device__ __forceinline__ ExtendPlan extend_plan(const ExtendArgs& a) {
  const int lane = threadIdx.x & (kWave - 1);
  ExtendPlan p;
  ExtendSeq s = {0, 0, 0};
  if (lane < a.B) s = extend_seq(a, lane);
  p.blocks = (int)(((int64_t)s.n * a.gs + ROWS - 1) / ROWS);
  const int step = max(1, kUnit * ROWS / (TILE * a.gs));  // new tiles that the next block of rows sees more
  const int n_new = div_up(s.n, TILE), first = div_up(div_up(ROWS, a.gs), TILE);
  const int paged = div_up(min(s.start, a.max_pages * kPage), TILE);
  const int ring = div_up(min(s.start, a.ring_cap), TILE);
  p.ret_a = (int64_t)kUnit * (kItemCost + paged + min(n_new, first));
  p.ret_c = step;
  // the band of a block has at most window + tokens of the block keys
  const int band = div_up(a.n_sink, TILE) + div_up(a.window, TILE) + first + 1;
  p.str_a = (int64_t)kUnit * (kItemCost + (a.evict ? ring + min(n_new, first) : min(ring + n_new, band)));
  p.str_c = a.evict ? step : 0;
  p.ret_head = places_of(p.ret_a, p.ret_c, p.blocks);
  p.str_head = places_of(p.str_a, p.str_c, p.blocks);
  const int64_t ret = a.n_ret * p.ret_head, str = a.n_str * p.str_head;
  const int64_t ret_to = lane_scan(ret), str_to = lane_scan(str);
  p.n_ret_places = from_lane(ret_to, kWave - 1);
  p.total = p.n_ret_places + from_lane(str_to, kWave - 1);
  p.ret0 = ret_to - ret;
  p.str0 = p.n_ret_places + str_to - str;
  p.range = max((p.total + a.wgs - 1) / a.wgs, (int64_t)a.min_tiles * kUnit);
  p.used = (int)((p.total + p.range - 1) / p.range);
  return p;
}

// Ranges go to the 8 XCDs (each with its own L2) in eight consecutive parts, so that the
// blocks of rows that share K/V run on one.  Returns the range of workgroup w, or -1.
__device__ __forceinline__ int range_of(int w, int used) {
  const int per = (used + 7) >> 3, r = (w & 7) * per + (w >> 3);
  return (w >> 3) < per && r < used ? r : -1;
}

struct ExtendItem {
  int b, kvl, rb;  // sequence, rank of the KV head in its cache, block of rows
  bool str;
  int64_t first, places;
};

// The item that holds place g < total.
__device__ __forceinline__ ExtendItem extend_item(const ExtendPlan& p, int64_t g, int n_ret, int n_str) {
  ExtendItem it;
  it.str = g >= p.n_ret_places;
  const int64_t at = it.str ? p.str0 : p.ret0, head = it.str ? p.str_head : p.ret_head;
  const uint64_t hit = __ballot(g >= at && g < at + head * (it.str ? n_str : n_ret));
  it.b = hit ? __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(hit)) : 0;
  const int64_t at_b = from_lane(at, it.b), head_b = from_lane(head, it.b);
  const int64_t a = from_lane(it.str ? p.str_a : p.ret_a, it.b);
  const int c = __builtin_amdgcn_readlane(it.str ? p.str_c : p.ret_c, it.b);
  it.kvl = (int)((g - at_b) / head_b);
  const int64_t base = at_b + it.kvl * head_b, off = g - base;
  int lo = 0, hi = __builtin_amdgcn_readlane(p.blocks, it.b);  // the last block that starts at or before off
  if (c == 0) {
    lo = (int)(off / a);
  } else {
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (places_of(a, c, mid) <= off) lo = mid;
      else hi = mid;
    }
  }
  it.rb = lo;
  it.first = base + places_of(a, c, lo);
  it.places = a + (int64_t)c * lo;
  return it;
}

// The tiles that an item's rows visit: up to three runs of cached tiles, then up to two of
// new ones.
struct Visits {
  int n_cached, n;          // visits of the cache, all visits
  int c1, c2, o0, o1, o2;   // cached: tile = visit + o0 below c1, + o1 below c2, + o2
  int d1, e0, e1;           // new: the same with the visit's place behind n_cached
  __device__ __forceinline__ int tile(int it) const {
    if (it < n_cached) return it + (it < c1 ? o0 : it < c2 ? o1 : o2);
    const int j = it - n_cached;
    return j + (j < d1 ? e0 : e1);
  }
};

// Rows of tokens t0 .. t1 of a sequence; cached: what its cache holds (positions, or slots).
template <int TILE>
__device__ __forceinline__ Visits visits_of(const ExtendArgs& a, bool str, int start, int cached, int t0, int t1) {
  Visits v;
  const int all = div_up(cached, TILE), n_new = t1 / TILE + 1;
  v.o0 = v.o1 = v.o2 = v.e0 = v.e1 = 0;
  if (!str) {
    v.n_cached = v.c1 = v.c2 = all;
    v.d1 = n_new;
    v.n = all + n_new;
    return v;
  }
  const int lo = a.evict ? start - a.window : start + t0 - a.window + 1;
  const int w0 = max(lo, a.n_sink);  // first cached position of the window
  const int sinks = div_up(min(a.n_sink, cached), TILE);
  int f1 = sinks, l1 = sinks, f2 = 0, l2 = 0;  // runs of window tiles
  if (w0 < start) {
    const int x = a.n_sink + (w0 - a.n_sink) % a.window, y = a.n_sink + (start - 1 - a.n_sink) % a.window;
    if (start - w0 >= a.window) {
      l1 = all;
    } else if (x <= y) {
      f1 = max(sinks, x / TILE);
      l1 = y / TILE + 1;
    } else {
      f1 = max(sinks, a.n_sink / TILE);
      l1 = y / TILE + 1;
      f2 = max(max(f1, l1), x / TILE);
      l2 = all;
    }
  }
  v.c1 = sinks;
  v.c2 = sinks + max(0, l1 - f1);
  v.n_cached = v.c2 + max(0, l2 - f2);
  v.o1 = f1 - v.c1;
  v.o2 = f2 - v.c2;
  const int d0 = max(0, lo - start) / TILE;  // first new tile of the window
  const int new_sinks = min(div_up(max(0, a.n_sink - start), TILE), d0);
  v.d1 = new_sinks;
  v.e1 = d0 - new_sinks;
  v.n = v.n_cached + new_sinks + n_new - d0;
  return v;
}

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
    const int n_cached = str ? min(s.start, a.ring_cap) : min(s.start, a.max_pages * kPage);
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
      for (int i = 0; i < kDims; ++i) o[i] *= alpha;
      for (int i = 0; i < kWave; ++i) {
        const int64_t at = s_at[wave][i];
        if (at < 0) continue;
        const bool cached = k0 + i < n_cached;
        vp = cached ? (str ? a.rv : a.pv) : a.v;
#pragma unroll
        for (int u = 0; u < kDims; ++u) o[u] += s_p[wave][i] * value(vp, at + (int64_t)(lane + kWave * u) * (cached ? kPage : 1));
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
        x += f * s_o[w][tid];
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
// Bound: the matrix cores, and the LDS reads that feed them.
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
// not 0 if it is not finite: the waves look for such values in the tiles that are masked,
// and a workgroup that has met one (or a page outside the cache) takes its range again in
// the careful loop.
template <int D, int ROWS>
struct TileShape {
  static constexpr int kThreads = 2 * ROWS;
  static constexpr bool kPair = ROWS == 256;
  static constexpr int kAhead = kPair ? 3 : 2;
  static constexpr int kKSlots = kPair ? 4 : D == 128 ? 2 : 3;
  static constexpr int kVSlots = kPair ? 4 : 3;
  static constexpr int kWavesPerSimd = D == 64 ? 3 : 2;
  static constexpr int kLoads = kBN * (D / 8) / kThreads;  // loads per thread and tile, K or V
  static constexpr int kWgsPerCu = kPair ? 1 : D == 64 ? 3 : 2;
};

template <int D, int ROWS>
struct TileRing {
  uint16_t k[TileShape<D, ROWS>::kKSlots][kBN * D];
  uint16_t v[TileShape<D, ROWS>::kVSlots][kBN * D];
};

// Largest sum of a lane's 32 exponentials of one tile, taken against the trailing
// reference max, that is accepted as it is.
constexpr float kSumHi = 65536.f;

// A block table entry, by a scalar load (the address is uniform): it is waited for with the
// LDS reads, not with the direct loads.
__device__ __forceinline__ int scalar_i32(const int32_t* p) {
  return *(const __attribute__((address_space(4))) int32_t*)(uintptr_t)p;
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
  auto k_operand = [&](uint32_t at, int s, int blk) __attribute__((always_inline)) {
    typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
    return *reinterpret_cast<lds_bf16x8*>((at ^ (32u * s)) + 64u * D * blk);
  };
  // cached: a tile of pages, else of new rows
  auto v_operand = [&](auto cached, uint32_t at, int ks, int mb) __attribute__((always_inline)) {
    if constexpr (decltype(cached)::value) {
      typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
      return *reinterpret_cast<lds_bf16x8*>(at + 32u * D * ks + 1024u * mb);
    } else {
      typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
      const uint32_t x = (at ^ (64u * mb)) + 32u * D * ks;
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

  bool again = false;
  int64_t g0 = -1;
#pragma unroll 1
  for (;;) {
    // The plan is made anew for every item, which costs less than the registers that would
    // hold it through the tiles.
    const ExtendPlan plan = extend_plan<ROWS, kBN>(a);
    const int rng = range_of(blockIdx.x, plan.used);
    if (rng < 0) return false;
    const int64_t g1 = min((rng + 1) * plan.range, plan.total);
    if (g0 < 0) g0 = rng * plan.range;
    if (g0 >= g1) return again;
    const ExtendItem item = extend_item(plan, g0, a.n_ret, a.n_str);
    const ExtendSeq seq = extend_seq(a, item.b);
    const bool str = item.str;
    const int g = a.kv_heads[str ? a.n_ret + item.kvl : item.kvl];
    const int start = __builtin_amdgcn_readfirstlane(seq.start), n_new = __builtin_amdgcn_readfirstlane(seq.n);
    const int n_rows = n_new * a.gs, row0 = item.rb * ROWS;
    const int cached = str ? min(start, a.ring_cap) : min(start, a.max_pages * kPage);
    const int t_first = row0 / a.gs, t_last = (min(row0 + ROWS, n_rows) - 1) / a.gs;
    const Visits vis = visits_of<kBN>(a, str, start, cached, t_first, t_last);
    // the share of the visits that this range stands for
    const int64_t s0 = g0 - item.first, s1 = min(g1 - item.first, item.places);
    const int v0 = (int)(s0 * vis.n / item.places), v1 = (int)(s1 * vis.n / item.places);
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

    // This lane's row, and the wave's first and last tokens.
    const int my_r = min(row0 + wave * 32 + l32, n_rows - 1);
    const int my_t = my_r / a.gs;
    const int w_t0 = min(row0 + wave * 32, n_rows - 1) / a.gs, w_t1 = min(row0 + wave * 32 + 31, n_rows - 1) / a.gs;
    // Without a window of its own (retrieval, or a window that no key has left) nothing is
    // below a row's first key.
    const bool band = str && !a.evict;
    const int lo_off = band ? start - a.window + 1 : INT32_MIN / 2;  // first key of token t's window: lo_off + t
    // ring: offset r behind the sinks holds position rbase + r, one window less behind r = rrem
    const int rlast = max(start - 1 - a.n_sink, 0), rrem = rlast % a.window, rbase = a.n_sink + rlast - rrem;
    const int64_t sb = a.cu_seqlens ? 0 : item.b, tok0 = a.cu_seqlens ? seq.row0 : 0;
    const uint16_t* kn = static_cast<const uint16_t*>(a.k) + sb * a.k_sb + tok0 * a.k_st + g * a.k_sh;
    const uint16_t* vn = static_cast<const uint16_t*>(a.v) + sb * a.v_sb + tok0 * a.v_st + g * a.v_sh;
    // cached tiles: units of 16 rows, `unit_step` apart from one page (block) to the next
    const int unit_step = str ? 1 : a.n_ret;
    const int64_t unit0 = str ? ((int64_t)item.b * a.n_str + item.kvl) * a.ring_blocks : item.kvl;
    const uint16_t* kc = static_cast<const uint16_t*>(str ? a.rk : a.pk) + unit0 * (kPage * D);
    const uint16_t* vc = static_cast<const uint16_t*>(str ? a.rv : a.pv) + unit0 * (kPage * D);
    const int32_t* table = str ? nullptr : a.block_table + (int64_t)item.b * a.max_pages;
    const int last_page = max(div_up(cached, kPage) - 1, 0);
    const int end_page = str ? a.ring_blocks : a.num_pages;

    // Direct loads of a tile: wave w fills kLoads blocks of 1 KB of K and of V, one
    // instruction each, which lie in one page of the tile (my_page).
    constexpr int kBlockRows = 512 / D;
    const int my_page = wave * Shape::kLoads * kBlockRows / kPage;
    bool bad = false;  // this wave has met a page outside the cache, or a V that the fast loop cannot take
    // Page of this wave's part of a cached tile: the block table's entry, read ahead of its use.
    auto entry_of = [&](int it) __attribute__((always_inline)) {
      const int pg = min(vis.tile(it) * (kBN / kPage) + my_page, last_page);
      return table ? scalar_i32(table + pg) : pg;
    };
    auto issue_cached = [&](int slot_k, int slot_v, int entry) __attribute__((always_inline)) {
      if (entry < 0 || entry >= end_page) {
        bad = true;
        entry = 0;
      }
      const int64_t unit = (int64_t)entry * unit_step * (kPage * D);
      const uint16_t* ku = kc + unit;
      const uint16_t* vu = vc + unit;
#pragma unroll
      for (int jj = 0; jj < Shape::kLoads; ++jj) {
        const int j = Shape::kLoads * wave + jj;
        const int r = kBlockRows * j + lane / Tile::kChunks;  // row of the tile
        lds_dma16(ku + (r % kPage) * D + 8 * ((lane % Tile::kChunks) ^ Tile::kx(r)), &ring.k[slot_k][512 * j]);
        const int dim = (32 * j + (lane >> 1)) % D;
        lds_dma16(vu + dim * kPage + 8 * ((lane & 1) ^ ((dim >> 3) & 1)), &ring.v[slot_v][512 * j]);
      }
    };
    auto issue_new = [&](int it, int slot_k, int slot_v) __attribute__((always_inline)) {
      const int kb = vis.tile(it) * kBN;
#pragma unroll
      for (int jj = 0; jj < Shape::kLoads; ++jj) {
        const int j = Shape::kLoads * wave + jj;
        const int r = kBlockRows * j + lane / Tile::kChunks, pc = lane % Tile::kChunks;
        const int64_t row = min(kb + r, n_new - 1);  // rows behind the last repeat it; no query sees them
        lds_dma16(kn + row * a.k_st + 8 * (pc ^ Tile::kx(r)), &ring.k[slot_k][512 * j]);
        lds_dma16(vn + row * a.v_st + 8 * (pc ^ Tile::vx(r)), &ring.v[slot_v][512 * j]);
      }
    };
    // V of a tile that this wave's loads have brought: zeroes tokens behind the cache's last
    // one, and looks for values that are not finite where a row does not see all keys.
    auto clean = [&](int it, int slot_v) __attribute__((always_inline)) {
      const int kb = vis.tile(it) * kBN;
      const bool of_cache = it < vis.n_cached;
      const bool tail = of_cache && kb + kBN > cached;
      const bool masked = of_cache ? band : kb + kBN - 1 > t_first || !(start + kb + kBN - 1 < a.n_sink || start + kb >= lo_off + t_last);
      if (!tail && !masked) return;
#pragma unroll
      for (int jj = 0; jj < Shape::kLoads; ++jj) {
        const int j = Shape::kLoads * wave + jj;
        u32x4* at = reinterpret_cast<u32x4*>(&ring.v[slot_v][512 * j + 8 * lane]);
        u32x4 x = *at;
        if (tail) {
          const int dim = (32 * j + (lane >> 1)) % D;
          const int left = cached - (kb + (32 * j / D) * kPage + 8 * ((lane & 1) ^ ((dim >> 3) & 1)));
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

    auto pv_part = [&](auto is_cached, int slot) __attribute__((always_inline)) {
      const uint32_t at = (decltype(is_cached)::value ? paddr0 : vaddr0) + (uint32_t)slot * Tile::kBytes;
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
#pragma unroll
        for (int mb = 0; mb < kMBlocks; ++mb) {
          const bf16x8 v = v_operand(is_cached, at, ks, mb);
#pragma unroll
          for (int i = PARTS - 1; i >= 0; --i) acc_o[mb] = mfma32(v, pop[i][ks], acc_o[mb]);
        }
    };
    auto qk_part = [&](int slot) __attribute__((always_inline)) {
      const uint32_t at = kaddr0 + (uint32_t)slot * Tile::kBytes;
#pragma unroll
      for (int blk = 0; blk < 2; ++blk)
#pragma unroll
        for (int i = 0; i < 16; ++i) sacc[blk][i] = 0.f;
#pragma unroll
      for (int s = 0; s < kKSteps; ++s)
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) sacc[blk] = mfma32(k_operand(at, s, blk), qreg[s], sacc[blk]);
    };
    // Steady-state MFMA phase, at raised wave priority: operands are read a few MFMAs ahead
    // of their products.
    auto mfma_phase = [&](auto is_cached, int slot_k, int slot_v) __attribute__((always_inline)) {
      __builtin_amdgcn_s_setprio(1);
      pv_part(is_cached, slot_v);
      qk_part(slot_k);
      constexpr int kReads = decltype(is_cached)::value ? 1 : 2;  // LDS reads of a V^T operand
      __builtin_amdgcn_sched_group_barrier(0x100, 4 * kReads, 0);
#pragma unroll
      for (int i = 0; i < D / 8 - 4; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, PARTS, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, kReads, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, PARTS, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
#pragma unroll
      for (int i = 0; i < D / 8 - 4; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(0);
    };

    // Key (place within the tile) of score i of block blk.
    auto key_of = [&](int blk, int i) __attribute__((always_inline)) { return 32 * blk + 16 * (i >> 3) + 8 * h2 + (i & 7); };
    // Whether this lane's row sees key j (position, slot, or new token).
    auto sees = [&](bool of_cache, int j) __attribute__((always_inline)) {
      if (of_cache) {
        const int r = j - a.n_sink;
        return j < cached && (r < 0 || rbase + r - (r > rrem ? a.window : 0) >= lo_off + my_t);
      }
      return j <= my_t && (start + j < a.n_sink || start + j >= lo_off + my_t);
    };
    auto apply_mask = [&](bool of_cache, int kb) __attribute__((always_inline)) {
#pragma unroll
      for (int blk = 0; blk < 2; ++blk)
#pragma unroll
        for (int i = 0; i < 16; ++i) sacc[blk][i] = sees(of_cache, kb + key_of(blk, i)) ? sacc[blk][i] : -INFINITY;
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
          psum[2 * blk + hf] = ((pf[0] + pf[1]) + (pf[2] + pf[3])) + ((pf[4] + pf[5]) + (pf[6] + pf[7]));
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
          for (int i = 0; i < 16; ++i) acc_o[mb][i] *= alpha;
        m_use = (m_run == -INFINITY) ? 0.f : m_run;
        tsum = exps();
      }
      l_run += tsum;
    };

    barrier();  // the ring's last use (the range's previous item) is over
    if constexpr (!CAREFUL) {
      auto valu_phase = [&](auto is_cached, int it) __attribute__((always_inline)) {
        constexpr bool of_cache = decltype(is_cached)::value;
        const int kb = vis.tile(it) * kBN;
        bool dead = false, mask;
        if constexpr (of_cache) {
          mask = kb + kBN > cached || band;
        } else {
          dead = kb > w_t1 || (start + kb >= a.n_sink && start + kb + kBN - 1 < lo_off + w_t0);
          mask = kb + kBN - 1 > w_t0 || !(start + kb + kBN - 1 < a.n_sink || start + kb >= lo_off + w_t1);
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
        if (mask) apply_mask(of_cache, kb);
        softmax_tile();
      };
      // Slots of the tile that is loaded next, of the tile whose K and of the one whose V is
      // read next.
      int in_k = 0, in_v = 0, at_k = 0, at_v = 0;
      auto next_k = [&](int& x) __attribute__((always_inline)) { x = x + 1 == Shape::kKSlots ? 0 : x + 1; };
      auto next_v = [&](int& x) __attribute__((always_inline)) { x = x + 1 == Shape::kVSlots ? 0 : x + 1; };
      int entry = 0;  // of the next tile that is loaded, if it is cached
      auto issue = [&](int it) __attribute__((always_inline)) {
        if (it < vis.n_cached) issue_cached(in_k, in_v, entry);
        else issue_new(it, in_k, in_v);
        next_k(in_k);
        next_v(in_v);
      };
      auto read_entry = [&](int it) __attribute__((always_inline)) {
        if (it < vis.n_cached && it < v1) entry = entry_of(it);
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
          clean(it + 1, s < 0 ? s + Shape::kVSlots : s);
        }
        __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
        barrier();
        if (it + Shape::kAhead < v1) issue(it + Shape::kAhead);
      };

      // Prologue: the first tiles and this wave's Q rows, then everything complete.
      for (int u = 0; u < Shape::kAhead && v0 + u < v1; ++u) {
        read_entry(v0 + u);
        issue(v0 + u);
      }
      {
        const int my_h = g * a.gs + my_r % a.gs;
        const uint16_t* qp = static_cast<const uint16_t*>(a.q) + sb * a.q_sb + (tok0 + my_t) * a.q_st + my_h * a.q_sh;
#pragma unroll
        for (int s = 0; s < kKSteps; ++s) qreg[s] = __builtin_bit_cast(bf16x8, ld16(qp + 8 * h2 + 16 * s));
      }
      __builtin_amdgcn_s_waitcnt(kWaitVm0);
      clean(v0, 0);
      read_entry(v0 + Shape::kAhead);
      __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
      barrier();

      // Every wave runs MFMA, vector phase, MFMA, ..: waves 0-3 take the barrier of a tile
      // after its vector phase, waves 4-7 after its MFMA phase.  A block table entry is read
      // while the vector phase runs.
      auto vector_phase = [&](auto is_cached, int it) __attribute__((always_inline)) {
        if (grp == 1) {
          sync_tile(it);
          read_entry(it + 1 + Shape::kAhead);
        }
        valu_phase(is_cached, it);
        if (grp == 0) {
          sync_tile(it);
          read_entry(it + 1 + Shape::kAhead);
        }
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
      const int mid = min(max(vis.n_cached, v0), v1);
      if (v0 < mid) run_tiles(kCached, v0, mid);
      if (mid < v1) run_tiles(kNew, mid, v1);

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
      const int my_h = g * a.gs + my_r % a.gs;
      const uint16_t* qp = static_cast<const uint16_t*>(a.q) + sb * a.q_sb + (tok0 + my_t) * a.q_st + my_h * a.q_sh;
#pragma unroll
      for (int s = 0; s < kKSteps; ++s) qreg[s] = __builtin_bit_cast(bf16x8, ld16(qp + 8 * h2 + 16 * s));
#pragma unroll 1
      for (int it = v0; it < v1; ++it) {
        const bool of_cache = it < vis.n_cached;
        const int kb = vis.tile(it) * kBN;
        __syncthreads();
        if (of_cache) issue_cached(0, 0, entry_of(it));
        else issue_new(it, 0, 0);
        __builtin_amdgcn_s_waitcnt(kWaitVm0);
        clean(it, 0);
        __syncthreads();
        uint32_t pages = 0;  // the tile's pages that are none
        if (of_cache && table)
          for (int i = 0; i < kBN / kPage; ++i) {
            const int e = table[min(kb / kPage + i, last_page)];
            if (e < 0 || e >= end_page) pages |= 1u << i;
          }
        auto seen = [&](int j) __attribute__((always_inline)) { return sees(of_cache, kb + j) && !((pages >> (j / kPage)) & 1u); };
        qk_part(0);
#pragma unroll
        for (int blk = 0; blk < 2; ++blk)
#pragma unroll
          for (int i = 0; i < 16; ++i) sacc[blk][i] = seen(key_of(blk, i)) ? sacc[blk][i] : -INFINITY;
        softmax_tile();
        // P.V with the finite values, and NaN where a row sees one that is not
#pragma unroll
        for (int mb = 0; mb < kMBlocks; ++mb) {
          f32x16 hits;
#pragma unroll
          for (int i = 0; i < 16; ++i) hits[i] = 0.f;
#pragma unroll
          for (int ks = 0; ks < 4; ++ks) {
            const bf16x8 v = of_cache ? v_operand(kCached, paddr0, ks, mb) : v_operand(kNew, vaddr0, ks, mb);
            const i16x8 bits = __builtin_bit_cast(i16x8, v);
            i16x8 fin;
            bf16x8 ind, on;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const bool out = (bits[e] & 0x7f80) == 0x7f80;
              fin[e] = out ? (short)0 : bits[e];
              ind[e] = (bf16)(out ? 1.f : 0.f);
              on[e] = (bf16)(seen(16 * ks + 8 * h2 + e) ? 1.f : 0.f);
            }
#pragma unroll
            for (int i = PARTS - 1; i >= 0; --i) acc_o[mb] = mfma32(__builtin_bit_cast(bf16x8, fin), pop[i][ks], acc_o[mb]);
            hits = mfma32(ind, on, hits);
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) acc_o[mb][i] = hits[i] > 0.f ? __builtin_nanf("") : acc_o[mb][i];
        }
      }
    }

    const float l_tot = xor32_sum(l_run);
    if (whole) {
      const float inv = 1.f / l_tot;
      if (row0 + wave * 32 + l32 < n_rows) {
        const int64_t at = sb * a.o_sb + (tok0 + my_t) * a.o_st + (int64_t)(g * a.gs + my_r % a.gs) * a.o_sh;
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
}

template <int D, int ROWS, int PARTS>
__global__ __launch_bounds__(2 * ROWS, (TileShape<D, ROWS>::kWavesPerSimd)) void extend_tile_kernel(ExtendArgs a) {
  __shared__ __align__(1024) TileRing<D, ROWS> ring;
  if (extend_range<D, ROWS, PARTS, false>(a, ring)) extend_range<D, ROWS, PARTS, true>(a, ring);
}

// ---------------------------------------------------------------------------
// Items that several workgroups share: one row a wave, its lanes over groups of partials
// and the dimensions.  The workgroups' x is the range that an item starts in.
template <int D, int ROWS, int TILE>
__global__ __launch_bounds__(256) void extend_merge_kernel(ExtendArgs a) {
  constexpr int kLanes = D / 4, kGroups = kWave / kLanes;
  const int lane = threadIdx.x & 63;
  const int row = blockIdx.y * 4 + (threadIdx.x >> 6);
  const ExtendPlan plan = extend_plan<ROWS, TILE>(a);
  const int rng = blockIdx.x;
  if (rng + 1 >= plan.used) return;
  const int64_t g0 = rng * plan.range, g1 = g0 + plan.range;
  const ExtendItem item = extend_item(plan, g1 - 1, a.n_ret, a.n_str);
  if (item.first < g0 || item.first + item.places <= g1) return;  // starts before this range, or ends in it
  const ExtendSeq seq = extend_seq(a, item.b);
  const int r = item.rb * ROWS + row;
  if (r >= seq.n * a.gs) return;
  const int last = (int)((item.first + item.places - 1) / plan.range);
  auto slot = [&](int w) { return (int64_t)(2 * w + (w == rng ? 1 : 0)) * ROWS + row; };
  // a partial without a key has m = -inf and l = 0 (keys with NaN scores leave a NaN sum)
  float M = -INFINITY;
  for (int w = rng + lane; w <= last; w += kWave) M = fmaxf(M, a.part_ml[slot(w) * 2]);
#pragma unroll
  for (int i = 1; i < kWave; i *= 2) M = wave_xor_max(M, i);
  float L = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int w = rng + lane / kLanes; w <= last; w += kGroups) {
    const int64_t at = slot(w);
    const float m = a.part_ml[at * 2], l = a.part_ml[at * 2 + 1];
    const float f = m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : fast_exp2(m - M);
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    if (m != -INFINITY || l != 0.f) x = *reinterpret_cast<const f32x4*>(a.part_acc + at * D + 4 * (lane % kLanes));
    L += f * l;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += f * x[e];
  }
#pragma unroll
  for (int i = kLanes; i < kWave; i *= 2) {
    L = wave_xor_sum(L, i);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = wave_xor_sum(o[e], i);
  }
  if (lane >= kLanes) return;
  const int g = a.kv_heads[item.str ? a.n_ret + item.kvl : item.kvl];
  const int64_t sb = a.cu_seqlens ? 0 : item.b, tok0 = a.cu_seqlens ? seq.row0 : 0;
  const int t = r / a.gs, h = g * a.gs + r % a.gs;
  const float inv = 1.f / L;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] *= inv;
  const int64_t at = sb * a.o_sb + (tok0 + t) * a.o_st + h * a.o_sh + 4 * lane;
  if (a.out_f32) store4<true>(a, at, o);
  else store4<false>(a, at, o);
}

template <int D, int ROWS>
static hipError_t launch_tiles(ExtendArgs a, hipStream_t s) {
  a.wgs = a.cus * TileShape<D, ROWS>::kWgsPerCu;
  a.min_tiles = 2;
  a.part_acc = static_cast<float*>(a.workspace);
  a.part_ml = a.part_acc + (int64_t)2 * a.wgs * ROWS * D;
  const dim3 grid((a.wgs + 7) / 8 * 8);
  if (a.out_f32) hipLaunchKernelGGL((extend_tile_kernel<D, ROWS, 3>), grid, dim3(2 * ROWS), 0, s, a);
  else hipLaunchKernelGGL((extend_tile_kernel<D, ROWS, 1>), grid, dim3(2 * ROWS), 0, s, a);
  if (hipError_t e = hipGetLastError()) return e;
  hipLaunchKernelGGL((extend_merge_kernel<D, ROWS, kBN>), dim3(a.wgs - 1, ROWS / 4), dim3(256), 0, s, a);
  return hipGetLastError();
}

// Bytes of the partials of the largest launch: two blocks of rows a workgroup.
size_t extend_workspace(int d, int cus) {
  const size_t rows = d == 64 ? 128 * 3 : 256;
  return (size_t)2 * cus * rows * (d + 2) * sizeof(float);
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
    if (d == 64) e = launch_tiles<64, 128>(x, s);
    else if ((int64_t)a.T * a.gs >= 256) e = launch_tiles<128, 256>(x, s);
    else e = launch_tiles<128, 128>(x, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace aoh
