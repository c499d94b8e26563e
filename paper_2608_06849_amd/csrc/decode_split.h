// Split passes of a decode step over its work space, shared by the caches'
// element types.
//
// A kernel here cuts the valid 16-token blocks of every (sequence, KV head) of
// both caches into ranges, has Body fold each wave's range into a softmax state,
// and joins the states.  Body gives
//   kD, kScores                      width; whether scores are kept (anchor layer)
//   kWaves, kPerSimd                 waves of a workgroup, and of a SIMD
//   kItemCost                        what starting a segment costs a wave, in blocks
//                                    (decode_many_kernel)
//   kWsItemCost                      what it costs a workgroup (decode_ws_kernel)
//   run(a, ring, b, kvl, len, blk0, blk_lim, acc, m, l, lds)
//     blocks [blk0, blk_lim) of the ring or paged cache row of (sequence b, KV head
//     kvl): the unnormalised sums acc (0 before), the maximum m in log2 units and
//     the sum l (left as they are when the range holds no token); lds: where the
//     wave's score codes pass (paged rows)
//   dim(t, G)                        first of the four consecutive output
//     dimensions that acc[t] holds in lane group G = lane / 16 (query head
//     lane % 16 of the group)
#pragma once
#include "aoh_device.h"
#include "aoh_internal.h"

namespace aoh {

// Four output dimensions d .. d + 3 of query head hq.
__device__ __forceinline__ void store_out4(const DecodeArgs& a, int b, int hq, int d, f32x4 o) {
  const int64_t at = (int64_t)b * a.o_sb + (int64_t)hq * a.o_sh + d;
  if (a.out_f32) {
    *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(a.out) + at) = o;
  } else {
    u32x2 w;
    w[0] = (uint32_t)f32_to_bf16_bits(o[0]) | ((uint32_t)f32_to_bf16_bits(o[1]) << 16);
    w[1] = (uint32_t)f32_to_bf16_bits(o[2]) | ((uint32_t)f32_to_bf16_bits(o[3]) << 16);
    *reinterpret_cast<u32x2*>(reinterpret_cast<uint16_t*>(a.out) + at) = w;
  }
}

// The waves' partial states (acc, m in log2 units, l) merged in
// LDS with log-sum-exp weights; lane (col, G) holds query head col of the
// group, and each wave writes a share of the dimension blocks of the merged
// partial to row `row` of part_acc / part_ml (lanes with lane_ok).  A wave
// without tokens has m = -inf and weight 0; if no wave has tokens the row gets
// m = -inf (the merge pass never reads such a row).  Starts with a barrier so
// a workgroup can call it once per segment.
template <class Body>
__device__ __forceinline__ void merge_waves_store(const DecodeArgs& a, f32x4 (&acc)[Body::kD / 16], float m, float l,
                                                  f32x4 (*s_acc)[Body::kD / 16][kWave], float (*s_m)[kWave],
                                                  float (*s_l)[kWave], bool lane_ok, int64_t row) {
  constexpr int D = Body::kD;
  constexpr int kDimBlocks = D / 16;
  constexpr int kWaves = Body::kWaves;
  constexpr int kPer = (kDimBlocks + kWaves - 1) / kWaves;  // dimension blocks of a wave
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & (kWave - 1);
  __syncthreads();
#pragma unroll
  for (int nb = 0; nb < kDimBlocks; ++nb) s_acc[wave][nb][lane] = acc[nb];
  s_m[wave][lane] = m;
  s_l[wave][lane] = l;
  __syncthreads();
  float M = -INFINITY;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) M = fmaxf(M, s_m[w][lane]);
  float wt[kWaves];
  float L = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const float mw = s_m[w][lane];
    wt[w] = (mw == -INFINITY) ? 0.f : fast_exp2(mw - M);
    L += wt[w] * s_l[w][lane];
  }
  if (lane_ok) {
    const int G = lane >> 4;
    float* pa = a.part_acc + row * D;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int nb = wave * kPer + k;
      if (kPer * kWaves > kDimBlocks && nb >= kDimBlocks) break;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const f32x4 x = s_acc[w][nb][lane];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] += wt[w] * x[i];
      }
      *reinterpret_cast<f32x4*>(pa + Body::dim(nb, G)) = o;
    }
    if (wave == 0 && G == 0) {
      a.part_ml[row * 2 + 0] = M;
      a.part_ml[row * 2 + 1] = L;
    }
  }
}

// ---------------------------------------------------------------------------
// Split pass over the step's work space (plain, anchor and fused-step
// decode of up to kWsMaxBatch sequences).
//
// Work space: the valid 16-token blocks of every item (cache type, sequence,
// KV head) laid end to end, paged items first, each type in (sequence, KV
// head) order, so one plan covers any mix of lengths and of the two cache
// types.  Every item is preceded by kWsItemCost places without a block, so that
// ranges of short items, which a workgroup takes one after the other, hold few of
// them.  Each workgroup takes one contiguous range of it and each of its
// waves a consecutive share of every item segment in that range; the waves'
// states are merged in LDS and the workgroup writes one partial per segment.
// The launch has two workgroups per CU: the first n_cu are placed one per CU,
// and a CU's second workgroup runs about a third slower (its waves lose issue
// arbitration on every SIMD to the older ones), so first-round ranges hold 4
// shares and second-round ranges 3, and both rounds end together.  Item i,
// covered by workgroups first_i..last_i, has its partials in slots
// first_i + i .. last_i + i (items are contiguous, so no two items share a
// slot): at most workgroups + items slots of gs heads each.
// Smallest range a workgroup takes: kWsShortBlocks while that leaves at most one
// workgroup per CU, kWsMinBlocks beyond.  A short step is a chain of memory
// latencies, which a wave with one 32-token chunk ends soonest; a long one pays
// for more partials.  28 layers of one sequence of 4093 tokens: 286-290 us with
// ranges of 4 blocks, 330 with 8, 374 with 16, 352 with 2 or 3; 16 layers of 4
// sequences of 2000-4000: 273 with at most one workgroup per CU, 281 with two.
constexpr int kWsShortBlocks = 4;
constexpr int kWsMinBlocks = 16;

__device__ __forceinline__ int ws_n_wg(int total, int n_cu, int max_wg) {
  const int many = (total + kWsShortBlocks - 1) / kWsShortBlocks;
  const int few = (total + kWsMinBlocks - 1) / kWsMinBlocks;
  return min(max_wg, max(1, max(few, min(many, n_cu))));
}

struct WsPlan {
  int nb_tot, nbr_tot;  // paged / ring places summed over the sequences
  int total;            // places of all items
  int n_old, n_young;   // workgroups of the first and second round
  int r_old, r_young;   // places per range of each round
  int g_young;          // first place of the second round's ranges
};

// The plan from the sequence lengths.  Every lane of a wave calls it; lane b
// gets sequence b's length, its places (blocks + COST, 0 without blocks) in the paged
// cache (nb) and the ring (nbr), and their exclusive prefix sums over the sequences
// (P, Q); lanes >= B get zeros.
template <int COST>
__device__ __forceinline__ WsPlan ws_plan(const int32_t* lens, int B, int max_pages, int n_ret, int ring_cap,
                                          int n_str, int n_cu, int& len, int& nb, int& nbr, int& P, int& Q) {
  const int lane = threadIdx.x & (kWave - 1);
  len = 0;
  nb = 0;
  nbr = 0;
  if (lane < B) {
    len = lens[lane];
    const int l = max(len, 0);
    if (n_ret) nb = (min(l, max_pages * kPage) + kPage - 1) / kPage;
    if (n_str) nbr = (min(l, ring_cap) + kPage - 1) / kPage;
    nb += nb ? COST : 0;
    nbr += nbr ? COST : 0;
  }
  int ip = nb, iq = nbr;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int tp = __shfl_up(ip, o, kWave), tq = __shfl_up(iq, o, kWave);
    if (lane >= o) {
      ip += tp;
      iq += tq;
    }
  }
  P = ip - nb;
  Q = iq - nbr;
  WsPlan p;
  p.nb_tot = __builtin_amdgcn_readlane(ip, kWave - 1);
  p.nbr_tot = __builtin_amdgcn_readlane(iq, kWave - 1);
  p.total = n_ret * p.nb_tot + n_str * p.nbr_tot;
  const int n_wg = ws_n_wg(p.total, n_cu, 2 * n_cu);
  p.n_old = min(n_wg, n_cu);
  p.n_young = n_wg - p.n_old;
  const int64_t weight = 4 * (int64_t)p.n_old + 3 * (int64_t)p.n_young;
  p.r_old = (int)((4 * (int64_t)p.total + weight - 1) / weight);
  p.g_young = min(p.total, p.n_old * p.r_old);
  p.r_young = p.n_young ? (p.total - p.g_young + p.n_young - 1) / p.n_young : 0;
  return p;
}

// Workgroup whose range holds place g (g < total).
__device__ __forceinline__ int ws_wg_of(int g, const WsPlan& p) {
  return g < p.g_young ? g / p.r_old : p.n_old + (g - p.g_young) / p.r_young;
}

// The item holding place g of the work space (g < total): its type, sequence,
// KV head rank, first place in the work space, valid blocks and item index.
struct WsItem {
  bool ring;
  int b, kvl, off, len, idx;
};

template <int COST>
__device__ __forceinline__ WsItem ws_item(int g, const WsPlan& p, int B, int n_ret, int n_str, int nb, int nbr, int P,
                                          int Q) {
  const int lane = threadIdx.x & (kWave - 1);
  WsItem it;
  const int paged_end = n_ret * p.nb_tot;
  it.ring = g >= paged_end;
  const int heads = it.ring ? n_str : n_ret;
  const int blocks = it.ring ? nbr : nb;
  const int start = (it.ring ? paged_end : 0) + heads * (it.ring ? Q : P);
  const uint64_t hit = __ballot(lane < B && g >= start && g < start + heads * blocks);
  if (hit == 0) {  // not reached for g < total
    it.b = it.kvl = it.off = it.idx = it.len = 0;
    return it;
  }
  it.b = __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(hit));
  const int first = __builtin_amdgcn_readlane(start, it.b);
  const int places = __builtin_amdgcn_readlane(blocks, it.b);
  it.kvl = (g - first) / places;
  it.off = first + it.kvl * places;
  it.len = places - COST;
  it.idx = it.ring ? B * n_ret + it.b * n_str + it.kvl : it.b * n_ret + it.kvl;
  return it;
}

template <class Body>
__global__ __launch_bounds__(Body::kWaves * kWave, Body::kPerSimd) void decode_ws_kernel(DecodeArgs a) {
  constexpr int D = Body::kD;
  constexpr int kDimBlocks = D / 16;
  constexpr int kWaves = Body::kWaves;
  __shared__ f32x4 s_acc[kWaves][kDimBlocks][kWave];
  // the score codes of each wave
  __shared__ f32x4 s_code[Body::kScores ? kWaves : 1][Body::kScores ? kDimBlocks * kWave : 1];
  __shared__ float s_m[kWaves][kWave];
  __shared__ float s_l[kWaves][kWave];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & (kWave - 1);
  int len_l, nb_l, nbr_l, P_l, Q_l;
  constexpr int kCost = Body::kWsItemCost;
  const WsPlan p = ws_plan<kCost>(a.lens, a.B, a.full.max_pages, a.full.n_kv, a.ring_cap, a.ring.n_kv, a.ws_cu, len_l, nb_l,
                           nbr_l, P_l, Q_l);
  const int w = blockIdx.x;
  int g0, g1;
  if (w < p.n_old) {
    g0 = w * p.r_old;
    g1 = min(g0 + p.r_old, p.g_young);
  } else {
    g0 = p.g_young + (w - p.n_old) * p.r_young;
    g1 = w < p.n_old + p.n_young ? min(g0 + p.r_young, p.total) : g0;
  }
  for (int g = g0; g < g1;) {  // uniform: every wave walks the same segments
    const WsItem it = ws_item<kCost>(g, p, a.B, a.full.n_kv, a.ring.n_kv, nb_l, nbr_l, P_l, Q_l);
    if (it.len == 0) break;
    const int s0 = max(0, g - it.off - kCost), s1 = min(g1 - it.off - kCost, it.len);
    g = it.off + kCost + s1;
    if (s0 >= s1) break;  // only places before the item's blocks: the range ends here
    const int len = __builtin_amdgcn_readlane(len_l, it.b);
    // This wave's consecutive share of the segment's 32-token chunks.
    const int per = ((s1 - s0 + 1) / 2 + kWaves - 1) / kWaves;
    const int c0 = min(s1, s0 + 2 * per * wave), c1 = min(s1, c0 + 2 * per);
    f32x4 acc[kDimBlocks];
#pragma unroll
    for (int nb = 0; nb < kDimBlocks; ++nb) acc[nb] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    if (c0 < c1) Body::run(a, it.ring, it.b, it.kvl, len, c0, c1, acc, m, l, s_code[Body::kScores ? wave : 0]);
    const int col = lane & 15;
    merge_waves_store<Body>(a, acc, m, l, s_acc, s_m, s_l, col < a.gs, (int64_t)(w + it.idx) * a.gs + col);
    if (s0 == 0 && threadIdx.x == 0) {
      // The workgroup holding the item's first block records where the item's
      // partials are for the merge pass: first slot and count.
      a.ws_items[2 * it.idx + 0] = w + it.idx;
      a.ws_items[2 * it.idx + 1] = ws_wg_of(it.off + kCost + it.len - 1, p) - w + 1;
    }
  }
}

// ---------------------------------------------------------------------------
// Split pass for steps of many items (up to kManyMaxBatch sequences): the same
// work space, in which every item is preceded by kItemCost places without a
// block: what starting a segment costs a wave (its first loads), in blocks, so
// that ranges of many short items hold fewer blocks.  Each workgroup takes one
// contiguous range and each of its waves a consecutive share of it.  An item
// that lies within one wave's share is finished and stored by that wave; the
// pieces of an item that several waves share meet in LDS (at most two a wave:
// the item its share starts in and the one it ends in), and those of several
// workgroups in the workspace, for the merge launch, which finds them through
// ws_items: by workgroup, the item that starts in it and goes on, if any.
//
// The ranges of the two rounds are those of decode_ws_kernel.  For few items
// that kernel's plan, which every wave holds in registers, starts faster (9.5
// us a launch against 12 for one sequence of 4093 tokens in ranges of 16
// blocks).  For many, its barriers and workspace partials at every item cost
// more, as do fixed splits of the capacity, of which most are empty when
// lengths differ: 96 sequences of 200-8000 tokens, 8 KV heads of width 128,
// capacity 8192: 160 us a step here, 333 with fixed splits; 64 of 200-400
// tokens: 28 us here, 51 with the other work-space kernel.  Bound: HBM, 5.4-6
// TB/s for full ranges.
struct ManyPlan {
  int paged_end;        // places of the paged items
  int total;            // places of all items
  int n_old, n_young;   // workgroups of the first and second round
  int r_old, r_young;   // places per range of each round
  int g_young;          // first place of the second round's ranges
};

// Lengths and, per cache type, the exclusive prefix sums over the sequences of
// an item's places (blocks + kItemCost; 0 for an item without blocks).
template <int WAVES>
struct ManyTables {
  int len[kManyMaxBatch];
  int pre[2][kManyMaxBatch + 4];
  int carry[2][WAVES];
};

// Fills the tables from the sequence lengths (thread t: sequences 4t .. 4t + 3)
// and derives the plan.  Ends with a barrier.
template <int WAVES, int COST>
__device__ __forceinline__ ManyPlan many_plan(const DecodeArgs& a, ManyTables<WAVES>& tb) {
  static_assert(kManyMaxBatch <= 4 * WAVES * kWave, "four sequences a thread");
  const int t = threadIdx.x, lane = t & (kWave - 1), wave = t / kWave;
  const bool many = a.B > 4 * kWave;  // uniform: more sequences than one wave takes
  if (wave == 0 || many) {
    int n[2][4], sum[2] = {0, 0};
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int b = 4 * t + u;
      const int len = b < a.B ? a.lens[b] : 0;
      const int l = max(len, 0);
      const int nb = a.full.n_kv ? (min(l, a.full.max_pages * kPage) + kPage - 1) / kPage : 0;
      const int nbr = a.ring.n_kv ? (min(l, a.ring_cap) + kPage - 1) / kPage : 0;
      n[0][u] = nb ? nb + COST : 0;
      n[1][u] = nbr ? nbr + COST : 0;
      if (b < a.B) tb.len[b] = len;
#pragma unroll
      for (int k = 0; k < 2; ++k) sum[k] += n[k][u];
    }
    int inc[2] = {sum[0], sum[1]};
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int y = __shfl_up(inc[k], o, kWave);
        if (lane >= o) inc[k] += y;
      }
    }
    if (many) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
        if (lane == kWave - 1) tb.carry[k][wave] = inc[k];
      __syncthreads();
      for (int w = 0; w < wave; ++w)
#pragma unroll
        for (int k = 0; k < 2; ++k) inc[k] += tb.carry[k][w];
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      int at = inc[k] - sum[k];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (4 * t + u < a.B) tb.pre[k][4 * t + u] = at;
        at += n[k][u];
      }
      if (4 * t < a.B && 4 * t + 4 >= a.B) tb.pre[k][a.B] = at;
    }
  }
  __syncthreads();
  ManyPlan p;
  p.paged_end = a.full.n_kv * __builtin_amdgcn_readfirstlane(tb.pre[0][a.B]);
  p.total = p.paged_end + a.ring.n_kv * __builtin_amdgcn_readfirstlane(tb.pre[1][a.B]);
  const int n_wg = ws_n_wg(p.total, a.ws_cu, a.many_wgs);
  p.n_old = min(n_wg, a.ws_cu);
  p.n_young = n_wg - p.n_old;
  const uint32_t weight = 4 * p.n_old + 3 * p.n_young;  // total < 2^29
  p.r_old = (int)((4 * (uint32_t)p.total + weight - 1) / weight);
  p.g_young = min(p.total, p.n_old * p.r_old);
  p.r_young = p.n_young ? (p.total - p.g_young + p.n_young - 1) / p.n_young : 0;
  return p;
}

// Workgroup whose range holds place g (g < total).
__device__ __forceinline__ int many_wg_of(int g, const ManyPlan& p) {
  return g < p.g_young ? g / p.r_old : p.n_old + (g - p.g_young) / p.r_young;
}

// The item holding place g of the work space (g < total): its type, sequence,
// KV head rank, first place and blocks.  A step of more than 64 sequences finds
// the 64 that hold the place first (trying 64 after 64 of them, 900 sequences of
// 10-200 tokens took 74 us a step where this takes 63, 300 of up to 900 62 and 57).
struct ManyItem {
  bool ring;
  int b, kvl, off, len;
};

template <int WAVES, int COST>
__device__ __forceinline__ ManyItem many_item(const DecodeArgs& a, int g, const ManyPlan& p,
                                              const ManyTables<WAVES>& tb) {
  const int lane = threadIdx.x & (kWave - 1);
  ManyItem it;
  it.ring = g >= p.paged_end;
  const int base = it.ring ? p.paged_end : 0;
  const int heads = it.ring ? a.ring.n_kv : a.full.n_kv;
  const int* pre = tb.pre[it.ring];
  int b0 = 0;
  if (a.B > kWave)  // the last 64 sequences whose first place is not behind it (lane 0's is 0)
    b0 = kWave * (__builtin_popcountll(__ballot(g - base >= heads * pre[min(kWave * lane, a.B)])) - 1);
  const int i = min(b0 + lane, a.B - 1);
  const uint64_t hit = __ballot(g - base >= heads * pre[i] && g - base < heads * pre[i + 1]);
  it.b = __builtin_amdgcn_readfirstlane(hit ? b0 + (int)__builtin_ctzll(hit) : 0);
  const int p0 = __builtin_amdgcn_readfirstlane(pre[it.b]);
  const int places = max(1, __builtin_amdgcn_readfirstlane(pre[it.b + 1]) - p0);
  it.kvl = (g - base - heads * p0) / places;
  it.off = base + heads * p0 + it.kvl * places;
  it.len = places - COST;
  return it;
}

__device__ __forceinline__ void store_ml(const DecodeArgs& a, int b, int hq, float m, float l) {
  a.ml_out[((int64_t)b * a.Hq + hq) * 2 + 0] = m;
  a.ml_out[((int64_t)b * a.Hq + hq) * 2 + 1] = l;
}

// Slot of the partial of an item's j-th workgroup, first + j.  A workgroup
// shares at most two items with others, the one its range starts in (j > 0) and
// the one it ends in.
__device__ __forceinline__ int many_slot(int first, int j) { return 2 * (first + j) + (j == 0 ? 1 : 0); }

template <class Body>
__global__ __launch_bounds__(Body::kWaves * kWave, Body::kPerSimd) void decode_many_kernel(DecodeArgs a) {
  constexpr int D = Body::kD;
  constexpr int kDimBlocks = D / 16;
  constexpr int kWaves = Body::kWaves;
  constexpr int kItemCost = Body::kItemCost;
  constexpr int kPieces = 2 * kWaves;
  __shared__ f32x4 s_acc[kPieces][kDimBlocks][kWave];
  __shared__ float s_m[kPieces][16], s_l[kPieces][16];
  __shared__ int s_g[kPieces];  // a place of the piece's segment; -1: no piece
  __shared__ i32x4 s_starts;
  __shared__ ManyTables<kWaves> tb;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & (kWave - 1);
  const int col = lane & 15, G = lane >> 4;
  if (threadIdx.x < kPieces) s_g[threadIdx.x] = -1;
  if (threadIdx.x == 0) s_starts = i32x4{0, 0, 0, 0};
  const ManyPlan p = many_plan<kWaves, kItemCost>(a, tb);
  const int w = blockIdx.x;

  int g0, g1;
  if (w < p.n_old) {
    g0 = min(w * p.r_old, p.g_young);
    g1 = min(g0 + p.r_old, p.g_young);
  } else {
    g0 = min(p.g_young + (w - p.n_old) * p.r_young, p.total);
    g1 = w < p.n_old + p.n_young ? min(g0 + p.r_young, p.total) : g0;
  }
  const int share = ((g1 - g0 + kWaves - 1) / kWaves + 1) & ~1;  // whole 32-token chunks
  const int e1 = min(g1, g0 + share * (wave + 1));
  for (int g = min(g1, g0 + share * wave); g < e1;) {
    const ManyItem it = many_item<kWaves, kItemCost>(a, g, p, tb);
    const int v0 = g - it.off, v1 = min(e1 - it.off, it.len + kItemCost);
    const int s0 = max(0, v0 - kItemCost), s1 = v1 - kItemCost;
    const int at = g;
    g = it.off + v1;
    if (s0 >= s1) continue;
    const int len = __builtin_amdgcn_readfirstlane(tb.len[it.b]);
    f32x4 acc[kDimBlocks];
#pragma unroll
    for (int nb = 0; nb < kDimBlocks; ++nb) acc[nb] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    // the score codes pass through the wave's second piece, which only its last segment fills
    Body::run(a, it.ring, it.b, it.kvl, len, s0, s1, acc, m, l, s_acc[2 * wave + 1]);
    if (s0 == 0 && s1 == it.len) {  // the whole item
      const int hq = (it.ring ? a.ring : a.full).kv_heads[it.kvl] * a.gs + col;
      if (col < a.gs) {
        const float inv = 1.f / l;
#pragma unroll
        for (int nb = 0; nb < kDimBlocks; ++nb) {
          f32x4 o;
#pragma unroll
          for (int i = 0; i < 4; ++i) o[i] = acc[nb][i] * inv;
          store_out4(a, it.b, hq, Body::dim(nb, G), o);
        }
        if (Body::kScores && !it.ring && G == 0) store_ml(a, it.b, hq, m, l);
      }
    } else {
      // the wave's last segment unless the item began before its share
      const int piece = 2 * wave + (s0 == 0 ? 1 : 0);
#pragma unroll
      for (int nb = 0; nb < kDimBlocks; ++nb) s_acc[piece][nb][lane] = acc[nb];
      if (G == 0) {
        s_m[piece][col] = m;
        s_l[piece][col] = l;
      }
      if (lane == 0) s_g[piece] = at;
    }
  }
  __syncthreads();

  // The pieces of an item are joined by the wave that has the first of them: one item
  // a wave, two where the workgroup's range starts inside one (300 sequences of
  // 100-1000 tokens, width 64: 41.5 us a step, 43.9 with the waves sharing the
  // dimensions of one item after the other; 65 of 29000-30000 over the bf16 caches, where
  // a range is one item: 1208 and 1211).  All statistics are read at once and the
  // loops over the pieces are unrolled (as loops with LDS reads in them they took 1.5 us more).
  const int g_l = s_g[lane & (kPieces - 1)];
  int g_q[kPieces];
  float m_q[kPieces], l_q[kPieces];
#pragma unroll
  for (int q = 0; q < kPieces; ++q) {
    g_q[q] = __builtin_amdgcn_readlane(g_l, q);
    m_q[q] = s_m[q][col];
    l_q[q] = s_l[q][col];
  }
  for (int mine = 2 * wave; mine < 2 * wave + 2; ++mine) {
    const int at = __builtin_amdgcn_readlane(g_l, mine);
    if (at < 0) continue;
    const ManyItem it = many_item<kWaves, kItemCost>(a, at, p, tb);
    const int end = it.off + it.len + kItemCost;
    bool first_here = true;
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int q = 0; q < kPieces; ++q) {
      if (g_q[q] >= it.off && g_q[q] < at) first_here = false;
      if (g_q[q] >= at && g_q[q] < end) M = fmaxf(M, m_q[q]);
    }
    if (!first_here) continue;
    f32x4 o[kDimBlocks];
#pragma unroll
    for (int nb = 0; nb < kDimBlocks; ++nb) o[nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < kPieces; ++q) {
      if (!(g_q[q] >= at && g_q[q] < end)) continue;  // uniform
      const float wt = m_q[q] == -INFINITY ? 0.f : fast_exp2(m_q[q] - M);
      L += wt * l_q[q];
#pragma unroll
      for (int nb = 0; nb < kDimBlocks; ++nb) {
        const f32x4 y = s_acc[q][nb][lane];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[nb][i] += wt * y[i];
      }
    }
    const int first = many_wg_of(it.off + kItemCost, p);
    const int ns = many_wg_of(end - 1, p) - first + 1;
    const int hq0 = (it.ring ? a.ring : a.full).kv_heads[it.kvl] * a.gs;
    if (col < a.gs) {
      const int64_t row = (int64_t)many_slot(first, w - first) * a.gs + col;
      const float inv = 1.f / L;
#pragma unroll
      for (int nb = 0; nb < kDimBlocks; ++nb) {
        const int d = Body::dim(nb, G);
        if (ns > 1) {
          *reinterpret_cast<f32x4*>(a.part_acc + row * D + d) = o[nb];
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) o[nb][i] *= inv;
          store_out4(a, it.b, hq0 + col, d, o[nb]);
        }
      }
      if (G == 0) {
        if (ns > 1) {
          a.part_ml[row * 2 + 0] = M;
          a.part_ml[row * 2 + 1] = L;
        } else if (Body::kScores && !it.ring) {
          store_ml(a, it.b, hq0 + col, M, L);
        }
      }
    }
    // the item shared with later workgroups that starts here: number of
    // workgroups (0: none), sequence, first query head, whether a ring
    if (w == first && ns > 1 && lane == 0) s_starts = i32x4{ns, it.b, hq0, it.ring};
  }
  __syncthreads();
  if (threadIdx.x == 0) *reinterpret_cast<i32x4*>(a.ws_items + 4 * w) = s_starts;

  // Rows without a key.
  for (int b = w; b < a.B; b += gridDim.x) {
    const bool none[2] = {tb.pre[0][b] == tb.pre[0][b + 1], tb.pre[1][b] == tb.pre[1][b + 1]};
    for (int k = 0; k < 2; ++k) {
      const CacheView& cv = k ? a.ring : a.full;
      if (!none[k]) continue;
      for (int e = threadIdx.x; e < cv.n_kv * a.gs * (D / 4); e += kWaves * kWave) {
        const int qh = e / (D / 4), hq = cv.kv_heads[qh / a.gs] * a.gs + qh % a.gs;
        store_out4(a, b, hq, 4 * (e % (D / 4)), f32x4{a.empty, a.empty, a.empty, a.empty});
        if (Body::kScores && k == 0 && e % (D / 4) == 0) store_ml(a, b, hq, -INFINITY, 0.f);
      }
    }
  }
}

}  // namespace aoh
