// Single-token decode over the 8-bit caches (layout and codes: q8.h; ranges,
// merging and output: decode_split.h).
//
// A wave folds a few blocks of its range at a time (a chunk: 64 tokens, 16 KB at
// d_head 128), the next ones loading meanwhile:
//   S^T[16 tokens x 16 heads] = K[16 x 32 dims] . Q^T       (D/32 steps a block)
//   O^T[16 dims x 16 heads]  += V^T[16 dims x 32 tokens] . P^T   (D/16 a block pair)
// with v_mfma_f32_16x16x32_bf16 on codes converted to bf16, exactly.  K's row
// scale multiplies the scores and V's the probabilities, exactly too.  A weight,
// probability times V's scale, is kept whole, as the sum of three bf16 numbers, which
// costs two more products.  us a step with weights rounded to bf16 / with two numbers
// (2^-16 of a weight lost) / whole: 8 sequences of 131072 tokens 187.1 / 187.5 / 188.1,
// 96 of 200-8000 91.4 / 91.9 / 92.3, one of 4093 10.1 / 10.4 / 10.5, 300 of up to 900
// (width 64, int8) 51.7 / 53.1 / 56.0; the error of a bf16 output against float64,
// relative to its norm, 1.68e-3 / 1.66e-3 / 1.66e-3 for the first of these, 1.89e-3 /
// 1.62e-3 / 1.62e-3 for the last, and up to a quarter less in steps of few tokens.
//   Bound: HBM.  8 sequences of 131072 tokens, 4 of 8 heads streaming, e4m3: 174-181
// us in the pass (1.09 GB of codes and scales, 1.03 times that fetched), 6.0-6.3 TB/s;
// a step with an exponential only for every fourth score 180.0 us, with all 179.7.
// Width 64, whose pieces of memory are half as long: 5.6-5.9 TB/s over a step of 16
// such sequences.  Short steps: a chain of memory latencies (lengths, block table, K,
// the join, the merge launch).  The registers decide: with two chunks in flight the
// width 128 body spilled, and the step above took 434 us.
//   Lane group G = lane / 16 receives the scores of rows 4G .. 4G + 3 of a block,
// and the k index of the second product is ordered so that it needs just those: P^T
// stays in its lanes, and the V operand of dimension block 4j + n is word n of two
// tiles (one of each block of the pair).  Row m of that operand is dimension
// 64 j + 4 m + n, so the lane's sums are transposed in registers at the end.
//   All addresses of a load are one uniform base and a constant offset of
// the lane.  Block table entries are loaded 64 at a time, one a lane.
#include <cfloat>
#include <type_traits>

#include "aoh_internal.h"
#include "decode_split.h"
#include "q8.h"

namespace aoh {

namespace {

// Codes and scales of the blocks that a wave folds at a time.
template <int D, int BLOCKS>
struct Q8Chunk {
  static constexpr int kBlocks = BLOCKS;
  u32x4 k[kBlocks][D / 64];
  u32x4 v[kBlocks][D / 64];
  u32x2 s[kBlocks];
};

// Stores the step's token (position len - 1 of sequence b, KV head g) as row
// `row` of a unit: lane t has D / 64 dimensions of K and of V.
template <int D, bool I8>
__device__ __forceinline__ void store_token(const DecodeArgs& a, uint8_t* uk, uint8_t* uv, uint8_t* us, int b, int g,
                                            int row) {
  constexpr int kPer = D / kWave;
  const int lane = threadIdx.x & (kWave - 1);
  uint32_t byte[2];
  uint32_t code[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const uint16_t* p = t == 0 ? reinterpret_cast<const uint16_t*>(a.k_new) + (int64_t)b * a.kn_sb + (int64_t)g * a.kn_sh
                               : reinterpret_cast<const uint16_t*>(a.v_new) + (int64_t)b * a.vn_sb + (int64_t)g * a.vn_sh;
    float x[4] = {};
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      x[i] = bf16_to_f32(p[kPer * lane + i]);
      amax = max(amax, __builtin_bit_cast(uint32_t, x[i]) & 0x7fffffffu);
    }
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, o, kWave));
    byte[t] = scale_byte<I8>(amax);
    code[t] = to_codes<I8>(x, inverse_scale(byte[t]), byte[t] == 255u);
  }
  if constexpr (kPer == 2) *reinterpret_cast<uint16_t*>(uk + row * D + 2 * lane) = (uint16_t)code[0];
  else uk[row * D + lane] = (uint8_t)code[0];
#pragma unroll
  for (int i = 0; i < kPer; ++i) uv[v_offset(kPer * lane + i, row)] = (uint8_t)(code[1] >> (8 * i));
  if (lane == 0) *reinterpret_cast<uint16_t*>(us + 2 * row) = (uint16_t)(byte[0] | (byte[1] << 8));
}

}  // namespace

template <int D, bool I8, int WAVES, int BLOCKS, int PER_SIMD>
struct Q8Body {
  static constexpr int kD = D;
  static constexpr bool kScores = false;
  static constexpr int kWaves = WAVES;
  static constexpr int kPerSimd = PER_SIMD;
  // 300 sequences of up to 900 tokens (width 64, int8): 56.6 us (63.8 with 4, 57.5 with 12); 96 of 200-8000: 82.7
  // (83.0, 85.0).
  static constexpr int kItemCost = 8;
  // Work-space pass, where a segment is the whole workgroup's: 8 heads of width 128, sequences of 1 and
  // 9532 tokens: 35.9 us with 0, 14.4 with 8, 14.2 with 16, 14.5 with 32; 16 heads of which 9 stream, of 58 and
  // 80104: 55.1, 33.7, 32.6, 33.0.
  static constexpr int kWsItemCost = 16;
  static constexpr int kBlocks = BLOCKS;
  static __device__ __forceinline__ int dim(int t, int G) { return 64 * (t >> 2) + 16 * G + 4 * (t & 3); }

  // q . k of the blocks of a chunk, unscaled by 1 / sqrt(D).
  static __device__ __forceinline__ void scores(const Q8Chunk<D, BLOCKS>& x, const bf16x8 (&q)[D / 32], float (&s)[kBlocks][4]) {
#pragma unroll
    for (int X = 0; X < kBlocks; ++X) {
      f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        sc = mfma16(codes_operand<I8>(x.k[X][i][0], x.k[X][i][1]), q[2 * i], sc);
        sc = mfma16(codes_operand<I8>(x.k[X][i][2], x.k[X][i][3]), q[2 * i + 1], sc);
      }
      s[X][0] = sc[0] * scale_of<0>(x.s[X][0]);
      s[X][1] = sc[1] * scale_of<2>(x.s[X][0]);
      s[X][2] = sc[2] * scale_of<0>(x.s[X][1]);
      s[X][3] = sc[3] * scale_of<2>(x.s[X][1]);
    }
  }

  // Folds scores, V codes and V scales of a chunk into the running softmax state
  // (m_run in units of q . k).  `left`: rows from the lane group's first one to
  // the end, where `partial`.
  static __device__ __forceinline__ void fold(const DecodeArgs& a, Q8Chunk<D, BLOCKS>& x, float (&s)[kBlocks][4],
                                              const u32x2 (&vs)[kBlocks], bool partial, int left,
                                              f32x4 (&acc)[D / 16], float& m_run, float& l_run) {
    float w[kBlocks][4];
#pragma unroll
    for (int X = 0; X < kBlocks; ++X) {
      w[X][0] = scale_of<1>(vs[X][0]);
      w[X][1] = scale_of<3>(vs[X][0]);
      w[X][2] = scale_of<1>(vs[X][1]);
      w[X][3] = scale_of<3>(vs[X][1]);
    }
    if (partial) {
      // Rows past the end may hold anything: score -inf, no V scale, no V code (it may be NaN).
#pragma unroll
      for (int X = 0; X < kBlocks; ++X) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool off = 16 * X + i >= left;
          s[X][i] = off ? -INFINITY : s[X][i];
          w[X][i] = off ? 0.f : w[X][i];
        }
        const int n = min(max(left - 16 * X, 0), 4);
        const uint32_t keep = n == 4 ? ~0u : (1u << (8 * n)) - 1u;
#pragma unroll
        for (int j = 0; j < D / 64; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) x.v[X][j][e] &= keep;
      }
    }
    float mx = s[0][0];
#pragma unroll
    for (int e = 1; e < 4 * kBlocks; ++e) mx = fmaxf(mx, s[e / 4][e % 4]);
    mx = wave_xor_max(mx, 16);
    mx = xor32_max(mx);
    if (__ballot(mx > m_run)) {  // in some head; rare after the first chunks
      const float m_new = fmaxf(m_run, mx);
      const float alpha = fast_exp2((m_run - m_new) * a.scale_log2);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int t = 0; t < D / 16; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[t][i] *= alpha;
    }
    float psum = 0.f;
    constexpr int kParts = 3;  // bf16 numbers of a weight
    u32x4 part[kBlocks / 2][kParts];
#pragma unroll
    for (int X = 0; X < kBlocks; ++X)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p = fast_exp2((s[X][i] - m_run) * a.scale_log2);  // the maximum's is 1 at any magnitude
        psum += p;
        w[X][i] *= p;
        if (!(i & 1)) continue;
        const int word = 2 * (X & 1) + i / 2;
        // the upper eight bits, the next eight of what is left, the last eight
        float w0 = w[X][i - 1], w1 = w[X][i];
#pragma unroll
        for (int n = 0; n < kParts; ++n) {
          const uint32_t b0 = __builtin_bit_cast(uint32_t, w0), b1 = __builtin_bit_cast(uint32_t, w1);
          part[X / 2][n][word] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
          w0 -= __builtin_bit_cast(float, b0 & 0xffff0000u);
          w1 -= __builtin_bit_cast(float, b1 & 0xffff0000u);
        }
      }
    l_run += psum;
    // acc += V^T . W^T
#pragma unroll
    for (int t = 0; t < D / 16; ++t)
#pragma unroll
      for (int P = 0; P < kBlocks / 2; ++P) {
        const bf16x8 v = codes_operand<I8>(x.v[2 * P][t >> 2][t & 3], x.v[2 * P + 1][t >> 2][t & 3]);
#pragma unroll
        for (int n = 0; n < kParts; ++n) acc[t] = mfma16(v, __builtin_bit_cast(bf16x8, part[P][n]), acc[t]);
      }
  }

  static __device__ __forceinline__ void run(const DecodeArgs& a, bool ring, int b, int kvl, int len, int blk0,
                                             int blk_lim, f32x4 (&acc)[D / 16], float& m_out, float& l_out, void*) {
    const CacheView& cv = ring ? a.ring : a.full;
    const int lane = threadIdx.x & (kWave - 1);
    const int col = lane & 15, G = lane >> 4;
    const int g = cv.kv_heads[kvl];
    // Lengths beyond the cache capacity are clamped so no read leaves the cache.
    const int n_valid = min(len, ring ? a.ring_cap : cv.max_pages * kPage);
    const int blk_end = min(blk_lim, (n_valid + kPage - 1) / kPage);
    if (blk0 >= blk_end) return;
    const int tok_end = min(n_valid, blk_end * kPage);

    // Unit of a block: unit0 + entry * step, with the page as the entry (an invalid
    // one reads page 0, never outside the cache) or the ring's block.  Entries of the
    // 64 blocks from `first` on, one a lane.
    const int64_t unit0 = ring ? ((int64_t)b * cv.n_kv + kvl) * cv.ring_blocks : kvl;
    const int step = ring ? 1 : cv.n_kv;
    const int32_t* bt = cv.block_table + (int64_t)b * cv.max_pages;
    auto entries = [&](int from) -> int {
      const int blk = min(from + lane, blk_end - 1);
      if (ring) return blk;
      const int page = bt[blk];
      return page < 0 || page >= cv.num_pages ? 0 : page;
    };
    static_assert(kWave % kBlocks == 0, "a chunk's entries are in one register");
    int first = blk0;
    int ent = entries(first);
    auto unit_of = [&](int blk) -> int64_t {
      return unit0 + (int64_t)__builtin_amdgcn_readlane(ent, blk - first) * step;
    };

    // Q^T operand: column = query head, dimensions in the order of the K loads.
    bf16x8 q[D / 32];
    {
      const uint16_t* qp = reinterpret_cast<const uint16_t*>(a.q) + (int64_t)b * a.q_sb + (int64_t)(g * a.gs + col) * a.q_sh;
#pragma unroll
      for (int i = 0; i < D / 64; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          u32x4 w = {0u, 0u, 0u, 0u};
          if (col < a.gs) w = ld16(qp + 64 * i + 16 * G + 8 * h);
          q[2 * i + h] = __builtin_bit_cast(bf16x8, w);
        }
    }

    const uint8_t* ck = reinterpret_cast<const uint8_t*>(cv.k);
    const uint8_t* cvv = reinterpret_cast<const uint8_t*>(cv.v);
    if (a.k_new && len <= kMaxPos) {
      // Fused step: the wave whose range holds the token's block stores it before
      // it reads the block; no other wave reads this unit.
      const int p = len - 1;
      const int slot = !ring || p < a.n_sink ? p : a.n_sink + (p - a.n_sink) % a.window;
      const int blk = slot / kPage;
      if (blk >= blk0 && blk < blk_end) {
        int64_t unit = unit0 + blk;
        if (!ring) {
          const int page = __builtin_amdgcn_readfirstlane(bt[blk]);
          unit = page >= 0 && page < cv.num_pages ? unit0 + (int64_t)page * step : -1;
        }
        if (unit >= 0) {
          store_token<D, I8>(a, const_cast<uint8_t*>(ck) + unit * (kPage * D), const_cast<uint8_t*>(cvv) + unit * (kPage * D),
                             const_cast<uint8_t*>(cv.scales) + unit * kScaleBytes, b, g, slot % kPage);
          // The stores must reach the cache before this wave's loads of it.
          asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
      }
    }

    const int k_off = col * D + 16 * G;   // K row `col`, 64 bytes of it a load
    const int v_off = col * 64 + 16 * G;  // V tile (dimension quad col, rows 4G .. 4G + 3)
    // Blocks c .. c + kBlocks - 1; what lies past the end stays as it is (masked).
    // K and V of a chunk are loaded into the registers of the chunk before it, each
    // as soon as those are used up.
    Q8Chunk<D, BLOCKS> x;
    auto load_k = [&](int c) {
#pragma unroll
      for (int X = 0; X < kBlocks; ++X) {
        if (c + X >= blk_end) break;
        const int64_t u = unit_of(c + X);
#pragma unroll
        for (int i = 0; i < D / 64; ++i) x.k[X][i] = ld16_stream(ck + u * (kPage * D) + k_off + 64 * i);
        x.s[X] = ld8(cv.scales + u * kScaleBytes + 8 * G);
      }
    };
    auto load_v = [&](int c) {
#pragma unroll
      for (int X = 0; X < kBlocks; ++X) {
        if (c + X >= blk_end) break;
        const int64_t u = unit_of(c + X);
#pragma unroll
        for (int i = 0; i < D / 64; ++i) x.v[X][i] = ld16_stream(cvv + u * (kPage * D) + v_off + 1024 * i);
      }
    };
#pragma unroll
    for (int X = 0; X < kBlocks; ++X) {
#pragma unroll
      for (int i = 0; i < D / 64; ++i) x.k[X][i] = x.v[X][i] = u32x4{0u, 0u, 0u, 0u};
      x.s[X] = u32x2{0u, 0u};
    }

    // Finite, so that tokens whose score is -inf have weight 0 however the range is cut.
    float m_run = -FLT_MAX, l_run = 0.f;

    load_k(blk0);
    load_v(blk0);
    for (int c = blk0; c < blk_end; c += kBlocks) {
      const bool partial = (c + kBlocks) * kPage > tok_end;
      const int left = tok_end - c * kPage - 4 * G;
      float s[kBlocks][4];
      scores(x, q, s);
      u32x2 vs[kBlocks];
#pragma unroll
      for (int X = 0; X < kBlocks; ++X) vs[X] = x.s[X];
      const int next = c + kBlocks;
      if (next < blk_end) {
        if (next == first + kWave) {
          first = next;
          ent = entries(first);
        }
        load_k(next);
      }
      fold(a, x, s, vs, partial, left, acc, m_run, l_run);
      if (next < blk_end) load_v(next);
    }

    // acc[4j + n][i] is dimension 64 j + 16 G + 4 i + n
#pragma unroll
    for (int j = 0; j < D / 64; ++j)
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int i = 0; i < n; ++i) {
          const float t = acc[4 * j + n][i];
          acc[4 * j + n][i] = acc[4 * j + i][n];
          acc[4 * j + i][n] = t;
        }
    float l_tot = wave_xor_sum(l_run, 16);
    l_tot = xor32_sum(l_tot);
    m_out = m_run * a.scale_log2;
    l_out = l_tot;
  }
};

namespace {

// Waves of a workgroup, blocks of a chunk and waves of a SIMD (registers).  Width
// 128: chunks of 16 KB in 250 registers, two workgroups of four waves a CU.  Width
// 64, work-space pass: two of six waves with chunks of 4 KB, which suits short steps
// (one sequence of 4093 tokens 8.8 us; 9.3 with four waves and 8 KB, 8.9 with eight
// and 4 KB; 8 of 300-2000, int8, 10.4, 11.5 and 10.5) and is 1-8% behind in long ones
// (16 of 131072, 4 of 8 heads streaming, e4m3 / int8: 187 / 197 us, 183 / 185, 181 / 187,
// and 229 with four waves and 4 KB; 16 of 2000-32000, int8, 40.0, 38.1 and 37.0).  The
// pass for many items keeps four waves, since more of them cut the items further (300
// sequences of up to 900 tokens, int8: 56.6 us, 82.5 with six waves).
template <int D, bool I8>
void launch_format(const DecodeArgs& a, hipStream_t s) {
  if (a.many_wgs) {
    using Body = Q8Body<D, I8, 4, 4, 2>;
    hipLaunchKernelGGL((decode_many_kernel<Body>), dim3(a.many_wgs), dim3(Body::kWaves * kWave), 0, s, a);
  } else {
    using Body = std::conditional_t<D == 64, Q8Body<D, I8, 6, 2, 4>, Q8Body<D, I8, 4, 4, 2>>;
    hipLaunchKernelGGL((decode_ws_kernel<Body>), dim3(2 * a.ws_cu), dim3(Body::kWaves * kWave), 0, s, a);
  }
}

}  // namespace

hipError_t launch_decode_q8_split(const DecodeArgs& a, int d, int format, hipStream_t s) {
  if (d == 64) {
    if (format == kFormatI8) launch_format<64, true>(a, s);
    else launch_format<64, false>(a, s);
  } else {
    if (format == kFormatI8) launch_format<128, true>(a, s);
    else launch_format<128, false>(a, s);
  }
  return hipGetLastError();
}

}  // namespace aoh
