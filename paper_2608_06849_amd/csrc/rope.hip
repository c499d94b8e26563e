// Head norms and position rotation, and appends to the caches that apply them on the
// way.
//
// A row x (one token, one query or key head, D values) becomes
//   y_d = x_d / sqrt(mean(x^2) + eps) w_d           (with a weight; else y = x)
//   (y_i, y_j) -> (y_i c - y_j s, y_j c + y_i s)    for its n rotated pairs, pair i =
//     (i, i + n) or (2 i, 2 i + 1), c and s = scale times cosine and sine of position
//     times inv_freq[i]; values behind the first 2 n stay.
// fp32 arithmetic, rounded once at the end.  The angle is reduced to a fraction of a turn
// in fp64: its error stays below 2^-51 of the angle however far the position (three
// roundings of half a step: position times frequency, the constant 1 / 2 pi, their product).
//
// A workgroup takes up to 16 tokens (appends: those of one 16-position block, so of one
// page) and a range of heads.  The tokens' cosines and sines are computed once into LDS;
// a thread keeps one token and one 16-byte piece of its rows, so it reads its pairs'
// values once and then goes over the heads, with the rows of the next two on their way.
// The partners of a half-split pair meet in LDS within the wave.  Values of several tokens
// pass through an LDS tile into the dimension-major V pages, single tokens are stored from
// the row.
// Bound: memory, for single tokens the chain positions -> angles -> stores.  Measured: norms
// and rotation of 8192 tokens (40 heads of 128, bf16) 52 us from HBM, 3.2 TB/s; 16 packed
// prompts of 64 to 2900 tokens (48 heads) into caches 134 us, 3.9 TB/s (191 us with one row
// on its way and three waves a SIMD); one token of 64 sequences 10 us.
#include <algorithm>
#include <type_traits>

#include "aoh_device.h"
#include "aoh_internal.h"

namespace aoh {

// Orders a wave's LDS writes before its reads of what other lanes wrote.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Cosine and sine of position p times frequency f, times scale.  The turn's fraction is
// exact to fp64; for fp32 rows the functions are taken in fp64 too, so that what they add
// stays below fp32's own rounding.
template <typename T>
__device__ __forceinline__ float2 turn(int64_t p, float f, float scale) {
  constexpr double kPerTurn = 0.15915494309189533577;  // 1 / (2 pi)
  const double t = ((double)p * (double)f) * kPerTurn;
  const double r = 2.0 * (t - rint(t));
  if constexpr (sizeof(T) == 4) {
    double s, c;
    sincospi(r, &s, &c);
    return float2{(float)(c * scale), (float)(s * scale)};
  } else {
    float s, c;
    sincospif((float)r, &s, &c);
    return float2{c * scale, s * scale};
  }
}

// Sum over LANES consecutive lanes, the same in each: within 16 by the data-parallel moves
// (neighbours, pairs, mirrored halves and rows), which need no LDS.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float x) {
  x += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0xB1, 0xF, 0xF, true));
  x += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x4E, 0xF, 0xF, true));
  x += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x141, 0xF, 0xF, true));
  if (LANES >= 16) x += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x140, 0xF, 0xF, true));
  if (LANES >= 32) x = wave_xor_sum(x, 16);
  return x;
}

// Two values as bf16, the first in the low half.
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

template <int D, typename T, bool APPEND>
__global__ __launch_bounds__(256, 4) void rope_kernel(RopeArgs a) {
  constexpr int kVec = 16 / sizeof(T);       // values of a thread's piece of a row
  constexpr int kLanes = D / kVec;           // threads of a row
  constexpr int kSlots = 256 / kLanes;       // rows at a time
  constexpr int kToks = kSlots < kPage ? kSlots : kPage;
  constexpr int kRowsAhead = 2;              // rows on their way: 3 cost registers, 16 packed prompts 139 us instead of 134
  __shared__ __align__(16) float2 s_cs[kPage][D / 2];
  __shared__ __align__(16) float s_y[256 * kVec + 4];  // and four zeros
  __shared__ __align__(16) T s_v[APPEND ? kPage : 1][D + kVec];

  const int tid = threadIdx.x;
  const int b = APPEND ? blockIdx.z : 0;
  // This workgroup's tokens: `rows` of the tensors from row0 on (APPEND: of sequence b),
  // at cache positions from p0 on.
  int row0, n_tok, p0 = 0, end = 0;
  if constexpr (APPEND) {
    const int start = a.start_pos ? a.start_pos[b] : 0;
    int n_new = a.T;
    row0 = 0;
    if (a.cu_seqlens) {
      const int c0 = min(max(a.cu_seqlens[b], 0), a.total), c1 = min(max(a.cu_seqlens[b + 1], c0), a.total);
      n_new = min(c1 - c0, a.T);
      row0 = c0;
    }
    if (start < 0 || start > kMaxPos) return;  // no such positions: nothing is written
    end = start + n_new;
    const int first = (start / kPage + (int)blockIdx.x) * kPage;
    const int lo = max(start, first), hi = min(end, first + kPage);
    if (lo >= hi) return;
    n_tok = hi - lo;
    p0 = lo;
    row0 += lo - start;
  } else {
    row0 = (int)blockIdx.x * kPage;
    n_tok = min(kPage, a.B * a.T - row0);
  }
  const int h0 = blockIdx.y * a.heads_per_wg, h1 = min(h0 + a.heads_per_wg, a.Hq + (APPEND ? 2 : 1) * a.Hkv);

  if (tid < 4) s_y[256 * kVec + tid] = 0.f;
  // Cosines and sines, token by token.
  if (a.n_pairs && h0 < a.Hq + a.Hkv) {
    for (int e = tid; e < n_tok * a.n_pairs; e += 256) {
      const int t = e / a.n_pairs, i = e - t * a.n_pairs;
      const int flat = APPEND && !a.cu_seqlens ? b * a.T + row0 + t : row0 + t;
      int64_t p;
      if (a.positions) p = a.positions[a.axis[i] * a.pos_stride + flat];
      else if (APPEND) p = p0 + t;
      else p = (int64_t)(a.start_pos ? a.start_pos[flat / a.T] : 0) + flat % a.T;
      s_cs[t][i] = turn<T>(p, a.inv_freq[i], a.scale);
    }
  }
  __syncthreads();

  const int vl = tid % kLanes, slot = tid / kLanes;
  const int d0 = vl * kVec;
  // Rows at a time: nt tokens (a power of two) of kSlots / nt heads.
  int nt = 1;
  while (nt < n_tok && nt < kToks) nt *= 2;
  const bool tile_v = n_tok > 1;  // values pass through LDS
  for (int t0 = 0; t0 < n_tok; t0 += nt) {
    const int t = t0 + slot % nt;
    const bool have = t < n_tok;
    // Element e turns with its partner z: out = y c + z sn.  Where nothing turns z is a zero
    // and sn minus zero, which leaves every y as it is.
    float c[kVec], sn[kVec];
    int mate[kVec / 4];  // half-split pairs: places in s_y of the partners of the four values from 4 i on
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const int d = d0 + e, n = a.n_pairs;
      if (e % 4 == 0) mate[e / 4] = 256 * kVec;
      c[e] = 1.f;
      sn[e] = -0.f;
      if (have && d < 2 * n) {
        const int i = a.interleaved ? d >> 1 : (d < n ? d : d - n);
        const bool second = a.interleaved ? (d & 1) : d >= n;
        const float2 x = s_cs[t][i];
        c[e] = x.x;
        sn[e] = second ? x.y : -x.y;
        if (e % 4 == 0) mate[e / 4] = slot * D + (second ? d - n : d + n);
      }
    }
    int64_t qoff, koff, voff, qo, ko;
    {
      const int row = row0 + t;
      const int64_t sb = APPEND ? b : row / a.T, tok = APPEND ? row : row % a.T;
      qoff = sb * a.q_sb + tok * a.q_st;
      koff = sb * a.k_sb + tok * a.k_st;
      voff = sb * a.v_sb + tok * a.v_st;
      qo = sb * a.qo_sb + tok * a.qo_st;
      ko = sb * a.ko_sb + tok * a.ko_st;
    }
    // Where the token goes: a row of a page, a slot of a ring (dropped where a later one of
    // this call takes it).
    int page = -1, slot_at = -1;
    const int p = p0 + t;
    if (APPEND && have) {
      if (a.n_ret && p / kPage < a.max_pages) {
        const int x = a.block_table[(int64_t)b * a.max_pages + p / kPage];
        if (x >= 0 && x < a.num_pages) page = x;
      }
      if (a.n_str && (p < a.n_sink || p >= end - a.window))
        slot_at = p < a.n_sink ? p : a.n_sink + (p - a.n_sink) % a.window;
    }
    // The heads of one kind (0: queries, 1: keys, 2: single tokens' values) in [lo, hi), the
    // rows of the next kRowsAhead heads on their way while one is worked on.
    auto heads = [&](auto kind_c, int lo, int hi, const T* src, int64_t sh, const void* norm, T* out, int64_t osh) {
      constexpr int kind = decltype(kind_c)::value;
      if (lo >= hi) return;
      float w[kVec];
      if (kind < 2 && norm) {
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          w[e] = a.norm_f32 || sizeof(T) == 4 ? static_cast<const float*>(norm)[d0 + e]
                                              : bf16_to_f32(static_cast<const uint16_t*>(norm)[d0 + e]);
      }
      // whether head g's row goes anywhere
      auto wanted = [&](int g) {
        if (!have || g >= hi) return false;
        return kind == 0 || !APPEND || (((a.streaming_mask >> g) & 1ull) ? slot_at : page) >= 0;
      };
      const int step = kSlots / nt;
      int g = lo + slot / nt;
      u32x4 raw = {0u, 0u, 0u, 0u}, ahead[kRowsAhead];
      const T* at_src = src + g * sh + d0;
      const int64_t src_step = step * sh;
      if (wanted(g)) raw = ld16(at_src);
#pragma unroll
      for (int u = 0; u + 1 < kRowsAhead; ++u) {
        ahead[u] = u32x4{0u, 0u, 0u, 0u};
        if (wanted(g + (u + 1) * step)) ahead[u] = ld16(at_src + (u + 1) * src_step);
      }
#pragma unroll 1
      for (int hb = lo; hb < hi; hb += step, g += step) {
        ahead[kRowsAhead - 1] = u32x4{0u, 0u, 0u, 0u};
        if (wanted(g + kRowsAhead * step)) ahead[kRowsAhead - 1] = ld16(at_src + kRowsAhead * src_step);
        at_src += src_step;
        if (kind < 2 && (norm || a.n_pairs)) {
          float y[kVec];
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            if constexpr (sizeof(T) == 4) y[e] = __builtin_bit_cast(float, (uint32_t)raw[e]);
            else y[e] = bf16_to_f32((uint16_t)(raw[e / 2] >> (16 * (e & 1))));
          }
          if (norm) {
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < kVec; ++e) ss = fmaf(y[e], y[e], ss);
            const float r = 1.f / sqrtf(lanes_sum<kLanes>(ss) * (1.f / D) + a.eps);
#pragma unroll
            for (int e = 0; e < kVec; ++e) y[e] = y[e] * r * w[e];
          }
          if (a.n_pairs) {
            float z[kVec];
            if (a.interleaved) {
#pragma unroll
              for (int e = 0; e < kVec; ++e) z[e] = d0 + e < 2 * a.n_pairs ? y[e ^ 1] : 0.f;
            } else {  // partners in other lanes of the row
#pragma unroll
              for (int e = 0; e < kVec; e += 4) *reinterpret_cast<f32x4*>(s_y + tid * kVec + e) = f32x4{y[e], y[e + 1], y[e + 2], y[e + 3]};
              wave_lds_fence();
              if (a.n_pairs % 4 == 0) {
#pragma unroll
                for (int e = 0; e < kVec; e += 4) {
                  const f32x4 x = *reinterpret_cast<const f32x4*>(s_y + mate[e / 4]);
#pragma unroll
                  for (int i = 0; i < 4; ++i) z[e + i] = x[i];
                }
              } else {
#pragma unroll
                for (int e = 0; e < kVec; ++e) {
                  const int d = d0 + e, n = a.n_pairs;
                  z[e] = s_y[d < n ? slot * D + d + n : d < 2 * n ? slot * D + d - n : 256 * kVec];
                }
              }
              wave_lds_fence();
            }
#pragma unroll
            for (int e = 0; e < kVec; ++e) y[e] = fmaf(y[e], c[e], z[e] * sn[e]);
          }
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            if constexpr (sizeof(T) == 4) raw[e] = __builtin_bit_cast(uint32_t, y[e]);
            else if (e & 1) raw[e / 2] = bf16_pair(y[e - 1], y[e]);
          }
        }
        if (wanted(g)) {
          if (kind == 0 || !APPEND) {
            st16(out + g * osh + d0, raw);
          } else {
            const bool str = (a.streaming_mask >> g) & 1ull;
            const int at = str ? slot_at : page;
            const int64_t unit = str ? ((int64_t)b * a.n_str + a.rank[g]) * a.ring_blocks + at / kPage : (int64_t)at * a.n_ret + a.rank[g];
            const int r = (str ? at : p) % kPage;
            if (kind == 1) {
              st16(static_cast<T*>(str ? a.rk : a.pk) + unit * (kPage * D) + r * D + d0, raw);
            } else {
              T* dst = static_cast<T*>(str ? a.rv : a.pv) + unit * (kPage * D);
              if (!str && a.v_token_major) {
                st16(dst + r * D + d0, raw);
              } else {
                T x[kVec];
                __builtin_memcpy(x, &raw, 16);
#pragma unroll
                for (int e = 0; e < kVec; ++e) dst[(d0 + e) * kPage + r] = x[e];
              }
            }
          }
        }
        raw = ahead[0];
#pragma unroll
        for (int u = 0; u + 1 < kRowsAhead; ++u) ahead[u] = ahead[u + 1];
      }
    };
    heads(std::integral_constant<int, 0>{}, h0, min(h1, a.Hq), static_cast<const T*>(a.q) + qoff, a.q_sh, a.q_norm,
          static_cast<T*>(a.q_out) + qo, a.qo_sh);
    heads(std::integral_constant<int, 1>{}, max(0, h0 - a.Hq), min(h1 - a.Hq, a.Hkv), static_cast<const T*>(a.k) + koff, a.k_sh, a.k_norm,
          static_cast<T*>(a.k_out) + ko, a.ko_sh);
    if (APPEND && !tile_v)
      heads(std::integral_constant<int, 2>{}, max(0, h0 - a.Hq - a.Hkv), h1 - a.Hq - a.Hkv, static_cast<const T*>(a.v) + voff, a.v_sh, nullptr,
            static_cast<T*>(nullptr), 0);
  }
  if constexpr (APPEND) {
    if (!tile_v) return;
    // Values of several tokens, head by head.
    const int lp = p0 / kPage;
    const int r0 = p0 % kPage;  // row of the first token in a page
    int page = -1;
    if (a.n_ret && lp < a.max_pages) {
      page = a.block_table[(int64_t)b * a.max_pages + lp];
      if (page >= a.num_pages) page = -1;
    }
    auto kept = [&](int p) { return p < a.n_sink || p >= end - a.window; };
    auto slot_of = [&](int p) { return p < a.n_sink ? p : a.n_sink + (p - a.n_sink) % a.window; };
    const bool some = kept(p0) || kept(p0 + n_tok - 1);
    // the first head from h on whose values go anywhere
    auto next_head = [&](int h) {
      while (h < h1 && !(((a.streaming_mask >> (h - a.Hq - a.Hkv)) & 1ull) ? some : page >= 0)) ++h;
      return h;
    };
    constexpr int kPieces = (kPage * kLanes + 255) / 256;  // of a thread, a head
    u32x4 piece[kPieces];
    auto load = [&](int h) {
      if (h >= h1) return;
      const T* src = static_cast<const T*>(a.v) + b * a.v_sb + row0 * a.v_st + (h - a.Hq - a.Hkv) * a.v_sh;
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const int e = tid + 256 * i;
        if (e < n_tok * kLanes) piece[i] = ld16(src + e / kLanes * a.v_st + e % kLanes * kVec);
      }
    };
    int h = next_head(max(h0, a.Hq + a.Hkv));
    load(h);
    for (int ahead; h < h1; h = ahead) {
      const int g = h - a.Hq - a.Hkv;
      const bool str = (a.streaming_mask >> g) & 1ull;
      ahead = next_head(h + 1);
      if (!str && a.v_token_major) {
        T* dst = static_cast<T*>(a.pv) + ((int64_t)page * a.n_ret + a.rank[g]) * (kPage * D);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          const int e = tid + 256 * i;
          if (e < n_tok * kLanes) st16(dst + (r0 + e / kLanes) * D + e % kLanes * kVec, piece[i]);
        }
        load(ahead);
        continue;
      }
      __syncthreads();  // the tile of the head before has been read
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const int e = tid + 256 * i;
        if (e < n_tok * kLanes) *reinterpret_cast<u32x4*>(&s_v[e / kLanes][e % kLanes * kVec]) = piece[i];
      }
      load(ahead);
      __syncthreads();
      // Whole 16-byte pieces where the tokens fill a page, or a block of the ring.
      bool whole = n_tok == kPage;
      int64_t unit = str ? ((int64_t)b * a.n_str + a.rank[g]) * a.ring_blocks : (int64_t)page * a.n_ret + a.rank[g];
      T* dst = static_cast<T*>(str ? a.rv : a.pv);
      if (str) {
        const int first = slot_of(p0);
        whole = whole && kept(p0) && first % kPage == 0 && slot_of(p0 + kPage - 1) == first + kPage - 1 &&
                (p0 + kPage <= a.n_sink || p0 >= max(a.n_sink, end - a.window));
        if (whole) unit += first / kPage;
      }
      dst += unit * (kPage * D);
      if (whole) {
        for (int e = tid; e < D * (kPage / kVec); e += 256) {
          const int d = e / (kPage / kVec), t = e % (kPage / kVec) * kVec;
          T x[kVec];
#pragma unroll
          for (int i = 0; i < kVec; ++i) x[i] = s_v[t + i][d];
          u32x4 y;
          __builtin_memcpy(&y, x, 16);
          st16(dst + d * kPage + t, y);
        }
      } else {
        for (int e = tid; e < D * kPage; e += 256) {
          const int d = e / kPage, t = e % kPage;
          if (t >= n_tok) continue;
          if (!str) {
            dst[d * kPage + r0 + t] = s_v[t][d];
          } else if (kept(p0 + t)) {
            const int at = slot_of(p0 + t);
            dst[(int64_t)(at / kPage) * (kPage * D) + d * kPage + at % kPage] = s_v[t][d];
          }
        }
      }
    }
  }
}

// Heads a workgroup: enough workgroups to fill the GPU first, then as many heads as
// possible for each computation of the angles.  Appends have sequences of different lengths
// and fewer key and value heads that go anywhere, and take more and smaller workgroups: 16
// packed prompts of 64 to 2900 tokens 134 us with 4096, 147 with 2048; a prompt of 8192
// tokens without caches 52 us with 1024, 70 with 4096, 57 with 512.
template <bool APPEND>
constexpr int kRopeWgs = APPEND ? 4096 : 1024;

template <int D, typename T, bool APPEND>
static hipError_t launch(RopeArgs a, int64_t tiles, hipStream_t s) {
  const int heads = a.Hq + (APPEND ? 2 : 1) * a.Hkv;
  const int64_t all = tiles * (APPEND ? a.B : 1);
  const int64_t groups = std::max<int64_t>(1, std::min<int64_t>((kRopeWgs<APPEND> + all - 1) / all, (heads + 3) / 4));
  a.heads_per_wg = (int)((heads + groups - 1) / groups);
  const int64_t gy = (heads + a.heads_per_wg - 1) / a.heads_per_wg;
  // The runtime takes a launch's work-items modulo 2^32, and a grid has at most 65535
  // layers: larger batches go in parts.
  const int64_t part = APPEND ? std::max<int64_t>(1, std::min<int64_t>(65535, (1ll << 31) / (tiles * gy * 256))) : a.B;
  for (int b0 = 0, B = a.B; b0 < B; b0 += (int)part) {
    RopeArgs x = a;
    if (APPEND) {
      x.B = (int)std::min<int64_t>(part, B - b0);
      x.q = static_cast<const T*>(a.q) + b0 * a.q_sb;
      x.q_out = static_cast<T*>(a.q_out) + b0 * a.qo_sb;
      x.k = static_cast<const T*>(a.k) + b0 * a.k_sb;
      x.v = static_cast<const T*>(a.v) + b0 * a.v_sb;
      if (a.positions && !a.cu_seqlens) x.positions += (int64_t)b0 * a.T;
      if (a.start_pos) x.start_pos += b0;
      if (a.cu_seqlens) x.cu_seqlens += b0;
      if (a.block_table) x.block_table += (int64_t)b0 * a.max_pages;
      const int64_t ring = (int64_t)b0 * a.n_str * a.ring_blocks * (kPage * D);
      if (a.n_str) {
        x.rk = static_cast<T*>(a.rk) + ring;
        x.rv = static_cast<T*>(a.rv) + ring;
      }
    }
    hipLaunchKernelGGL((rope_kernel<D, T, APPEND>), dim3((unsigned)tiles, (unsigned)gy, APPEND ? x.B : 1), dim3(256), 0, s, x);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

hipError_t launch_rope(const RopeArgs& a, int dtype, int d, bool append, hipStream_t s) {
  // an append's tokens may begin anywhere in a page
  const int64_t tiles = append ? ((int64_t)a.T + kPage - 1 + (a.start_pos ? kPage - 1 : 0)) / kPage
                               : ((int64_t)a.B * a.T + kPage - 1) / kPage;
  if (append) {
    if (dtype == 1) return d == 64 ? launch<64, float, true>(a, tiles, s) : launch<128, float, true>(a, tiles, s);
    return d == 64 ? launch<64, uint16_t, true>(a, tiles, s) : launch<128, uint16_t, true>(a, tiles, s);
  }
  if (dtype == 1) return d == 64 ? launch<64, float, false>(a, tiles, s) : launch<128, float, false>(a, tiles, s);
  return d == 64 ? launch<64, uint16_t, false>(a, tiles, s) : launch<128, uint16_t, false>(a, tiles, s);
}

}  // namespace aoh
