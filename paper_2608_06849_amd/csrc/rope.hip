// Head norms and position rotation, and appends to the caches that apply them on the
// way.
//
// A row x (one token, one query or key head, D values) becomes
//   y_d = x_d / sqrt(mean(x^2) + eps) w_d           (with a weight; else y = x)
//   (y_i, y_j) -> (y_i c - y_j s, y_j c + y_i s)    for its n rotated pairs, pair i =
//     (i, i + n) or (2 i, 2 i + 1), c and s = scale times cosine and sine of position
//     times inv_freq[i]; values behind the first 2 n stay.
// fp32 arithmetic, rounded once at the end.  The angle is reduced to a fraction of a turn
// in fp64: its error stays below 2^-52 of the angle however far the position.
//
// A workgroup takes up to 16 tokens (appends: those of one 16-position block, so of one
// page) and a range of heads.  The tokens' cosines and sines are computed once into LDS;
// a thread keeps one token and one 16-byte piece of its rows, so it reads its pairs'
// values once and then goes over the heads.  The partners of a half-split pair meet in
// LDS within the wave.  Values of several tokens pass through an LDS tile into the
// dimension-major V pages, single tokens are stored from the row.
// Bound: memory, for single tokens the chain positions -> angles -> stores.
#include <algorithm>

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

template <int D, typename T, bool APPEND>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  constexpr int kVec = 16 / sizeof(T);       // values of a thread's piece of a row
  constexpr int kLanes = D / kVec;           // threads of a row
  constexpr int kSlots = 256 / kLanes;       // rows at a time
  constexpr int kToks = kSlots < kPage ? kSlots : kPage;
  __shared__ __align__(16) float2 s_cs[kPage][D / 2];
  __shared__ __align__(16) float s_y[256][kVec];
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
  float w[2][kVec];  // weights of this thread's values: queries, keys
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const void* p = i ? a.k_norm : a.q_norm;
    if (!p) continue;
#pragma unroll
    for (int e = 0; e < kVec; ++e)
      w[i][e] = a.norm_f32 || sizeof(T) == 4 ? static_cast<const float*>(p)[d0 + e]
                                              : bf16_to_f32(static_cast<const uint16_t*>(p)[d0 + e]);
  }

  const bool tile_v = n_tok > 1;  // values pass through LDS
  const int h_rows = APPEND && !tile_v ? h1 : min(h1, a.Hq + a.Hkv);
  for (int t0 = 0; t0 < n_tok; t0 += nt) {
    const int t = t0 + slot % nt;
    const bool have = t < n_tok;
    // element e turns with its partner: out = y c + partner sn
    float c[kVec], sn[kVec];
    int mate[kVec];  // partner's dimension, or -1
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const int d = d0 + e, n = a.n_pairs;
      mate[e] = -1;
      c[e] = 1.f;
      sn[e] = 0.f;
      if (have && d < 2 * n) {
        const int i = a.interleaved ? d >> 1 : (d < n ? d : d - n);
        const bool second = a.interleaved ? (d & 1) : d >= n;
        const float2 x = s_cs[t][i];
        c[e] = x.x;
        sn[e] = second ? x.y : -x.y;
        mate[e] = a.interleaved ? d ^ 1 : second ? d - n : d + n;
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
    for (int hb = h0; hb < h_rows; hb += kSlots / nt) {
      const int h = hb + slot / nt;
      const bool on = have && h < h_rows;
      const int kind = h < a.Hq ? 0 : h < a.Hq + a.Hkv ? 1 : 2;  // query, key, value
      const int g = kind == 0 ? h : kind == 1 ? h - a.Hq : h - a.Hq - a.Hkv;
      u32x4 raw = {0u, 0u, 0u, 0u};
      if (on) {
        const T* src = kind == 0 ? static_cast<const T*>(a.q) + qoff + g * a.q_sh
                                 : kind == 1 ? static_cast<const T*>(a.k) + koff + g * a.k_sh
                                             : static_cast<const T*>(a.v) + voff + g * a.v_sh;
        raw = ld16(src + d0);
      }
      const bool norm = kind == 0 ? a.q_norm != nullptr : kind == 1 && a.k_norm != nullptr;
      if (a.n_pairs || a.q_norm || a.k_norm) {
        float y[kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          if constexpr (sizeof(T) == 4) y[e] = __builtin_bit_cast(float, (uint32_t)raw[e]);
          else y[e] = bf16_to_f32((uint16_t)(raw[e / 2] >> (16 * (e & 1))));
        }
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < kVec; ++e) ss = fmaf(y[e], y[e], ss);
#pragma unroll
        for (int m = 1; m < kLanes; m *= 2) ss = wave_xor_sum(ss, m);
        if (norm) {
          const float r = 1.f / sqrtf(ss * (1.f / D) + a.eps);
#pragma unroll
          for (int e = 0; e < kVec; ++e) y[e] = y[e] * r * (kind ? w[1][e] : w[0][e]);
        }
        float z[kVec];
        if (a.n_pairs) {
          if (!a.interleaved) {  // partners in other lanes of the row
#pragma unroll
            for (int e = 0; e < kVec; e += 4) *reinterpret_cast<f32x4*>(&s_y[tid][e]) = f32x4{y[e], y[e + 1], y[e + 2], y[e + 3]};
            wave_lds_fence();
            const float* line = &s_y[slot * kLanes][0];
#pragma unroll
            for (int e = 0; e < kVec; ++e) z[e] = line[mate[e] < 0 ? 0 : mate[e]];
            wave_lds_fence();
          } else {
#pragma unroll
            for (int e = 0; e < kVec; ++e) z[e] = y[e ^ 1];
          }
#pragma unroll
          for (int e = 0; e < kVec; ++e)
            if (mate[e] >= 0 && kind < 2) y[e] = fmaf(y[e], c[e], z[e] * sn[e]);
        }
        if (kind < 2 && (norm || a.n_pairs)) {
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            if constexpr (sizeof(T) == 4) raw[e] = __builtin_bit_cast(uint32_t, y[e]);
            else if (e & 1) raw[e / 2] = (uint32_t)f32_to_bf16_bits(y[e - 1]) | ((uint32_t)f32_to_bf16_bits(y[e]) << 16);
          }
        }
      }
      if (!on) continue;
      if (kind == 0) {
        st16(static_cast<T*>(a.q_out) + qo + g * a.qo_sh + d0, raw);
      } else if (!APPEND) {
        st16(static_cast<T*>(a.k_out) + ko + g * a.ko_sh + d0, raw);
      } else {
        const bool str = (a.streaming_mask >> g) & 1ull;
        const int at = str ? slot_at : page;
        if (at < 0) continue;
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
    for (int h = max(h0, a.Hq + a.Hkv); h < h1; ++h) {
      const int g = h - a.Hq - a.Hkv;
      const bool str = (a.streaming_mask >> g) & 1ull;
      if (str ? !(kept(p0) || kept(p0 + n_tok - 1)) : page < 0) continue;  // uniform
      const T* src = static_cast<const T*>(a.v) + b * a.v_sb + row0 * a.v_st + g * a.v_sh;
      if (!str && a.v_token_major) {
        T* dst = static_cast<T*>(a.pv) + ((int64_t)page * a.n_ret + a.rank[g]) * (kPage * D);
        for (int e = tid; e < n_tok * kLanes; e += 256) {
          const int t = e / kLanes, d = e % kLanes * kVec;
          st16(dst + (r0 + t) * D + d, ld16(src + t * a.v_st + d));
        }
        continue;
      }
      __syncthreads();  // the tile of the head before has been read
      for (int e = tid; e < n_tok * kLanes; e += 256) {
        const int t = e / kLanes, d = e % kLanes * kVec;
        *reinterpret_cast<u32x4*>(&s_v[t][d]) = ld16(src + t * a.v_st + d);
      }
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
// possible for each computation of the angles.
constexpr int kRopeWgs = 1024;

template <int D, typename T, bool APPEND>
static hipError_t launch(RopeArgs a, int64_t tiles, hipStream_t s) {
  const int heads = a.Hq + (APPEND ? 2 : 1) * a.Hkv;
  const int64_t all = tiles * (APPEND ? a.B : 1);
  const int64_t groups = std::max<int64_t>(1, std::min<int64_t>((kRopeWgs + all - 1) / all, (heads + 3) / 4));
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
