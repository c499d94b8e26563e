// Attention of new tokens over the caches and over themselves (paper Sec. 5,
// chunked-prefill stage: retrieval heads see the whole cached prefix, streaming heads what
// their sink + recent cache holds).
//
// Query t of sequence b stands at position start_pos[b] + t.  Its keys are the cached
// positions below start_pos[b] (paged cache, or the ring's slots) and the new tokens
// 0 .. t, whose K/V come from the call's tensors: the append runs after the attention, so
// the ring still holds what the first new queries see of the window.
#include <algorithm>

#include "aoh_device.h"
#include "aoh_internal.h"

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

// A wave takes 64 keys at a time, one a lane, then the lanes take the output's dimensions.
template <int D, typename T>
__global__ __launch_bounds__(256) void extend_simple_kernel(ExtendArgs a) {
#pragma clang fp contract(off)
  constexpr int kDims = D / kWave;
  __shared__ float s_q[D];
  __shared__ int64_t s_at[4][kWave];
  __shared__ float s_p[4][kWave];
  __shared__ float s_o[4][D], s_m[4], s_l[4];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  auto value = [](const void* p, int64_t i) {
    if constexpr (sizeof(T) == 4) return static_cast<const float*>(p)[i];
    else return bf16_to_f32(static_cast<const uint16_t*>(p)[i]);
  };
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
      if (a.out_f32 || sizeof(T) == 4) static_cast<float*>(a.out)[at] = x;
      else static_cast<uint16_t*>(a.out)[at] = f32_to_bf16_bits(x);
    }
  }
}

template <int D, typename T>
static hipError_t launch_simple(const ExtendArgs& a, hipStream_t s) {
  const int64_t rows = (int64_t)a.B * a.T * a.Hq;
  hipLaunchKernelGGL((extend_simple_kernel<D, T>), dim3((unsigned)std::min<int64_t>(rows, 1 << 16)), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_extend(const ExtendArgs& a, int dtype, int d, hipStream_t s) {
  if (dtype == 1) return d == 64 ? launch_simple<64, float>(a, s) : launch_simple<128, float>(a, s);
  return d == 64 ? launch_simple<64, uint16_t>(a, s) : launch_simple<128, uint16_t>(a, s);
}

}  // namespace aoh
