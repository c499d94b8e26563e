// Writing the 8-bit caches and reading them back (layout and codes: q8.h).
//
// Both passes give a workgroup the 16 positions of a logical page of one
// (sequence, KV head), 2 D threads: thread t has dimensions 8 (t % (D / 8)) .. + 7
// of position t / (D / 8), one 16-byte load of bf16 for K and one for V.  The
// largest magnitude of a row is found among the D / 8 lanes that hold it.  V
// codes pass through LDS, which turns rows into the unit's 4 x 4 tiles, wherever
// the 16 positions are one whole unit; elsewhere (the ends of an append, a ring
// whose blocks are not page-aligned) they are single bytes.
// The start positions and lengths are read on the device, so the grid depends
// on the number of tokens only.
#include <algorithm>

#include "aoh_internal.h"
#include "q8.h"

namespace aoh {

namespace {

// Rows of 20 words: 16 for the unit's rows, padded so that 16-byte reads of four
// rows stay aligned and the writes of a wave spread over the banks.
constexpr int kTileStride = 20;

template <int D>
using VTiles = uint32_t[D / 4][kTileStride];

// 4 x 4 bytes transposed: byte j of out[i] is byte i of in[j].
__device__ __forceinline__ u32x4 transpose4(u32x4 r) {
  const uint32_t t0 = __builtin_amdgcn_perm(r[1], r[0], 0x05010400u), t1 = __builtin_amdgcn_perm(r[1], r[0], 0x07030602u);
  const uint32_t u0 = __builtin_amdgcn_perm(r[3], r[2], 0x05010400u), u1 = __builtin_amdgcn_perm(r[3], r[2], 0x07030602u);
  return u32x4{__builtin_amdgcn_perm(u0, t0, 0x05040100u), __builtin_amdgcn_perm(u0, t0, 0x07060302u),
               __builtin_amdgcn_perm(u1, t1, 0x05040100u), __builtin_amdgcn_perm(u1, t1, 0x07060302u)};
}

// Eight consecutive values as fp32.
__device__ __forceinline__ void load8(const uint16_t* p, float (&x)[8]) {
  const u32x4 w = ld16(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __builtin_bit_cast(float, w[i] << 16);
    x[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = a[i];
    x[4 + i] = b[i];
  }
}

// Eight values code * scale; both types hold them exactly.
template <bool I8>
__device__ __forceinline__ void store8(uint16_t* p, u32x2 w, float scale) {
  u32x4 o;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    f32x4 x = codes_to_f32<I8>(w[h]);
    uint32_t f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __builtin_bit_cast(uint32_t, x[i] * scale);
    o[2 * h] = __builtin_amdgcn_perm(f[1], f[0], 0x07060302u);
    o[2 * h + 1] = __builtin_amdgcn_perm(f[3], f[2], 0x07060302u);
  }
  st16(p, o);
}
template <bool I8>
__device__ __forceinline__ void store8(float* p, u32x2 w, float scale) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    f32x4 x = codes_to_f32<I8>(w[h]);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] *= scale;
    *reinterpret_cast<f32x4*>(p + 4 * h) = x;
  }
}

// 2^E of a scale byte, NaN for 255.
__device__ __forceinline__ float row_scale(uint32_t byte) {
  return __builtin_bit_cast(float, byte == 255u ? 0x7fc00000u : byte << 23);
}

// Codes and scale byte of the row that D / 8 neighbouring lanes hold.
template <int D, bool I8>
__device__ __forceinline__ u32x2 quantise8(const float (&x)[8], uint32_t& byte) {
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) amax = max(amax, __builtin_bit_cast(uint32_t, x[i]) & 0x7fffffffu);
#pragma unroll
  for (int o = 1; o < D / 8; o <<= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, o, kWave));
  byte = scale_byte<I8>(amax);
  const float inv = inverse_scale(byte);
  return u32x2{to_codes<I8>(x, inv, byte == 255u), to_codes<I8>(x + 4, inv, byte == 255u)};
}

__device__ __forceinline__ int ring_slot(int p, int n_sink, int window) {
  return p < n_sink ? p : n_sink + (p - n_sink) % window;
}

}  // namespace

template <int D, typename T, bool I8>
__global__ __launch_bounds__(2 * D) void append_q8_kernel(Q8Args a) {
  __shared__ __align__(16) VTiles<D> vt;
  const int g = blockIdx.y, b = blockIdx.z;
  int64_t row0 = 0;  // first row of the sequence in a packed tensor
  int n = a.n;
  if (a.cu_seqlens) {
    const int lo = min(max(a.cu_seqlens[b], 0), a.total), hi = min(max(a.cu_seqlens[b + 1], 0), a.total);
    row0 = lo;
    n = min(n, hi - lo);
  }
  const int start = a.start_pos ? a.start_pos[b] : 0;
  if (start < 0 || start >= kMaxPos || n <= 0) return;  // an invalid start position writes nothing
  const int end = start + n;
  const int lp = start / kPage + a.chunk0 + (int)blockIdx.x;
  const int p_lo = max(lp * kPage, start), p_hi = min(lp * kPage + kPage, end);
  if (p_lo >= p_hi) return;
  const bool streaming = (a.streaming_mask >> g) & 1ull;
  // ring: a later position of this call overwrites all others
  auto kept = [&](int p) { return !streaming || p < a.n_sink || p >= end - a.window; };
  if (!kept(p_lo) && !kept(p_hi - 1)) return;
  if (!streaming && lp >= a.max_pages) return;  // beyond the block table

  const int tid = threadIdx.x;
  const int row = tid / (D / 8), c = tid % (D / 8);
  const int p = lp * kPage + row;
  const bool on = p >= p_lo && p < p_hi && kept(p);
  float kx[8] = {}, vx[8] = {};
  if (on) {
    const int64_t t = row0 + (p - start);
    load8(reinterpret_cast<const T*>(a.k) + (int64_t)b * a.k_sb + t * a.k_st + (int64_t)g * a.k_sh + 8 * c, kx);
    load8(reinterpret_cast<const T*>(a.v) + (int64_t)b * a.v_sb + t * a.v_st + (int64_t)g * a.v_sh + 8 * c, vx);
  }

  int64_t unit;
  int r = row;
  bool whole = p_hi - p_lo == kPage;  // the 16 positions are one unit
  uint8_t *ck, *cv, *cs;
  if (!streaming) {
    const int page = a.block_table[(int64_t)b * a.max_pages + lp];
    if (page < 0 || page >= a.num_pages) return;  // unmapped
    unit = (int64_t)page * a.n_ret + a.rank[g];
    ck = a.pk;
    cv = a.pv;
    cs = a.ps;
  } else {
    if (whole) {
      const int first = ring_slot(p_lo, a.n_sink, a.window);
      whole = first % kPage == 0 && ring_slot(p_hi - 1, a.n_sink, a.window) == first + kPage - 1 &&
              (p_hi <= a.n_sink || p_lo >= max(a.n_sink, end - a.window));
    }
    const int slot = ring_slot(p, a.n_sink, a.window);
    unit = ((int64_t)b * a.n_str + a.rank[g]) * a.ring_blocks + slot / kPage;
    r = slot % kPage;
    ck = a.rk;
    cv = a.rv;
    cs = a.rs;
  }

  uint32_t kb, vb;
  const u32x2 kw = quantise8<D, I8>(kx, kb), vw = quantise8<D, I8>(vx, vb);
  if (on) {
    *reinterpret_cast<u32x2*>(ck + unit * (kPage * D) + r * D + 8 * c) = kw;
    if (c == 0) *reinterpret_cast<uint16_t*>(cs + unit * kScaleBytes + 2 * r) = (uint16_t)(kb | (vb << 8));
  }
  uint8_t* uv = cv + unit * (kPage * D);
  if (whole) {  // uniform; row r of the unit is row `row`
    vt[2 * c][row] = vw[0];
    vt[2 * c + 1][row] = vw[1];
    __syncthreads();
    if (tid < D) st16(uv + 16 * tid, transpose4(ld16(&vt[tid >> 2][4 * (tid & 3)])));
  } else if (on) {
#pragma unroll
    for (int i = 0; i < 8; ++i) uv[v_offset(8 * c + i, r)] = (uint8_t)(vw[i >> 2] >> (8 * (i & 3)));
  }
}

template <int D, typename T, bool I8>
__global__ __launch_bounds__(2 * D) void read_q8_kernel(Q8Args a) {
  __shared__ __align__(16) VTiles<D> vt;
  const int g = blockIdx.y, b = blockIdx.z;
  const int start = a.start_pos ? a.start_pos[b] : 0;
  if (start < 0 || start >= kMaxPos) return;
  const int len = a.lens[b];
  const int end = min(start + a.n, len);
  const int lp = start / kPage + a.chunk0 + (int)blockIdx.x;
  const int p_lo = max(lp * kPage, start), p_hi = min(lp * kPage + kPage, end);
  if (p_lo >= p_hi) return;
  const bool streaming = (a.streaming_mask >> g) & 1ull;
  auto held = [&](int p) { return !streaming || p < a.n_sink || p >= len - a.window; };
  if (!held(p_lo) && !held(p_hi - 1)) return;
  if (!streaming && lp >= a.max_pages) return;

  const int tid = threadIdx.x;
  const int row = tid / (D / 8), c = tid % (D / 8);
  const int p = lp * kPage + row;
  const bool on = p >= p_lo && p < p_hi && held(p);
  int64_t unit;
  int r = row;
  bool whole = true;
  const uint8_t *ck, *cv, *cs;
  if (!streaming) {
    const int page = a.block_table[(int64_t)b * a.max_pages + lp];
    if (page < 0 || page >= a.num_pages) return;
    unit = (int64_t)page * a.n_ret + a.rank[g];
    ck = a.pk;
    cv = a.pv;
    cs = a.ps;
  } else {
    const int first = ring_slot(p_lo, a.n_sink, a.window);
    whole = p_hi - p_lo == kPage && first % kPage == 0 && held(p_lo) && held(p_hi - 1) &&
            ring_slot(p_hi - 1, a.n_sink, a.window) == first + kPage - 1 &&
            (p_hi <= a.n_sink || p_lo >= max(a.n_sink, len - a.window));
    const int slot = ring_slot(p, a.n_sink, a.window);
    unit = ((int64_t)b * a.n_str + a.rank[g]) * a.ring_blocks + slot / kPage;
    r = slot % kPage;
    ck = a.rk;
    cv = a.rv;
    cs = a.rs;
  }
  u32x2 kw = {0u, 0u}, vw = {0u, 0u};
  uint32_t sw = 0;
  if (on) {
    kw = *reinterpret_cast<const u32x2*>(ck + unit * (kPage * D) + r * D + 8 * c);
    sw = *reinterpret_cast<const uint16_t*>(cs + unit * kScaleBytes + 2 * r);
  }
  const uint8_t* uv = cv + unit * (kPage * D);
  if (whole) {  // uniform
    if (tid < D) *reinterpret_cast<u32x4*>(&vt[tid >> 2][4 * (tid & 3)]) = transpose4(ld16(uv + 16 * tid));
    __syncthreads();
    vw = u32x2{vt[2 * c][row], vt[2 * c + 1][row]};
  } else if (on) {
#pragma unroll
    for (int i = 0; i < 8; ++i) vw[i >> 2] |= (uint32_t)uv[v_offset(8 * c + i, r)] << (8 * (i & 3));
  }
  if (on) {
    const int64_t t = p - start;
    store8<I8>(reinterpret_cast<T*>(const_cast<void*>(a.k)) + (int64_t)b * a.k_sb + t * a.k_st + (int64_t)g * a.k_sh + 8 * c,
               kw, row_scale(sw & 0xffu));
    store8<I8>(reinterpret_cast<T*>(const_cast<void*>(a.v)) + (int64_t)b * a.v_sb + t * a.v_st + (int64_t)g * a.v_sh + 8 * c,
               vw, row_scale(sw >> 8));
  }
}

namespace {

template <int D, typename T, bool I8>
void launch_part(const Q8Args& a, bool write, dim3 grid, hipStream_t s) {
  if (write) hipLaunchKernelGGL((append_q8_kernel<D, T, I8>), grid, dim3(2 * D), 0, s, a);
  else hipLaunchKernelGGL((read_q8_kernel<D, T, I8>), grid, dim3(2 * D), 0, s, a);
}

template <int D>
void launch_width(const Q8Args& a, int dtype, int format, bool write, dim3 grid, hipStream_t s) {
  if (dtype == 1) {
    if (format == kFormatI8) launch_part<D, float, true>(a, write, grid, s);
    else launch_part<D, float, false>(a, write, grid, s);
  } else {
    if (format == kFormatI8) launch_part<D, uint16_t, true>(a, write, grid, s);
    else launch_part<D, uint16_t, false>(a, write, grid, s);
  }
}

}  // namespace

// The runtime takes a launch's work-items modulo 2^32, so a grid of 2^31 and more
// goes in parts: of the chunks of one sequence, or of whole sequences.
hipError_t launch_q8(const Q8Args& a, int dtype, int format, int d, bool write, hipStream_t s) {
  const int64_t per_chunk = (int64_t)a.Hkv * 2 * d;
  const int64_t most = ((int64_t)1 << 31) / per_chunk;  // chunks of a launch
  const int64_t chunks = ((int64_t)a.n + kPageTokens - 1) / kPageTokens + 1;
  const int64_t seqs = std::min<int64_t>(std::max<int64_t>(1, most / chunks), 65535);
  const int es = dtype == 1 ? 4 : 2;
  for (int64_t b0 = 0; b0 < a.B; b0 += seqs) {
    Q8Args p = a;
    if (a.cu_seqlens) {
      p.cu_seqlens += b0;
    } else {
      p.k = static_cast<const char*>(a.k) + b0 * a.k_sb * es;
      p.v = static_cast<const char*>(a.v) + b0 * a.v_sb * es;
    }
    if (a.start_pos) p.start_pos += b0;
    if (a.lens) p.lens += b0;
    if (a.block_table) p.block_table += b0 * a.max_pages;
    const int64_t ring = b0 * a.n_str * a.ring_blocks;  // units of the rings before
    if (a.rk) {
      p.rk += ring * kPageTokens * d;
      p.rv += ring * kPageTokens * d;
      p.rs += ring * 2 * kPageTokens;
    }
    for (int64_t c0 = 0; c0 < chunks; c0 += most) {
      p.chunk0 = (int)c0;
      const dim3 grid((unsigned)std::min(most, chunks - c0), (unsigned)a.Hkv, (unsigned)std::min<int64_t>(seqs, a.B - b0));
      if (d == 64) launch_width<64>(p, dtype, format, write, grid, s);
      else launch_width<128>(p, dtype, format, write, grid, s);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

}  // namespace aoh
