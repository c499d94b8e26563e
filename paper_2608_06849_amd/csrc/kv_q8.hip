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
// on the number of tokens only: a workgroup for each chunk of positions (or pair of
// chunks) of a paged head, and for a ring only for as many as its sinks and its
// window can touch.  A chunk's rows are loaded before its block table entry is
// known.
// Bound: memory.  One prompt of 65536 tokens, 8 paged heads of width 128, bf16: 91 us
// to read (4.4 TB/s moved), 89 to write; a large copy moves 4.65 TB/s on the card.
// Heads of a page side by side in the grid, or several of them a workgroup, were
// slower: the scale bytes of a page's heads share lines, which then several XCDs
// write at a time.
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

// Eight consecutive values of a row as they are loaded.
template <typename T>
struct Row8;
template <>
struct Row8<uint16_t> {
  u32x4 w;
  __device__ __forceinline__ void load(const uint16_t* p) { w = ld16(p); }
  // as fp32; 0 for a row that is not `on`
  __device__ __forceinline__ void values(float (&x)[8], bool on) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = on ? __builtin_bit_cast(float, w[i] << 16) : 0.f;
      x[2 * i + 1] = on ? __builtin_bit_cast(float, w[i] & 0xffff0000u) : 0.f;
    }
  }
};
template <>
struct Row8<float> {
  f32x4 w[2];
  __device__ __forceinline__ void load(const float* p) {
    w[0] = *reinterpret_cast<const f32x4*>(p);
    w[1] = *reinterpret_cast<const f32x4*>(p + 4);
  }
  __device__ __forceinline__ void values(float (&x)[8], bool on) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = on ? w[i >> 2][i & 3] : 0.f;
  }
};

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

// The head that a workgroup of a launch handles, its rank in its cache, and the
// number of its first chunk: of the sequence's chunks from `start` on, or of the
// ring's (sink chunks first, then those of the window that ends at `end`).
struct Work {
  bool streaming;
  int g, rank, chunk;
};
template <int CHUNKS>
__device__ __forceinline__ Work work_of(const Q8Args& a) {
  Work w;
  int x = a.x0 + (int)blockIdx.x;
  w.streaming = x >= a.n_ret * a.groups;
  if (w.streaming) x -= a.n_ret * a.groups;
  const int per = w.streaming ? a.ring_groups : a.groups;
  w.rank = x / per;
  w.chunk = (x - w.rank * per) * CHUNKS;
  w.g = w.streaming ? a.str[w.rank] : a.ret[w.rank];
  return w;
}
// Logical page of a chunk; negative for none.
__device__ __forceinline__ int page_of(const Q8Args& a, bool streaming, int chunk, int start, int end) {
  const int first = start / kPage;
  if (!streaming || a.ring_sinks < 0) return first + chunk;
  // the pages up to the sinks' end, then those of the window that come after them
  const int sink_end = max(first, a.ring_sinks);
  if (chunk < a.ring_sinks) return first + chunk < sink_end ? first + chunk : -1;
  return max(sink_end, max(start, end - a.window) / kPage) + chunk - a.ring_sinks;
}

// The positions [lo, hi) of a chunk, and where this thread's position p lives: unit
// and row, and whether the chunk is one whole unit.
struct Chunk {
  int lp, lo, hi, page;
  bool live;  // uniform: there is something to do
};
struct Place {
  int64_t unit;
  int row;
  bool whole;
};
// `oldest`: the least position after the sinks that the ring keeps.
__device__ __forceinline__ Place place_of(const Q8Args& a, const Work& w, const Chunk& x, int b, int p, int oldest) {
  Place at;
  at.whole = x.hi - x.lo == kPage;
  if (!w.streaming) {
    at.unit = (int64_t)x.page * a.n_ret + w.rank;
    at.row = p % kPage;
    return at;
  }
  if (at.whole) {
    const int first = ring_slot(x.lo, a.n_sink, a.window);
    at.whole = first % kPage == 0 && ring_slot(x.hi - 1, a.n_sink, a.window) == first + kPage - 1 &&
               (x.hi <= a.n_sink || x.lo >= max(a.n_sink, oldest));
  }
  const int slot = ring_slot(p, a.n_sink, a.window);
  at.unit = ((int64_t)b * a.n_str + w.rank) * a.ring_blocks + slot / kPage;
  at.row = slot % kPage;
  return at;
}

}  // namespace

// CHUNKS chunks a workgroup, whose rows are all loaded before the first is stored.
template <int D, typename T, bool I8, int CHUNKS>
__global__ __launch_bounds__(2 * D) void append_q8_kernel(Q8Args a) {
  __shared__ __align__(16) VTiles<D> tiles[CHUNKS > 1 ? 2 : 1];
  const int b = blockIdx.y;
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
  const Work w = work_of<CHUNKS>(a);
  // ring: a later position of this call overwrites all others
  auto kept = [&](int p) { return !w.streaming || p < a.n_sink || p >= end - a.window; };

  const int tid = threadIdx.x;
  const int row = tid / (D / 8), c = tid % (D / 8);
  const T* k = reinterpret_cast<const T*>(a.k) + (int64_t)b * a.k_sb + (int64_t)w.g * a.k_sh + 8 * c;
  const T* v = reinterpret_cast<const T*>(a.v) + (int64_t)b * a.v_sb + (int64_t)w.g * a.v_sh + 8 * c;
  Chunk x[CHUNKS];
  Row8<T> kx[CHUNKS], vx[CHUNKS];
  bool on[CHUNKS];
#pragma unroll
  for (int u = 0; u < CHUNKS; ++u) {
    x[u].lp = page_of(a, w.streaming, w.chunk + u, start, end);
    x[u].lo = max(x[u].lp * kPage, start);
    x[u].hi = min(x[u].lp * kPage + kPage, end);
    // nothing beyond the block table
    x[u].live = x[u].lo < x[u].hi && (kept(x[u].lo) || kept(x[u].hi - 1)) && (w.streaming || x[u].lp < a.max_pages);
    const int p = x[u].lp * kPage + row;
    on[u] = x[u].live && p >= x[u].lo && p < x[u].hi && kept(p);
    if (on[u]) {
      const int64_t t = row0 + (p - start);
      kx[u].load(k + t * a.k_st);
      vx[u].load(v + t * a.v_st);
    }
  }
  // block table entries are needed only when the rows have come
#pragma unroll
  for (int u = 0; u < CHUNKS; ++u)
    x[u].page = !w.streaming && x[u].live ? a.block_table[(int64_t)b * a.max_pages + x[u].lp] : 0;
#pragma unroll
  for (int u = 0; u < CHUNKS; ++u) {
    if (!x[u].live || (!w.streaming && (x[u].page < 0 || x[u].page >= a.num_pages))) continue;  // uniform; unmapped
    const Place at = place_of(a, w, x[u], b, x[u].lp * kPage + row, end - a.window);
    float f[8];
    uint32_t kb, vb;
    kx[u].values(f, on[u]);
    const u32x2 kw = quantise8<D, I8>(f, kb);
    vx[u].values(f, on[u]);
    const u32x2 vw = quantise8<D, I8>(f, vb);
    if (on[u]) {
      *reinterpret_cast<u32x2*>((w.streaming ? a.rk : a.pk) + at.unit * (kPage * D) + at.row * D + 8 * c) = kw;
      if (c == 0)
        *reinterpret_cast<uint16_t*>((w.streaming ? a.rs : a.ps) + at.unit * kScaleBytes + 2 * at.row) =
            (uint16_t)(kb | (vb << 8));
    }
    uint8_t* uv = (w.streaming ? a.rv : a.pv) + at.unit * (kPage * D);
    if (at.whole) {  // uniform; row r of the unit is row `row`
      VTiles<D>& vt = tiles[CHUNKS > 1 ? u & 1 : 0];  // in turn: one barrier a chunk
      vt[2 * c][row] = vw[0];
      vt[2 * c + 1][row] = vw[1];
      __syncthreads();
      if (tid < D) st16(uv + 16 * tid, transpose4(ld16(&vt[tid >> 2][4 * (tid & 3)])));
    } else if (on[u]) {
#pragma unroll
      for (int i = 0; i < 8; ++i) uv[v_offset(8 * c + i, at.row)] = (uint8_t)(vw[i >> 2] >> (8 * (i & 3)));
    }
  }
}

template <int D, typename T, bool I8, int CHUNKS>
__global__ __launch_bounds__(2 * D) void read_q8_kernel(Q8Args a) {
  __shared__ __align__(16) VTiles<D> tiles[CHUNKS > 1 ? 2 : 1];
  const int b = blockIdx.y;
  const int start = a.start_pos ? a.start_pos[b] : 0;
  if (start < 0 || start >= kMaxPos) return;
  const int len = a.lens[b];
  const int end = min(start + a.n, len);
  const Work w = work_of<CHUNKS>(a);
  auto held = [&](int p) { return !w.streaming || p < a.n_sink || p >= len - a.window; };

  const int tid = threadIdx.x;
  const int row = tid / (D / 8), c = tid % (D / 8);
  Chunk x[CHUNKS];
#pragma unroll
  for (int u = 0; u < CHUNKS; ++u) {
    x[u].lp = page_of(a, w.streaming, w.chunk + u, start, len);
    x[u].lo = max(x[u].lp * kPage, start);
    x[u].hi = min(x[u].lp * kPage + kPage, end);
    x[u].live = x[u].lo < x[u].hi && (held(x[u].lo) || held(x[u].hi - 1)) && (w.streaming || x[u].lp < a.max_pages);
    x[u].page = !w.streaming && x[u].live ? a.block_table[(int64_t)b * a.max_pages + x[u].lp] : 0;
  }
  u32x2 kw[CHUNKS], vw[CHUNKS];
  u32x4 tile[CHUNKS];
  uint32_t sw[CHUNKS];
  bool on[CHUNKS], whole[CHUNKS];
#pragma unroll
  for (int u = 0; u < CHUNKS; ++u) {
    x[u].live = x[u].live && x[u].page >= 0 && (w.streaming || x[u].page < a.num_pages);
    if (!x[u].live) continue;
    const int p = x[u].lp * kPage + row;
    const Place at = place_of(a, w, x[u], b, p, len - a.window);
    on[u] = p >= x[u].lo && p < x[u].hi && held(p);
    whole[u] = at.whole || !w.streaming;  // a page is read whole wherever the chunk lies in it
    const uint8_t* uv = (w.streaming ? a.rv : a.pv) + at.unit * (kPage * D);
    if (on[u]) {
      kw[u] = ld8((w.streaming ? a.rk : a.pk) + at.unit * (kPage * D) + at.row * D + 8 * c);
      sw[u] = *reinterpret_cast<const uint16_t*>((w.streaming ? a.rs : a.ps) + at.unit * kScaleBytes + 2 * at.row);
    }
    if (whole[u]) {
      if (tid < D) tile[u] = ld16(uv + 16 * tid);
    } else if (on[u]) {
      vw[u] = u32x2{0u, 0u};
#pragma unroll
      for (int i = 0; i < 8; ++i) vw[u][i >> 2] |= (uint32_t)uv[v_offset(8 * c + i, at.row)] << (8 * (i & 3));
    }
  }
  T* k = reinterpret_cast<T*>(const_cast<void*>(a.k)) + (int64_t)b * a.k_sb + (int64_t)w.g * a.k_sh + 8 * c;
  T* v = reinterpret_cast<T*>(const_cast<void*>(a.v)) + (int64_t)b * a.v_sb + (int64_t)w.g * a.v_sh + 8 * c;
#pragma unroll
  for (int u = 0; u < CHUNKS; ++u) {
    if (!x[u].live) continue;
    if (whole[u]) {  // uniform
      VTiles<D>& vt = tiles[CHUNKS > 1 ? u & 1 : 0];  // in turn: one barrier a chunk
      if (tid < D) *reinterpret_cast<u32x4*>(&vt[tid >> 2][4 * (tid & 3)]) = transpose4(tile[u]);
      __syncthreads();
      vw[u] = u32x2{vt[2 * c][row], vt[2 * c + 1][row]};
    }
    if (on[u]) {
      const int64_t t = x[u].lp * kPage + row - start;
      store8<I8>(k + t * a.k_st, kw[u], row_scale(sw[u] & 0xffu));
      store8<I8>(v + t * a.v_st, vw[u], row_scale(sw[u] >> 8));
    }
  }
}

namespace {

template <int D, typename T, bool I8, int CHUNKS>
void launch_chunks(const Q8Args& a, bool write, dim3 grid, hipStream_t s) {
  if (write) hipLaunchKernelGGL((append_q8_kernel<D, T, I8, CHUNKS>), grid, dim3(2 * D), 0, s, a);
  else hipLaunchKernelGGL((read_q8_kernel<D, T, I8, CHUNKS>), grid, dim3(2 * D), 0, s, a);
}

template <int D, typename T>
void launch_type(const Q8Args& a, int format, bool pairs, bool write, dim3 grid, hipStream_t s) {
  if (format == kFormatI8) {
    if (pairs) launch_chunks<D, T, true, 2>(a, write, grid, s);
    else launch_chunks<D, T, true, 1>(a, write, grid, s);
  } else {
    if (pairs) launch_chunks<D, T, false, 2>(a, write, grid, s);
    else launch_chunks<D, T, false, 1>(a, write, grid, s);
  }
}

template <int D>
void launch_width(const Q8Args& a, int dtype, int format, bool pairs, bool write, dim3 grid, hipStream_t s) {
  if (dtype == 1) launch_type<D, float>(a, format, pairs, write, grid, s);
  else launch_type<D, uint16_t>(a, format, pairs, write, grid, s);
}

}  // namespace

// The runtime takes a launch's work-items modulo 2^32, so a grid of 2^31 and more
// goes in parts: of whole sequences, or of one sequence's workgroups.
hipError_t launch_q8(const Q8Args& a, int dtype, int format, int d, bool write, hipStream_t s) {
  const int64_t most = ((int64_t)1 << 31) / (2 * d);  // workgroups of a launch
  const int64_t chunks = ((int64_t)a.n + kPageTokens - 1) / kPageTokens + 1;
  // pages that hold sinks, and pages that a window touches
  const int64_t sinks = ((int64_t)a.n_sink + kPageTokens - 1) / kPageTokens;
  const int64_t touched = sinks + ((int64_t)a.window + kPageTokens - 1) / kPageTokens + 1;
  const int64_t ring_chunks = std::min(chunks, touched);
  // Two chunks a workgroup where a sequence has no more than those (64 x 1 token,
  // written and read back 6.6 us, 7.5 with one), and in large packed writes, where
  // many workgroups find their sequence ended (16 prompts of 512-24576 tokens,
  // written and read back 296 us, 304 with one); else one, since fewer workgroups fill
  // the GPU less evenly (4 x 4096: 33.3 us, 33.8 with two, 38.6 with four; 8 x 1000
  // written: 22.4, 23.4, 27.1).
  const bool pairs = chunks == 2 || (a.cu_seqlens && (chunks * a.n_ret + ring_chunks * a.n_str) * a.B >= 32768);
  const int per = pairs ? 2 : 1;
  const int64_t groups = (chunks + per - 1) / per, ring_groups = (ring_chunks + per - 1) / per;
  const int64_t per_seq = groups * a.n_ret + ring_groups * a.n_str;
  const int64_t seqs = std::min<int64_t>(std::max<int64_t>(1, most / per_seq), 65535);
  const int es = dtype == 1 ? 4 : 2;
  for (int64_t b0 = 0; b0 < a.B; b0 += seqs) {
    Q8Args p = a;
    p.groups = (int)groups;
    p.ring_groups = (int)ring_groups;
    p.ring_sinks = touched < chunks ? (int)sinks : -1;
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
    for (int64_t x0 = 0; x0 < per_seq; x0 += most) {
      p.x0 = (int)x0;
      const dim3 grid((unsigned)std::min(most, per_seq - x0), (unsigned)std::min<int64_t>(seqs, a.B - b0));
      if (d == 64) launch_width<64>(p, dtype, format, pairs, write, grid, s);
      else launch_width<128>(p, dtype, format, pairs, write, grid, s);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

}  // namespace aoh
